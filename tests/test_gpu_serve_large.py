"""Sizes of the serving operators at which a launch or an index runs out of 32 bits."""
import numpy as np
import pytest

import serve_oracle as so
from test_gpu_serve import dev, harp, host, say  # noqa: F401  (harp: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d,dtype", [((1 << 24) + 3, 16, "bf16"), ((1 << 22) + 1, 8200, "bf16")])
def test_quantize_more_rows_than_a_launch_has(harp, n, d, dtype):
    """256 threads a row, and 1024: 2^32 threads and more.  Row i holds row i % 1021 of a small matrix."""
    import torch
    say("quantize", n, d, dtype)
    r = np.random.default_rng(d)
    period = 1021
    x = dev(r.standard_normal((period, d)).astype(np.float32) * r.uniform(0.1, 9, (period, 1)).astype(np.float32), dtype)
    codes, scales = so.quantize_rows(host(x))
    X = torch.empty(n, d, dtype=x.dtype, device="cuda")
    whole = n // period * period
    X[:whole].view(-1, period, d).copy_(x.expand(whole // period, -1, -1))
    X[whole:] = x[:n - whole]
    out = torch.full((n, d), 55, dtype=torch.int8, device="cuda")
    s = torch.full((n,), -1.0, device="cuda")
    harp.harp_quantize_rows(X, out, s)
    codes, scales = dev(codes), dev(scales)
    assert bool((out[:whole].view(-1, period, d) == codes).all()) and torch.equal(out[whole:], codes[:n - whole])
    assert bool((s[:whole].view(-1, period) == scales).all()) and torch.equal(s[whole:], scales[:n - whole])
