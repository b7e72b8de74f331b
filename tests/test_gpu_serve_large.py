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


@pytest.mark.parametrize("n,d_out,d_in,pitch", [(65535 * 64 + 70, 3, 5, 5), ((1 << 21) + 5, 20, 32, 32), (2, (1 << 24) + 40, 16, 16),
                                                (40, (1 << 24) + 40, 16, 16), (40, (1 << 24) + 40, 5, 7)])
def test_products_in_more_than_one_part(harp, n, d_out, d_in, pitch):
    """More than 2^16 tiles of 64 unaligned rows, more rows and more channels than one launch takes.  Sums are below 2^24: exact in float32."""
    import torch
    say("matmul", n, d_out, d_in, pitch)
    g = torch.Generator(device="cuda").manual_seed(n % 1000 + d_in)
    codes = lambda rows: torch.randint(-128, 128, (rows, pitch), device="cuda", generator=g, dtype=torch.int8)[:, :d_in]   # noqa: E731
    scale = lambda rows: torch.rand(rows, device="cuda", generator=g) + 0.5   # noqa: E731
    a, sa, w, sw = codes(n), scale(n), codes(d_out), scale(d_out)
    y = torch.full((n, d_out), 3.0, dtype=torch.bfloat16, device="cuda")
    harp.harp_matmul_int8(a, sa, w, sw, y)
    for j in range(0, d_out, 1 << 20):      # (the library's product of 2^24 columns at once has wrong sums)
        part = slice(j, j + (1 << 20))
        sums = a.float().contiguous() @ w[part].float().t().contiguous()
        assert torch.equal(y[:, part], ((sums * sa[:, None]) * sw[part]).bfloat16())


def test_unaligned_products_need_no_workspace(harp):
    """Sizes that are cut into slices where the operands are aligned; the kernel of unaligned ones has no slices."""
    import torch
    n, d_out, d_in = 48, 256, 2048
    r = np.random.default_rng(3)
    a, w = (dev(r.integers(-128, 128, (rows, d_in + 1)).astype(np.int8)) for rows in (n, d_out))
    sa, sw, y = torch.ones(n, device="cuda"), torch.ones(d_out, device="cuda"), torch.zeros(n, d_out, device="cuda")
    assert harp.harp_matmul_int8_workspace_size(n, d_out, d_in) > 0
    status = harp.lib.harp_matmul_int8(a.data_ptr(), d_in + 1, sa.data_ptr(), w.data_ptr(), d_in + 1, sw.data_ptr(), n, d_out, d_in, y.data_ptr(),
                                       d_out, harp.HARP_F32, None, 0, torch.cuda.current_stream().cuda_stream)
    assert status == harp.HARP_OK
    assert np.array_equal(host(y), so.matmul(host(a[:, :d_in]), np.ones(n, np.float32), host(w[:, :d_in]), np.ones(d_out, np.float32)))


def test_more_sequences_than_a_launch_has_slots(harp):
    """One new token for each of 2^24 sequences (two slots each in the cache's kernels, one in attention's).  All have one page of 16 tokens, of 251 that they
    share, for gathers and attention; the appends write a page of their own for each."""
    import torch
    batch, shared, dh = (1 << 24) + 5, 251, 64
    say("sequences", batch)
    g = torch.Generator(device="cuda").manual_seed(1)
    starts = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    lens = (torch.arange(batch, device="cuda") % shared % 16 + 1).int()
    table = (torch.arange(batch, device="cuda") % shared).int()[:, None]
    small = harp.kv_cache(shared, 1, dh, 16)
    for t in small[:2]:
        t.copy_(torch.randint(-127, 128, t.shape, device="cuda", generator=g))
    for t in small[2:]:
        t.copy_(torch.rand(t.shape, device="cuda", generator=g) * 0.02 + 0.01)
    first = slice(0, shared)

    def periodic(x, want):
        whole = batch // shared * shared
        return torch.equal(x[:whole].view(-1, shared, dh), want.view(1, shared, dh).expand(whole // shared, -1, -1)) and \
            torch.equal(x[whole:, 0], want[:batch - whole, 0])

    q = torch.randn(shared, 1, dh, device="cuda", generator=g).bfloat16()
    many = q.repeat(batch // shared + 1, 1, 1)[:batch]
    out = torch.full_like(many, 7.0)
    harp.harp_attention_int8(small, table, starts, lens, many, out)
    want = harp.harp_attention_int8(small, table[first], starts[:shared + 1], lens[first], q)
    assert periodic(out, want) and bool(torch.isfinite(want).all()) and bool(want.any())
    k, v = out, torch.full_like(many, 7.0)
    harp.harp_kv_gather(small, table, starts, lens, batch, k, v)
    want = harp.harp_kv_gather(small, table[first], starts[:shared + 1], lens[first], shared)
    assert periodic(k, want[0]) and periodic(v, want[1])
    del k, v, out
    own = harp.kv_cache(batch, 1, dh, 16)
    each = torch.arange(batch, dtype=torch.int32, device="cuda")[:, None]
    ones = torch.ones(batch, dtype=torch.int32, device="cuda")
    for t in own:
        t.zero_()
    harp.harp_kv_append(own, each, starts, ones, many, many)
    top = q.float().abs().amax(2) / torch.full((), 127.0, device="cuda")
    codes = torch.round(q.float()[:, 0] / top).to(torch.int8)
    whole = batch // shared * shared
    assert torch.equal(own.k_scale[:whole].view(-1, shared), top.view(1, -1).expand(whole // shared, -1)) and torch.equal(own.k_scale, own.v_scale)
    assert periodic(own.k[:, :, 0], codes[:, None]) and periodic(own.v[:, :, 0, :, 0], codes[:, None])
