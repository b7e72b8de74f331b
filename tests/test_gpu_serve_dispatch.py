"""The serving operators where the choice of a kernel decides what is computed how: test_serve_dispatch.py says which kernels these sizes reach."""
import numpy as np
import pytest

import serve_oracle as so
from test_gpu_serve import check_attention, dev, harp, host, make_batch, rounded, say  # noqa: F401  (harp: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d_out,d_in", [(700, 4100, 16400)])
def test_matmul_largest_tiles_in_slices(harp, n, d_out, d_in):
    import torch
    say("matmul", n, d_out, d_in)
    r = np.random.default_rng(n + d_out)
    a, w = r.integers(-128, 128, (n, d_in)).astype(np.int8), r.integers(-128, 128, (d_out, d_in)).astype(np.int8)
    sa, sw = r.uniform(0.01, 2, n).astype(np.float32), r.uniform(0.01, 2, d_out).astype(np.float32)
    want = so.matmul(a, sa, w, sw)
    for dtype, td in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        assert np.array_equal(host(harp.harp_matmul_int8(dev(a), dev(sa), dev(w), dev(sw), dtype=td)), rounded(want, dtype)), dtype


# Rows at negative positions, whole tiles of them, and a sequence whose only page is not there, in every attention kernel
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,total,page,heads,group,dh", [([200, 300, 130], [100, 330, 16], 16, 28, 2, 64), ([300, 130], [200, 16], 32, 28, 2, 128),
                                                           ([200, 130, 129], [100, 1300, 16], 64, 8, 4, 128), ([260, 150], [100, 1400], 16, 16, 2, 64),
                                                           ([130, 9, 2], [2, 40, 16], 16, 2, 1, 64), ([140, 3], [12, 90], 32, 1, 1, 128),
                                                           ([150, 2], [6, 1500], 64, 1, 1, 64), ([1, 135], [2000, 5], 128, 2, 1, 128)])
def test_attention_rows_without_keys(harp, new, total, page, heads, group, dh, dtype):
    say("rows without keys", new, total, page, heads, group, dh, dtype)
    r = np.random.default_rng(sum(total) + page + dh)
    cache, table, row_start, kv_len, angles = make_batch(r, new, total, page, heads, dh, missing=((len(new) - 1, 0, -1),) if total[-1] == 16 else ())
    Q = rounded(r.standard_normal((int(row_start[-1]), heads * group, dh)) * 1.5, dtype)
    out = host(check_attention(harp, cache, table, row_start, kv_len, Q, angles, dh == 64, dtype, longest=max(total)))
    for b, (n, t) in enumerate(zip(new, total)):
        none = n if total[-1] == 16 and b == len(new) - 1 else max(n - t, 0)
        assert not out[row_start[b]:row_start[b] + none].any()


@pytest.mark.parametrize("new,heads", [([3, 2], 1), ([200, 90], 28)])
def test_no_pages_at_all(harp, new, heads):
    """A table of no columns and a rotation of no positions: no row has a place, results are zeros and nothing is read or stored."""
    import torch
    rows = sum(new)
    row_start, kv_len = dev(np.cumsum([0] + new).astype(np.int32)), dev(np.zeros(2, np.int32))
    table = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    rope = torch.zeros(0, 32, device="cuda"), torch.zeros(0, 32, device="cuda")
    c = harp.kv_cache(2, heads, 64, 16)
    c.k_scale.fill_(3)
    x = torch.ones(rows, 2 * heads, 64, device="cuda")
    out = torch.full_like(x, 7.0)
    harp.harp_kv_append(c, table, row_start, kv_len, x[:, :heads], x[:, heads:], rope=rope)
    harp.harp_attention_int8(c, table, row_start, kv_len, x, out, rope=rope)
    assert not bool(out.any()) and bool((c.k_scale == 3).all())
    assert not any(bool(t.any()) for t in harp.harp_kv_gather(c, table, row_start, kv_len, rows))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,total,heads", [([3], [40], 2), ([140, 150], [130, 170], 28)])
def test_an_infinite_query_is_nan(harp, new, total, heads, dtype):
    """Softmax of scores that are all -inf has no value; results are NaN as for a NaN query, not the zeros of a row without keys."""
    r = np.random.default_rng(15)
    cache, table, row_start, kv_len, _ = make_batch(r, new, total, 16, heads, 64)
    np.clip(np.abs(cache[0]), 1, 127, out=cache[0])                 # no key has a coordinate of 0
    Q = rounded(r.standard_normal((sum(new), 4 * heads, 64)), dtype)
    Q[1, 0, 5], Q[-1, 1, 7], Q[-1, 2, 9] = -np.inf, np.inf, -np.inf
    with np.errstate(invalid="ignore"):
        O, _, _ = so.attention(cache, table, row_start, kv_len, Q, None, False, 0.125)
    out = host(harp.harp_attention_int8(harp.KVCache(*(dev(a) for a in cache)), dev(table), dev(row_start), dev(kv_len), dev(Q, dtype)))
    assert np.array_equal(np.isnan(out), np.isnan(O)) and np.isnan(out).any()
    assert np.isnan(out[-1, 1]).all() and np.isnan(out[-1, 2]).all() and not np.isnan(out[-1, 0]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** 115, 1e-29])
@pytest.mark.parametrize("new,total,heads,group", [([1], [400], 1, 4), ([1], [700], 1, 4), ([1], [6000], 1, 2), ([130], [1300], 28, 2), ([260], [300], 28, 2)])
def test_attention_of_very_large_and_small_values(harp, new, total, heads, group, size, dtype):
    """Values near 2^117, whose sums over the keys stay within float32, and ones of 10^-29: few rows by four waves and eight, many rows, pieces of both."""
    r = np.random.default_rng(16)
    cache, table, row_start, kv_len, angles = make_batch(r, new, total, 64, heads, 64)
    cache[3][...] *= np.float32(size)
    Q = rounded(r.standard_normal((sum(new), heads * group, 64)), dtype)
    check_attention(harp, cache, table, row_start, kv_len, Q, angles, False, dtype, longest=max(total))
