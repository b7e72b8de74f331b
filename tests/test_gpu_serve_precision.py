"""How exact the serving operators are where test_gpu_serve.py's worst-case bounds leave room."""
import numpy as np
import pytest

import serve_oracle as so
from test_gpu_serve import dev, harp, host, make_batch, rounded, say  # noqa: F401  (harp: the fixture)

pytestmark = pytest.mark.gpu


def half_step(x, dtype):
    """Half the distance of neighbouring numbers of the type at |x|, x in float64."""
    bits = 8 if dtype == "bf16" else 24
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 1e-300))) - bits)


def attend(harp, cache, table, row_start, kv_len, Q, rope, dtype, longest=None):
    out = harp.harp_attention_int8(harp.KVCache(*(dev(a) for a in cache)), dev(table), dev(row_start), dev(kv_len), dev(Q, dtype),
                                   rope=None if rope is None else tuple(dev(a) for a in rope), max_kv_len=longest)
    return host(out).astype(np.float64)


def two_halves_bound(A, S, dh, keys):
    """What 22 bits of queries and weights and float32 sums leave: test_gpu_serve.py's derivation."""
    return 2 * A * (2.0 ** -21 * (1 + 2 * S) + (dh + keys) * 2.0 ** -24)


@pytest.mark.parametrize("new,total,page,heads,group,dh", [([1], [40], 16, 8, 4, 64), ([1] * 6, [64, 65, 3, 50, 31, 17], 32, 4, 4, 128), ([9, 3], [60, 20], 16, 4, 7, 64),
                                                           ([1, 1], [300, 700], 64, 4, 8, 128), ([1], [1500], 128, 2, 8, 64)])
def test_few_rows_of_bfloat16_are_the_rounded_result(harp, new, total, page, heads, group, dh):
    """Between the exact result and a bfloat16 one of few rows stands the result's own rounding, and what two halves leave."""
    say("few rows, bf16", new, total, page, heads, group, dh)
    r = np.random.default_rng(sum(total) + dh + group)
    cache, table, row_start, kv_len, angles = make_batch(r, new, total, page, heads, dh)
    Q = rounded(r.standard_normal((int(row_start[-1]), heads * group, dh)) * 1.5, "bf16")
    O, A, S = so.attention(cache, table, row_start, kv_len, Q, angles, False, dh ** -0.5)
    got = attend(harp, cache, table, row_start, kv_len, Q, angles, "bf16", max(total))
    bound = two_halves_bound(A, S, dh, table.shape[1] * page)
    tol = half_step(np.abs(O) + bound, "bf16") + bound
    assert (np.abs(got - O) <= tol).all(), (int((np.abs(got - O) > tol).sum()), float(np.max(np.abs(got - O) / tol)))


@pytest.mark.parametrize("new,heads", [(1, 1), (129, 28)])
@pytest.mark.parametrize("apart", [8, 16, 18, 20])
def test_float32_pages_of_very_different_magnitudes(harp, apart, new, heads):
    """The first page's values are 2^apart times as large and its keys weigh 2^-apart as much, so both count alike.  Scores come from one
    product each, exact but for three roundings of a score of `apart` (base 2); sums of n keys and the 22 bits add."""
    say("scales apart", apart, new, heads)
    r = np.random.default_rng(apart)
    dh, total = 64, max(new + 3, 32)
    cache, table, row_start, kv_len, _ = make_batch(r, [new], [total], 16, heads, dh)
    k, v, ks, vs = cache
    k[:], ks[:], vs[:] = 0, 1, r.uniform(0.5, 1, vs.shape)
    k[table[0, 0], :, :, 0] = -127
    ks[table[0, 0]] = apart * np.log(2) / 127
    vs[table[0, 0]] *= 2.0 ** apart
    Q = np.zeros((new, 4 * heads, dh), np.float32)
    Q[:, :, 0] = 1
    O, A, _ = so.attention(cache, table, row_start, kv_len, Q, None, False, 1.0)
    out = harp.harp_attention_int8(harp.KVCache(*(dev(a) for a in cache)), dev(table), dev(row_start), dev(kv_len), dev(Q), scale=1.0, max_kv_len=total)
    keys = (total - new + 1 + np.arange(new))[:, None, None]
    tol = 2.0 ** -23 * np.abs(O) + 2 * A * 2.0 ** -24 * (8 + 4 * apart + keys)
    off = np.abs(host(out) - O)
    assert (off <= tol).all(), float(np.max(off / tol))


def spread(cache, table, row_start, kv_len, Q, scale):
    """(O, E) in float64: the result, and the r.m.s. that independent roundings of queries and weights to one half (each within 2^-11 of itself,
    r.m.s. 2^-11 / sqrt(3) at most) leave in it.  A score's is s_j^2 = sum_i (q_i k_ij scale)^2 2^-22 / 3; it moves the weight in both sums, so o by
    w_j (V_j - o) times it.  The sum of weights is taken before they are rounded, so a weight's own rounding moves o by w_j V_j times it."""
    _, heads, size, dh = cache[0].shape
    group = Q.shape[1] // heads
    O, E = np.zeros(Q.shape), np.zeros(Q.shape)
    for b in range(len(kv_len)):
        total, n = int(kv_len[b]), int(row_start[b + 1] - row_start[b])
        K, V, there = so.tokens(cache, table, b, total)
        assert there.all()
        for j in range(n):
            see, t = total - n + j + 1, int(row_start[b]) + j
            for h in range(Q.shape[1]):
                k, v, x = K[:see, h // group], V[:see, h // group], Q[t, h].astype(np.float64) * scale
                w = np.exp(k @ x - (k @ x).max())
                w /= w.sum()
                o = w @ v
                c = w * w * ((k * k) @ (x * x))
                moved = np.maximum(c @ (v * v) - 2 * o * (c @ v) + o * o * c.sum(), 0) + (w * w) @ (v * v)
                O[t, h], E[t, h] = o, np.sqrt(moved * 2.0 ** -22 / 3)
    return O, E


@pytest.mark.parametrize("new,total,page,heads,group,dh", [([600], [600], 128, 8, 3, 64), ([130], [2600], 64, 7, 4, 128), ([300, 200], [300, 450], 32, 8, 4, 128),
                                                           ([128], [4000], 32, 1, 16, 64), ([1], [9000], 32, 1, 4, 64), ([2, 1, 1], [1500, 900, 64], 16, 4, 4, 128)])
def test_bfloat16_errors_are_those_of_independent_roundings(harp, new, total, page, heads, group, dh):
    """No entry is further off than half a step of bfloat16 and six times the r.m.s. of what the roundings leave (of 10^6 normal numbers one
    in a thousand runs has one beyond), and all together not further than their r.m.s.  The roundings to one half bound what two halves leave, too."""
    say("errors", new, total, page, heads, group, dh)
    r, dtype = np.random.default_rng(sum(total) + dh), "bf16"
    cache, table, row_start, kv_len, _ = make_batch(r, new, total, page, heads, dh)
    Q = rounded(r.standard_normal((int(row_start[-1]), heads * group, dh)) * 0.7, dtype)
    O, E = spread(cache, table, row_start, kv_len, Q, dh ** -0.5)
    off = np.abs(attend(harp, cache, table, row_start, kv_len, Q, None, dtype, max(total)) - O)
    h = half_step(np.abs(O) + 6 * E, dtype)
    assert (off <= h + 6 * E).all(), float(np.max(off / (h + 6 * E)))
    assert np.mean(off ** 2) <= 1.1 * np.mean(h ** 2 / 3 + E ** 2), float(np.mean(off ** 2) / np.mean(h ** 2 / 3 + E ** 2))
