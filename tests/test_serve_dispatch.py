"""Which kernels the sizes of the device tests reach: the choice is host arithmetic, so no GPU is needed.  A threshold that moves
must not leave a kernel without its tests."""
import pytest

import test_gpu_serve as gpu
import test_gpu_serve_dispatch as more
from paper_2605_29843_amd import harp

P = 1 << 20     # stands for a device address; these calls never use it


def attention_kernel(new, total, page, heads, group, dh, longest=None):
    width = max(1, max(-(-max(t, 0) // page) for t in total) + 1)      # as the tests' make_batch lays out its table
    cache = harp._CacheArgs(P, P, P, P, 1000, heads, dh, page)
    batch = harp._BatchArgs(P, width, P, P, sum(new), len(new), width)
    name = harp.lib.harp_attention_int8_kernel_name(cache, batch, heads * group, max(total) if longest is None else longest)
    return name.decode()


def parameters(test, names):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and m.args[0] == names)


SIZES = "new,total,page,heads,group,dh"


def test_every_product_kernel_is_tested():
    sizes = parameters(gpu.test_matmul, "n,d_out,d_in") + parameters(gpu.test_matmul_tiles, "n,d_out,d_in") + \
        parameters(more.test_matmul_largest_tiles_in_slices, "n,d_out,d_in")
    tiles = ["tile_32x128", "tile_64x64", "tile_128x128", "tile_192x256", "tile_256x256"]
    assert {harp.harp_matmul_int8_kernel_name(*s) for s in sizes} >= {"few", *tiles, *(t + "_sliced" for t in tiles)}
    for s in parameters(more.test_matmul_largest_tiles_in_slices, "n,d_out,d_in"):
        assert harp.harp_matmul_int8_kernel_name(*s) == "tile_256x256_sliced"


def test_every_attention_kernel_is_tested():
    assert all(attention_kernel(*s).startswith("few_rows") for s in parameters(gpu.test_attention, SIZES))
    reached = {}
    for s in parameters(more.test_attention_rows_without_keys, SIZES):
        # a row at a negative position, and at least one whole tile of rows without a key
        new, total, _, _, group, _ = s
        assert max((n - t) * group for n, t in zip(new, total)) >= 128
        reached.setdefault(attention_kernel(*s), set()).add(s[5])
    assert reached == {"many_rows": {64, 128}, "many_rows_pieces": {64, 128}, "few_rows": {64, 128}, "few_rows_pieces": {64, 128}}
    many = [attention_kernel(*s) for s in parameters(gpu.test_attention_many_rows, SIZES)]
    assert many.count("many_rows") >= 2 and many.count("many_rows_pieces") >= 2


def test_names_of_refused_arguments():
    assert harp.harp_matmul_int8_kernel_name(4, 8, 0) == "none" and harp.harp_matmul_int8_kernel_name(4, 8, 131072) == "none"
    assert harp.lib.harp_attention_int8_kernel_name(None, None, 4, 80) == b"none"


@pytest.mark.parametrize("n,name", [(1, "few"), (2048, "tile_192x256")])
def test_product_names(n, name):
    assert harp.harp_matmul_int8_kernel_name(n, 11008, 4096) == name


def test_a_table_without_pages_takes_a_rotation_without_positions():
    cache, batch = harp._CacheArgs(P, P, P, P, 3, 2, 64, 16), harp._BatchArgs(None, 0, P, P, 0, 2, 0)
    for rope, status in ((harp._RopeArgs(None, None, 0, 0), harp.HARP_OK), (harp._RopeArgs(None, None, 0, 2), harp.HARP_ERR_INVALID_ARG),
                         (harp._RopeArgs(None, None, -1, 0), harp.HARP_ERR_INVALID_ARG)):
        assert harp.lib.harp_attention_int8(cache, batch, None, 256, 64, None, 256, 64, 4, 1, 0.1, rope, 0, None, 0, None) == status
        assert harp.lib.harp_kv_append(cache, batch, None, 128, 64, None, 128, 64, 1, rope, None) == status
