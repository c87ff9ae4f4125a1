"""CPU checks of the rules that choose a kernel, through the library's own
functions (no GPU work)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2011_11188_amd as m
    return C.CDLL(m.LIB_PATH)


def test_column_sums_one_launch_rule(lib):
    """One launch of 1024-thread blocks: only above one 256-row chunk (below,
    most of its row lanes would have no row) and within a launch's 2^32 threads."""
    f = lib["_ZN4mdnn16column_sums_onceEll"]
    f.argtypes, f.restype = [C.c_int64, C.c_int64], C.c_bool
    for cols in (8, 64, 1000, 1 << 20):
        assert not any(f(rows, cols) for rows in (0, 1, 32, 255, 256, 1025, 5000))
        assert all(f(rows, cols) for rows in (257, 1000, 1024))
    assert not f(1024, 7)
    for cols in ((1 << 28) - 64, (1 << 28) - 63, 1 << 28, (1 << 28) + 70, 1 << 40):
        assert not f(300, cols) or -(-cols // 64) * 1024 < 2 ** 32


class _Geom(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "h", "w", "c", "k", "r", "s", "pad", "ho", "wo")]


class _Plan(C.Structure):
    _fields_ = [("splits", C.c_int), ("k_per_split", C.c_int64)]


def _geom(n, h, w, c, k, r, pad):
    return _Geom(n, h, w, c, k, r, r, pad, h + 2 * pad - r + 1, w + 2 * pad - r + 1)


def test_direct_to_lds_filter_gradient_offsets_fit_32_bits(lib):
    """Few pixels and very many output channels: dy's byte offsets up to the end
    of the padded last K step (64 pixels) stay below 2^32, where the range check
    turns them into zeros (past it they would wrap to valid rows, and an Inf
    there would reach the sums as 0 * Inf)."""
    f = lib["_ZN4mdnn21conv_pipe_filter_planERKNS_8ConvGeomE"]
    f.argtypes, f.restype = [C.POINTER(_Geom)], _Plan
    taken = 0
    for n in (1, 2, 3, 15, 16, 31, 32, 33, 63, 64, 65, 129):
        for k in [8, 64, 1 << 20] + [(1 << p) + d for p in (24, 25, 26) for d in (-8, 0, 8)]:
            if f(C.byref(_geom(n, 1, 1, 8, k, 1, 0))).splits:
                taken += 1
                assert -(-n // 64) * 64 * k * 2 <= 2 ** 32, (n, k)
    assert taken > 40


def test_direct_to_lds_convolution_launches_stay_below_2_32_threads(lib):
    """More output pixels than 512 threads per 128 x 128 or 256 x 64 tile leave
    room for go to the general kernel, whose launch still holds them."""
    fit = lib["_ZN4mdnn18conv_pipe_runs_fitEll"]
    fit.argtypes, fit.restype = [C.c_int64, C.c_int64], C.c_bool
    taken = 0
    for n in (1, 64, 65, 72, 128, 129, 1000):
        for m in [64, 1 << 20] + [(1 << p) + d for p in (27, 28, 29, 30, 31) for d in (-300, -1, 0)]:
            if fit(m, n):
                taken += 1
                assert 512 * max(-(-m // 128) * -(-n // 128), -(-m // 256) * -(-n // 64)) < 2 ** 32, (m, n)
    assert taken > 30 and all(fit(1 << 20, n) for n in (1, 64, 200, 1000))


class _I8Order(C.Structure):
    _fields_ = [("by_cols", C.c_bool), ("group", C.c_uint32)]


def _i8_order(lib, M, N, ldd, elem_bytes, K=4096):
    f = lib["_ZN4mdnn13i8_tile_orderElllll"]
    f.argtypes, f.restype = [C.c_int64] * 5, _I8Order
    return f(M, N, K, ldd, elem_bytes)


def _walk(order, tiles_m, tiles_n):
    """The tiles (row, column) of consecutive workgroups: groups of `group` tile columns row by row, or of tile rows
    column by column."""
    major, minor = (tiles_n, tiles_m) if order.by_cols else (tiles_m, tiles_n)
    for g in range(0, major, order.group):
        for b in range(minor):
            for a in range(g, min(g + order.group, major)):
                yield (b, a) if order.by_cols else (a, b)


@pytest.mark.parametrize("M,N", [(256, 4096), (512, 2048), (1024, 1024), (1024, 2048), (4096, 512)])
def test_int8_tiles_of_an_xcd_share_their_panels(lib, M, N):
    """Grids of 64 x 64 tiles of a few to a CU: the 32 workgroups that an XCD starts with read 12 panels of the
    operands, the fewest that 32 tiles in whole rows of 4 or 8 have (in groups of 16 columns they read 18)."""
    order = _i8_order(lib, M, N, N, 2)
    at = list(_walk(order, M // 64, N // 64))
    assert len(set(at)) == len(at) == (M // 64) * (N // 64)
    for x in range(0, len(at), 32):
        rows, cols = {r for r, _ in at[x:x + 32]}, {c for _, c in at[x:x + 32]}
        assert len(rows) + len(cols) <= 12, (x, rows, cols)


def test_int8_tile_order_by_the_size_of_d(lib):
    """Wide D: 8 tile columns below 256 MB, 16 from there on and up to four steps; tall D: 4 tile rows where its rows are whole pages and
    it is not far above N, 8 elsewhere."""
    for es, n in ((2, 1 << 14), (4, 1 << 13)):
        at = (1 << 28) // es // n
        assert (_i8_order(lib, at - 1, n, n, es).by_cols, _i8_order(lib, at - 1, n, n, es).group) == (True, 8)
        assert (_i8_order(lib, at, n, n, es).by_cols, _i8_order(lib, at, n, n, es).group) == (True, 16)
        assert (_i8_order(lib, at - 1, n, n, es, 512).group, _i8_order(lib, at - 1, n, n, es, 513).group) == (16, 8)
    for args, group in (((16384, 8192, 8192, 2), 4), ((65536, 4096, 4096, 2), 8), ((12000, 5000, 5000, 2), 8),
                        ((20, 10, 10, 4), 8)):
        o = _i8_order(lib, *args)
        assert (o.by_cols, o.group) == (False, group)


I8_64, I8_128, I8_128X8, I8_256X128, I8_256 = range(5)


F32, F16, BF16 = range(3)


def _i8_choice(lib, M, N, K, d_type=F16):
    f = lib["_ZN4mdnn14i8_tile_choiceEllll12mdnn_dtype_t"]
    f.argtypes, f.restype = [C.c_int64] * 4 + [C.c_int], C.c_int
    return f(M, N, K, N, d_type)


@pytest.mark.parametrize("size,tile", [
    # 128 tiles of 128 x 128 and one more; 160 of them, one more, and one step more
    ((1024, 2048, 4096), I8_64), ((1152, 2048, 4096), I8_128), ((1280, 2048, 2048), I8_64), ((1280, 2048, 2049), I8_128),
    ((1408, 2048, 1024), I8_128X8),
    # 256 of them, and one more
    ((2048, 2048, 1536), I8_128X8), ((2048, 2048, 1537), I8_128), ((2049, 2048, 1537), I8_128X8),
    # 160 tiles of 256 x 128 and more, 256 and more
    ((1024, 5120, 4096), I8_128X8), ((1100, 4099, 1536), I8_128X8), ((1100, 4099, 1537), I8_256X128),
    ((2048, 4096, 4096), I8_256X128), ((2500, 2500, 1152), I8_128X8), ((30000, 300, 1537), I8_256X128),
    # whole rounds of 256 x 256 tiles, and nearly whole ones; four steps and one byte more
    ((4096, 4096, 128), I8_256), ((16384, 8192, 8192), I8_256), ((13000, 13000, 320), I8_256),
    ((9600, 13952, 512), I8_128X8), ((9600, 13952, 513), I8_256), ((14000, 5000, 512), I8_128X8),
    # bf16, and tall fp32 D in rows of whole pages, up to four steps; wide, other rows, more steps
    ((4096, 4096, 512, BF16), I8_128X8), ((4096, 4096, 513, BF16), I8_256),
    ((10240, 8192, 512, F32), I8_128X8), ((10240, 8192, 513, F32), I8_256), ((8192, 8192, 512, F32), I8_256),
    ((14176, 6848, 128, F32), I8_256), ((10240, 8192, 512, F16), I8_256),
    # five, six and seven rounds of 128 x 128 for two of 256 x 256, below and above K = 1024
    ((4100, 4100, 4096), I8_128X8), ((5184, 4544, 1024), I8_128X8), ((5184, 4544, 1025), I8_256),
    ((5000, 5500, 640), I8_256)])
def test_int8_tile_choice(lib, size, tile):
    """Both sides of the rule's lines."""
    assert _i8_choice(lib, *size) == tile


def test_int8_tests_reach_every_tile(lib):
    """The sizes of the product's GPU tests run every tile of rows on 16 bytes with whole last steps and with partial
    ones (two different kernels each)."""
    from tests import test_gpu_int8 as g

    def sizes(test):
        return [size[:3] for mark in test.pytestmark if mark.args[0] == "M,N,K" for size in mark.args[1]]

    assert {_i8_choice(lib, *s) for s in sizes(g.test_product_whole_steps)} == set(range(5))
    assert all(s[2] % 128 == 0 for s in sizes(g.test_product_whole_steps))
    partial = [s for s in sizes(g.test_product_each_tile) if s[2] % 128]
    assert {_i8_choice(lib, *s) for s in partial} == set(range(5))
