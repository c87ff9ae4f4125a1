"""CPU checks of how a call of the last layer's cross entropy runs, through the
library's own function: no GPU work."""
import ctypes as C

import pytest

NN, NT = 0, 1
F32, F16, BF16 = 0, 1, 2
TILED, PACKED, STAGED, GENERAL = range(4)
BASE = 1 << 20  # an address on 16 bytes, never read


class _Way(C.Structure):
    _fields_ = [("way", C.c_int32), ("classes", C.c_int64)]


@pytest.fixture(scope="module")
def way():
    import paper_2011_11188_amd as m
    f = C.CDLL(m.LIB_PATH)["_ZN4mdnn8xent_wayE13mdnn_layout_tllllPKvl12mdnn_dtype_tb"]
    f.argtypes = [C.c_int] + [C.c_int64] * 4 + [C.c_void_p, C.c_int64, C.c_int, C.c_bool]
    f.restype = _Way

    def call(layout, M, N, K, t, backward, pad=0, w=BASE):
        r = f(layout, M, N, K, K, w, (N if layout == NN else K) + pad, t, backward)
        return r.way, r.classes

    return call


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("M", [1, 7, 64, 300, 1000])
@pytest.mark.parametrize("N,K", [(250880, 14336), (256000, 18432), (1 << 20, 4096), (5 << 20, 1024)])
def test_tables_past_the_loaders_reach(way, M, N, K, backward):
    """Tables of 2^31 elements and more are taken in products that 32-bit offsets reach, by the tiles, not through logits
    in the workspace."""
    assert N * K >= 2 ** 31
    for t in (F16, BF16):
        for pad in (0, 8, 64):
            got, classes = way(NT, M, N, K, t, backward, pad)
            assert got == TILED and classes % 256 == 0 and (classes + 255) * (K + pad) < 2 ** 31
        assert way(NT, M, N, K, t, backward, 3)[0] == STAGED  # (rows on any element)
    for pad in (0, 1, 64):
        got, classes = way(NT, M, N, K, F32, backward, pad)
        assert got == STAGED and classes % 256 == 0 and (classes + 255) * (K + pad) < 2 ** 30


@pytest.mark.parametrize("backward", [False, True])
def test_smaller_tables_are_whole(way, backward):
    """Below the reach a table of few rows is one product, as far as the rows allow."""
    for N, K in ((131072, 4096), (250880, 8000), (262144, 7168)):
        for M in (1, 64):
            assert way(NT, M, N, K, BF16, backward) == (TILED, N)
            assert way(NN, M, N, K, BF16, backward) == (TILED, N)
    assert way(NT, 8, 250880, 4000, F32, backward) == (STAGED, 250880)


def _tile_row_pieces(N, classes):
    return [min(classes, N - lo) for lo in range(0, N, classes)]


@pytest.mark.parametrize("M,N,K,t,backward", [
    (16384, N, 64, F32, True) for N in (8191, 8192, 8193, 8194, 8195, 8196, 16383, 16385, 16387, 16388)] + [
    (1 << 20, N, 64, F32, True) for N in (256, 257, 259, 2304, 2305, 2307, 2308, 4609)] + [
    (200, (1 << 19) + d, 65, F16, True) for d in (-1, 0, 1, 7, 8)] + [
    (1 << 20, (1 << 11) + d, 33, F32, False) for d in (-1, 0, 1, 3, 4)] + [
    (1 << 24, N, 40, F32, False) for N in (257, 513, 1027, 2050)])
def test_a_short_last_piece_does_not_change_the_way(way, M, N, K, t, backward):
    """Class-contiguous W whose classes leave one to seven (fp32: three) past whole pieces: every piece holds a 16-byte chunk,
    so that the register-staged tiles take all of them."""
    got, classes = way(NN, M, N, K, t, backward)
    assert got == STAGED
    assert min(_tile_row_pieces(N, classes)) >= (4 if t == F32 else 8)
