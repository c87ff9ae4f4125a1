"""Host checks of the 8-bit and norm entry points: every refusal below comes
before any GPU work, so it runs without a GPU."""
import pytest

FAKE = 0x10000  # never dereferenced


@pytest.fixture(scope="module")
def m():
    import paper_2011_11188_amd as mdnn
    return mdnn


def _refuses(m, status, f, *args):
    with pytest.raises(m.MdnnError) as e:
        f(*args, stream=0)
    assert e.value.status == status, args
    assert m.last_error()


@pytest.mark.parametrize("args,status", [
    # rows, cols, x, ldx, type, q, ldq, scale
    ((-1, 4, FAKE, 4, 0, FAKE, 4, FAKE), 2),
    ((4, -1, FAKE, 4, 0, FAKE, 4, FAKE), 2),
    ((4, (1 << 29) + 1, FAKE, 1 << 30, 0, FAKE, 1 << 30, FAKE), 2),
    ((4, 4, FAKE, 4, 3, FAKE, 4, FAKE), 4),
    ((4, 4, None, 4, 0, FAKE, 4, FAKE), 1),
    ((4, 4, FAKE, 4, 0, None, 4, FAKE), 1),
    ((4, 4, FAKE, 4, 0, FAKE, 4, None), 1),
    ((4, 4, FAKE, 3, 0, FAKE, 4, FAKE), 3),
    ((4, 4, FAKE, 4, 0, FAKE, 3, FAKE), 3),
    ((4, 4, FAKE + 2, 4, 0, FAKE, 4, FAKE), 5),
    ((4, 4, FAKE + 1, 4, 1, FAKE, 4, FAKE), 5),
    ((4, 4, FAKE, 4, 0, FAKE, 4, FAKE + 2), 5),
])
def test_quantize_refuses(m, args, status):
    _refuses(m, status, m.mdnn_quantize_i8, *args)
    need = m.mdnn_quantize_i8_t_workspace(args[0], args[1])
    _refuses(m, status, m.mdnn_quantize_i8_t, *args, FAKE, need)


def test_quantize_columns_refuses_workspaces(m):
    need = m.mdnn_quantize_i8_t_workspace(300, 40)
    assert need == 10 * 40 * 4 and m.mdnn_quantize_i8_t_workspace(-1, 4) == 0 and m.mdnn_quantize_i8_t_workspace(0, 4) == 0
    assert m.mdnn_quantize_i8_t_workspace(128, 40) == 0 and m.mdnn_quantize_i8_t_workspace(129, 40) > 0  # one tile of rows
    for ws, nb in ((None, need), (FAKE, need - 1), (FAKE + 4, need)):
        _refuses(m, m.ERR_WORKSPACE, m.mdnn_quantize_i8_t, 300, 40, FAKE, 40, 0, FAKE, 300, FAKE, ws, nb)
    _refuses(m, m.ERR_LAYOUT, m.mdnn_quantize_i8_t, 300, 40, FAKE, 40, 0, FAKE, 299, FAKE, FAKE, need)


@pytest.mark.parametrize("args,status", [
    # M, N, K, A, lda, a_scale, B, ldb, b_scale, bias, act, D, ldd, type
    ((-1, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 4, 0), 2),
    ((4, 4, 131072, FAKE, 131072, FAKE, FAKE, 131072, FAKE, None, 0, FAKE, 4, 0), 2),
    ((1 << 40, 1 << 40, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 1 << 40, 0), 2),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 4, 3), 4),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 2, FAKE, 4, 0), 4),
    ((4, 4, 4, None, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 4, 0), 1),
    ((4, 4, 4, FAKE, 4, None, FAKE, 4, FAKE, None, 0, FAKE, 4, 0), 1),
    ((4, 4, 4, FAKE, 4, FAKE, None, 4, FAKE, None, 0, FAKE, 4, 0), 1),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, None, None, 0, FAKE, 4, 0), 1),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, None, 4, 0), 1),
    ((4, 4, 4, FAKE, 3, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 4, 0), 3),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 3, FAKE, None, 0, FAKE, 4, 0), 3),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 3, 0), 3),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE + 2, 4, 0), 5),
    ((4, 4, 4, FAKE, 4, FAKE + 1, FAKE, 4, FAKE, None, 0, FAKE, 4, 1), 5),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, FAKE + 2, 0, FAKE, 4, 1), 5),
    ((4, 4, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, 4, 1, FAKE + 8, 64), 5),
])
def test_gemm_i8_refuses(m, args, status):
    _refuses(m, status, m.mdnn_gemm_i8, *args)


def test_gemm_i8_workspace_of_bad_sizes(m):
    assert m.mdnn_gemm_i8_workspace(-1, 4, 4) == 0 and m.mdnn_gemm_i8_workspace(4, 4, 1 << 20) == 0


def test_gemm_i8_workspace_is_for_copies_of_large_odd_operands(m):
    ws = m.mdnn_gemm_i8_workspace
    assert ws(4095, 4095, 4095) == (4095 + 4095) * 4096
    # whole 16-byte rows, few rows or columns, small products: no copy
    for size in ((4096, 4096, 4096), (4096, 4096, 4000), (64, 100000, 4095), (100000, 32, 4095), (1000, 777, 1531),
                 (4096, 4096, 15), (0, 4096, 4095)):
        assert ws(*size) == 0, size
    # the first size above 256 tiles of 256 x 128 (16 x 16 of them at 4096 x 2048)
    assert ws(4096, 2048, 33) == 0 and ws(4097, 2048, 33) == (4097 + 2048) * 128
    # a copy's chunks are counted in 32 bits
    assert ws((1 << 31) // 8 + 1, 64, 100) == 0 and ws(1 << 28, 64, 100) > 0


NORM = dict(rows=4, cols=8, x=FAKE, ldx=8, res=FAKE, ldr=8, gamma=FAKE, eps=1e-6, h=FAKE, ldh=8)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(cols=(1 << 29) + 1), 2), (dict(eps=0.0), 2), (dict(eps=-1.0), 2),
    (dict(eps=float("nan")), 2), (dict(eps=float("inf")), 2), (dict(x=None), 1), (dict(ldx=7), 3), (dict(ldr=7), 3),
    (dict(ldh=7), 3), (dict(x=FAKE + 1), 5), (dict(res=FAKE + 1), 5), (dict(h=FAKE + 1), 5), (dict(gamma=FAKE + 2), 5)])
def test_norm_refuses(m, change, status):
    a = tuple({**NORM, **change}.values())
    _refuses(m, status, m.mdnn_rmsnorm_fwd, *a, FAKE, 1 << 30, m.F16)
    _refuses(m, status, m.mdnn_rmsnorm_i8_fwd, *a, FAKE, 1 << 30, FAKE, m.F16)


def test_norm_refuses_outputs(m):
    a = tuple(NORM.values())
    for out, ld, t, status in ((None, 8, 1, m.ERR_NULL), (FAKE, 7, 1, m.ERR_LAYOUT), (FAKE, 8, 5, m.ERR_DTYPE)):
        _refuses(m, status, m.mdnn_rmsnorm_fwd, *a, out, ld, t)
        _refuses(m, status, m.mdnn_rmsnorm_i8_fwd, *a, out, ld, FAKE, t)
    _refuses(m, m.ERR_MISALIGNED, m.mdnn_rmsnorm_fwd, *a, FAKE + 1, 8, 1)
    _refuses(m, m.ERR_NULL, m.mdnn_rmsnorm_i8_fwd, *a, FAKE, 8, None, 1)
    _refuses(m, m.ERR_MISALIGNED, m.mdnn_rmsnorm_i8_fwd, *a, FAKE, 8, FAKE + 2, 1)


BWD = dict(rows=4, cols=8, dy=FAKE, lddy=8, h=FAKE, ldh=8, gamma=FAKE, eps=1e-6, dres=FAKE, lddr=8, dx=FAKE, lddx=8,
           dgamma=FAKE, dtype=1, ws=FAKE, nb=1 << 20)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(eps=0.0), 2), (dict(eps=float("nan")), 2), (dict(dtype=7), 4),
    (dict(dy=None), 1), (dict(h=None), 1), (dict(lddy=7), 3), (dict(ldh=7), 3), (dict(lddr=7), 3), (dict(lddx=7), 3),
    (dict(dy=FAKE + 1), 5), (dict(h=FAKE + 1), 5), (dict(dres=FAKE + 1), 5), (dict(dx=FAKE + 1), 5),
    (dict(gamma=FAKE + 2), 5), (dict(dgamma=FAKE + 2), 5), (dict(ws=None), 6), (dict(ws=FAKE + 16), 6), (dict(nb=8), 6)])
def test_norm_gradients_refuse(m, change, status):
    _refuses(m, status, m.mdnn_rmsnorm_bwd, *{**BWD, **change}.values())


def test_workspace_sizes(m):
    assert m.mdnn_rmsnorm_bwd_workspace(0, 8) == 0 and m.mdnn_rmsnorm_bwd_workspace(4, 0) == 0
    assert m.mdnn_rmsnorm_bwd_workspace(4, 8) >= 8 * 4
    # the blocks' sums do not grow with the rows without end
    assert m.mdnn_rmsnorm_bwd_workspace(1 << 40, 4096) == m.mdnn_rmsnorm_bwd_workspace(1 << 30, 4096)


@pytest.mark.parametrize("M,N", [((1 << 30) - 127, 64), (64, (1 << 30) - 127), (1 << 18, 1 << 18), (1 << 62, 1),
                                 (1, (1 << 63) - 1)])
def test_gemm_i8_refuses_more_tiles_than_a_launch_holds(m, M, N):
    """The documented limit, 2^24 - 2 tiles of 64 x 64: the first sizes above it, and sizes whose count would wrap."""
    _refuses(m, m.ERR_SHAPE, m.mdnn_gemm_i8, M, N, 4, FAKE, 4, FAKE, FAKE, 4, FAKE, None, 0, FAKE, N, 0)
