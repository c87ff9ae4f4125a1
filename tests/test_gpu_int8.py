"""8-bit codes and their product against the oracle: quantisers (bitwise, codes
and scales are defined down to the rounding), and the product over tile, step
and chunk edges, strides, types, empty and extreme operands."""
import numpy as np
import pytest

from oracle import rowwise as R
from tests.helpers import dev, host64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
GUARD = 77


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _values(rows, cols, seed, dtype, pad=0, offset=0):
    """A [rows, cols] device view with `pad` spare elements a row, starting `offset` elements into
    its memory (the rest NaN), and its values as fp32."""
    import torch
    g = np.random.default_rng(seed)
    v = (g.standard_normal((rows, cols)) * np.exp(g.standard_normal((rows, 1)))).astype(np.float32)
    base = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=_t(dtype), device="cuda")
    x = base[offset:].view(rows, cols + pad)[:, :cols]
    x.copy_(torch.from_numpy(v).cuda())
    return x, x.float().cpu().numpy()


def _code_room(rows, cols, ld, offset):
    import torch
    base = torch.full((offset + rows * ld + 64,), GUARD, dtype=torch.int8, device="cuda")
    return base, base[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def _untouched(base, view):
    """Every byte of base outside view still holds the guard."""
    keep = base.clone()
    keep.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(GUARD)
    return bool((keep == GUARD).all())


COLS = [1, 2, 7, 8, 9, 15, 16, 100, 127, 128, 129, 505, 512, 513, 1531, 2047, 2048, 2056, 4097, 8185, 8200, 16391,
        32768, 32769, 40003]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_quantize_rows(mdnn, cols, dtype):
    import torch
    for rows, pad, offset in ((1, 0, 0), (5, 3, 1), (35, 0, 0)):
        x, v = _values(rows, cols, cols + rows, dtype, pad, offset)
        v[rows // 2] = 0
        x[rows // 2] = 0
        q, s = R.codes(v)
        base, room = _code_room(rows, cols, cols + pad, offset)
        _, scale = mdnn.quantize_i8(x, q=room)
        assert (room.cpu().numpy() == q).all()
        assert (scale.cpu().numpy() == s).all()
        assert _untouched(base, room)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (300, 1), (3, 5), (31, 63), (32, 64), (33, 65), (127, 255),
                                       (128, 256), (129, 257), (777, 130), (4097, 67), (2050, 1000), (70001, 3)])
def test_quantize_columns(mdnn, rows, cols, dtype):
    for pad, offset in ((0, 0), (3, 1)):
        x, v = _values(rows, cols, rows + cols, dtype, pad, offset)
        x[:, cols // 2] = 0
        v[:, cols // 2] = 0
        q, s = R.codes(np.ascontiguousarray(v.T))
        base, room = _code_room(cols, rows, rows + pad, offset)
        _, scale = mdnn.quantize_i8(x, transpose=True, q=room)
        assert (room.cpu().numpy() == q).all()
        assert (scale.cpu().numpy() == s).all()
        assert _untouched(base, room)


def _special(cols):
    inf, nan = np.inf, np.nan
    v = np.random.default_rng(5).standard_normal((12, cols)).astype(np.float32)
    v[0, 0], v[1, -1], v[2, cols // 2] = nan, inf, -inf
    v[3] = 0
    v[4] *= np.float32(2.0 ** -110)
    v[5] *= np.float32(2.0 ** -140)
    with np.errstate(over="ignore"):
        v[6] = np.clip(v[6] * np.float32(1e38), -3e38, 3e38)
    v[7] = np.float32(2.0 ** -100)
    v[8] = -0.0
    v[9] = np.resize(np.float32([127, 0.5, 1.5, 2.5, -0.5, -1.5, -126.5]), cols)
    v[10], v[10, -1] = 0, nan
    return v


@pytest.mark.parametrize("cols", [5, 9, 130, 1000, 3000, 40000])
def test_quantize_special_rows(mdnn, cols):
    import torch
    v = _special(cols)
    q, s = R.codes(v)
    x = torch.from_numpy(v).cuda()
    got, scale = mdnn.quantize_i8(x)
    assert (got.cpu().numpy() == q).all()
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    got, scale = mdnn.quantize_i8(x.t().contiguous(), transpose=True)
    assert (got.cpu().numpy() == q).all()
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)


def test_quantize_empty(mdnn):
    import torch
    floor = np.float32(2.0 ** -100) / np.float32(127)
    q, s = mdnn.quantize_i8(torch.empty((3, 0), device="cuda"))
    assert s.cpu().numpy().tolist() == [floor] * 3
    q, s = mdnn.quantize_i8(torch.empty((0, 5), device="cuda"))
    assert s.numel() == 0
    q, s = mdnn.quantize_i8(torch.empty((0, 5), device="cuda"), transpose=True)
    assert s.cpu().numpy().tolist() == [floor] * 5


# ---------------------------------------------------------------- product

def _codes(rows, cols, seed, ld, offset=0, lo=-127):
    import torch
    v = np.random.default_rng(seed).integers(lo, 128, (rows, cols), dtype=np.int8)
    base = torch.full((offset + rows * ld + 16,), 113, dtype=torch.int8, device="cuda")
    t = base[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    t.copy_(torch.from_numpy(v).cuda())
    return t, v


def _check(mdnn, M, N, K, out, padded=True, bias=True, relu=True, offset=0, ldd_pad=0, ws=True, seed=0, lo=-127):
    import torch
    ld = (K + 15) // 16 * 16 if padded else K
    a, av = _codes(M, K, seed + 1, ld, offset, lo)
    b, bv = _codes(N, K, seed + 2, ld, offset, lo)
    g = np.random.default_rng(seed + 3)
    sa = np.exp(g.standard_normal(M)).astype(np.float32) * np.float32(1e-2)
    sb = np.exp(g.standard_normal(N)).astype(np.float32) * np.float32(1.0 / np.sqrt(max(K, 1)) / 100)
    bi = g.standard_normal(N).astype(np.float32) if bias else None
    room = torch.full((M, N + ldd_pad), 1e3, dtype=_t(out), device="cuda")
    d = room[:, :N]
    mdnn.gemm_i8(a, dev(sa, "f32"), b, dev(sb, "f32"), dev(bi, "f32") if bias else None,
                 mdnn.ACT_RELU if relu else mdnn.ACT_NONE, out=d, workspace=True if ws else None)
    acc = av.astype(np.float64) @ bv.astype(np.float64).T  # exact: below 2^53
    prod = acc * sa[:, None].astype(np.float64) * sb.astype(np.float64)
    exact = prod + (bi.astype(np.float64) if bias else 0.0)
    # the sum's conversion and two products each round once, the addition of the bias once; then the storage
    tol = 3.01 * U * np.abs(prod) + 1.01 * U * np.abs(exact) + 1.01 * HALF[out] * np.abs(exact) + TINY[out]
    if relu:
        exact = np.maximum(exact, 0.0)
    err = np.abs(host64(d) - exact)
    assert (err <= tol).all(), (M, N, K, float((err - tol).max()))
    assert ldd_pad == 0 or bool((room[:, N:] == 1e3).all())
    return d


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [1, 3, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 143, 255, 256, 257, 300, 511, 513, 1025])
def test_product_depths(mdnn, K, out):
    for M, N in ((1, 1), (3, 70), (70, 5), (129, 130)):
        for padded in (True, False):
            _check(mdnn, M, N, K, out, padded, bias=K % 2 == 0, relu=K % 3 == 0, seed=K)


@pytest.mark.parametrize("M", [1, 2, 8, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 100, 128, 200])
@pytest.mark.parametrize("N,K", [(1, 4096), (7, 130), (16, 512), (33, 1000), (64, 64), (65, 2048), (1000, 777),
                                 (4096, 256)])
def test_product_few_rows(mdnn, M, N, K):
    for padded, ws in ((True, True), (True, False), (False, True)):
        _check(mdnn, M, N, K, "f16", padded, ws=ws, seed=M)


@pytest.mark.parametrize("M,N,K", [(256, 256, 128), (257, 255, 384), (300, 4096, 256), (513, 1025, 640),
                                   (1000, 777, 1531), (2048, 2048, 512), (4100, 260, 1040), (1024, 1024, 4096),
                                   (130, 9000, 2064), (5000, 64, 512), (64, 5000, 512), (4096, 4096, 272)])
def test_product_tiles(mdnn, M, N, K):
    for out, padded, offset in (("f32", True, 0), ("bf16", True, 16), ("f16", False, 0), ("f32", True, 5)):
        _check(mdnn, M, N, K, out, padded, bias=out != "f32", relu=out == "bf16", offset=offset, ldd_pad=3, seed=N)


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1000, 783, 333), (1500, 1502, 1000), (1700, 1701, 300), (4100, 1985, 129),
                                   (1100, 4099, 1700), (1800, 1803, 1605), (2500, 2500, 1101), (4090, 4086, 605)])
def test_product_each_tile(mdnn, M, N, K, out):
    """Every tile of rows on 16 bytes, in each type, over the edges of D (by the sizes: 64 x 64, 128 x 128 of both
    kinds, 256 x 128, 256 x 256), and the same sizes as rows on any byte."""
    for padded in (True, False):
        _check(mdnn, M, N, K, out, padded, bias=padded, relu=not padded, ldd_pad=3 if padded else 0, ws=False, seed=K)


@pytest.mark.parametrize("M,N,K", [(4200, 4300, 131), (8200, 2100, 45), (1025, 16500, 16 * 9 + 1)])
def test_product_rows_copied(mdnn, M, N, K):
    """Large products with unaligned rows copy them into the workspace; one operand or both; a workspace too small,
    or none, gives the same result, and nothing past it is written."""
    import torch
    need = mdnn.mdnn_gemm_i8_workspace(M, N, K)
    assert need == (M + N) * ((K + 127) // 128 * 128)
    g = np.random.default_rng(K)
    sa, sb = dev(g.random(M).astype(np.float32), "f32"), dev(g.random(N).astype(np.float32), "f32")
    for a_pad, b_pad in ((False, False), (True, False), (False, True)):
        a, av = _codes(M, K, 1, (K + 15) // 16 * 16 if a_pad else K, 0 if a_pad else 3)
        b, bv = _codes(N, K, 2, (K + 15) // 16 * 16 if b_pad else K + 5, 0 if b_pad else 1)
        ws = torch.full((need + 64,), GUARD, dtype=torch.uint8, device="cuda")
        d = mdnn.gemm_i8(a, sa, b, sb, workspace=ws[:need])
        assert bool((ws[need:] == GUARD).all())
        assert torch.equal(d, mdnn.gemm_i8(a, sa, b, sb))
        assert torch.equal(d, mdnn.gemm_i8(a, sa, b, sb, workspace=ws[:need - 16]))
        acc = torch.from_numpy(av.astype(np.float64)).cuda() @ torch.from_numpy(bv.astype(np.float64)).cuda().T
        want = acc * sa.double()[:, None] * sb.double()
        assert bool(((d.double() - want).abs() <= 3.01 * U * want.abs()).all())


def test_product_strided_rows(mdnn):
    """Rows far apart, outputs inside a wider matrix; what lies between stays."""
    for ldd_pad in (1, 4, 5):
        _check(mdnn, 130, 131, 260, "bf16", padded=True, ldd_pad=ldd_pad)
        _check(mdnn, 40, 131, 260, "f32", padded=False, ldd_pad=ldd_pad)
        _check(mdnn, 1, 131, 260, "f16", padded=False, ldd_pad=ldd_pad)


@pytest.mark.parametrize("M,N", [(1, 64), (17, 40), (130, 140), (300, 300)])
def test_product_extreme_sums(mdnn, M, N):
    """The largest sums that 32 bits hold, and codes of -128."""
    import torch
    K = 131071
    for va, vb in ((-128, -128), (-128, 127), (127, 127)):
        a = torch.full((M, K + 1), va, dtype=torch.int8, device="cuda")[:, :K]
        b = torch.full((N, K + 1), vb, dtype=torch.int8, device="cuda")[:, :K]
        one = torch.ones(max(M, N), device="cuda")
        d = mdnn.gemm_i8(a, one[:M], b, one[:N], workspace=True)
        assert bool((d == float(np.float32(K * va * vb))).all())
    a, av = _codes(M, 4096, 1, 4096, lo=-128)
    _check(mdnn, M, N, 4096, "f32", lo=-128, bias=False, relu=False)


def test_product_zero_sizes(mdnn):
    import torch
    one = torch.ones(8, device="cuda")
    z = lambda r, c: torch.zeros((r, c), dtype=torch.int8, device="cuda")
    bias = torch.arange(8, device="cuda", dtype=torch.float32) - 3
    d = mdnn.gemm_i8(z(5, 0), one[:5], z(8, 0), one, bias)
    assert torch.equal(d, bias.expand(5, 8))
    assert mdnn.gemm_i8(z(0, 4), one[:0], z(8, 4), one).shape == (0, 8)
    assert mdnn.gemm_i8(z(5, 4), one[:5], z(0, 4), one[:0]).shape == (5, 0)


@pytest.mark.parametrize("M", [1, 20, 300])
def test_product_of_a_row_without_a_scale(mdnn, M):
    """A NaN scale (a row that held Inf or NaN) makes that row NaN and no other, through ReLU too."""
    import torch
    a, _ = _codes(M, 200, 3, 208)
    b, _ = _codes(90, 200, 4, 208)
    sa, sb = torch.ones(M, device="cuda"), torch.ones(90, device="cuda")
    sa[M - 1] = float("nan")
    sb[7] = float("nan")
    d = mdnn.gemm_i8(a, sa, b, sb, act=mdnn.ACT_RELU).isnan()
    want = torch.zeros_like(d)
    want[M - 1], want[:, 7] = True, True
    assert torch.equal(d, want)


def test_product_overflow_and_large_scales(mdnn):
    """fp16 outputs past 65504 are Inf; small scales in both factors do not vanish in their product."""
    import torch
    a, _ = _codes(3, 64, 5, 64)
    b, _ = _codes(9, 64, 6, 64)
    acc = a.cpu().numpy().astype(np.int64) @ b.cpu().numpy().astype(np.int64).T
    one = torch.ones(9, device="cuda")
    d = mdnn.gemm_i8(a, one[:3] * 1e6, b, one, out_dtype=torch.float16)
    assert torch.equal(d.cpu(), torch.from_numpy(np.sign(acc) * np.inf).half())
    d = mdnn.gemm_i8(a, one[:3] * 2.0 ** 100, b, one * 2.0 ** -130)
    assert np.array_equal(d.cpu().numpy(), (acc * 2.0 ** -30).astype(np.float32))
    d = mdnn.gemm_i8(a, one[:3] * 2.0 ** -80, b, one * 2.0 ** -60)
    assert np.array_equal(d.cpu().numpy(), (acc * 2.0 ** -140).astype(np.float32))


@pytest.mark.parametrize("M,N,padded", [(3, 64, True), (3, 64, False), (200, 300, True)])
def test_product_far_rows(mdnn, M, N, padded):
    """Rows whose offsets pass 2^31 and 2^32 bytes."""
    import torch
    K = 500
    far = (2 ** 32 // (M - 1) // 16 + 7) * 16 + (0 if padded else 3)
    base = torch.zeros(far * (M - 1) + 512, dtype=torch.int8, device="cuda")
    a = base.as_strided((M, K), (far, 1))
    v = np.random.default_rng(9).integers(-127, 128, (M, K), dtype=np.int8)
    a.copy_(torch.from_numpy(v).cuda())
    b, bv = _codes(N, K, 10, 512)
    one = torch.ones(max(M, N), device="cuda")
    want = v.astype(np.int64) @ bv.astype(np.int64).T
    assert np.array_equal(mdnn.gemm_i8(a, one[:M], b, one[:N], workspace=True).cpu().numpy(), want)
    assert np.array_equal(mdnn.gemm_i8(b, one[:N], a, one[:M], workspace=True).cpu().numpy(), want.T)


@pytest.mark.parametrize("M,N,K", [(4_200_000, 16, 4), (1, (1 << 27) + 5, 4), (20, (1 << 26) + 1, 3)])
def test_product_more_tiles_than_a_grid_side(mdnn, M, N, K):
    """More row or column tiles than the few-rows kernels' grid holds."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randint(-127, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    b = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    d = mdnn.gemm_i8(a, torch.ones(M, device="cuda"), b, torch.ones(N, device="cuda"), out_dtype=torch.float32)
    for m in {0, M // 2, M - 1}:
        assert torch.equal(d[m], (b.float() * a[m].float()).sum(1))
    for n in {0, N // 2, N - 1}:
        assert torch.equal(d[:, n], (a.float() * b[n].float()).sum(1))


def test_product_layer_of_a_trained_net(mdnn):
    """As it is used: weights of a layer quantised by output channel, a batch normalised into codes, the layer's
    product with bias and ReLU, its result quantised, the next layer's product; against the oracle step by step."""
    import torch
    B, I, H, O = 37, 200, 330, 50
    g = np.random.default_rng(11)
    w1, w2 = (g.standard_normal((I, H)) * np.sqrt(2 / I)).astype(np.float32), (g.standard_normal((H, O)) / 18).astype(np.float32)
    b1, gamma = (0.1 * g.standard_normal(H)).astype(np.float32), (1 + 0.1 * g.standard_normal(I)).astype(np.float32)
    x, res = _values(B, I, 12, "bf16")[0], _values(B, I, 13, "bf16")[0]
    q1, s1 = mdnn.quantize_i8(dev(w1, "f32"), transpose=True)
    q2, s2 = mdnn.quantize_i8(dev(w2, "f32"), transpose=True)
    qx, sx, h = mdnn.rmsnorm_i8(x, dev(gamma, "f32"), res)
    y = mdnn.gemm_i8(qx, sx, q1, s1, dev(b1, "f32"), mdnn.ACT_RELU, out_dtype=torch.bfloat16, workspace=True)
    qy, sy = mdnn.quantize_i8(y)
    z = mdnn.gemm_i8(qy, sy, q2, s2, workspace=True)

    rq, rs = R.rmsnorm_codes(x.float().cpu().numpy(), res.float().cpu().numpy(), gamma, 1e-6)
    assert (qx.cpu().numpy() == rq).all()
    wq1, ws1 = R.codes(np.ascontiguousarray(w1.T))
    ry = R.gemm_i8(rq, rs, wq1, ws1, b1, relu=True)
    assert np.abs(host64(y) - ry).max() <= (HALF["bf16"] + 64 * U) * np.abs(ry).max()
    ryq, rys = R.codes(y.float().cpu().numpy())  # from the stored y: codes are defined from it
    assert (qy.cpu().numpy() == ryq).all() and (sy.cpu().numpy() == rys).all()
    wq2, ws2 = R.codes(np.ascontiguousarray(w2.T))
    rz = R.gemm_i8(ryq, rys, wq2, ws2)
    assert np.abs(host64(z) - rz).max() <= 4 * U * np.abs(rz).max()
    # and the whole against the layers in full precision: 8 bits' worth of agreement
    hh = host64(x) + host64(res)
    full = np.maximum(R.rmsnorm(hh, gamma, 1e-6) @ w1.astype(np.float64) + b1, 0) @ w2.astype(np.float64)
    assert np.linalg.norm(host64(z) - full) <= 0.05 * np.linalg.norm(full)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (30, 1000, 2000), (300, 300, 4096)])
def test_product_streams_and_graphs(mdnn, M, N, K):
    """On another stream, and captured with its quantiser and norm and replayed on new data."""
    import torch
    x = torch.randn(M, K, device="cuda").half()
    w = torch.randn(K, N, device="cuda")
    gamma = torch.ones(K, device="cuda")
    qw, sw = mdnn.quantize_i8(w, transpose=True)
    qx, sx = mdnn.rmsnorm_i8(x, gamma)
    ws = torch.empty(max(mdnn.mdnn_gemm_i8_workspace(M, N, K), 16), dtype=torch.uint8, device="cuda")
    out = torch.empty(M, N, device="cuda")

    def step():
        mdnn.rmsnorm_i8(x, gamma, q=qx, scale=sx)
        mdnn.gemm_i8(qx, sx, qw, sw, out=out, workspace=ws)

    step()
    want = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn(M, K, device="cuda").half())
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(7)
        step()
        assert torch.equal(out, got), i


@pytest.mark.parametrize("handle", [False, True])
def test_own_workspaces_follow_the_stream(mdnn, handle):
    """A workspace that a wrapper allocates is not handed to other work while the call's stream still waits."""
    import torch
    x = torch.randn(2000, 500, device="cuda")
    g = torch.randn(2000, 500, device="cuda")
    a = torch.randint(-127, 128, (4100, 33), dtype=torch.int8, device="cuda")
    b = torch.randint(-127, 128, (8300, 33), dtype=torch.int8, device="cuda")
    sa, sb = torch.rand(4100, device="cuda"), torch.rand(8300, device="cuda")
    assert mdnn.mdnn_gemm_i8_workspace(4100, 8300, 33) > 0
    calls = [(mdnn.mdnn_quantize_i8_t_workspace(2000, 500), lambda **k: mdnn.quantize_i8(x, transpose=True, **k)),
             (mdnn.mdnn_rmsnorm_bwd_workspace(2000, 500), lambda **k: mdnn.rmsnorm_bwd(g, x, **k)),
             (mdnn.mdnn_gemm_i8_workspace(4100, 8300, 33),
              lambda **k: (mdnn.gemm_i8(a, sa, b, sb, workspace=True, **k),))]
    side = torch.cuda.Stream()
    for nbytes, call in calls:
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = call(stream=side.cuda_stream if handle else side)
        other = [torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert all((o == 255).all() for o in other)
        assert all(torch.equal(w, v) for w, v in zip(want, got))


def test_api_refuses(mdnn):
    import torch
    a = torch.zeros((4, 32), dtype=torch.int8, device="cuda")
    one = torch.ones(4, device="cuda")
    for bad in (lambda: mdnn.gemm_i8(a.t(), one, a, one), lambda: mdnn.gemm_i8(a, one[:3], a, one),
                lambda: mdnn.gemm_i8(a, one.half(), a, one), lambda: mdnn.gemm_i8(a, one, a[:, :16], one),
                lambda: mdnn.gemm_i8(a.float(), one, a, one), lambda: mdnn.gemm_i8(a, one, a.cpu(), one),
                lambda: mdnn.gemm_i8(a, one, a, one, bias=one[:2]),
                lambda: mdnn.gemm_i8(a, one, a, one, workspace=torch.zeros(64, device="cuda")),
                lambda: mdnn.quantize_i8(a.float().t()), lambda: mdnn.quantize_i8(a.float(), q=a[:, :8]),
                lambda: mdnn.quantize_i8(a.float(), scale=one[:2]), lambda: mdnn.quantize_i8(a.float().cpu())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mdnn.MdnnError):
        mdnn.gemm_i8(a, one, a, one, workspace=torch.zeros(33, dtype=torch.uint8, device="cuda")[1:])


def test_wrappers_on_the_default_streams_handle(mdnn):
    """The default stream given as its handle, which is 0, from another current stream: what is allocated lies in the
    default stream's memory, and the results are those of the call without a stream."""
    import torch
    assert torch.cuda.default_stream().cuda_stream == 0
    x, dy = torch.randn(2000, 500, device="cuda"), torch.randn(2000, 500, device="cuda")
    side = torch.cuda.Stream()
    for call in (lambda **k: mdnn.quantize_i8(x, transpose=True, **k), lambda **k: mdnn.rmsnorm_bwd(dy, x, **k)):
        want = call()
        with torch.cuda.stream(side):
            got = call(stream=0)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        for t in got:
            at = t.untyped_storage().data_ptr()
            owner = [g["stream"] for g in torch.cuda.memory_snapshot()
                     if g["address"] <= at < g["address"] + g["total_size"]]
            assert owner == [0]


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1000, 783, 384), (1000, 783, 1152),     # 64 x 64
                                   (2500, 2500, 256), (2500, 2500, 640),    # 128 x 128, eight waves
                                   (1800, 1803, 1664), (1800, 1803, 2048),  # 128 x 128, four waves
                                   (1100, 4099, 1792), (1100, 4099, 1920),  # 256 x 128
                                   (4090, 4086, 640), (4090, 4086, 1280)])  # 256 x 256
def test_product_whole_steps(mdnn, M, N, K, out):
    """Depths of whole 128-byte steps, whose loads are not checked against the row's end, on every tile of rows on 16
    bytes, over the edges of D and with an even and an odd count of steps after the steady rounds."""
    assert K % 128 == 0
    _check(mdnn, M, N, K, out, True, bias=out != "f16", relu=out != "f32", ldd_pad=3, ws=False, seed=K)


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [1040, 1111, 1407])
def test_product_ragged_depths_of_the_largest_tile(mdnn, K, out):
    """256 x 256 tiles whose last step is a partial one: whole 16-byte chunks, and bytes beyond them."""
    _check(mdnn, 4090, 4086, K, out, True, bias=True, relu=False, ldd_pad=5, ws=False, seed=K)


@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("K", [1021, 1660])
def test_product_rows_copied_to_whole_steps(mdnn, K, out):
    """Copied rows of more than 512 bytes, which the 256 x 256 tiles take."""
    assert mdnn.mdnn_gemm_i8_workspace(4095, 4095, K) == 2 * 4095 * ((K + 127) // 128 * 128)
    _check(mdnn, 4095, 4095, K, out, False, bias=True, relu=True, offset=3, seed=K)


@pytest.mark.parametrize("K", [1792, 1791])
def test_product_bits_are_those_of_the_definition_in_every_kernel(mdnn, K):
    """The sum's conversion, its product with the row's scale, and the column's scale with the bias in one rounding:
    the same bits from every tile, few-rows and any-byte kernel and with copied rows."""
    import torch
    M, N = 3840, 4099
    a, av = _codes(M, K, 1, 1792)
    b, bv = _codes(N, K, 2, 1792)
    a1, _ = _codes(M, K, 1, 1793, 5)  # the same codes in rows on any byte
    b1, _ = _codes(N, K, 2, 1793, 3)
    g = np.random.default_rng(3)
    sa, sb = np.exp(g.standard_normal(M)).astype(np.float32), np.exp(g.standard_normal(N)).astype(np.float32) / 1000
    bias = (100 * g.standard_normal(N)).astype(np.float32)
    acc = torch.from_numpy(av).cuda().double() @ torch.from_numpy(bv).cuda().double().T
    p = acc.float() * dev(sa, "f32")[:, None]
    exact = p.double() * dev(sb, "f32").double()  # (48 bits)
    hi = exact + dev(bias, "f32").double()
    back = hi - exact
    lo = (exact - (hi - back)) + (dev(bias, "f32").double() - back)
    # hi rounds to fp32 as the whole sum does unless it lies on a midpoint that lo moves it off
    sure = (lo == 0) | ((hi.view(torch.int64) & 0x1fffffff) != 0x10000000)
    want, plain = hi.float(), exact.float()
    dsa, dsb, dbias = dev(sa, "f32"), dev(sb, "f32"), dev(bias, "f32")
    for rows, cols in ((3840, 4099), (1100, 4099), (900, 4099), (1800, 1803), (300, 4099), (100, 4099), (40, 4099),
                       (17, 500), (16, 4099), (1, 4099), (1000, 20)):
        for x, y in ((a, b), (a1, b1), (a, b1)):
            for ws in (None, True):
                args = (x[:rows], dsa[:rows], y[:cols], dsb[:cols])
                d = mdnn.gemm_i8(*args, dbias[:cols], workspace=ws)
                assert bool(((d == want[:rows, :cols]) | ~sure[:rows, :cols]).all()), (rows, cols)
                assert torch.equal(mdnn.gemm_i8(*args, workspace=ws), plain[:rows, :cols]), (rows, cols)
