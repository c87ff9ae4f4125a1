"""Root-mean-square norm, its 8-bit output and its gradients against the oracle
in 64 bits.

Tolerances, with u = 2^-24: a sum of a row's n terms is taken by at most 1024
threads, each adding ceil(n / 1024) + 32 terms at most, and combined in a tree
and a chain of at most 22 more; with the roundings of the terms themselves
every sum is within S(n) = (64 + n / 1024) u of the sum of its terms'
magnitudes.  1 / rms is then within S / 2 + 6 u (mean, eps, root, quotient),
and each product rounds once."""
import numpy as np
import pytest

from oracle import rowwise as R
from tests.helpers import dev, host64
from tests.test_gpu_int8 import COLS, GUARD, HALF, TINY, U, _code_room, _special, _t, _untouched, _values

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _sum_bound(n):
    return (64 + n / 1024) * U


def _gamma(cols, seed=1):
    return (1 + 0.2 * np.random.default_rng(seed).standard_normal(cols)).astype(np.float32)


def _room(rows, cols, dtype, pad, offset):
    import torch
    base = torch.full((offset + rows * (cols + pad),), 1e3, dtype=_t(dtype), device="cuda")
    return base, base[offset:].view(rows, cols + pad)[:, :cols]


def _kept(base, view):
    keep = base.clone()
    keep.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(1e3)
    return bool((keep == 1e3).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_norm(mdnn, cols, dtype):
    gamma = _gamma(cols)
    for rows, pad, offset, with_res, with_gamma in ((1, 0, 0, True, True), (5, 3, 1, True, True), (35, 0, 0, False, True),
                                                    (18, 8, 0, True, False)):
        x, xv = _values(rows, cols, cols + rows, dtype, pad, offset)
        res, rv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        xv[rows // 2], rv[rows // 2] = 0, 0
        x[rows // 2], res[rows // 2] = 0, 0
        g = gamma if with_gamma else np.ones(cols, np.float32)
        base, y = _room(rows, cols, dtype, pad, offset)
        hbase, h = _room(rows, cols, dtype, pad, offset)
        mdnn.rmsnorm(x, dev(gamma, "f32") if with_gamma else None, res if with_res else None, EPS,
                     h_out=h if with_res else None, out=y)
        hv = xv.astype(np.float64) + (rv.astype(np.float64) if with_res else 0.0)
        want = R.rmsnorm(hv, g, EPS)
        k = _sum_bound(cols) / 2 + 9 * U
        assert (np.abs(host64(y) - want) <= (k + 1.001 * HALF[dtype]) * np.abs(want) + TINY[dtype]).all()
        assert _kept(base, y)
        if with_res:
            assert (np.abs(host64(h) - hv) <= (1.001 * HALF[dtype] + U) * np.abs(hv) + TINY[dtype]).all()
            assert _kept(hbase, h)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_norm_codes(mdnn, cols, dtype):
    gamma = _gamma(cols)
    for rows, pad, offset, with_res, with_gamma in ((1, 0, 0, True, True), (5, 3, 1, True, True), (35, 0, 0, False, True),
                                                    (18, 8, 0, True, False)):
        x, xv = _values(rows, cols, cols + rows, dtype, pad, offset)
        res, rv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        base, q = _code_room(rows, cols, cols + pad, offset)
        hbase, h = _room(rows, cols, dtype, pad, offset)
        out = mdnn.rmsnorm_i8(x, dev(gamma, "f32") if with_gamma else None, res if with_res else None, EPS,
                              h_out=h if with_res else None, q=q)
        rq, rs = R.rmsnorm_codes(xv, rv if with_res else None, gamma if with_gamma else None, EPS)
        assert (q.cpu().numpy() == rq).all()
        assert (np.abs(host64(out[1]) - rs) <= (_sum_bound(cols) / 2 + 8 * U) * rs).all()
        assert _untouched(base, q)
        if with_res:
            hv = xv.astype(np.float64) + rv
            assert (np.abs(host64(h) - hv) <= (1.001 * HALF[dtype] + U) * np.abs(hv) + TINY[dtype]).all()
            assert _kept(hbase, h)


@pytest.mark.parametrize("cols", [5, 9, 130, 1000, 3000, 40000])
def test_norm_special_rows(mdnn, cols):
    """Rows with Inf or NaN, or whose squares overflow: all NaN, codes 0 and scale NaN; rows of nothing: zeros."""
    import torch
    v = _special(cols)
    x, gamma = torch.from_numpy(v).cuda(), torch.ones(cols, device="cuda")
    y = mdnn.rmsnorm(x, gamma, eps=EPS).cpu().numpy()
    q, s = (t.cpu().numpy() for t in mdnn.rmsnorm_i8(x, gamma, eps=EPS))
    bad = [0, 1, 2, 6, 10]
    for r in range(12):
        assert np.isnan(y[r]).all() == (r in bad) and np.isnan(y[r]).any() == (r in bad)
        assert np.isnan(s[r]) == (r in bad)
    assert (q[bad] == 0).all() and (q[3] == 0).all() and (q[8] == 0).all()
    assert (y[3] == 0).all() and (y[8] == 0).all()
    ok = [r for r in range(12) if r not in bad]
    rq, _ = R.codes(v[ok])
    assert (q[ok] == rq).all()
    # h * gamma overflows though h does not: the codes have no scale
    x = torch.full((2, cols), 1e10, device="cuda")
    gamma[cols - 1] = 1e30
    q, s = mdnn.rmsnorm_i8(x, gamma, eps=EPS)
    assert bool(s.isnan().all()) and bool((q == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_gradients(mdnn, cols, dtype):
    import torch
    gamma = _gamma(cols)
    for rows, pad, offset, with_res, with_gamma in ((1, 0, 0, True, True), (5, 3, 1, True, True), (35, 0, 0, False, True),
                                                    (18, 8, 0, True, False), (1100, 0, 0, True, True)):
        if rows * cols > 1 << 22:
            continue
        h, hv = _values(rows, cols, cols + rows, dtype, pad, offset)
        dy, dv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        dr, rv = _values(rows, cols, cols + rows + 2, dtype, pad, offset)
        hv[rows // 2] = 0
        h[rows // 2] = 0
        g = gamma if with_gamma else np.ones(cols, np.float32)
        base, dx = _room(rows, cols, dtype, pad, offset)
        _, dg = mdnn.rmsnorm_bwd(dy, h, dev(gamma, "f32") if with_gamma else None, EPS, dr if with_res else None, dx=dx)
        want, want_g = R.rmsnorm_bwd(dv, hv, g, EPS, rv if with_res else None)
        hv, dv, g = hv.astype(np.float64), dv.astype(np.float64), g.astype(np.float64)
        r = 1 / np.sqrt(np.mean(hv * hv, axis=1, keepdims=True) + EPS)
        # the terms' magnitudes, each within two sums' error (rms and mean) and a few roundings
        size = r * (np.abs(g * dv) + np.abs(hv * r) * np.mean(np.abs(g * dv * hv * r), axis=1, keepdims=True))
        size = size + (np.abs(rv) if with_res else 0.0)
        tol = (2 * _sum_bound(cols) + 12 * U) * size + 1.01 * HALF[dtype] * np.abs(want) + TINY[dtype]
        assert (np.abs(host64(dx) - want) <= tol).all()
        assert _kept(base, dx)
        # a sum of `rows` terms in any order, each term within the rms' error
        tol = ((rows + 8) * U + _sum_bound(cols) / 2 + 8 * U) * np.sum(np.abs(dv * hv * r), axis=0) + TINY["f32"]
        assert (np.abs(host64(dg) - want_g) <= tol).all()


def test_gradients_one_at_a_time(mdnn):
    import torch
    for rows, cols in ((700, 200), (33, 4096), (3, 20000)):
        h, _ = _values(rows, cols, 1, "bf16")
        dy, _ = _values(rows, cols, 2, "bf16")
        dx, dg = mdnn.rmsnorm_bwd(dy, h)
        only_x, none = mdnn.rmsnorm_bwd(dy, h, with_dgamma=False)
        assert none is None and torch.equal(only_x, dx)
        ws = torch.empty(mdnn.mdnn_rmsnorm_bwd_workspace(rows, cols), dtype=torch.uint8, device="cuda")
        only_g = torch.empty_like(dg)
        mdnn.mdnn_rmsnorm_bwd(rows, cols, dy, cols, h, cols, None, 1e-6, None, 0, None, 0, only_g, mdnn.BF16, ws,
                              ws.numel())
        assert torch.equal(only_g, dg)
    dg = torch.ones(77, device="cuda")
    mdnn.rmsnorm_bwd(torch.empty((0, 77), device="cuda"), torch.empty((0, 77), device="cuda"), dgamma=dg)
    assert bool((dg == 0).all())


def test_gradients_by_differences(mdnn):
    """dx and dgamma against differences of the forward pass itself."""
    import torch
    rows, cols = 3, 19
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.randn(rows, cols, generator=g, device="cuda")
    dy = torch.randn(rows, cols, generator=g, device="cuda")
    gamma = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    dx, dg = mdnn.rmsnorm_bwd(dy, h, gamma, 1e-3)
    # step 2^-7: the quotient's error is e^2 / 6 times third derivatives (of order 10 / r^3 with r about 1, times
    # |dy| sums of order 10) plus rounding 2^-24 * sum |dy y| / e: below 0.02
    e = 2.0 ** -7
    loss = lambda a, b: float((dy.double() * mdnn.rmsnorm(a, b, eps=1e-3).double()).sum())
    for i in range(rows):
        for j in range(0, cols, 5):
            d = torch.zeros_like(h)
            d[i, j] = e
            assert abs((loss(h + d, gamma) - loss(h - d, gamma)) / (2 * e) - float(dx[i, j])) <= 0.02
    for j in range(cols):
        d = torch.zeros_like(gamma)
        d[j] = e
        assert abs((loss(h, gamma + d) - loss(h, gamma - d)) / (2 * e) - float(dg[j])) <= 0.02


@pytest.mark.parametrize("cols", [5, 100, 1000, 1531, 4096, 9000, 16392, 40000])
def test_in_place(mdnn, cols):
    """Outputs exactly in place of inputs give what separate ones do."""
    import torch
    for dtype in ("f32", "bf16"):
        x, _ = _values(37, cols, 1, dtype)
        res, _ = _values(37, cols, 2, dtype)
        gamma = dev(_gamma(cols), "f32")
        y, h = mdnn.rmsnorm(x, gamma, res, EPS)
        q, s, h2 = mdnn.rmsnorm_i8(x, gamma, res, EPS)
        dx, dg = mdnn.rmsnorm_bwd(x, res, gamma, EPS, y)
        assert torch.equal(h, h2)
        a, b = x.clone(), res.clone()
        mdnn.rmsnorm(a, gamma, b, EPS, h_out=b, out=a)
        assert torch.equal(a, y) and torch.equal(b, h)
        a, b = x.clone(), res.clone()
        mdnn.rmsnorm(a, gamma, b, EPS, h_out=a, out=b)
        assert torch.equal(a, h) and torch.equal(b, y)
        b = res.clone()
        q2, s2, _ = mdnn.rmsnorm_i8(x, gamma, b, EPS, h_out=b)
        assert torch.equal(q2, q) and torch.equal(s2, s) and torch.equal(b, h)
        for k in range(3):
            t = [x.clone(), res.clone(), y.clone()]
            _, dg2 = mdnn.rmsnorm_bwd(t[0], t[1], gamma, EPS, t[2], dx=t[k])
            assert torch.equal(t[k], dx) and torch.equal(dg2, dg)


def test_deterministic_and_captured(mdnn):
    """A training step's forward and backward norm, captured and replayed on new data."""
    import torch
    rows, cols = 700, 1531
    x = torch.randn(rows, cols, device="cuda").bfloat16()
    res, dy = torch.randn_like(x), torch.randn_like(x)
    gamma = torch.rand(cols, device="cuda") + 0.5
    y, h, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dg = torch.empty(cols, device="cuda")
    ws = torch.empty(mdnn.mdnn_rmsnorm_bwd_workspace(rows, cols), dtype=torch.uint8, device="cuda")

    def step():
        mdnn.rmsnorm(x, gamma, res, EPS, h_out=h, out=y)
        mdnn.rmsnorm_bwd(dy, h, gamma, EPS, y, dx=dx, dgamma=dg, workspace=ws)

    step()
    first = [t.clone() for t in (y, h, dx, dg)]
    for _ in range(3):
        step()
        assert all(torch.equal(a, b) for a, b in zip(first, (y, h, dx, dg)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.copy_(torch.randn(rows, cols, device="cuda").bfloat16())
        dy.copy_(torch.randn(rows, cols, device="cuda").bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, h, dx, dg)]
        for t in (y, h, dx, dg):
            t.zero_()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, h, dx, dg)))


def test_many_rows(mdnn):
    """More rows than one launch has blocks for."""
    import torch
    rows, cols = (1 << 20) * 16 + 5, 9
    x = torch.randn(rows, cols, device="cuda").half()
    y = mdnn.rmsnorm(x, None, eps=EPS)
    q, s = mdnn.quantize_i8(x)
    xf = x.double()
    # in pieces, with the definition in 64 bits on the GPU
    for lo in range(0, rows, 1 << 22):
        p = xf[lo:lo + (1 << 22)]
        want = p / torch.sqrt((p * p).mean(1, keepdim=True) + EPS)
        err = (y[lo:lo + (1 << 22)].double() - want).abs()
        assert bool((err <= (1.001 * HALF["f16"] + 80 * U) * want.abs() + TINY["f16"]).all())
        a = p.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
        inv = (torch.full_like(a, 127.0) / a).float().double()
        assert torch.equal(q[lo:lo + (1 << 22)], (p * inv).float().round().to(torch.int8))
        assert torch.equal(s[lo:lo + (1 << 22)], (a / torch.full_like(a, 127.0)).float()[:, 0])


@pytest.mark.parametrize("rows,cols", [(1, (1 << 27) + 40), (2, (1 << 25) + 72)])
def test_widest_gamma_gradient(mdnn, rows, cols):
    """One row, whose sums are the gradient, and more columns than the gamma gradient's launch has blocks for."""
    import torch
    h = torch.randn(rows, cols, device="cuda").half()
    dy = torch.randn(rows, cols, device="cuda").half()
    _, dg = mdnn.rmsnorm_bwd(dy, h)
    square = sum(p.double().square().sum(1, keepdim=True) for p in h.split(1 << 24, 1))
    rstd = 1 / torch.sqrt(square / cols + 1e-6)
    for lo in range(0, cols, 1 << 24):
        terms = dy[:, lo:lo + (1 << 24)].double() * h[:, lo:lo + (1 << 24)].double() * rstd
        err = (dg[lo:lo + (1 << 24)].double() - terms.sum(0)).abs()
        # the sum of squares: at most 2^17 terms a thread
        assert bool((err <= _sum_bound(cols) * terms.abs().sum(0) + 1e-30).all())


@pytest.mark.parametrize("rows,cols", [(96, 112), (97, 112), (16, 1000), (17, 1000), (4, 4096), (5, 4096), (2, 9000),
                                       (257, 40000)])
def test_gradients_by_blocks(mdnn, rows, cols):
    """The most rows that one block takes, whose sums are the gradient, one row more, and more long rows than blocks."""
    import torch
    h = torch.randn(rows, cols, device="cuda")
    dy = torch.randn(rows, cols, device="cuda")
    dx, dg = mdnn.rmsnorm_bwd(dy, h, eps=EPS)
    h, dy = h.double(), dy.double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    terms = dy * h * r
    tol = ((rows + 8) * U + _sum_bound(cols) / 2 + 8 * U) * terms.abs().sum(0)
    assert bool(((dg.double() - terms.sum(0)).abs() <= tol).all())
    want = r * (dy - h * r * terms.mean(1, keepdim=True))
    size = r * (dy.abs() + (h * r).abs() * terms.abs().mean(1, keepdim=True))
    tol = (2 * _sum_bound(cols) + 12 * U) * size + 1.01 * HALF["f32"] * want.abs()
    assert bool(((dx.double() - want).abs() <= tol).all())


def test_far_rows(mdnn):
    """Rows whose offsets pass 2^32 bytes."""
    import torch
    cols, far = 700, 2 ** 31 + 24
    base = torch.zeros(2 * far + cols, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((3, cols), (far, 1))
    v, vals = _values(3, cols, 3, "bf16")
    x.copy_(v)
    gamma = dev(_gamma(cols), "f32")
    y, h = mdnn.rmsnorm(v, gamma, v, EPS)
    q, s, _ = mdnn.rmsnorm_i8(v, gamma, v, EPS)
    dx, dg = mdnn.rmsnorm_bwd(v, v, gamma, EPS, v)
    y2, _ = mdnn.rmsnorm(x, gamma, x, EPS)
    q2, s2, _ = mdnn.rmsnorm_i8(x, gamma, x, EPS)
    dx2, dg2 = mdnn.rmsnorm_bwd(x, x, gamma, EPS, x)
    for a, b in ((y, y2), (q, q2), (s, s2), (dx, dx2), (dg, dg2)):
        assert torch.equal(a, b)
    assert torch.equal(mdnn.quantize_i8(x)[0], mdnn.quantize_i8(v)[0])
    assert torch.equal(mdnn.quantize_i8(x, transpose=True)[0], mdnn.quantize_i8(v, transpose=True)[0])
    out = base.as_strided((3, cols), (far, 1))
    mdnn.rmsnorm(x, gamma, x, EPS, h_out=out)
    assert torch.equal(out, h)


def test_api_refuses(mdnn):
    import torch
    x = torch.zeros((4, 32), device="cuda")
    g = torch.ones(32, device="cuda")
    for bad in (lambda: mdnn.rmsnorm(x.t(), g), lambda: mdnn.rmsnorm(x, g[:8]), lambda: mdnn.rmsnorm(x, g, x[:, :8]),
                lambda: mdnn.rmsnorm(x, g, x.half()), lambda: mdnn.rmsnorm(x, g.half()), lambda: mdnn.rmsnorm(x.cpu(), g),
                lambda: mdnn.rmsnorm_bwd(x, x[:2], g), lambda: mdnn.rmsnorm_bwd(x, None, g),
                lambda: mdnn.rmsnorm_i8(x, g, q=torch.zeros((4, 32), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mdnn.MdnnError):
        mdnn.rmsnorm(x, g, eps=0.0)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(40001, 128), (40001, 200), (9000, 512), (9001, 1000), (2600, 2000), (2601, 3999),
                                       (1100, 8192), (1101, 8185), (700, 16384), (701, 9001), (600, 20000)])
def test_gradients_of_many_rows(mdnn, rows, cols, dtype):
    """Every shape of the gradients' kernels with several rows to a block in turn, the last turn a partial one, with
    gamma and the residual's gradient; in 64 bits on the GPU."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    make = lambda: (torch.randn(rows, cols, generator=g, device="cuda")
                    * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(_t(dtype))
    h, dy, dres = make(), make(), make()
    gamma = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    dx, dg = mdnn.rmsnorm_bwd(dy, h, gamma, EPS, dres)
    h, dy, dres, gamma = h.double(), dy.double(), dres.double(), gamma.double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    xh, along = h * r, gamma * dy
    want = r * (along - xh * (along * xh).mean(1, keepdim=True)) + dres
    size = r * (along.abs() + xh.abs() * (along * xh).abs().mean(1, keepdim=True)) + dres.abs()
    tol = (2 * _sum_bound(cols) + 12 * U) * size + 1.01 * HALF[dtype] * want.abs() + TINY[dtype]
    assert bool(((dx.double() - want).abs() <= tol).all())
    # a column's sum: 256 thread groups at least take the rows in turn, at most 32 of them are joined in a block, and
    # the blocks' sums in chains of at most 16 and 32; each term within the rms' error and two products
    terms = dy * xh
    chain = -(-rows // 256) + 32 + 16 + 32
    tol = (chain * U + _sum_bound(cols) / 2 + 8 * U) * terms.abs().sum(0)
    assert bool(((dg.double() - terms.sum(0)).abs() <= tol).all())


@pytest.mark.parametrize("rows,cols", [((1 << 20) + 5, 5), ((1 << 24) + 5, 130), ((1 << 22) + 5, 264), ((1 << 20) + 5, 1032),
                                       ((1 << 20) + 5, 4104)])
def test_more_rows_than_blocks(mdnn, rows, cols):
    """Blocks that walk on to a second row: each half of the rows by itself, one row a block, gives the same."""
    import torch
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda").normal_()
    gamma = dev(_gamma(cols), "f32")
    for f in (lambda t: (mdnn.rmsnorm(t, gamma, eps=EPS),), lambda t: mdnn.rmsnorm_i8(t, gamma, eps=EPS),
              lambda t: mdnn.quantize_i8(t)):
        whole = f(x)
        for half in (slice(0, rows // 2), slice(rows // 2, rows)):
            assert all(torch.equal(a[half], b) for a, b in zip(whole, f(x[half])))


# The sums of the kernels for long rows, whatever the length: eight terms at a time in fp32 and those sums in 64 bits,
# a rounding to fp32, and the tree and chain of at most 26 additions over the threads.
LONG_SUM = (8 + 1 + 26) * U


@pytest.mark.parametrize("value", [1.1, 0.1, 1.37])
def test_long_rows_of_one_magnitude(mdnn, value):
    """Terms of one size, whose roundings all fall to one side: the sums do not lose bits with the row's length."""
    import torch
    rows, cols = 2, (1 << 26) + 3
    h = torch.full((rows, cols), value, device="cuda")
    h[1] *= -2
    hd = h[:, :1].double()
    y = mdnn.rmsnorm(h, None, eps=EPS)
    want = hd / torch.sqrt(hd * hd + EPS)
    assert bool(((y.double() - want).abs() <= (LONG_SUM / 2 + 9 * U + 1.01 * HALF["f32"]) * want.abs()).all())
    q, s = mdnn.rmsnorm_i8(h, None, eps=EPS)
    want = (hd.abs() / 127 / torch.sqrt(hd * hd + EPS))[:, 0]
    assert bool(((s.double() - want).abs() <= (LONG_SUM / 2 + 9 * U) * want).all())
    # every other gradient 0: mean(dy xh) is not lost in dx's difference
    dy = torch.zeros(rows, cols, device="cuda")
    dy[:, ::2] = 0.7
    d = dy[:, :2].double()
    r = 1 / torch.sqrt(hd * hd + EPS)
    mean = d[:, :1] * hd * r * ((cols + 1) // 2) / cols
    dx, dg = mdnn.rmsnorm_bwd(dy, h, eps=EPS)
    size = r * (d.abs() + (hd * r).abs() * mean.abs())
    for c in (0, 1):
        want = r * (d[:, c:c + 1] - hd * r * mean)
        assert bool(((dx[:, c::2].double() - want).abs() <= (2 * LONG_SUM + 13 * U) * size[:, c:c + 1]).all())
        terms = d[:, c:c + 1] * hd * r
        assert bool(((dg[c::2].double() - terms.sum(0)).abs() <= (LONG_SUM / 2 + 10 * U) * terms.abs().sum(0)).all())


@pytest.mark.parametrize("rows,cols", [(1 << 22, 1), ((1 << 24) + 3, 4), (1 << 22, 7)])
def test_gamma_gradient_of_many_narrow_rows(mdnn, rows, cols):
    """Millions of rows below eight columns, all terms of one sign and size: a column's sum is taken in 64 bits over a
    block's rows, rounded once, and the blocks' sums are added in chains of at most 8 and 32; each term is a rounded
    product of dy and h / rms, whose root's error is that of a sum of fewer than eight terms."""
    import torch
    h = torch.full((rows, cols), 1.1, device="cuda")
    dy = torch.full((rows, cols), 0.7, device="cuda")
    dx, dg = mdnn.rmsnorm_bwd(dy, h, eps=EPS)
    hd, d = h[0].double(), dy[0].double()
    r = 1 / torch.sqrt(hd * hd + EPS)
    want = rows * d * hd * r
    assert bool(((dg.double() - want).abs() <= (1 + 8 + 32 + 16) * U * want.abs()).all())
    # the blocks' rows in turn, the last ones included
    first, *_ = mdnn.rmsnorm_bwd(dy[:5], h[:5], eps=EPS)
    assert bool((dx == first[0]).all())
