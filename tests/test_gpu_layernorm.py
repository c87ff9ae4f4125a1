"""Dropout and layer norm, forward and backward, against the oracle in 64 bits.

Tolerances, with u = 2^-24.  Every sum over a row's n terms is within S(n) =
(64 + n / 1024) u of the sum of the terms' magnitudes: a thread adds at most
ceil(n / 1024) + 32 of them in fp32, at most 22 more additions join the threads
(rows past the registers: eight at a time in fp32, then in 64 bits).
With d = h - mean(h), the kernel's difference is off by the rounding of h
itself (u |h|, and u for the product of dropout), its mean over the row, the
rounding of the differences and S times the mean of |d| (the mean's error
cancels: it is taken out again by the mean of the differences).  The variance is
then within S and twice the mean of |d| times that error; 1 / deviation is half
of it, relative, and six roundings (quotients, eps, root); every product and sum
after it rounds once."""
import numpy as np
import pytest

from oracle import blocks as B
from tests.helpers import dev, host64

pytestmark = pytest.mark.gpu
EPS = 1e-5
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
SEED, STEP, SITE = 0x9E3779B97F4A7C15, 2 ** 32 + 17, 5
COLS = [1, 2, 7, 8, 9, 15, 16, 100, 127, 128, 129, 505, 512, 513, 1531, 2047, 2048, 2056, 4097, 8185, 8200, 16384, 16391,
        32768, 32769, 40003]
SHAPES = ((1, 0, 0, True, True), (5, 3, 1, True, True), (35, 0, 0, False, True), (18, 8, 0, True, False))


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _sum_bound(n):
    return (64 + n / 1024) * U


def _vec(cols, seed, at):
    return (at + 0.2 * np.random.default_rng(seed).standard_normal(cols)).astype(np.float32)


def _values(rows, cols, seed, dtype, pad=0, offset=0):
    """A [rows, cols] device view with `pad` spare elements a row, `offset` elements into its memory (the rest NaN), and
    its values; rows of different size and offset, one of zeros."""
    import torch
    g = np.random.default_rng(seed)
    v = (g.standard_normal((rows, cols)) + 2 * g.standard_normal((rows, 1))) * np.exp(g.standard_normal((rows, 1)))
    if rows > 2:
        v[rows // 2] = 0
    base = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=_t(dtype), device="cuda")
    x = base[offset:].view(rows, cols + pad)[:, :cols]
    x.copy_(torch.from_numpy(v.astype(np.float32)).cuda())
    return x, x.double().cpu().numpy()


def _room(rows, cols, dtype, pad, offset):
    import torch
    base = torch.full((offset + rows * (cols + pad),), 1e3, dtype=_t(dtype), device="cuda")
    return base, base[offset:].view(rows, cols + pad)[:, :cols]


def _kept(base, view):
    keep = base.clone()
    keep.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(1e3)
    return bool((keep == 1e3).all())


@pytest.fixture(scope="module")
def rng(mdnn):
    return mdnn.make_rng(SEED, STEP)


def _stats(h, size):
    """d, 1 / deviation, the error of d and the relative error of 1 / deviation; size: what h's own rounding goes by."""
    n = h.shape[1]
    mean = lambda v: np.mean(v, axis=1, keepdims=True)
    d = h - mean(h)
    e = 1.01 * (U * (size + mean(size)) + 6 * U * np.abs(d) + _sum_bound(n) * mean(np.abs(d)) + 2 * U * np.abs(mean(d)))
    # (second order: the mean's own error, S mean |h|, goes through the rounding of the differences)
    e = e + 8 * U * _sum_bound(n) * mean(np.abs(h))
    r = 1 / np.sqrt(mean(d * d) + EPS)
    return d, r, e, r * r * mean(np.abs(d) * e) + _sum_bound(n) / 2 + 7 * U


def _norm_room(h, size, gamma, want, beta, half):
    d, r, e, rho = _stats(h, size)
    return np.abs(gamma) * r * e + np.abs(want - beta) * (rho + 4 * U) + 2 * U * np.abs(want) + 1.01 * half * np.abs(want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_dropout(mdnn, rng, cols, dtype):
    for (rows, pad, offset, with_res, _), p in zip(SHAPES, (0.1, 0.5, 0.25, 0.9)):
        x, xv = _values(rows, cols, cols + rows, dtype, pad, offset)
        res, rv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        keep = B.kept(rows, cols, p, SEED, STEP, SITE)
        base, y = _room(rows, cols, dtype, pad, offset)
        mdnn.dropout(x, p, rng, SITE, res if with_res else None, out=y)
        want = keep * xv + (rv if with_res else 0.0)
        tol = 2 * U * np.abs(keep * xv) + U * np.abs(want) + 1.01 * HALF[dtype] * np.abs(want) + TINY[dtype]
        assert (np.abs(host64(y) - want) <= tol).all()
        assert _kept(base, y)
        assert ((host64(y) == 0) >= ((keep == 0) & (not with_res))).all()  # dropped: exactly 0
        base, dx = _room(rows, cols, dtype, pad, offset)
        mdnn.dropout_bwd(x, p, rng, SITE, dx=dx)
        tol = (2 * U + 1.01 * HALF[dtype]) * np.abs(keep * xv) + TINY[dtype]
        assert (np.abs(host64(dx) - keep * xv) <= tol).all()
        assert _kept(base, dx)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_dropout_of_no_and_every_element(mdnn, rng, dtype):
    import torch
    x, _ = _values(9, 77, 1, dtype)
    res, _ = _values(9, 77, 2, dtype)
    x[3, 4], x[5, 6] = float("inf"), float("nan")
    assert torch.equal(mdnn.dropout(x, 0.0).nan_to_num(7.0), x.nan_to_num(7.0))
    assert torch.equal(mdnn.dropout(x, 1e-6, rng).nan_to_num(7.0), x.nan_to_num(7.0))  # t = 0: nothing is drawn
    assert bool((mdnn.dropout(x, 1.0, rng) == 0).all()) and torch.equal(mdnn.dropout(x, 1.0, rng, 0, res), res)
    # what is dropped may hold anything
    x.fill_(float("nan"))
    keep = torch.from_numpy(B.kept(9, 77, 0.5, SEED, STEP, SITE)).cuda()
    y = mdnn.dropout(x, 0.5, rng, SITE)
    assert torch.equal(y.isnan(), keep > 0) and bool((y[keep == 0] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_norm(mdnn, rng, cols, dtype):
    for (rows, pad, offset, with_res, affine), p in zip(SHAPES, (0.0, 0.3, 0.5, 0.0)):
        x, xv = _values(rows, cols, cols + rows, dtype, pad, offset)
        res, rv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        gamma, beta = (_vec(cols, 1, 1), _vec(cols, 2, 0)) if affine else (np.ones(cols, np.float32), np.zeros(cols, np.float32))
        base, y = _room(rows, cols, dtype, pad, offset)
        hbase, h = _room(rows, cols, dtype, pad, offset)
        stored = with_res or p > 0
        mdnn.layernorm(x, dev(gamma, "f32") if affine else None, dev(beta, "f32") if affine else None,
                       res if with_res else None, EPS, p, rng, SITE, h_out=h if stored else None, out=y)
        dropped = B.kept(rows, cols, p, SEED, STEP, SITE) * xv
        hv = dropped + (rv if with_res else 0.0)
        size = (2 * np.abs(dropped) if p > 0 else 0.0) + (np.abs(hv) if with_res else 0.0) * np.ones_like(hv)
        want = B.layernorm(hv, gamma, beta, EPS)
        tol = _norm_room(hv, size, gamma, want, beta, HALF[dtype]) + TINY[dtype]
        assert (np.abs(host64(y) - want) <= tol).all(), (rows, p)
        assert _kept(base, y)
        if stored:
            assert (np.abs(host64(h) - hv) <= U * size + 1.01 * HALF[dtype] * np.abs(hv) + TINY[dtype]).all()
            assert _kept(hbase, h)


@pytest.mark.parametrize("cols", [8, 100, 1531, 9000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_norm_stores_what_dropout_does(mdnn, rng, cols, dtype):
    import torch
    x, _ = _values(33, cols, 1, dtype)
    res, _ = _values(33, cols, 2, dtype)
    _, h = mdnn.layernorm(x, residual=res, p=0.3, rng=rng, site=SITE)
    assert torch.equal(h, mdnn.dropout(x, 0.3, rng, SITE, res))


@pytest.mark.parametrize("cols", [5, 9, 130, 1000, 3000, 40000])
def test_norm_special_rows(mdnn, cols):
    """Inf and NaN make their row NaN and no other; rows of one value, however far from 0, give beta."""
    import torch
    x = torch.randn(12, cols, device="cuda")
    x[0, 0], x[1, cols - 1], x[2, cols // 2] = float("inf"), float("nan"), float("-inf")
    x[3], x[4], x[5], x[6] = 0.0, 1000.1, -3e7, 1e-30
    x[7], x[7, ::2] = 3e38, -3e38  # (the sum of squares passes fp32)
    beta = torch.randn(cols, device="cuda")
    y = mdnn.layernorm(x, None, beta)
    bad = [0, 1, 2, 7]
    for r in range(12):
        assert bool(y[r].isnan().all()) == (r in bad) and bool(y[r].isnan().any()) == (r in bad), r
    # a row of one value: what is left of the differences is below n roundings of roundings
    for r in (3, 4, 5, 6):
        left = float(x[r, 0].abs()) * 4 * _sum_bound(cols) * U / EPS ** 0.5 * 40
        assert float((y[r] - beta).abs().max()) <= left + 2 * U * float(beta.abs().max()), r


@pytest.mark.parametrize("offset", [0.0, 100.0, 1e4])
@pytest.mark.parametrize("cols", [64, 1531, 8192, 40000])
def test_norm_of_rows_far_from_zero(mdnn, cols, offset):
    """The variance is that of the differences: an offset does not cancel it away."""
    import torch
    x = torch.randn(16, cols, device="cuda") + offset
    y = mdnn.layernorm(x)
    xd = x.double()
    d = xd - xd.mean(1, keepdim=True)
    want = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    # the differences are exact to u |d| and the mean's correction; no term goes by the offset but the second-order one
    tol = (2 * _sum_bound(cols) + 20 * U) * (want.abs() + 1) + 40 * U * _sum_bound(cols) * offset
    assert bool(((y.double() - want).abs() <= tol).all())


def _check_gradients(dx, dh, dg, db, dy, h, gamma, dres, keep, rows, cols, dtype):
    want, want_g, want_b = B.layernorm_bwd(dy, h, gamma, EPS, dres)
    S = _sum_bound(cols)
    mean = lambda v: np.mean(v, axis=1, keepdims=True)
    d, r, e, rho = _stats(h, np.zeros_like(h))
    xh, g = d * r, dy * gamma
    e_x = r * e + np.abs(xh) * (rho + 3 * U)
    mg, mgx = mean(np.abs(g)), np.abs(mean(g * xh))
    e_m = r * ((2 * S + 8 * U) * mean(np.abs(g * d)) + mean(np.abs(g) * e) + S * mean(np.abs(d)) * mg) + mgx * (rho + 6 * U)
    tol = r * ((4 * U) * np.abs(g) + (S + 6 * U) * mg + e_x * mgx + np.abs(xh) * e_m + 4 * U * np.abs(xh) * mgx)
    tol = tol + r * (np.abs(g) + mg + np.abs(xh) * mgx) * (rho + 6 * U) + U * np.abs(want)
    if dres is not None:
        tol = tol + U * np.abs(dres)
    if dh is not None:
        assert (np.abs(host64(dh) - want) <= tol + 1.01 * HALF[dtype] * np.abs(want) + TINY[dtype]).all()
    if dx is not None:
        at = keep * want
        assert (np.abs(host64(dx) - at) <= keep * tol + (2 * U + 1.01 * HALF[dtype]) * np.abs(at) + TINY[dtype]).all()
    # a column's sum: 256 thread groups at least take the rows in turn, at most 32 of them are joined in a block, and the
    # blocks' sums in chains of at most 16 and 32
    chain = -(-rows // 256) + 32 + 16 + 32
    tol = np.sum(np.abs(dy) * e_x, axis=0) + (chain + 2) * U * np.sum(np.abs(dy * xh), axis=0) + TINY["f32"]
    assert (np.abs(host64(dg) - want_g) <= tol).all()
    assert (np.abs(host64(db) - want_b) <= chain * U * np.sum(np.abs(dy), axis=0) + TINY["f32"]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_gradients(mdnn, rng, cols, dtype):
    for (rows, pad, offset, with_res, affine), p in zip(SHAPES + ((1100, 0, 0, True, True),), (0.0, 0.3, 0.5, 0.0, 0.1)):
        if rows * cols > 1 << 21:
            continue
        h, hv = _values(rows, cols, cols + rows, dtype, pad, offset)
        dy, dv = _values(rows, cols, cols + rows + 1, dtype, pad, offset)
        dr, rv = _values(rows, cols, cols + rows + 2, dtype, pad, offset)
        gamma = _vec(cols, 1, 1) if affine else np.ones(cols, np.float32)
        base, dx = _room(rows, cols, dtype, pad, offset)
        hbase, dh = _room(rows, cols, dtype, pad, offset)
        _, _, dg, db = mdnn.layernorm_bwd(dy, h, dev(gamma, "f32") if affine else None, EPS, dr if with_res else None, p,
                                          rng, SITE, dx=dx, dh=dh)
        _check_gradients(dx, dh, dg, db, dv, hv, gamma.astype(np.float64), rv if with_res else None,
                         B.kept(rows, cols, p, SEED, STEP, SITE), rows, cols, dtype)
        assert _kept(base, dx) and _kept(hbase, dh)


@pytest.mark.parametrize("rows,cols", [(96, 112), (97, 112), (3, 40), (16, 1000), (17, 1000), (4, 4096), (5, 4096),
                                       (2, 9000), (700, 9000), (257, 20000), (5000, 200), (40001, 16), (3000, 2000)])
def test_gradients_by_blocks(mdnn, rng, rows, cols):
    """The most rows that one block takes, whose sums are the gradients, one row more, and more rows than blocks."""
    h, hv = _values(rows, cols, 1, "bf16")
    dy, dv = _values(rows, cols, 2, "bf16")
    gamma = _vec(cols, 3, 1)
    dx, dh, dg, db = mdnn.layernorm_bwd(dy, h, dev(gamma, "f32"), EPS, None, 0.25, rng, SITE)
    _check_gradients(dx, dh, dg, db, dv, hv, gamma.astype(np.float64), None, B.kept(rows, cols, 0.25, SEED, STEP, SITE),
                     rows, cols, "bf16")


def test_gradients_one_at_a_time(mdnn, rng):
    import torch
    for rows, cols in ((700, 200), (33, 4096), (3, 20000), (900, 5)):
        h, _ = _values(rows, cols, 1, "bf16")
        dy, _ = _values(rows, cols, 2, "bf16")
        dx, dh, dg, db = mdnn.layernorm_bwd(dy, h, p=0.5, rng=rng, site=2)
        only = mdnn.layernorm_bwd(dy, h, p=0.5, rng=rng, site=2, with_sums=False)
        assert only[2] is None and only[3] is None and torch.equal(only[0], dx) and torch.equal(only[1], dh)
        ws = torch.empty(max(256, mdnn.mdnn_layernorm_bwd_workspace(rows, cols)), dtype=torch.uint8, device="cuda")
        for k, want in enumerate((dx, dh, dg, db)):
            out = [None] * 4
            out[k] = torch.empty_like(want)
            mdnn.mdnn_layernorm_bwd(rows, cols, dy, cols, h, cols, None, 1e-5, None, 0, 0.5, rng, 2, out[0], cols, out[1],
                                    cols, out[2], out[3], mdnn.BF16, ws, ws.numel())
            assert torch.equal(out[k], want)
        plain, same, _, _ = mdnn.layernorm_bwd(dy, h)
        assert same is plain and torch.equal(plain, dh)
    dg, db = torch.ones(77, device="cuda"), torch.ones(77, device="cuda")
    mdnn.layernorm_bwd(torch.empty((0, 77), device="cuda"), torch.empty((0, 77), device="cuda"), dgamma=dg, dbeta=db)
    assert bool((dg == 0).all()) and bool((db == 0).all())


def test_gradients_by_differences(mdnn, rng):
    """Every gradient against differences of the forward pass itself, dropout and residual in it."""
    import torch
    rows, cols = 3, 19
    g = torch.Generator(device="cuda").manual_seed(4)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, res, dy, dres = (make(rows, cols) for _ in range(4))
    gamma, beta = 1 + 0.2 * make(cols), make(cols)

    def loss(x, res, gamma, beta):
        y, h = mdnn.layernorm(x, gamma, beta, res, 1e-3, 0.3, rng, 1)
        return float((dy.double() * y.double()).sum() + (dres.double() * h.double()).sum())

    _, h = mdnn.layernorm(x, gamma, beta, res, 1e-3, 0.3, rng, 1)
    got = mdnn.layernorm_bwd(dy, h, gamma, 1e-3, dres, 0.3, rng, 1)
    # step 2^-7: the quotient's error is e^2 / 6 times third derivatives (of order 10 s^3 / r^3, s < 1.5, r about 1, times
    # sums of |dy| of order 20) plus rounding 2^-24 * sum |dy y| / e: below 0.03
    e = 2.0 ** -7
    args = [x, res, gamma, beta]
    for k, grad in enumerate(got):
        for at in np.ndindex(tuple(grad.shape)):
            if len(at) == 2 and at[1] % 5:
                continue
            d = torch.zeros_like(args[k])
            d[at] = e
            up, down = ([a + (s * d if i == k else 0) for i, a in enumerate(args)] for s in (1, -1))
            assert abs((loss(*up) - loss(*down)) / (2 * e) - float(grad[at])) <= 0.03, (k, at)


@pytest.mark.parametrize("cols", [5, 100, 1000, 1531, 4096, 9000, 16392, 40000])
def test_in_place(mdnn, rng, cols):
    """Outputs exactly in place of inputs give what separate ones do."""
    import torch
    for dtype in ("f32", "bf16"):
        x, _ = _values(37, cols, 1, dtype)
        res, _ = _values(37, cols, 2, dtype)
        gamma = dev(_vec(cols, 1, 1), "f32")
        k = dict(eps=EPS, p=0.3, rng=rng, site=1)
        y, h = mdnn.layernorm(x, gamma, gamma, res, **k)
        dx, dh, dg, db = mdnn.layernorm_bwd(x, res, gamma, dres=y, **k)
        a, b = x.clone(), res.clone()
        mdnn.layernorm(a, gamma, gamma, b, h_out=b, out=a, **k)
        assert torch.equal(a, y) and torch.equal(b, h)
        a, b = x.clone(), res.clone()
        mdnn.layernorm(a, gamma, gamma, b, h_out=a, out=b, **k)
        assert torch.equal(a, h) and torch.equal(b, y)
        for i in range(3):
            for j in range(3):
                if i == j:
                    continue
                t = [x.clone(), res.clone(), y.clone()]
                _, _, dg2, db2 = mdnn.layernorm_bwd(t[0], t[1], gamma, dres=t[2], dx=t[i], dh=t[j], **k)
                assert torch.equal(t[i], dx) and torch.equal(t[j], dh) and torch.equal(dg2, dg) and torch.equal(db2, db)
        a = x.clone()
        assert torch.equal(mdnn.dropout(a, 0.3, rng, 1, res, out=a), mdnn.dropout(x, 0.3, rng, 1, res))


def test_captured_steps_draw_anew(mdnn):
    """Forward and backward in a graph: each replay is the eager pass at the step that the state holds."""
    import torch
    rows, cols = 700, 1531
    x = torch.randn(rows, cols, device="cuda").bfloat16()
    res, dy = torch.randn_like(x), torch.randn_like(x)
    gamma = torch.rand(cols, device="cuda") + 0.5
    rng = mdnn.make_rng(42)
    y, h, dx, dh = (torch.empty_like(x) for _ in range(4))
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mdnn.mdnn_layernorm_bwd_workspace(rows, cols), dtype=torch.uint8, device="cuda")

    def step():
        mdnn.layernorm(x, gamma, None, res, p=0.2, rng=rng, site=1, h_out=h, out=y)
        mdnn.layernorm_bwd(dy, h, gamma, dres=y, p=0.2, rng=rng, site=1, dx=dx, dh=dh, dgamma=dg, dbeta=db, workspace=ws)

    outs = (y, h, dx, dh, dg, db)
    step()
    first = [t.clone() for t in outs]
    for _ in range(3):
        step()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    seen = [first[1]]
    for _ in range(3):
        rng[1] += 1
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert not any(torch.equal(got[1], s) for s in seen)
        seen.append(got[1])
        for t in outs:
            t.zero_()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
    # back at the first step: its results again
    rng[1] = 0
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))


def test_side_stream(mdnn, rng):
    import torch
    x = torch.randn(300, 777, device="cuda").half()
    want = mdnn.layernorm(x, p=0.2, rng=rng, site=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mdnn.layernorm(x, p=0.2, rng=rng, site=9, stream=side)
    drop = mdnn.dropout(x, 0.2, rng, 9, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(drop, want[1])


@pytest.mark.parametrize("rows,cols", [((1 << 20) + 5, 5), ((1 << 24) + 5, 40), ((1 << 20) + 5, 1032)])
def test_more_rows_than_blocks(mdnn, rng, rows, cols):
    """Blocks that walk on: the first and last rows by themselves, one row a block, give the same; without dropout, which
    goes by the row."""
    import torch
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda").normal_()
    whole, n = mdnn.layernorm(x), 1000
    assert torch.equal(whole[:n], mdnn.layernorm(x[:n])) and torch.equal(whole[-n:], mdnn.layernorm(x[-n:]))
    y = mdnn.dropout(x, 0.5, rng, SITE)
    for lo in (0, rows - n):
        keep = torch.from_numpy(B.kept(n, cols, 0.5, SEED, STEP, SITE, row0=lo)).cuda()
        assert torch.equal(y[lo:lo + n], (keep * x[lo:lo + n].double()).half())


def test_far_rows(mdnn, rng):
    """Rows whose offsets pass 2^32 bytes."""
    import torch
    cols, far = 700, 2 ** 31 + 24
    base = torch.zeros(2 * far + cols, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((3, cols), (far, 1))
    v, _ = _values(3, cols, 3, "bf16")
    x.copy_(v)
    gamma = dev(_vec(cols, 1, 1), "f32")
    k = dict(p=0.3, rng=rng, site=1)
    for a, b in zip(mdnn.layernorm(v, gamma, gamma, v, **k) + mdnn.layernorm_bwd(v, v, gamma, dres=v, **k),
                    mdnn.layernorm(x, gamma, gamma, x, **k) + mdnn.layernorm_bwd(x, x, gamma, dres=x, **k)):
        assert torch.equal(a, b)
    assert torch.equal(mdnn.dropout(x, 0.3, rng, 1, x), mdnn.dropout(v, 0.3, rng, 1, v))


@pytest.mark.parametrize("value", [1.1, 0.1])
def test_long_rows_of_two_values(mdnn, value):
    """Terms of one size, whose roundings all fall to one side: no sum loses bits with the row's length."""
    import torch
    cols = (1 << 25) + 6
    x = torch.full((2, cols), value, device="cuda")
    x[:, ::2] = -3 * value
    y = mdnn.layernorm(x)
    a, b = x[0, 0].double(), x[0, 1].double()
    mean = (a + b) / 2
    want = torch.stack((a - mean, b - mean)) / torch.sqrt((a - b) ** 2 / 4 + 1e-5)
    for c in (0, 1):
        # sums: 8 terms in fp32, then 64 bits; the rest as in the module's note
        assert bool(((y[:, c::2].double() - want[c]).abs() <= (8 + 20) * U * want[c].abs() * 2).all())


@pytest.mark.parametrize("rows,cols", [(1 << 22, 1), ((1 << 22) + 3, 4), (1 << 20, 7)])
def test_sums_of_many_narrow_rows(mdnn, rows, cols):
    """Millions of rows below eight columns of one value: beta's gradient, a sum of equal terms, is taken in 64 bits over a
    block's rows, rounded once, and the blocks' sums are added in chains of at most 64 and 32."""
    import torch
    h = torch.randn(rows, cols, device="cuda")
    dy = torch.full((rows, cols), 0.1, device="cuda")
    _, _, _, db = mdnn.layernorm_bwd(dy, h)
    want = dy[0, 0].double() * rows
    assert bool(((db.double() - want).abs() <= 100 * U * want).all())
