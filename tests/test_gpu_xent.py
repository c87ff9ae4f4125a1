"""The last layer's cross entropy in pieces of the classes, forward and
backward, against the oracle in 64 bits.

Tolerances, with u = 2^-24.  A logit is a sum of K products in fp32 and a bias:
within e_z = (K + 2) u sum |x w| + 2 u |bias|.  An exponential of a difference d is
within 2^-21 + 2 |d| u, relative (its argument's rounding and product with log2
e, and the instruction's last place).  A row's sum of exponentials is joined from
at most N / 256 + 64 partial sums in turn, four roundings and one exponential
each, so lse is within the largest e_z of the row, weighted by the
probabilities, plus those, plus the logarithm's roundings (2 u |lse| + 2^-21).
A gradient G = p - [label] is within p (e_z + e_lse + 2^-21 + 2 |z - lse| u) and one
rounding to the storage type (half a step; fp16 is scaled by 2^15, so its
smallest step is 2^-39), and each product adds its depth's roundings."""
import numpy as np
import pytest

from oracle import blocks as B
from oracle.rounding import round_to
from tests.helpers import dev, host64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
IGNORED = -7


def _t(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def _view(v, dtype, pad, offset):
    """A device view of the values v (rounded to dtype) with `pad` spare elements a row, `offset` elements into its memory
    (the rest NaN), and the values it holds."""
    import torch
    rows, cols = v.shape
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


class Problem:
    def __init__(self, m, n, k, dtype, by_class, bias=True, pad=0, offset=0, seed=0, scale=2.0):
        import torch
        g = np.random.default_rng(seed + m + n + k)
        self.m, self.n, self.k, self.dtype, self.by_class = m, n, k, dtype, by_class
        w = g.standard_normal((k, n)) * scale / np.sqrt(k)
        self.w, wv = _view(w.T if by_class else w, dtype, pad, offset)
        self.wv = wv.T if by_class else wv
        labels = g.integers(0, n, m)
        x = g.standard_normal((m, k)) + g.random((m, 1)) * self.wv[:, labels].T
        self.x, self.xv = _view(x, dtype, pad, offset)
        self.bias = (0.5 * g.standard_normal(n)).astype(np.float32) if bias else None
        if m > 3:
            labels[g.random(m) < 0.2] = IGNORED
            labels[0], labels[1], labels[m - 1] = IGNORED, 0, n - 1
        self.labels = labels.astype(np.int32)
        self.dlabels = torch.from_numpy(self.labels).cuda()
        self.pad, self.offset = pad, offset

    def args(self, mdnn):
        bias = None if self.bias is None else dev(self.bias, "f32")
        return bias, dict(layout=mdnn.NT if self.by_class else mdnn.NN, ignored=IGNORED)

    def e_z(self):
        b = 0.0 if self.bias is None else 2 * U * np.abs(np.nan_to_num(self.bias.astype(np.float64), posinf=0, neginf=0))
        return (self.k + 2) * U * (np.abs(self.xv) @ np.abs(self.wv)) + b

    def forward(self, mdnn):
        bias, kw = self.args(mdnn)
        return mdnn.linear_xent(self.x, self.w, self.dlabels, bias, **kw)

    def check_forward(self, mdnn):
        got = [host64(t) for t in self.forward(mdnn)]
        loss, row, lse, z = B.linear_xent(self.xv, self.wv, self.bias, self.labels, IGNORED)
        p = np.exp(z - lse[:, None])
        away = np.where(p > 0, np.abs(z - z.max(axis=1, keepdims=True)), 0.0)
        e_z = self.e_z()
        steps = self.n / 256 + 64
        seen = np.where(p > 2.0 ** -60, e_z, 0.0)  # (a class below that adds nothing in any rounding)
        e_lse = (np.sum(p * (seen + 2 * U * away), axis=1) + steps * (4 * U + 2.0 ** -21) + seen.max(axis=1) * 1e-3
                 + 2 * U * np.abs(lse) + 2.0 ** -21)
        assert (np.abs(got[2] - lse) <= e_lse).all()
        inside = np.where(self.labels == IGNORED, 0, self.labels)
        e_row = e_lse + e_z[np.arange(self.m), inside] + 2 * U * np.abs(row)
        assert (np.abs(got[1] - row) <= e_row).all()
        assert (got[1][self.labels == IGNORED] == 0).all()
        assert abs(got[0][0] - loss) <= e_row.max() + 2 * U * abs(loss)
        return z, lse, e_lse

    def check_backward(self, mdnn, loss_scale=None, dw_type=None):
        import torch
        bias, kw = self.args(mdnn)
        lse64 = B.linear_xent(self.xv, self.wv, self.bias, self.labels, IGNORED)[2]
        lse = lse64.astype(np.float32)
        z = self.xv @ self.wv + (0.0 if self.bias is None else self.bias)
        g = B.linear_xent_grad(z, lse, self.labels, IGNORED)
        s = 1.0 if loss_scale is None else loss_scale
        want = B.linear_xent_bwd(self.xv, self.wv, g, self.labels, IGNORED, s)
        dw_type = dw_type or "f32"
        xb, dx = _room(self.m, self.k, self.dtype, self.pad, self.offset)
        wb, dw = _room(*self.w.shape, dw_type, self.pad, self.offset)
        db = None if self.bias is None else torch.empty(self.n, device="cuda")
        mdnn.linear_xent_bwd(self.x, self.w, self.dlabels, dev(lse, "f32"), bias,
                             loss_scale=None if loss_scale is None else torch.full((1,), loss_scale, device="cuda"), dx=dx,
                             dw=dw, db=db, **kw)
        a = s / max(1, int(np.sum(self.labels != IGNORED)))
        counted = (self.labels != IGNORED)[:, None]
        p = np.where(counted, np.exp(z - lse[:, None].astype(np.float64)), 0.0)
        off = np.where(p > 0, self.e_z() + 2.0 ** -21 + 2 * U * np.abs(z - lse[:, None]), 0.0)  # (0 * Inf is 0 here)
        exact = p * off + U * np.abs(g)
        stored = exact + HALF[self.dtype] * (np.abs(g) + exact) + (2.0 ** -40 if self.dtype == "f16" else 2.0 ** -134)
        stored = np.where(counted, stored, 0.0)
        xa, wa, ga = np.where(counted, np.abs(self.xv), 0.0), np.abs(self.wv), np.abs(g)
        pieces = 4  # (at most, here: a sum's pieces are joined in fp32)
        tol = a * ((stored + (self.n + 64 + pieces) * U * ga) @ wa.T) + 4 * U * np.abs(want[0])
        tol = tol + 1.01 * HALF[self.dtype] * np.abs(want[0]) + TINY[self.dtype]
        assert (np.abs(host64(dx) - want[0]) <= tol).all()
        assert (host64(dx)[~counted[:, 0]] == 0).all()
        tol = a * (xa.T @ (stored + (self.m + 64) * U * ga)) + 4 * U * np.abs(want[1])
        tol = tol + 1.01 * HALF[dw_type] * np.abs(want[1]) + TINY[dw_type]
        got = host64(dw).T if self.by_class else host64(dw)
        assert (np.abs(got - want[1]) <= tol).all()
        assert _kept(xb, dx) and _kept(wb, dw)
        if db is not None:
            tol = a * np.sum(np.where(counted, exact, 0.0) + (self.m + 8) * U * ga, axis=0) + 4 * U * np.abs(want[2])
            assert (np.abs(host64(db) - want[2]) <= tol + TINY["f32"]).all()


SIZES = [(1, 1, 1), (1, 2, 3), (2, 5, 8), (1, 1000, 64), (3, 4097, 40), (5, 300, 333), (16, 2048, 256), (17, 1001, 129),
         (33, 515, 64), (64, 1024, 128), (65, 1030, 72), (100, 3001, 200), (128, 256, 512), (200, 777, 1000),
         (257, 2000, 96), (300, 1536, 320), (512, 512, 64),
         (40, 1500, 1100), (5, 300, 2100), (1, 999, 520), (70, 513, 777), (600, 130, 600),
         (7, 3000, 1000), (8, 515, 4100), (3, 9000, 65), (2, 70, 2100), (4, 8, 8), (8, 2049, 17)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_forward(mdnn, size, by_class, dtype):
    for bias, pad, offset in ((True, 0, 0), (False, 3, 1), (True, 8, 8)):
        Problem(*size, dtype, by_class, bias, pad, offset).check_forward(mdnn)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("size", SIZES)
def test_gradients(mdnn, size, by_class, dtype):
    for bias, pad, offset, scale, dw in ((True, 0, 0, None, dtype), (False, 3, 1, 1024.0, "f32"), (True, 8, 8, 0.25, "f32")):
        Problem(*size, dtype, by_class, bias, pad, offset).check_backward(mdnn, scale, dw)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (3, 1)])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k", [(9, 5003, 1000), (33, 1031, 1100), (64, 4097, 520), (130, 4097, 520)])
def test_gradients_of_a_few_dozen_rows(mdnn, m, n, k, by_class, wide, pad, offset, dtype):
    Problem(m, n, k, dtype, by_class, pad=pad, offset=offset).check_backward(mdnn, dw_type="f32" if wide else dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k", [(700, 5003, 1301), (401, 12008, 901), (385, 9024, 1300)])
def test_odd_sizes_of_large_products(mdnn, m, n, k, by_class, pad, offset, dtype):
    p = Problem(m, n, k, dtype, by_class, pad=pad, offset=offset)
    p.check_forward(mdnn)
    p.check_backward(mdnn, dw_type=dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k,by_class", [(4100, 9000, 64, False), (4096, 8192, 128, True), (9000, 20011, 32, True),
                                            (1000, 70001, 40, False), (20000, 4100, 72, False), (70, 131072, 520, True),
                                            (1 << 20, 2305, 64, False), (1 << 20, 2368, 64, True), (4, 70001, 264, True),
                                            (3, 70001, 264, False)])
def test_large(mdnn, m, n, k, by_class, dtype):
    """Several pieces, row blocks and tiles; against 64 bits on the GPU, by the module's bounds."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(m + n)
    x = torch.randn(m, k, generator=g, device="cuda").to(_t(dtype))
    w = (torch.randn(*((n, k) if by_class else (k, n)), generator=g, device="cuda") * 2 / k ** 0.5).to(_t(dtype))
    bias = torch.randn(n, generator=g, device="cuda")
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(m, generator=g, device="cuda") < 0.1] = IGNORED
    kw = dict(layout=mdnn.NT if by_class else mdnn.NN, ignored=IGNORED)
    loss, row, lse = mdnn.linear_xent(x, w, labels, bias, **kw)
    dx, dw, db = mdnn.linear_xent_bwd(x, w, labels, lse, bias, **kw)
    wd = w.double().t().contiguous() if by_class else w.double()
    counted = labels != IGNORED
    a = 1.0 / int(counted.sum())
    dw_want, db_want, total = torch.zeros_like(wd), torch.zeros(n, dtype=torch.float64, device="cuda"), 0.0
    dw_tol, db_tol = torch.zeros_like(wd), torch.zeros_like(db_want)
    step = 2000 if m < 1 << 20 else 1 << 14
    for lo in range(0, m, step):
        rows = slice(lo, min(m, lo + step))
        xd, c = x[rows].double(), counted[rows, None]
        z = xd @ wd + bias.double()
        want = torch.logsumexp(z, 1)
        p = (z - want[:, None]).exp()
        e_z = (k + 2) * U * (xd.abs() @ wd.abs()) + 2 * U * bias.double().abs()
        away = (z - z.amax(1, keepdim=True)).abs()
        e_lse = ((p * (e_z + 2 * U * away)).sum(1) + (n / 256 + 64) * (4 * U + 2.0 ** -21) + e_z.amax(1) * 1e-3
                 + 2 * U * want.abs() + 2.0 ** -21)
        assert bool(((lse[rows].double() - want).abs() <= e_lse).all())
        at = labels[rows].clamp(min=0).long()[:, None]
        r = torch.where(c[:, 0], want - z.gather(1, at)[:, 0], 0.0)
        assert bool(((row[rows].double() - r).abs() <= e_lse + e_z.gather(1, at)[:, 0] + 2 * U * r.abs()).all())
        total += float(r.sum())
        l = lse[rows].double()[:, None]
        p = torch.where(c, (z - l).exp(), 0.0)
        gr = p.clone()
        gr.scatter_add_(1, at, -c.double())
        exact = p * (e_z + 2.0 ** -21 + 2 * U * (z - l).abs()) + U * gr.abs()
        stored = torch.where(c, exact + HALF[dtype] * (gr.abs() + exact) + (2.0 ** -40 if dtype == "f16" else 2.0 ** -134), 0.0)
        wt = wd.t().contiguous()
        dx_want = a * (gr @ wt)
        tol = a * ((stored + (n + 68) * U * gr.abs()) @ wt.abs()) + (4 * U + 1.01 * HALF[dtype]) * dx_want.abs() + TINY[dtype]
        assert bool(((dx[rows].double() - dx_want).abs() <= tol).all())
        xm = torch.where(c, xd, 0.0).t().contiguous()
        dw_want += a * (xm @ gr)
        dw_tol += a * (xm.abs() @ (stored + (m + 64) * U * gr.abs()))
        db_want += a * gr.sum(0)
        db_tol += a * (torch.where(c, exact, 0.0) + (m + 8) * U * gr.abs()).sum(0)
    assert abs(float(loss) - a * total) <= 1e-4 * abs(a * total)
    got = dw.double().t() if by_class else dw.double()
    assert bool(((got - dw_want).abs() <= dw_tol + 6 * U * dw_want.abs()).all())
    assert bool(((db.double() - db_want).abs() <= db_tol + 4 * U * db_want.abs()).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k", [(6, 600, 64), (70, 2048, 128), (300, 1031, 40)])
def test_masked_classes(mdnn, m, n, k, by_class, dtype):
    """A bias of -Inf (whole tiles of them) or of the type's lowest value takes classes out: no probability, no gradient."""
    import torch
    for low in (-np.inf, float(np.finfo(np.float32).min)):
        p = Problem(m, n, k, dtype, by_class)
        p.bias[: n // 2] = low
        p.bias[n - 3:] = low
        p.labels[p.labels != IGNORED] = n // 2 + 1
        p.dlabels = torch.from_numpy(p.labels).cuda()
        p.check_forward(mdnn)
        p.check_backward(mdnn)
        bias, kw = p.args(mdnn)
        lse = p.forward(mdnn)[2]
        _, dw, db = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, lse, bias, **kw)
        out = torch.isinf(bias) | (bias < -1e38)
        assert bool((db[out] == 0).all()) and bool(((dw if by_class else dw.t())[out] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(6, 600, 64), (70, 2048, 128), (300, 1031, 40)])
def test_rows_without_a_distribution(mdnn, m, n, k, dtype):
    """Every class masked: lse -Inf and no loss, also no NaN in the other rows' place; ignored rows count nowhere, whatever
    they hold; a label that is no class makes its row NaN."""
    import torch
    p = Problem(m, n, k, dtype, True)
    p.bias[:] = -np.inf
    _, row, lse = p.forward(mdnn)
    assert bool((lse == -float("inf")).all()) and bool(row[p.dlabels != IGNORED].isnan().all())
    assert bool((row[p.dlabels == IGNORED] == 0).all())
    # ignored rows hold Inf and NaN
    p = Problem(m, n, k, dtype, True)
    clean_f, bias_kw = p.forward(mdnn), p.args(mdnn)
    clean_b = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, clean_f[2], bias_kw[0], **bias_kw[1])
    skip = p.dlabels == IGNORED
    assert bool(skip.any())
    p.x[skip] = float("nan")
    p.x[int(skip.nonzero()[0, 0]), 0] = float("inf")
    loss, row, lse = p.forward(mdnn)
    assert torch.equal(loss, clean_f[0]) and torch.equal(row, clean_f[1]) and torch.equal(lse[~skip], clean_f[2][~skip])
    got = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, lse, bias_kw[0], **bias_kw[1])
    assert all(torch.equal(a, b) for a, b in zip(got, clean_b))
    # all ignored: nothing
    none = torch.full_like(p.dlabels, IGNORED)
    loss, row, lse = mdnn.linear_xent(p.x, p.w, none, bias_kw[0], **bias_kw[1])
    assert float(loss) == 0.0 and bool((row == 0).all())
    got = mdnn.linear_xent_bwd(p.x, p.w, none, lse, bias_kw[0], **bias_kw[1])
    assert all(bool((t == 0).all()) for t in got)
    # labels that are no class
    p = Problem(m, n, k, dtype, True)
    bad = p.dlabels.clone()
    bad[1], bad[2] = n, -1
    loss, row, lse = mdnn.linear_xent(p.x, p.w, bad, bias_kw[0], **bias_kw[1])
    assert bool(loss.isnan()) and bool(row[1:3].isnan().all()) and not bool(row[3:].isnan().any())
    dx, dw, db = mdnn.linear_xent_bwd(p.x, p.w, bad, lse, bias_kw[0], **bias_kw[1])
    assert bool(dx[1:3].isnan().all()) and not bool(dx[3:].isnan().any()) and bool(dw.isnan().all()) and bool(db.isnan().all())


def test_no_rows_and_some_outputs(mdnn):
    import torch
    x, labels = torch.empty((0, 64), device="cuda").half(), torch.empty((0,), dtype=torch.int32, device="cuda")
    w = torch.randn(64, 100, device="cuda").half()
    bias = torch.zeros(100, device="cuda")
    loss, row, lse = mdnn.linear_xent(x, w, labels, bias)
    assert float(loss) == 0.0 and row.numel() == 0
    for t in (torch.float32, torch.float16):
        dx, dw, db = mdnn.linear_xent_bwd(x, w, labels, lse, bias, dw_dtype=t)
        assert bool((dw == 0).all()) and bool((db == 0).all())
    p = Problem(70, 1030, 72, "bf16", False)
    bias, kw = p.args(mdnn)
    full = p.forward(mdnn)
    ws = torch.empty(mdnn.mdnn_linear_xent_bwd_workspace(mdnn.NN, 70, 1030, 72, mdnn.BF16)
                     + mdnn.mdnn_linear_xent_fwd_workspace(mdnn.NN, 70, 1030, 72, mdnn.BF16), dtype=torch.uint8, device="cuda")
    for k in range(3):
        out = [None] * 3
        out[k] = torch.empty_like(full[k])
        mdnn.mdnn_linear_xent_fwd(mdnn.NN, 70, 1030, 72, p.x, 72, p.w, 1030, mdnn.BF16, bias, p.dlabels, IGNORED, *out, ws,
                                  ws.numel())
        assert torch.equal(out[k], full[k])
    full = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, full[2], bias, **kw)
    lse = p.forward(mdnn)[2]
    for k in range(3):
        out = [None] * 3
        out[k] = torch.empty_like(full[k])
        mdnn.mdnn_linear_xent_bwd(mdnn.NN, 70, 1030, 72, p.x, 72, p.w, 1030, mdnn.BF16, bias, p.dlabels, IGNORED, lse, None,
                                  out[0], 72, out[1], 1030, mdnn.F32, out[2], ws, ws.numel())
        assert torch.equal(out[k], full[k])


def test_gradients_by_differences(mdnn):
    """dx, dw and db against differences of the forward loss."""
    import torch
    p = Problem(5, 37, 19, "f32", False)
    bias, kw = p.args(mdnn)
    loss, _, lse = p.forward(mdnn)
    got = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, lse, bias, **kw)
    # step 2^-6: e^2 / 6 times a third derivative below 8 (|w|^3 or |x|^3 times p's, below 3^3 / 4), plus rounding
    # 2^-22 * loss / e: below 2e-3
    e, args = 2.0 ** -6, [p.x, p.w, bias]
    for k, grad in enumerate(got):
        for at in list(np.ndindex(tuple(grad.shape)))[::7]:
            d = torch.zeros_like(args[k])
            d[at] = e
            up, down = ([a + (s * d if i == k else 0) for i, a in enumerate(args)] for s in (1, -1))
            f = lambda v: float(mdnn.linear_xent(v[0], v[1], p.dlabels, v[2], **kw)[0])
            assert abs((f(up) - f(down)) / (2 * e) - float(grad[at])) <= 2e-3, (k, at)


def test_the_loss_scale_does_not_move_the_rounding(mdnn):
    """Times a power of two, fp16 gradients far below its range without the scale keep the same bits."""
    import torch
    p = Problem(300, 2000, 96, "f16", True)
    bias, kw = p.args(mdnn)
    lse = p.forward(mdnn)[2]
    one = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, lse, bias, **kw)
    big = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, lse, bias, loss_scale=torch.full((1,), 4096.0, device="cuda"), **kw)
    assert torch.equal(one[1] * 4096, big[1]) and torch.equal(one[2] * 4096, big[2])


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 300, 2048, 128), ("f32", 130, 1001, 77), ("f16", 4, 5000, 256)])
def test_deterministic_and_captured(mdnn, dtype, m, n, k):
    """Both passes in one graph that shares a workspace, replayed on new rows with eager work in between."""
    import torch
    p = Problem(m, n, k, dtype, True)
    bias, kw = p.args(mdnn)
    code = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
    ws = torch.empty(max(f(mdnn.NT, m, n, k, code) for f in (mdnn.mdnn_linear_xent_fwd_workspace,
                                                             mdnn.mdnn_linear_xent_bwd_workspace)),
                     dtype=torch.uint8, device="cuda")
    loss, row, lse = torch.empty(1, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    dx, dw, db = torch.empty_like(p.x), torch.empty_like(p.w), torch.empty(n, device="cuda")
    outs = (loss, row, lse, dx, dw, db)

    def step():
        mdnn.mdnn_linear_xent_fwd(mdnn.NT, m, n, k, p.x, k, p.w, k, code, bias, p.dlabels, IGNORED, loss, row, lse, ws,
                                  ws.numel())
        mdnn.mdnn_linear_xent_bwd(mdnn.NT, m, n, k, p.x, k, p.w, k, code, bias, p.dlabels, IGNORED, lse, None, dx, k, dw, k,
                                  code, db, ws, ws.numel())

    step()
    first = [t.clone() for t in outs]
    for _ in range(3):
        ws.fill_(255)
        step()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        p.x.copy_(torch.randn(m, k, device="cuda"))
        p.dlabels.copy_(torch.randint(0, n, (m,), device="cuda"))
        if m > 8:
            p.dlabels[i:8] = IGNORED
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_side_stream(mdnn):
    import torch
    p = Problem(200, 777, 1000, "f16", False)
    bias, kw = p.args(mdnn)
    want = p.forward(mdnn)
    grads = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, want[2], bias, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mdnn.linear_xent(p.x, p.w, p.dlabels, bias, stream=side, **kw)
    back = mdnn.linear_xent_bwd(p.x, p.w, p.dlabels, got[2], bias, stream=side, **kw)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want + grads, got + back))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_and_its_loss_together(mdnn, dtype):
    """The operators as a step uses them: a layer's output dropped out, added to the residual and normed, the last layer's
    loss, and all gradients back through them, against the oracle's chain on the values that each operator stored."""
    import torch
    rows, cols, n, p_drop = 150, 264, 1500, 0.2
    g = np.random.default_rng(8)
    rng = mdnn.make_rng(77, 3)
    x, xv = _view(g.standard_normal((rows, cols)), dtype, 0, 0)
    res, rv = _view(g.standard_normal((rows, cols)), dtype, 0, 0)
    w, wv = _view(g.standard_normal((n, cols)) * 2 / np.sqrt(cols), dtype, 0, 0)
    gamma, beta = ((a + 0.2 * g.standard_normal(cols)).astype(np.float32) for a in (1, 0))
    labels = g.integers(0, n, rows).astype(np.int32)
    labels[:9] = IGNORED
    dl = torch.from_numpy(labels).cuda()
    y, h = mdnn.layernorm(x, dev(gamma, "f32"), dev(beta, "f32"), res, p=p_drop, rng=rng, site=1)
    loss, _, lse = mdnn.linear_xent(y, w, dl, layout=mdnn.NT, ignored=IGNORED)
    dy, dw, _ = mdnn.linear_xent_bwd(y, w, dl, lse, layout=mdnn.NT, ignored=IGNORED)
    dx, dh, dg, db = mdnn.layernorm_bwd(dy, h, dev(gamma, "f32"), p=p_drop, rng=rng, site=1)
    keep = B.kept(rows, cols, p_drop, 77, 3, 1)
    hv = keep * xv + rv
    yv = B.layernorm(hv, gamma, beta, 1e-5)
    want, _, l64, z = B.linear_xent(yv, wv.T, None, labels, IGNORED)
    dyv, dwv, _ = B.linear_xent_bwd(yv, wv.T, B.linear_xent_grad(z, l64, labels, IGNORED), labels, IGNORED)
    dhv, dgv, dbv = B.layernorm_bwd(dyv, hv, gamma, 1e-5)
    # the chain in exact numbers: every stored tensor on the way (h, y, dy, and G inside) adds its half step, relative in
    # the norm of what it feeds, and the logits' share enters through p (|z| errors of |y| |w| times half a step, about 2
    # here); ten such half steps bound each of the results in norm
    near = lambda a, b: np.linalg.norm(host64(a) - b) <= 10 * HALF[dtype] * np.linalg.norm(b) + 2e-5 * np.linalg.norm(b)
    assert abs(float(loss) - want) <= 10 * HALF[dtype] * abs(want) + 2e-5
    for a, b in ((dy, dyv), (dw, dwv.T), (dx, keep * dhv), (dh, dhv), (dg, dgv), (db, dbv)):
        assert near(a, b)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 1), (5, 300, 333), (64, 1024, 128), (300, 1031, 40), (600, 777, 200),
                                  (4100, 9000, 64), (600, 70001, 72), (9000, 20011, 32)])
def test_the_workspace_is_enough(mdnn, size, dtype):
    """Nothing is written past the bytes that the query names."""
    import torch
    m, n, k = size
    code = {"f32": 0, "f16": 1, "bf16": 2}[dtype]
    for layout in (mdnn.NN, mdnn.NT):
        x = torch.randn(m, k, device="cuda").to(_t(dtype))
        w = torch.randn(*((k, n) if layout == mdnn.NN else (n, k)), device="cuda").to(_t(dtype))
        labels = torch.randint(0, n, (m,), device="cuda", dtype=torch.int32)
        loss, row, lse = torch.empty(1, device="cuda"), torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, device="cuda")
        for backward in (False, True):
            f = mdnn.mdnn_linear_xent_bwd_workspace if backward else mdnn.mdnn_linear_xent_fwd_workspace
            need = f(layout, m, n, k, code)
            ws = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
            if backward:
                mdnn.mdnn_linear_xent_bwd(layout, m, n, k, x, k, w, w.shape[1], code, None, labels, -1, lse, None, dx, k, dw,
                                          w.shape[1], code, db, ws, need)
            else:
                mdnn.mdnn_linear_xent_fwd(layout, m, n, k, x, k, w, w.shape[1], code, None, labels, -1, loss, row, lse, ws,
                                          need)
            assert bool((ws[need:] == 0xA5).all())
