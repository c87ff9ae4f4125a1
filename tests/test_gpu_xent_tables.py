"""The last layer's cross entropy over tables of classes past what one product's
32-bit offsets reach, both ways, against 64 bits on the GPU; bounds as in
test_gpu_xent.py's note."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
IGNORED = -7


def _check(mdnn, m, n, k, dtype, pad=0, step=1 << 14, by_class=True):
    import torch
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(m + n)
    x = torch.randn(m, k, generator=g, device="cuda").to(t)
    rows, cols = (n, k) if by_class else (k, n)
    w = torch.randn(rows, cols + pad, generator=g, device="cuda", dtype=t)[:, :cols]
    w *= 2 / k ** 0.5
    table = lambda v, lo: (v[lo:lo + step] if by_class else v[:, lo:lo + step].t()).double()  # noqa: E731
    bias = torch.randn(n, generator=g, device="cuda")
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    labels[0] = n - 1
    if m > 3:
        labels[1], labels[2], labels[3] = 0, IGNORED, n // 2
    kw = dict(layout=mdnn.NT if by_class else mdnn.NN, ignored=IGNORED)
    loss, row, lse = mdnn.linear_xent(x, w, labels, bias, **kw)
    dx, dw, db = mdnn.linear_xent_bwd(x, w, labels, lse, bias, dw_dtype=t, **kw)
    xd, counted = x.double(), labels != IGNORED
    a, l, at = 1.0 / int(counted.sum()), lse.double()[:, None], labels.long()

    def pieces():
        for lo in range(0, n, step):
            wd = table(w, lo).contiguous()
            z = xd @ wd.t() + bias[lo:lo + step].double()
            yield lo, wd, z, (k + 2) * U * (xd.abs() @ wd.abs().t()) + 2 * U * bias[lo:lo + step].double().abs()

    parts = []
    zl, el, off, most = (torch.zeros(m, dtype=torch.float64, device="cuda") for _ in range(4))
    for lo, wd, z, e in pieces():
        parts.append(torch.logsumexp(z, 1))
        off += ((z - l).exp() * (e + 2 * U * (z - l).abs())).sum(1)
        most = torch.maximum(most, e.amax(1))
        here = (at >= lo) & (at < lo + z.shape[1])
        r = here.nonzero()[:, 0]
        zl[r], el[r] = z[r, at[r] - lo], e[r, at[r] - lo]
    want = torch.logsumexp(torch.stack(parts), 0)
    e_lse = off * 1.01 + (n / 256 + 64) * (4 * U + 2.0 ** -21) + most * 1e-3 + 2 * U * want.abs() + 2.0 ** -21
    assert bool(((lse.double() - want).abs() <= e_lse).all())
    r = torch.where(counted, want - zl, 0.0)
    assert bool(((row.double() - r).abs() <= e_lse + el + 2 * U * r.abs()).all())
    assert abs(float(loss) - float(row.double().sum()) * a) <= 2 * U * abs(float(loss))
    xm = torch.where(counted[:, None], xd, 0.0)
    dx_want, dx_tol = 0.0, 0.0
    for lo, wd, z, e in pieces():
        p = torch.where(counted[:, None], (z - l).exp(), 0.0)
        exact = p * (e + 2.0 ** -21 + 2 * U * (z - l).abs())
        q = (counted & (at >= lo) & (at < lo + z.shape[1])).nonzero()[:, 0]
        p[q, at[q] - lo] -= 1.0
        exact += U * p.abs()
        stored = exact + HALF[dtype] * (p.abs() + exact) + (2.0 ** -40 if dtype == "f16" else 2.0 ** -134)
        stored = torch.where(counted[:, None], stored, 0.0)
        dx_want = dx_want + a * (p @ wd)
        dx_tol = dx_tol + a * ((stored + (n + 68) * U * p.abs()) @ wd.abs())
        w_want = a * (p.t() @ xm)
        tol = a * ((stored + (m + 64) * U * p.abs()).t() @ xm.abs()) + TINY[dtype]
        tol = tol + (6 * U + 1.01 * HALF[dtype]) * w_want.abs()
        assert bool(((table(dw, lo) - w_want).abs() <= tol).all()), lo
        b_want = a * p.sum(0)
        tol = a * (exact + (m + 8) * U * p.abs()).sum(0) + 4 * U * b_want.abs() + TINY["f32"]
        assert bool(((db[lo:lo + step].double() - b_want).abs() <= tol).all()), lo
    dx_tol = dx_tol + (4 * U + 1.01 * HALF[dtype]) * dx_want.abs() + TINY[dtype]
    assert bool(((dx.double() - dx_want).abs() <= dx_tol).all())


@pytest.mark.parametrize("m,n,k,dtype,pad", [(3, 250880, 8704, "bf16", 0), (70, 250880, 8704, "bf16", 0),
                                             (200, 250881, 8704, "f16", 8), (5, 250880, 8707, "f16", 0),
                                             (2, 4300000, 256, "f32", 0), (20, 4300001, 257, "f32", 0)])
def test_tables_of_2_31_elements(mdnn, m, n, k, dtype, pad):
    assert n * k >= 2 ** (30 if dtype == "f32" else 31)
    _check(mdnn, m, n, k, dtype, pad, 1 << (19 if k < 1000 else 14))


@pytest.mark.parametrize("m,n,k,dtype,pad", [(70, 250880, 8704, "bf16", 0), (20, 250881, 8704, "f16", 0),
                                             (3, 250880, 8704, "bf16", 8), (20, 262144, 4200, "f32", 4)])
def test_class_contiguous_weights_of_2_31_elements(mdnn, m, n, k, dtype, pad):
    assert n * k >= 2 ** (30 if dtype == "f32" else 31)
    _check(mdnn, m, n, k, dtype, pad, by_class=False)


def _check_rows(mdnn, m, n, k, dtype):
    """Class-contiguous W and many rows, a piece of the rows at a time."""
    import torch
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.empty(m, k, dtype=t, device="cuda").normal_(generator=g)
    w = (torch.randn(k, n, generator=g, device="cuda") * 2 / k ** 0.5).to(t)
    bias = torch.randn(n, generator=g, device="cuda")
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    labels[::7], labels[1], labels[2] = IGNORED, n - 1, n // 256 * 256
    loss, row, lse = mdnn.linear_xent(x, w, labels, bias, ignored=IGNORED)
    dx, dw, db = mdnn.linear_xent_bwd(x, w, labels, lse, bias, ignored=IGNORED)
    counted = labels != IGNORED
    a, wd = 1.0 / int(counted.sum()), w.double()
    dw_want, dw_tol = torch.zeros_like(wd), torch.zeros_like(wd)
    db_want, db_tol = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    wt = wd.t().contiguous()
    step = max(40, (1 << 25) // max(n, k))
    for lo in range(0, m, step):
        rows = slice(lo, min(m, lo + step))
        xd, c = x[rows].double(), counted[rows, None]
        z, e_z = xd @ wd + bias.double(), (k + 2) * U * (xd.abs() @ wd.abs()) + 2 * U * bias.double().abs()
        want = torch.logsumexp(z, 1)
        p = (z - want[:, None]).exp()
        e = ((p * (e_z + 2 * U * (z - z.amax(1, keepdim=True)).abs())).sum(1) + (n / 256 + 64) * (4 * U + 2.0 ** -21)
             + e_z.amax(1) * 1e-3 + 2 * U * want.abs() + 2.0 ** -21)
        assert bool(((lse[rows].double() - want).abs() <= e).all())
        at = labels[rows].clamp(min=0).long()[:, None]
        r = torch.where(c[:, 0], want - z.gather(1, at)[:, 0], 0.0)
        assert bool(((row[rows].double() - r).abs() <= e + e_z.gather(1, at)[:, 0] + 2 * U * r.abs()).all())
        l = lse[rows].double()[:, None]
        p = torch.where(c, (z - l).exp(), 0.0)
        exact = p * (e_z + 2.0 ** -21 + 2 * U * (z - l).abs())
        p.scatter_add_(1, at, -c.double())
        exact += U * p.abs()
        least = 2.0 ** -40 if dtype == "f16" else 2.0 ** -134
        stored = torch.where(c, exact + HALF[dtype] * (p.abs() + exact) + least, 0.0)
        dx_want = a * (p @ wt)
        tol = a * ((stored + (n + 68) * U * p.abs()) @ wt.abs()) + TINY[dtype]
        tol = tol + (4 * U + 1.01 * HALF[dtype]) * dx_want.abs()
        assert bool(((dx[rows].double() - dx_want).abs() <= tol).all())
        xm = torch.where(c, xd, 0.0).t().contiguous()
        dw_want += a * (xm @ p)
        dw_tol += a * (xm.abs() @ (stored + (m + 64) * U * p.abs()))
        db_want += a * p.sum(0)
        db_tol += a * (torch.where(c, exact, 0.0) + (m + 8) * U * p.abs()).sum(0)
    assert bool(((dw.double() - dw_want).abs() <= dw_tol + 6 * U * dw_want.abs()).all())
    assert bool(((db.double() - db_want).abs() <= db_tol + 4 * U * db_want.abs()).all())
    assert abs(float(loss) - float(row.double().sum()) * a) <= 2 * U * abs(float(loss))


@pytest.mark.parametrize("m,n,k,dtype", [(16384, 8193, 40, "f32"), (16384, 16387, 24, "f32"), (1 << 19, 515, 64, "f32"),
                                         (200, (1 << 19) + 3, 65, "f16"), (1 << 20, 2051, 33, "f32")])
def test_short_last_pieces(mdnn, m, n, k, dtype):
    """Classes that leave less than a 16-byte chunk past whole pieces."""
    _check_rows(mdnn, m, n, k, dtype)


@pytest.mark.parametrize("m,n,k,dtype", [(540000, 520, 4096, "bf16"), (530001, 261, 4100, "f16"),
                                         (270000, 300, 4096, "f32")])
def test_rows_of_2_31_elements(mdnn, m, n, k, dtype):
    """x past what 32-bit offsets reach."""
    assert m * k >= 2 ** (30 if dtype == "f32" else 31)
    _check_rows(mdnn, m, n, k, dtype)
