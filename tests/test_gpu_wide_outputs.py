"""Products with more columns than a grid's second dimension counts tiles of
(65535 x 64), which fp32 products of few steps or of narrow operands put on
their vector kernel, and the last layer's gradients that make such products.

Tolerance: a chain of k fp32 products is within k u sum |a b| of it, u = 2^-24;
the result's factor and rounding add 2 u |d|."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
WIDE = 65535 * 64


def _close(got, a, b):
    """got against a b in 64 bits, a piece of the columns at a time."""
    for lo in range(0, b.shape[1], 1 << 20):
        p = b[:, lo:lo + (1 << 20)].double()
        want, tol = a.double() @ p, (a.shape[1] * U) * (a.double().abs() @ p.abs())
        if not bool(((got[:, lo:lo + (1 << 20)].double() - want).abs() <= tol + 2 * U * want.abs()).all()):
            return False
    return True


@pytest.mark.parametrize("n", [WIDE, WIDE + 4, WIDE + 64 * 7 + 12, 5000000])
@pytest.mark.parametrize("m,k", [(5, 8), (100, 8), (70, 16)])
def test_nn(mdnn, m, n, k):
    import torch
    a, b = torch.randn(m, k, device="cuda"), torch.randn(k, n, device="cuda")
    assert _close(mdnn.gemm(mdnn.NN, a, b), a, b)


@pytest.mark.parametrize("layout", ["NT", "TN"])
def test_other_layouts(mdnn, layout):
    import torch
    m, n, k = 9, WIDE + 1000, 12
    a = torch.randn(m, k, device="cuda")
    b = torch.randn(k, n, device="cuda")
    if layout == "NT":
        got = mdnn.gemm(mdnn.NT, a, b.t().contiguous())
    else:
        got = mdnn.gemm(mdnn.TN, a.t().contiguous(), b)
    assert _close(got, a, b)


@pytest.mark.parametrize("m,k", [(16, 8), (20, 64)])
def test_gradients_of_millions_of_classes(mdnn, m, k):
    """fp32 rows by feature: dW is one product of m steps with all the classes' columns."""
    import torch
    n = 5000000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(m, k, generator=g, device="cuda")
    w = torch.randn(k, n, generator=g, device="cuda") * 0.5
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    _, _, lse = mdnn.linear_xent(x, w, labels)
    dx, dw, _ = mdnn.linear_xent_bwd(x, w, labels, lse)
    xd, dx_want, dx_tol = x.double(), 0.0, 0.0
    for lo in range(0, n, 1 << 20):
        wd = w[:, lo:lo + (1 << 20)].double()
        z = xd @ wd
        p = (z - lse.double()[:, None]).exp()
        # logits k + 2 products' roundings, the exponential 2^-21 and its argument's 2 |z - lse| u (module note of the
        # cross entropy's tests), G's own rounding; the products' chains
        e = p * ((k + 2) * U * (xd.abs() @ wd.abs()) + 2.0 ** -21 + 2 * U * (z - lse.double()[:, None]).abs())
        at = labels.long() - lo
        here = ((at >= 0) & (at < wd.shape[1])).nonzero()[:, 0]
        p[here, at[here]] -= 1.0
        e = (e + U * p.abs()) / m
        p = p / m
        want, tol = xd.t() @ p, xd.abs().t() @ (e + (m + 4) * U * p.abs())
        assert bool(((dw[:, lo:lo + (1 << 20)].double() - want).abs() <= tol + 2.0 ** -149).all())
        dx_want = dx_want + p @ wd.t()
        dx_tol = dx_tol + (e + (n + 70) * U * p.abs()) @ wd.abs().t()
    assert bool(((dx.double() - dx_want).abs() <= dx_tol).all())
