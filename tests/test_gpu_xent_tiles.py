"""Kernels of the last layer's cross entropy that only larger sizes reach, each
in both forms of W; problems and bounds of test_gpu_xent.py."""
import pytest

from tests import test_gpu_xent as X

pytestmark = pytest.mark.gpu
IGNORED = X.IGNORED


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k,pad,offset", [(4096, 4096, 192, 0, 0), (4090, 4100, 190, 3, 1), (3900, 4352, 256, 8, 8)])
def test_largest_tiles(mdnn, m, n, k, pad, offset, by_class, dtype):
    """Tiles of 256 x 256 (from one a compute unit on, K above 128), W as it is and copied."""
    assert -(-m // 256) * -(-n // 256) >= 256 and k > 128
    p = X.Problem(m, n, k, dtype, by_class, pad=pad, offset=offset)
    p.check_forward(mdnn)
    p.check_backward(mdnn, dw_type=dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k", [(385, 9024, 1300), (700, 12007, 1301), (1000, 10001, 1283), (600, 3001, 1001),
                                   (321, 5002, 1030), (1024, 4096, 640)])
def test_fp32_gradients_of_hundreds_of_rows(mdnn, m, n, k, by_class, pad, offset, dtype):
    """dW in fp32 from 16-bit operands in whole rows: 128 x 128 tiles with one step in LDS (768 and more) and with two."""
    X.Problem(m, n, k, dtype, by_class, pad=pad, offset=offset).check_backward(mdnn, dw_type="f32")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("by_class", [False, True])
@pytest.mark.parametrize("m,n,k", [(1100, 2900, 1000), (1100, 3100, 1000), (520, 5600, 1024), (520, 5900, 1024)])
def test_split_depths(mdnn, m, n, k, by_class, dtype):
    """dx whole and in parts of its depth (the classes), on both sides of the rule's lines."""
    X.Problem(m, n, k, dtype, by_class).check_backward(mdnn, dw_type=dtype)


@pytest.mark.parametrize("m,n,k,dtype", [(1025, 300, 40, "f32"), (4100, 1001, 64, "f16"), (70001, 515, 24, "bf16"),
                                         (1 << 20, 300, 32, "bf16")])
def test_the_mean_over_many_blocks(mdnn, m, n, k, dtype):
    """More than 1024 rows, whose mean the last block takes: the rows' own losses over those that count (a sum in 64 bits, a
    quotient and one rounding), with workspaces of any content, in every run."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(m)
    x, w = (torch.randn(s, generator=g, device="cuda").to(X._t(dtype)) for s in ((m, k), (k, n)))
    labels = torch.randint(0, n, (m,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(m, generator=g, device="cuda") < 0.3] = IGNORED
    labels[m - 1] = 0
    ws = torch.empty(mdnn.mdnn_linear_xent_fwd_workspace(mdnn.NN, m, n, k, mdnn.dtype_of(x)), dtype=torch.uint8,
                     device="cuda")
    seen = []
    for fill in (0, 255, 1):
        ws.fill_(fill)
        loss, row, _ = mdnn.linear_xent(x, w, labels, ignored=IGNORED, workspace=ws)
        want = float(row.double().sum()) / int((labels != IGNORED).sum())
        # one rounding to fp32; the sums in 64 bits differ by their order, m u^2 of it
        assert abs(float(loss) - want) <= 2.0 ** -24 * abs(want) * (1 + 2.0 ** -5)
        seen.append((float(loss), row))
    assert all(a == seen[0][0] and torch.equal(b, seen[0][1]) for a, b in seen)


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 4100, 1001, 64), ("f32", 1500, 520, 33), ("f16", 2048, 4160, 192)])
def test_captured_with_many_rows(mdnn, dtype, m, n, k):
    X.test_deterministic_and_captured(mdnn, dtype, m, n, k)
