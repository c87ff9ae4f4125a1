"""The cross entropy's workspaces stay bounded whatever the classes: a piece of
G is at most 2^27 elements (its rows padded to 64 in 16 bits), a piece of stored
logits 2^24 forward and 2^25 backward, beside what goes by M, N or K alone."""
import pytest


@pytest.mark.parametrize("M", [1, 7, 64, 1000, 16384])
@pytest.mark.parametrize("N", [1 << 22, 1 << 25, (1 << 26) + 5, (1 << 31) - 1])
def test_many_classes(M, N):
    import paper_2011_11188_amd as m
    K = 64
    for layout in (m.NN, m.NT):
        for t, es in ((m.F32, 4), (m.F16, 2), (m.BF16, 2)):
            rows = max(64, -(-M // 64) * 64)
            forward = m.mdnn_linear_xent_fwd_workspace(layout, M, N, K, t)
            backward = m.mdnn_linear_xent_bwd_workspace(layout, M, N, K, t)
            # forward: logits or pairs of 64 columns at least (2^25 of a row block's 64), W's copy of at most 2^27 elements
            assert forward <= (1 << 26) + (8 << 25) + (es << 27) + 64 * M * K + (1 << 20)
            # backward: G, logits, W's copy, x's copy, column sums and products' parts of 64 MB at most each
            assert backward <= (es << 27) + (4 << 25) + (es << 27) + rows * K * 12 + (1 << 28)
