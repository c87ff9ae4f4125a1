"""Whole numbers that their C argument does not hold are refused by the binding:
cut off to 32 bits, a site would draw another one's bits and an ignored label
would name a class.  Refusals come before any GPU work."""
import pytest

from tests.test_abi_blocks import BWD, DROP, FWD, NORM, XBWD


@pytest.mark.parametrize("site", [-1, 1 << 32, (1 << 32) + 3])
def test_sites(site):
    import paper_2011_11188_amd as m
    bare = {k: v for k, v in DROP.items() if k not in ("res", "ldr")}
    for f, args in ((m.mdnn_dropout_fwd, DROP), (m.mdnn_dropout_bwd, bare), (m.mdnn_layernorm_fwd, NORM),
                    (m.mdnn_layernorm_bwd, {**BWD, "dgamma": None, "dbeta": None})):
        nothing = {**args, "rows": 0}  # (no rows: nothing would run)
        with pytest.raises(ValueError, match="site"):
            f(*{**nothing, "site": site}.values(), stream=0)
        for ok in (0, (1 << 32) - 1):
            f(*{**nothing, "site": ok}.values(), stream=0)


@pytest.mark.parametrize("ignored", [1 << 31, -(1 << 31) - 1, 1 << 32, (1 << 32) - 1])
def test_ignored_labels(ignored):
    import paper_2011_11188_amd as m
    for f, args, none in ((m.mdnn_linear_xent_fwd, FWD, ("loss", "row_loss", "lse")),
                          (m.mdnn_linear_xent_bwd, XBWD, ("dx", "dw", "db"))):
        nothing = {**args, **dict.fromkeys(none)}  # (no output: nothing would run)
        with pytest.raises(ValueError, match="ignored"):
            f(*{**nothing, "ignored": ignored}.values(), stream=0)
        for ok in (-(1 << 31), (1 << 31) - 1):
            f(*{**nothing, "ignored": ok}.values(), stream=0)
