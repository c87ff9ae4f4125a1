"""Host checks of dropout, layer norm and the last layer's cross entropy: every
refusal below comes before any GPU work, so it runs without a GPU."""
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


DROP = dict(rows=4, cols=8, x=FAKE, ldx=8, res=FAKE, ldr=8, p=0.5, rng=FAKE, site=0, y=FAKE, ldy=8, dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=-1), 2), (dict(cols=(1 << 29) + 1), 2), (dict(p=-0.1), 2), (dict(p=1.1), 2),
    (dict(p=float("nan")), 2), (dict(rows=(1 << 32) + 1), 2), (dict(dtype=3), 4), (dict(x=None), 1), (dict(y=None), 1),
    (dict(rng=None), 1), (dict(ldx=7), 3), (dict(ldr=7), 3), (dict(ldy=7), 3), (dict(x=FAKE + 1), 5),
    (dict(res=FAKE + 1), 5), (dict(y=FAKE + 1), 5), (dict(rng=FAKE + 4), 5)])
def test_dropout_refuses(m, change, status):
    a = {**DROP, **change}
    _refuses(m, status, m.mdnn_dropout_fwd, *a.values())
    if not set(change) & {"res", "ldr"}:
        _refuses(m, status, m.mdnn_dropout_bwd, *(v for k, v in a.items() if k not in ("res", "ldr")))


def test_dropout_of_nothing(m):
    for change in (dict(rows=0), dict(cols=0)):
        assert m.mdnn_dropout_fwd(*{**DROP, **change, "x": None, "y": None}.values(), stream=0) == 0


NORM = dict(rows=4, cols=8, x=FAKE, ldx=8, res=FAKE, ldr=8, p=0.5, rng=FAKE, site=0, gamma=FAKE, beta=FAKE, eps=1e-5,
            h=FAKE, ldh=8, y=FAKE, ldy=8, dtype=1)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(cols=(1 << 29) + 1), 2), (dict(eps=0.0), 2), (dict(eps=float("nan")), 2),
    (dict(eps=float("inf")), 2), (dict(p=-1e-3), 2), (dict(p=2.0), 2), (dict(dtype=9), 4), (dict(x=None), 1),
    (dict(y=None), 1), (dict(rng=None), 1), (dict(ldx=7), 3), (dict(ldr=7), 3), (dict(ldh=7), 3), (dict(ldy=7), 3),
    (dict(x=FAKE + 1), 5), (dict(res=FAKE + 1), 5), (dict(h=FAKE + 1), 5), (dict(y=FAKE + 1), 5),
    (dict(gamma=FAKE + 2), 5), (dict(beta=FAKE + 2), 5), (dict(rng=FAKE + 2), 5)])
def test_layernorm_refuses(m, change, status):
    _refuses(m, status, m.mdnn_layernorm_fwd, *{**NORM, **change}.values())


BWD = dict(rows=400, cols=8, dy=FAKE, lddy=8, h=FAKE, ldh=8, gamma=FAKE, eps=1e-5, dres=FAKE, lddr=8, p=0.5, rng=FAKE,
           site=0, dx=FAKE, lddx=8, dh=FAKE, lddh=8, dgamma=FAKE, dbeta=FAKE, dtype=1, ws=FAKE, nb=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 2), (dict(cols=0), 2), (dict(eps=-1.0), 2), (dict(p=1.5), 2), (dict(dtype=7), 4), (dict(dy=None), 1),
    (dict(h=None), 1), (dict(rng=None), 1), (dict(lddy=7), 3), (dict(ldh=7), 3), (dict(lddr=7), 3), (dict(lddx=7), 3),
    (dict(lddh=7), 3), (dict(dy=FAKE + 1), 5), (dict(h=FAKE + 1), 5), (dict(dres=FAKE + 1), 5), (dict(dx=FAKE + 1), 5),
    (dict(dh=FAKE + 1), 5), (dict(gamma=FAKE + 2), 5), (dict(dgamma=FAKE + 2), 5), (dict(dbeta=FAKE + 2), 5),
    (dict(ws=None), 6), (dict(ws=FAKE + 16), 6), (dict(nb=8), 6)])
def test_layernorm_gradients_refuse(m, change, status):
    _refuses(m, status, m.mdnn_layernorm_bwd, *{**BWD, **change}.values())


def test_layernorm_workspace(m):
    ws = m.mdnn_layernorm_bwd_workspace
    assert ws(0, 8) == 0 and ws(4, 0) == 0 and ws(-1, 8) == 0 and ws(4, (1 << 29) + 1) == 0
    assert ws(1, 4096) == 0  # a block alone
    assert ws(1 << 40, 4096) == ws(1 << 30, 4096) > 0  # the blocks' sums do not grow with the rows without end


FWD = dict(layout=0, M=4, N=16, K=8, x=FAKE, ldx=8, w=FAKE, ldw=16, dtype=1, bias=FAKE, labels=FAKE, ignored=-1,
           loss=FAKE, row_loss=FAKE, lse=FAKE, ws=FAKE, nb=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(layout=2), 3), (dict(layout=5), 3), (dict(M=-1), 2), (dict(M=(1 << 24) + 1), 2), (dict(N=0), 2),
    (dict(N=1 << 31), 2), (dict(K=0), 2), (dict(K=1 << 31), 2), (dict(dtype=4), 4), (dict(x=None), 1), (dict(w=None), 1),
    (dict(labels=None), 1), (dict(ldx=7), 3), (dict(ldw=15), 3), (dict(layout=1, ldw=7), 3), (dict(x=FAKE + 1), 5),
    (dict(w=FAKE + 1), 5), (dict(bias=FAKE + 2), 5), (dict(labels=FAKE + 2), 5), (dict(loss=FAKE + 2), 5),
    (dict(row_loss=FAKE + 2), 5), (dict(lse=FAKE + 2), 5), (dict(ws=None), 6), (dict(ws=FAKE + 128), 6), (dict(nb=64), 6)])
def test_cross_entropy_refuses(m, change, status):
    _refuses(m, status, m.mdnn_linear_xent_fwd, *{**FWD, **change}.values())


XBWD = dict(layout=0, M=4, N=16, K=8, x=FAKE, ldx=8, w=FAKE, ldw=16, dtype=1, bias=FAKE, labels=FAKE, ignored=-1,
            lse=FAKE, scale=FAKE, dx=FAKE, lddx=8, dw=FAKE, lddw=16, dw_type=0, db=FAKE, ws=FAKE, nb=1 << 40)


@pytest.mark.parametrize("change,status", [
    (dict(layout=2), 3), (dict(M=-1), 2), (dict(M=(1 << 24) + 1), 2), (dict(N=0), 2), (dict(K=0), 2), (dict(dtype=4), 4),
    (dict(dw_type=2), 4), (dict(dw_type=9), 4), (dict(dtype=0, dw_type=1, x=FAKE), 4), (dict(x=None), 1),
    (dict(w=None), 1), (dict(labels=None), 1), (dict(lse=None), 1), (dict(ldx=7), 3), (dict(ldw=15), 3),
    (dict(lddx=7), 3), (dict(lddw=15), 3), (dict(layout=1, ldw=8, lddw=7), 3), (dict(x=FAKE + 1), 5),
    (dict(w=FAKE + 1), 5), (dict(bias=FAKE + 2), 5), (dict(labels=FAKE + 2), 5), (dict(lse=FAKE + 2), 5),
    (dict(scale=FAKE + 2), 5), (dict(dx=FAKE + 1), 5), (dict(dw=FAKE + 2), 5), (dict(db=FAKE + 2), 5),
    (dict(ws=None), 6), (dict(ws=FAKE + 128), 6), (dict(nb=64), 6)])
def test_cross_entropy_gradients_refuse(m, change, status):
    _refuses(m, status, m.mdnn_linear_xent_bwd, *{**XBWD, **change}.values())


def test_cross_entropy_workspaces(m):
    for f in (m.mdnn_linear_xent_fwd_workspace, m.mdnn_linear_xent_bwd_workspace):
        assert f(2, 4, 16, 8, 1) == 0 and f(0, -1, 16, 8, 1) == 0 and f(0, 4, 0, 8, 1) == 0 and f(0, 4, 16, 8, 7) == 0
        assert f(0, 0, 16, 8, 1) == 0 and f(1, 4, 16, 8, 1) > 0
        # pieces: no logits of all classes (fp32 ones would be 32 GB)
        for t in (0, 1, 2):
            assert f(1, 16384, 1 << 19, 256, t) < 4 << 30
    assert m.mdnn_linear_xent_fwd(*{**FWD, "M": 4, "loss": None, "row_loss": None, "lse": None}.values(), stream=0) == 0
    assert m.mdnn_linear_xent_bwd(*{**XBWD, "dx": None, "dw": None, "db": None}.values(), stream=0) == 0


def test_the_generators_state_wraps(monkeypatch):
    import torch
    import paper_2011_11188_amd as m
    for seed in (0, 1, 2 ** 63 - 1, 2 ** 63, 2 ** 64 - 1):
        t = m.make_rng(seed, 2 ** 32 + 5, device="cpu")
        assert t.dtype == torch.int64 and [int(v) % 2 ** 64 for v in t.tolist()] == [seed, 2 ** 32 + 5]
