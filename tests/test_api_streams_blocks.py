"""Whose memory the wrappers of dropout, layer norm and the cross entropy
allocate, on the host (see test_api_streams.py for the records)."""
import pytest

from tests.test_api_streams import SIDE, Stream, streams  # noqa: F401


def _calls(m, new):
    """(call, shapes of its results) of every wrapper of these operators that takes a stream."""
    import torch
    x, w, v20 = new((6, 20)), new((20, 9)), new((20,))
    labels, lse, bias, rng = new((6,), torch.int32), new((6,)), new((9,)), new((2,), torch.int64)
    drop = dict(p=0.5, rng=rng)
    return {
        "dropout": (lambda **k: m.dropout(x, **drop, **k), [(6, 20)]),
        "dropout_bwd": (lambda **k: m.dropout_bwd(x, **drop, **k), [(6, 20)]),
        "layernorm": (lambda **k: m.layernorm(x, v20, v20, x, **drop, **k), [(6, 20), (6, 20)]),
        "layernorm_bwd": (lambda **k: m.layernorm_bwd(x, x, v20, **drop, **k), [(6, 20), (6, 20), (20,), (20,)]),
        "linear_xent": (lambda **k: m.linear_xent(x, w, labels, bias, **k), [(1,), (6,), (6,)]),
        "linear_xent_bwd": (lambda **k: m.linear_xent_bwd(x, w, labels, lse, bias, **k), [(6, 20), (20, 9), (9,)]),
    }


@pytest.mark.parametrize("given,owner", [(None, "current"), (7, "current"), (Stream("current"), "current"),
                                         (0, "default"), (64, ("external", 64)), (SIDE, "side")])
@pytest.mark.parametrize("name", ["dropout", "dropout_bwd", "layernorm", "layernorm_bwd", "linear_xent",
                                  "linear_xent_bwd"])
def test_results_belong_to_the_calls_stream(streams, monkeypatch, name, given, owner):  # noqa: F811
    import paper_2011_11188_amd as m
    from paper_2011_11188_amd import api
    for f in dir(api):
        if f.startswith("mdnn_") and not f.endswith("_workspace"):
            monkeypatch.setattr(api, f, lambda *a, **k: None)
    call, results = _calls(m, streams.tensor)[name]
    call(stream=given)
    assert len(streams.made) >= len(results) and all(o == owner for _, o in streams.made), streams.made
    assert sorted(streams.also_used) == ([] if owner == "current" else sorted((r, "current") for r in results))
    assert streams.stack == ["current"]


def test_wrappers_refuse(streams):  # noqa: F811
    import torch
    import paper_2011_11188_amd as m
    new = streams.tensor
    x, w, labels, rng = new((6, 20)), new((20, 9)), new((6,), torch.int32), new((2,), torch.int64)
    for bad in (lambda: m.dropout(x, 0.5), lambda: m.dropout(x, 0.5, new((2,))), lambda: m.dropout(x, 0.5, rng, 0, x[:3]),
                lambda: m.dropout_bwd(x, 0.5, new((3,), torch.int64)), lambda: m.layernorm(x, new((19,))),
                lambda: m.layernorm(x, p=0.1), lambda: m.layernorm_bwd(x, None), lambda: m.layernorm_bwd(x, x[:, :8]),
                lambda: m.linear_xent(x, w, labels.long()), lambda: m.linear_xent(x, w, labels[:3]),
                lambda: m.linear_xent(x, w, labels, layout=m.NT), lambda: m.linear_xent(x, w, labels, layout=m.TN),
                lambda: m.linear_xent(x, w.half(), labels), lambda: m.linear_xent(x, w, labels, new((20,))),
                lambda: m.linear_xent_bwd(x, w, labels, new((5,))),
                lambda: m.linear_xent_bwd(x, w, labels, new((6,)), dw=new((9, 20)))):
        with pytest.raises(ValueError):
            bad()
