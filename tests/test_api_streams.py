"""Whose memory the tensor-level wrappers allocate, on the host: torch's
streams and the launches are replaced by records, so nothing runs on a GPU."""
import contextlib

import pytest


class Stream(str):
    """A stream by its name; its handle is the name's."""

    @property
    def cuda_stream(self):
        return {"current": 7, "side": 8}[self]


class Streams:
    """The stack of streams that allocations belong to, and what was asked for."""

    def __init__(self):
        self.stack = [Stream("current")]

    @contextlib.contextmanager
    def use(self, stream):
        self.stack.append(stream)
        try:
            yield
        finally:
            self.stack.pop()


@pytest.fixture
def streams(monkeypatch):
    import torch
    from paper_2011_11188_amd import api
    s = Streams()

    def external(handle):
        assert handle != 0, "a zero handle does not name the default stream here: torch takes a stream of its pool"
        return ("external", handle)

    monkeypatch.setattr(torch.cuda, "stream", s.use)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: "default")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: s.stack[-1])
    monkeypatch.setattr(api, "_s", lambda stream: s.stack[-1].cuda_stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)  # (a host tensor's device index)
    empty = torch.empty
    s.made = []
    s.also_used = []

    class Device(torch.Tensor):
        """A host tensor that the wrappers take for one of the current GPU."""
        is_cuda = True

        def record_stream(self, stream):
            s.also_used.append((tuple(self.shape), stream))

    def record(*args, **kw):
        t = empty(*args, **kw).as_subclass(Device)
        s.made.append((tuple(t.shape), s.stack[-1]))
        return t

    s.tensor = lambda shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype).as_subclass(Device)

    monkeypatch.setattr(torch, "empty", record)
    return s


def _calls(m, new):
    """(call, shapes of its results) of every wrapper that takes a stream."""
    import torch
    x, w = new((6, 20)), new((9, 20))
    img, filt, dy = new((2, 8, 8, 4), torch.float16), new((5, 3, 3, 4), torch.float16), new((2, 8, 8, 5), torch.float16)
    codes, wcodes = new((6, 20), torch.int8), new((9, 20), torch.int8)
    v6, v9, v20 = new((6,)), new((9,)), new((20,))
    return {
        "quantize_i8": (lambda **k: m.quantize_i8(x, **k), [(6, 20), (6,)]),
        "quantize_i8 columns": (lambda **k: m.quantize_i8(x, transpose=True, **k), [(20, 6), (20,)]),
        "gemm_i8": (lambda **k: m.gemm_i8(codes, v6, wcodes, v9, workspace=True, **k), [(6, 9)]),
        "rmsnorm": (lambda **k: m.rmsnorm(x, v20, x, **k), [(6, 20), (6, 20)]),
        "rmsnorm_i8": (lambda **k: m.rmsnorm_i8(x, v20, x, **k), [(6, 20), (6, 20), (6,)]),
        "rmsnorm_bwd": (lambda **k: m.rmsnorm_bwd(x, x, v20, **k), [(6, 20), (20,)]),
        "gemm": (lambda **k: m.gemm(m.NT, x, w, workspace=True, **k), [(6, 9)]),
        "split_f16": (lambda **k: m.split_f16(x, 0.0, **k), [(6, 20), (6, 20), (1,)]),
        "gemm_split3": (lambda **k: m.gemm_split3(m.NT, x, w, **k), [(6, 9)]),
        "conv2d_fwd": (lambda **k: m.conv2d_fwd(img, filt, 1, **k), [(2, 8, 8, 5)]),
        "conv2d_fwd_algo": (lambda **k: m.conv2d_fwd_algo(img, filt, 1, m.CONV_AUTO, **k), [(2, 8, 8, 5)]),
        "conv2d_fwd_winograd": (lambda **k: m.conv2d_fwd_winograd(img, filt, 1, **k), [(2, 8, 8, 5)]),
        "conv2d_bwd_data": (lambda **k: m.conv2d_bwd_data(dy, filt, 1, 8, 8, **k), [(2, 8, 8, 4)]),
        "conv2d_bwd_filter": (lambda **k: m.conv2d_bwd_filter(img, dy, 3, 3, 1, **k), [(5, 3, 3, 4), (5,)]),
    }


NAMES = ["quantize_i8", "quantize_i8 columns", "gemm_i8", "rmsnorm", "rmsnorm_i8", "rmsnorm_bwd", "gemm", "split_f16",
         "gemm_split3", "conv2d_fwd", "conv2d_fwd_algo", "conv2d_fwd_winograd", "conv2d_bwd_data", "conv2d_bwd_filter"]


SIDE = Stream("side")


@pytest.mark.parametrize("given,owner", [(None, "current"), (7, "current"), (Stream("current"), "current"),
                                         (0, "default"), (64, ("external", 64)), (SIDE, "side")])
@pytest.mark.parametrize("name", NAMES)
def test_results_belong_to_the_calls_stream(streams, monkeypatch, name, given, owner):
    """What a wrapper allocates, workspaces too, is the memory of the stream that writes it, and its results are also
    kept for the stream that was current, where the caller uses them; the current stream by name needs neither."""
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


def test_a_stream_given_by_position(streams, monkeypatch):
    import paper_2011_11188_amd as m
    from paper_2011_11188_amd import api
    monkeypatch.setattr(api, "mdnn_quantize_i8_t", lambda *a, **k: None)
    m.quantize_i8(streams.tensor((300, 20)), True, None, None, None, SIDE)
    assert [o for _, o in streams.made] == ["side"] * 3  # codes, scales and the workspace


def test_the_stream_is_current_again_after_an_error(streams):
    import paper_2011_11188_amd as m
    with pytest.raises(ValueError):
        m.rmsnorm(streams.tensor((6, 20)), streams.tensor((7,)), stream=SIDE)
    assert streams.stack == ["current"]
