"""Results that the tensor-level wrappers allocate for a call on a given
stream: whose memory they are, and how long they are kept."""
import pytest

pytestmark = pytest.mark.gpu


def _owner(t):
    """The stream whose memory t lies in."""
    import torch
    at = t.untyped_storage().data_ptr()
    return [g["stream"] for g in torch.cuda.memory_snapshot() if g["address"] <= at < g["address"] + g["total_size"]]


def _calls(m):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(2000, 500, generator=g, device="cuda") for _ in range(2))
    gamma = torch.rand(500, generator=g, device="cuda")
    codes = torch.randint(-127, 128, (4100, 33), generator=g, dtype=torch.int8, device="cuda")
    wide = torch.randint(-127, 128, (8300, 33), generator=g, dtype=torch.int8, device="cuda")
    sa, sb = torch.rand(4100, generator=g, device="cuda"), torch.rand(8300, generator=g, device="cuda")
    half = x.half()
    img, grad = (torch.randn(64, 28, 28, c, generator=g, device="cuda").half() for c in (32, 64))
    filt = torch.randn(64, 3, 3, 32, generator=g, device="cuda").half()
    return {"quantize_i8": lambda **k: m.quantize_i8(x, **k),
            "quantize_i8 columns": lambda **k: m.quantize_i8(x, transpose=True, **k),
            "gemm_i8": lambda **k: (m.gemm_i8(codes, sa, wide, sb, workspace=True, **k),),
            "rmsnorm": lambda **k: m.rmsnorm(x, gamma, dy, **k),
            "rmsnorm_i8": lambda **k: m.rmsnorm_i8(x, gamma, dy, **k),
            "rmsnorm_bwd": lambda **k: m.rmsnorm_bwd(dy, x, gamma, **k),
            "gemm": lambda **k: (m.gemm(m.NT, half, half, workspace=True, **k),),
            "split_f16": lambda **k: m.split_f16(x, 0.0, **k),
            "gemm_split3": lambda **k: (m.gemm_split3(m.NT, x, dy, **k),),
            "conv2d_fwd": lambda **k: (m.conv2d_fwd(img, filt, 1, **k),),
            "conv2d_fwd_algo": lambda **k: (m.conv2d_fwd_algo(img, filt, 1, m.CONV_IM2COL_GEMM, **k),),
            "conv2d_fwd_winograd": lambda **k: (m.conv2d_fwd_winograd(img, filt, 1, **k),),
            "conv2d_bwd_data": lambda **k: (m.conv2d_bwd_data(grad, filt, 1, 28, 28, **k),),
            "conv2d_bwd_filter": lambda **k: m.conv2d_bwd_filter(img, grad, 3, 3, 1, **k)}


NAMES = ["quantize_i8", "quantize_i8 columns", "gemm_i8", "rmsnorm", "rmsnorm_i8", "rmsnorm_bwd", "gemm", "split_f16",
         "gemm_split3", "conv2d_fwd", "conv2d_fwd_algo", "conv2d_fwd_winograd", "conv2d_bwd_data", "conv2d_bwd_filter"]


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_results_of_a_call_on_a_given_stream(mdnn, name, handle):
    import torch
    call = _calls(mdnn)[name]
    want = call()
    side = torch.cuda.Stream()
    given = side.cuda_stream if handle else side
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=given)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # the memory of the stream that writes them: what the current stream has released is not in it
    assert all(_owner(t) == [side.cuda_stream] for t in got)
    # dropped while the current stream still reads them, they are not handed to the side stream's next work
    sums = lambda ts: [t.sum(dtype=torch.float64) for t in ts]
    first = sums(want)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    asleep = torch.cuda.Event()
    asleep.record()
    kept = sums(got)
    at = {t.untyped_storage().data_ptr() for t in got}
    sizes = [t.untyped_storage().nbytes() for t in got]
    del got
    with torch.cuda.stream(side):
        other = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
    assert not asleep.query(), "the reads were over before the memory was asked for"
    assert not at & {t.data_ptr() for t in other}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, kept))


def test_chain_on_a_given_stream_with_dropped_intermediates(mdnn):
    """A serving block whose calls all run on one given stream, nothing kept between them: the codes are not handed
    to the current stream's work while the given stream still waits to read them."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    x, res = (torch.randn(300, 2000, generator=g, device="cuda").half() for _ in range(2))
    w, gamma = torch.randn(2000, 700, generator=g, device="cuda"), torch.rand(2000, generator=g, device="cuda")

    def block(**k):
        qw, sw = mdnn.quantize_i8(w, transpose=True, **k)
        qx, sx, _ = mdnn.rmsnorm_i8(x, gamma, res, **k)
        y = mdnn.gemm_i8(qx, sx, qw, sw, act=mdnn.ACT_RELU, out_dtype=torch.float16, workspace=True, **k)
        del qx, sx, qw, sw
        if k:  # (work of the current stream that takes memory of the codes' sizes)
            junk.extend(torch.full((300 * 2048,), 85, dtype=torch.int8, device="cuda") for _ in range(6))
        return mdnn.quantize_i8(y, **k)

    junk = []
    want = block()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = block(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert all(bool((j == 85).all()) for j in junk)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("joined", [False, True])
def test_results_allocated_under_capture(mdnn, handle, joined):
    """A norm and its quantiser captured with the stream named in the calls: the capturing one, or a side stream joined
    to the capture; replayed on new data."""
    import torch
    x, gamma = torch.randn(70, 1531, device="cuda").half(), torch.rand(1531, device="cuda")
    side = torch.cuda.Stream()

    def step(stream):
        given = stream.cuda_stream if handle else stream
        y = mdnn.rmsnorm(x, gamma, stream=given)
        return mdnn.quantize_i8(y, transpose=True, stream=given)

    want = step(torch.cuda.current_stream())  # (loads the kernels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        now = torch.cuda.current_stream()
        if joined:
            side.wait_stream(now)
        got = step(side if joined else now)
        if joined:
            now.wait_stream(side)
    for _ in range(3):
        x.copy_(torch.randn(70, 1531, device="cuda").half())
        want = step(torch.cuda.current_stream())
        junk = torch.full((1 << 20,), 85, dtype=torch.uint8, device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert bool((junk == 85).all())
