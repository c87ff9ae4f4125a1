"""Tensor-level conveniences over the C ABI (argument marshalling only).

These derive sizes and leading dimensions from torch tensor shapes, allocate
outputs and workspaces with torch, and call the ``mdnn_*`` entry points.
With a ``stream`` argument (a torch stream or a handle; None: the current one)
the call runs on that stream and what it allocates is that stream's memory;
results are kept, too, until the current stream's work at their release is done.
Ordering the two streams is the caller's, as with torch's own operations.
"""
from __future__ import annotations

import ctypes as C
import functools
import inspect
from typing import Optional, Sequence

from . import (_s, ACT_NONE, BF16, F16, F32, LAYER_CONV, LAYER_FC, LAYER_MAXPOOL2, LOSS_MSE, LOSS_XENT,
               NN, NT, TN, ConvShape, LayerDesc, Scaler, TrainCfg, dtype_of, mdnn_conv2d_bwd_data,
               mdnn_conv2d_bwd_filter, mdnn_conv2d_bwd_filter_workspace, mdnn_conv2d_fwd,
               mdnn_gemm_mixed, mdnn_gemm_mixed_ws, mdnn_gemm_workspace, mdnn_gemm_split3,
               mdnn_gemm_split3_workspace, mdnn_net_activation, mdnn_net_output_grad, mdnn_net_bind, mdnn_net_create, mdnn_net_destroy, mdnn_net_sizes, mdnn_net_sync_lowp,
               mdnn_split_f16, mdnn_train_step, mdnn_train_step_async, mdnn_train_graph_create,
               mdnn_graph_launch, mdnn_graph_destroy, mdnn_conv2d_fwd_winograd,
               mdnn_conv2d_fwd_winograd_workspace, mdnn_conv2d_fwd_algo, mdnn_conv2d_fwd_algo_workspace,
               mdnn_quantize_i8, mdnn_quantize_i8_t, mdnn_quantize_i8_t_workspace, mdnn_gemm_i8,
               mdnn_gemm_i8_workspace, mdnn_rmsnorm_fwd, mdnn_rmsnorm_i8_fwd, mdnn_rmsnorm_bwd,
               mdnn_rmsnorm_bwd_workspace)

__all__ = ["torch_dtype", "gemm", "split_f16", "gemm_split3", "conv_shape", "conv2d_fwd",
           "conv2d_fwd_winograd", "conv2d_fwd_algo", "conv2d_bwd_data", "conv2d_bwd_filter", "make_scaler", "read_scaler", "Net", "StepGraph",
           "quantize_i8", "gemm_i8", "rmsnorm", "rmsnorm_i8", "rmsnorm_bwd"]


def torch_dtype(code: int):
    import torch
    return {F32: torch.float32, F16: torch.float16, BF16: torch.bfloat16}[code]


def _on_its_stream(wrapper):
    """A wrapper whose call on a given stream is made with that stream current:
    what it allocates is that stream's memory, which no pending work of another
    one still uses.  Its results are kept, besides, until the work that the
    caller's own stream has at their release is done."""
    names = list(inspect.signature(wrapper).parameters)
    at = names.index("stream")

    @functools.wraps(wrapper)
    def call(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None or (stream if isinstance(stream, int) else stream.cuda_stream) == _s(None):
            return wrapper(*args, **kw)
        import torch
        own = torch.cuda.current_stream()
        if isinstance(stream, int):  # (0 is the default stream; an ExternalStream of 0 would be one of torch's pool)
            stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
        with torch.cuda.stream(stream):
            results = wrapper(*args, **kw)
        for t in results if isinstance(results, tuple) else (results,):
            if t is not None:
                t.record_stream(own)
        return results

    return call


@_on_its_stream
def gemm(layout: int, A, B, out_dtype=None, bias=None, act: int = ACT_NONE, mask=None,
         alpha: float = 1.0, beta: float = 0.0, Cm=None, out=None, stream=None, workspace=None,
         nonfinite=None):
    """D = epi(alpha op(A) op(B) + beta C) for row-major 2-D tensors A, B.
    workspace: None (mdnn_gemm_mixed), True (allocate what
    mdnn_gemm_workspace asks for) or a device byte tensor (mdnn_gemm_mixed_ws).
    nonfinite: a device int32 tensor set to 1 when a stored value of the fp32
    D is Inf or NaN (mdnn_gemm_mixed_ws; implies a workspace, empty if None)."""
    import torch
    if layout == TN:
        K, M = A.shape
    else:
        M, K = A.shape
    N = B.shape[0] if layout == NT else B.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype or torch.float32, device=A.device)
    args = (layout, M, N, K, alpha, A, A.stride(0), B, B.stride(0), dtype_of(A), beta, Cm,
            Cm.stride(0) if Cm is not None else 0, out, out.stride(0), dtype_of(out), bias,
            act, mask, mask.stride(0) if mask is not None else 0)
    if workspace is None and nonfinite is None:
        mdnn_gemm_mixed(*args, stream)
        return out
    if workspace is True:
        nb = mdnn_gemm_workspace(dtype_of(A), M, N, K)
        workspace = torch.empty((max(nb, 16),), dtype=torch.uint8, device=A.device)
    mdnn_gemm_mixed_ws(*args, workspace, workspace.numel() if workspace is not None else 0, stream,
                       nonfinite=nonfinite)
    return out


@_on_its_stream
def split_f16(x, scale: float = 1.0, stream=None, scale_out=None):
    """(hi, lo) fp16 tensors of the two-term split of a 2-D fp32 tensor.
    scale 0 lets the library choose the power of two on the device; it is
    written to ``scale_out`` (a one-element fp32 device tensor, allocated when
    not given, returned as the third value)."""
    import torch
    rows, cols = x.shape
    hi = torch.empty((rows, cols), dtype=torch.float16, device=x.device)
    lo = torch.empty((rows, cols), dtype=torch.float16, device=x.device)
    if scale == 0.0 and scale_out is None:
        scale_out = torch.empty((1,), dtype=torch.float32, device=x.device)
    mdnn_split_f16(rows, cols, x, x.stride(0), scale, scale_out, hi, cols, lo, cols, stream)
    return (hi, lo, scale_out) if scale == 0.0 else (hi, lo)


@_on_its_stream
def gemm_split3(layout: int, A, B, a_scale: float = 1.0, b_scale: float = 1.0, alpha: float = 1.0,
                beta: float = 0.0, Cm=None, out=None, stream=None):
    """fp32 D = alpha op(A) op(B) + beta C through three fp16 MFMA products
    (a scale of 0: chosen on the device from the operand's largest magnitude)."""
    import torch
    if layout == TN:
        K, M = A.shape
    else:
        M, K = A.shape
    N = B.shape[0] if layout == NT else B.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=A.device)
    ws_bytes = mdnn_gemm_split3_workspace(M, N, K)
    ws = torch.empty((max(ws_bytes, 256),), dtype=torch.uint8, device=A.device)
    mdnn_gemm_split3(layout, M, N, K, alpha, A, A.stride(0), a_scale, B, B.stride(0), b_scale, beta, Cm,
                     Cm.stride(0) if Cm is not None else 0, out, out.stride(0), ws, ws_bytes, stream)
    return out


def conv_shape(x_shape: Sequence[int], c_out: int, r: int, s: int, pad: int) -> ConvShape:
    n, h, w, c = x_shape
    return ConvShape(n, h, w, c, c_out, r, s, pad)


@_on_its_stream
def conv2d_fwd(x, w, pad: int, bias=None, act: int = ACT_NONE, out_dtype=None, stream=None):
    import torch
    k, r, s, c = w.shape
    sh = conv_shape(x.shape, k, r, s, pad)
    ho, wo = sh.h + 2 * pad - r + 1, sh.w + 2 * pad - s + 1
    y = torch.empty((sh.n, ho, wo, k), dtype=out_dtype or x.dtype, device=x.device)
    mdnn_conv2d_fwd(sh, x, w, dtype_of(x), bias, act, y, dtype_of(y), stream)
    return y


@_on_its_stream
def conv2d_fwd_algo(x, w, pad: int, algo: int, bias=None, act: int = ACT_NONE, out_dtype=None, workspace=None,
                    stream=None):
    """conv2d_fwd through a chosen algorithm (CONV_AUTO: the library's
    per-layer choice for the given workspace; a workspace of the algorithm's
    size is allocated when none is given)."""
    import torch
    k, r, s, c = w.shape
    sh = conv_shape(x.shape, k, r, s, pad)
    ho, wo = sh.h + 2 * pad - r + 1, sh.w + 2 * pad - s + 1
    y = torch.empty((sh.n, ho, wo, k), dtype=out_dtype or x.dtype, device=x.device)
    io = dtype_of(x)
    if workspace is None:
        need = mdnn_conv2d_fwd_algo_workspace(sh, io, algo)
        workspace = torch.empty((max(need, 256),), dtype=torch.uint8, device=x.device)
    mdnn_conv2d_fwd_algo(sh, x, w, io, bias, act, y, dtype_of(y), algo, workspace, workspace.numel(), stream)
    return y


@_on_its_stream
def conv2d_fwd_winograd(x, w, pad: int, bias=None, act: int = ACT_NONE, out_dtype=None, workspace=None,
                        stream=None):
    """conv2d_fwd through Winograd F(2x2, 3x3) (3x3 filters, fp16 / bf16)."""
    import torch
    k, r, s, c = w.shape
    sh = conv_shape(x.shape, k, r, s, pad)
    ho, wo = sh.h + 2 * pad - r + 1, sh.w + 2 * pad - s + 1
    y = torch.empty((sh.n, ho, wo, k), dtype=out_dtype or x.dtype, device=x.device)
    nb = mdnn_conv2d_fwd_winograd_workspace(sh, dtype_of(x))
    if workspace is None:
        workspace = torch.empty((max(nb, 256),), dtype=torch.uint8, device=x.device)
    mdnn_conv2d_fwd_winograd(sh, x, w, dtype_of(x), bias, act, y, dtype_of(y), workspace, workspace.numel(), stream)
    return y


@_on_its_stream
def conv2d_bwd_data(dy, w, pad: int, h: int, wd: int, mask=None, out_dtype=None, stream=None):
    import torch
    k, r, s, c = w.shape
    sh = ConvShape(dy.shape[0], h, wd, c, k, r, s, pad)
    dx = torch.empty((sh.n, h, wd, c), dtype=out_dtype or dy.dtype, device=dy.device)
    mdnn_conv2d_bwd_data(sh, dy, w, dtype_of(dy), mask, dx, dtype_of(dx), stream)
    return dx


@_on_its_stream
def conv2d_bwd_filter(x, dy, r: int, s: int, pad: int, with_db: bool = True, stream=None):
    import torch
    n, h, wd, c = x.shape
    k = dy.shape[3]
    sh = ConvShape(n, h, wd, c, k, r, s, pad)
    dw = torch.empty((k, r, s, c), dtype=torch.float32, device=x.device)
    db = torch.empty((k,), dtype=torch.float32, device=x.device) if with_db else None
    ws_bytes = mdnn_conv2d_bwd_filter_workspace(sh, dtype_of(x))
    ws = torch.empty((max(ws_bytes, 16),), dtype=torch.uint8, device=x.device)
    mdnn_conv2d_bwd_filter(sh, x, dy, dtype_of(x), dw, db, ws, ws_bytes, stream)
    return dw, db


def _rows_of(t, name: str):
    """(rows, cols, leading dimension) of a 2-D device tensor whose rows are
    contiguous, on the current device (whose stream the call runs on)."""
    import torch
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name} must be 2-D with contiguous rows")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is not on the current GPU")
    rows, cols = t.shape
    return rows, cols, max(t.stride(0), cols) if rows <= 1 else t.stride(0)


def _vector_of(t, n: int, name: str):
    """A contiguous fp32 vector of n elements on the current device."""
    import torch
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} contiguous fp32 values")
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is not on the current GPU")
    return t


def _like(t, x, name: str):
    """(tensor, leading dimension) of an operand with x's shape and type."""
    if t is None:
        return None, x.shape[1]
    if t.shape != x.shape or t.dtype != x.dtype:
        raise ValueError(f"{name} must have the shape and type of the first operand")
    return t, _rows_of(t, name)[2]


def _codes_like(q, rows: int, cols: int, device):
    """Room for [rows, cols] codes; allocated rows start on 128 bytes (a cache line)."""
    import torch
    if q is None:
        q = torch.empty((rows, (cols + 127) // 128 * 128), dtype=torch.int8, device=device)[:, :cols]
    elif q.dtype != torch.int8 or tuple(q.shape) != (rows, cols):
        raise ValueError(f"q must be int8 [{rows}, {cols}]")
    return q, _rows_of(q, "q")[2]


def _bytes_of(ws):
    """(tensor, bytes) of an optional workspace on the current device."""
    import torch
    if ws is None:
        return None, 0
    if ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device.index != torch.cuda.current_device():
        raise ValueError("workspace must be contiguous bytes on the current GPU")
    return ws, ws.numel()


@_on_its_stream
def quantize_i8(x, transpose: bool = False, q=None, scale=None, workspace=None, stream=None):
    """(codes, scales) of a 2-D tensor: int8 codes with an fp32 scale for each
    row, or with transpose for each column, the codes stored [cols, rows] (a
    layer's weights W[in, out] as gemm_i8's operand B)."""
    import torch
    rows, cols, ldx = _rows_of(x, "x")
    n = cols if transpose else rows
    q, ldq = _codes_like(q, n, rows if transpose else cols, x.device)
    scale = torch.empty((n,), dtype=torch.float32, device=x.device) if scale is None else _vector_of(scale, n, "scale")
    if not transpose:
        mdnn_quantize_i8(rows, cols, x, ldx, dtype_of(x), q, ldq, scale, stream)
        return q, scale
    if workspace is None:
        need = mdnn_quantize_i8_t_workspace(rows, cols)
        workspace = torch.empty((max(need, 16),), dtype=torch.uint8, device=x.device)
    mdnn_quantize_i8_t(rows, cols, x, ldx, dtype_of(x), q, ldq, scale, *_bytes_of(workspace), stream)
    return q, scale


@_on_its_stream
def gemm_i8(A, a_scale, B, b_scale, bias=None, act: int = ACT_NONE, out_dtype=None, out=None, workspace=None,
            stream=None):
    """D = act((A B^T) * a_scale[:, None] * b_scale + bias) of int8 codes A [M, K],
    B [N, K].  workspace: None, True (allocate what mdnn_gemm_i8_workspace
    asks for) or a device byte tensor."""
    import torch
    M, K, lda = _rows_of(A, "A")
    N, KB, ldb = _rows_of(B, "B")
    if A.dtype != torch.int8 or B.dtype != torch.int8 or KB != K:
        raise ValueError("A and B must be int8 codes of one depth")
    _vector_of(a_scale, M, "a_scale"), _vector_of(b_scale, N, "b_scale"), _vector_of(bias, N, "bias")
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype or torch.float32, device=A.device)
    elif tuple(out.shape) != (M, N):
        raise ValueError(f"out must be [{M}, {N}]")
    if workspace is True:
        workspace = torch.empty((max(mdnn_gemm_i8_workspace(M, N, K), 16),), dtype=torch.uint8, device=A.device)
    mdnn_gemm_i8(M, N, K, A, lda, a_scale, B, ldb, b_scale, bias, act, out, _rows_of(out, "out")[2], dtype_of(out),
                 *_bytes_of(workspace), stream)
    return out


@_on_its_stream
def rmsnorm(x, gamma=None, residual=None, eps: float = 1e-6, h_out=None, out=None, stream=None):
    """y = h * gamma / sqrt(mean(h^2) + eps) of the rows of h = x + residual.
    Returns y, or (y, h) with a residual (h_out is allocated then)."""
    import torch
    rows, cols, ldx = _rows_of(x, "x")
    residual, ldr = _like(residual, x, "residual")
    if residual is not None and h_out is None:
        h_out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    h_out, ldh = _like(h_out, x, "h_out")
    out, ldy = _like(torch.empty((rows, cols), dtype=x.dtype, device=x.device) if out is None else out, x, "out")
    mdnn_rmsnorm_fwd(rows, cols, x, ldx, residual, ldr, _vector_of(gamma, cols, "gamma"), eps, h_out, ldh, out, ldy,
                     dtype_of(x), stream)
    return (out, h_out) if h_out is not None else out


@_on_its_stream
def rmsnorm_i8(x, gamma=None, residual=None, eps: float = 1e-6, h_out=None, q=None, scale=None, stream=None):
    """rmsnorm with its result as int8 codes and an fp32 scale for each row.
    Returns (q, scale), or (q, scale, h) with a residual."""
    import torch
    rows, cols, ldx = _rows_of(x, "x")
    residual, ldr = _like(residual, x, "residual")
    if residual is not None and h_out is None:
        h_out = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
    h_out, ldh = _like(h_out, x, "h_out")
    q, ldq = _codes_like(q, rows, cols, x.device)
    scale = (torch.empty((rows,), dtype=torch.float32, device=x.device) if scale is None
             else _vector_of(scale, rows, "scale"))
    mdnn_rmsnorm_i8_fwd(rows, cols, x, ldx, residual, ldr, _vector_of(gamma, cols, "gamma"), eps, h_out, ldh, q, ldq,
                        scale, dtype_of(x), stream)
    return (q, scale, h_out) if h_out is not None else (q, scale)


@_on_its_stream
def rmsnorm_bwd(dy, h, gamma=None, eps: float = 1e-6, dres=None, dx=None, with_dgamma: bool = True, dgamma=None,
                workspace=None, stream=None):
    """(dx, dgamma) of rmsnorm at the stored h; dres is the gradient that
    reaches h along the residual.  dgamma is None without with_dgamma."""
    import torch
    rows, cols, lddy = _rows_of(dy, "dy")
    if h is None:
        raise ValueError("h is required")
    h, ldh = _like(h, dy, "h")
    dres, lddr = _like(dres, dy, "dres")
    dx, lddx = _like(torch.empty((rows, cols), dtype=dy.dtype, device=dy.device) if dx is None else dx, dy, "dx")
    if not with_dgamma:
        dgamma = None
    elif dgamma is None:
        dgamma = torch.empty((cols,), dtype=torch.float32, device=dy.device)
    else:
        _vector_of(dgamma, cols, "dgamma")
    if with_dgamma and workspace is None:
        need = mdnn_rmsnorm_bwd_workspace(rows, cols)
        workspace = torch.empty((max(need, 256),), dtype=torch.uint8, device=dy.device)
    mdnn_rmsnorm_bwd(rows, cols, dy, lddy, h, ldh, _vector_of(gamma, cols, "gamma"), eps, dres, lddr, dx, lddx, dgamma,
                     dtype_of(dy), *_bytes_of(workspace), stream)
    return dx, dgamma


def make_scaler(scale: float, growth_interval: int = 2000, growth: float = 2.0,
                backoff: float = 0.5, min_scale: float = 1.0, device="cuda"):
    """A device copy of an mdnn_scaler_t (32 bytes)."""
    import torch
    s = Scaler(scale, 0, 0, growth_interval, growth, backoff, min_scale, 0)
    raw = bytes(memoryview(s))
    return torch.frombuffer(bytearray(raw), dtype=torch.uint8).to(device)


def read_scaler(t) -> dict:
    raw = bytes(t.cpu().numpy().tobytes())
    s = Scaler.from_buffer_copy(raw)
    return {f: getattr(s, f) for f, _ in Scaler._fields_}


class Net:
    """A bound train-step handle: parameter, gradient, momentum, low-precision
    and workspace buffers are torch allocations owned by this object."""

    def __init__(self, layers, batch: int, dtype: int, loss: int, lr: float,
                 momentum: float = 0.0, loss_scaling: bool = False, init_scale: float = 1.0,
                 n_classes: int = 10, device="cuda", shared_master=None, fuse_update: bool = False):
        """shared_master: another Net's `master` tensor to bind instead of a
        private one (asynchronous workers; step with step_async only).
        fuse_update: the train config's fuse_update (eligible FC layers
        updated inside their weight-gradient products)."""
        import torch
        descs = [LayerDesc(l.kind, l.act, l.c_in, l.h, l.w, l.c_out, l.r, l.s, l.pad) for l in layers]
        self.cfg = TrainCfg(dtype, loss, lr, momentum, 1 if loss_scaling else 0,
                            n_classes if loss == LOSS_XENT else 0, 1 if fuse_update else 0)
        self.handle = mdnn_net_create(descs, batch, self.cfg)
        self.batch = batch
        self.dtype = dtype
        self.n_params, self.ws_bytes = mdnn_net_sizes(self.handle)
        dev = torch.device(device)
        if shared_master is not None:
            if shared_master.numel() != self.n_params or shared_master.dtype != torch.float32:
                raise ValueError("shared_master must be fp32 with this net's parameter count")
            self.master = shared_master
        else:
            self.master = torch.zeros(self.n_params, dtype=torch.float32, device=dev)
        self.grads = torch.zeros(self.n_params, dtype=torch.float32, device=dev)
        self.mom = torch.zeros(self.n_params, dtype=torch.float32, device=dev) if momentum else None
        self.lowp = (torch.zeros(self.n_params, dtype=torch_dtype(dtype), device=dev)
                     if dtype != F32 else None)
        self.ws = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=dev)
        self.scaler = make_scaler(init_scale, device=dev) if loss_scaling else None
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        mdnn_net_bind(self.handle, self.master, self.grads, self.mom, self.lowp, self.ws,
                      self.ws.numel(), self.scaler)

    def set_params(self, params, stream=None):
        """Copy fp32 master parameters (any array-like) and derive the
        low-precision working copy."""
        import torch
        self.master.copy_(torch.as_tensor(params, dtype=torch.float32))
        mdnn_net_sync_lowp(self.handle, stream)

    def step(self, x, target, loss_out=None, stream=None):
        out = self.loss if loss_out is None else loss_out
        mdnn_train_step(self.handle, x, target, out, stream)
        return out

    def record_step(self, x, target, loss_out=None) -> "StepGraph":
        """Record one step on these exact buffers into a HIP graph (see
        mdnn_train_graph_create); replay it with .launch()."""
        out = self.loss if loss_out is None else loss_out
        return StepGraph(mdnn_train_graph_create(self.handle, x, target, out), (self, x, target, out))

    def step_async(self, x, target, loss_out=None, stream=None):
        """Asynchronous step (section 3.1) on a master vector shared with other
        workers: see mdnn_train_step_async."""
        out = self.loss if loss_out is None else loss_out
        mdnn_train_step_async(self.handle, x, target, out, stream)
        return out

    def activation_ptr(self, i: int) -> Optional[int]:
        return mdnn_net_activation(self.handle, i)

    def output_grad_ptr(self, which: int) -> Optional[int]:
        return mdnn_net_output_grad(self.handle, which)

    def close(self):
        if getattr(self, "handle", None):
            mdnn_net_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class StepGraph:
    """A recorded train step.  Holds references to the net and the buffers
    the graph reads and writes, so they outlive it."""

    def __init__(self, handle: int, keep):
        self.handle = handle
        self._keep = keep

    def launch(self, stream=None):
        mdnn_graph_launch(self.handle, stream)

    def close(self):
        if getattr(self, "handle", None):
            mdnn_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
