"""Cases by which the 8-bit product, its quantisers and the root-mean-square norm are measured.

Each case is one pass through one operator:

  gemm      D = act(a_scale[m] * b_scale[n] * sum_k A[m, k] B[n, k] + bias[n]) of 8-bit integer codes: a trained fully
            connected layer in serving, for one sample up to large batches (``mdnn_gemm_i8``);
  norm      h = x + residual, y = gamma * h / sqrt(mean(h^2) + eps), with y in the inputs' type
            (``mdnn_rmsnorm_fwd``) or as 8-bit codes with a scale for each row, the next product's
            operand (``mdnn_rmsnorm_i8_fwd``);
  norm_bwd  the norm's gradients: with respect to h (plus the gradient that arrives along the residual) and to gamma
            (``mdnn_rmsnorm_bwd``);
  quant     8-bit codes with a scale for each row (activations) or for each column, stored transposed (a
            layer's weights [in, out], laid out for the product) (``mdnn_quantize_i8``, ``mdnn_quantize_i8_t``).

Codes are whole numbers -127..127 and part of the operators' definition down to the rounding: with a = max|t| over the
row (at least 2^-100), the code of t is fl32(t * fl32(127 / a)) rounded to the nearest whole number, ties to even,
and the scale is fl32(a / 127).  For the norm t is fl32(h * gamma), h = fl32(x + residual): the row's
1 / rms is common to all its elements, so it belongs to the scale alone.  Codes therefore depend on no order of
summation and are returned as the whole numbers they are, beside the fp32 scales.

``listed`` covers the smallest calls (one row), ordinary and the largest ones, with sizes that are multiples of the
tiles and sizes that are not; ``draw`` takes sizes from the same ranges.
"""
import math

import torch

own = False

DEV = "cuda"
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CODE = {"f32": 0, "f16": 1, "bf16": 2}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
A_MIN = 2.0 ** -100


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _gemm(name, m, n, k, out, act=True, bias=True, padded=True):
    return {"name": name, "kind": "gemm", "m": m, "n": n, "k": k, "out": out, "act": act, "bias": bias,
            "padded": padded}


def _norm(name, rows, cols, dtype, i8, residual=True):
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "i8": i8, "residual": residual}


def _bwd(name, rows, cols, dtype, residual=True):
    return {"name": name, "kind": "norm_bwd", "rows": rows, "cols": cols, "dtype": dtype, "residual": residual}


def _quant(name, rows, cols, dtype, by):
    return {"name": name, "kind": "quant", "rows": rows, "cols": cols, "dtype": dtype, "by": by}


def listed():
    return [
        # one sample through a hidden layer of the wide network: the weights' read is all there is
        _gemm("gemm_i8_m1_4096x4096", 1, 4096, 4096, "f16"),
        # a few dozen requests gathered into one call, a wider layer
        _gemm("gemm_i8_m40_8192x4096", 40, 8192, 4096, "bf16", act=False),
        # sizes that divide by nothing, rows packed without padding, an fp32 output layer
        _gemm("gemm_i8_m1000_777x1531_packed", 1000, 777, 1531, "f32", act=False, padded=False),
        # the wide network's hidden layer at its training batch
        _gemm("gemm_i8_m4096_4096x4096", 4096, 4096, 4096, "f16"),
        # offline scoring of a large batch, the largest product
        _gemm("gemm_i8_m16384_8192x8192", 16384, 8192, 8192, "bf16", bias=False),
        # one sample between two layers: latency
        _norm("norm_i8_1x4096", 1, 4096, "f16", True),
        # the training batch's rows handed to an 8-bit layer
        _norm("norm_i8_4096x4096", 4096, 4096, "bf16", True),
        # a training step's forward norm of a large batch
        _norm("norm_16384x8192", 16384, 8192, "bf16", False),
        # its gradient at the wide network's batch
        _bwd("norm_bwd_4096x4096", 4096, 4096, "f16"),
        # a last batch of odd size in full precision
        _bwd("norm_bwd_1000x1531", 1000, 1531, "f32"),
        # an activation of odd width between two 8-bit layers
        _quant("quant_rows_1000x1531", 1000, 1531, "f16", "rows"),
        # a trained layer's fp32 master weights, once per layer at deployment
        _quant("quant_channels_4096x4096", 4096, 4096, "f32", "channels"),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is spread evenly; half of them multiples of a power of two (as sizes mostly are)."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        q = 8 if v < 128 else 64
        v = max(q, v // q * q) if v >= q else v
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "norm", "norm", "norm_bwd", "norm_bwd", "quant", "quant"])
    if kind == "gemm":
        while True:
            c = _gemm("", _log(rng, 1, 16384), _log(rng, 16, 8192), _log(rng, 32, 8192),
                      rng.choice(["f32", "f16", "bf16"]), rng.random() < 0.5, rng.random() < 0.7, rng.random() < 0.75)
            if c["m"] * c["n"] * c["k"] <= 1 << 38:
                break
    else:
        dtype = rng.choice(["f32", "f16", "bf16"])
        most = 1 << 26 if dtype == "f32" else 1 << 27
        while True:
            rows, cols = _log(rng, 1, 65536), _log(rng, 32, 16384)
            if rows * cols <= most:
                break
        if kind == "norm":
            c = _norm("", rows, cols, dtype, rng.random() < 0.5, rng.random() < 0.7)
        elif kind == "norm_bwd":
            c = _bwd("", rows, cols, dtype, rng.random() < 0.7)
        else:
            c = _quant("", min(rows, 16384), cols, dtype, rng.choice(["rows", "channels"]))
    c.pop("name")
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

class _Rng:
    """Draws on the GPU, from the seed alone."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, scale=1.0, dtype="f32"):
        return (torch.randn(shape, generator=self.g, device=DEV) * scale).to(TORCH[dtype])

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def stream(self, rows, cols, dtype):
        """Activations along a residual: a spread of magnitudes over the rows, a few columns much larger than the
        rest, and about one row in 64 that is padding (zeros)."""
        x = torch.randn((rows, cols), generator=self.g, device=DEV)
        x *= torch.exp(torch.randn((rows, 1), generator=self.g, device=DEV))
        x *= torch.where(self.uniform(1, cols) < 0.005, 20.0, 1.0)
        if rows > 1:
            x *= (self.uniform(rows, 1) >= 1.0 / 64).float()
        return x.to(TORCH[dtype])


def _codes(g, rows, cols, padded, heavy):
    """Codes as the quantiser leaves them (normal data, or a ReLU's with half of it zero) and their scales."""
    width = (cols + 15) // 16 * 16 if padded else cols
    q = torch.empty((rows, width), dtype=torch.int8, device=DEV)
    x = torch.randn((rows, width), generator=g.g, device=DEV)
    if heavy:
        x = x.clamp_(min=0)
    a = x[:, :cols].abs().amax(1, keepdim=True).clamp_(min=1e-3)
    q.copy_((x * (127.0 / a)).round_().clamp_(-127, 127))
    return q[:, :cols], (a[:, 0] / 127.0).contiguous()


def prepare(case, seed):
    kind, g = case["kind"], _Rng(seed)
    s = {"case": case}
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["a_scale"] = _codes(g, m, k, case["padded"], True)
        s["b"], s["b_scale"] = _codes(g, n, k, case["padded"], False)
        s["b_scale"] *= math.sqrt(2.0 / k)
        s["bias"] = g.normal(n, scale=0.1) if case["bias"] else None
        s["d"] = torch.empty((m, n), dtype=TORCH[case["out"]], device=DEV)
        return s
    rows, cols, dt = case["rows"], case["cols"], case["dtype"]
    if kind == "quant":
        if case["by"] == "rows":
            s["x"] = g.stream(rows, cols, dt)
            s["q"] = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=DEV)[:, :cols]
        else:
            s["x"] = g.normal(rows, cols, scale=math.sqrt(2.0 / rows), dtype=dt)
            s["q"] = torch.empty((cols, (rows + 15) // 16 * 16), dtype=torch.int8, device=DEV)[:, :rows]
        s["scale"] = torch.empty(s["q"].shape[0], device=DEV)
        return s
    s["gamma"] = 1.0 + g.normal(cols, scale=0.1)
    if kind == "norm":
        s["x"] = g.normal(rows, cols, dtype=dt) if case["residual"] else g.stream(rows, cols, dt)
        if case["residual"]:
            s["res"] = g.stream(rows, cols, dt)
            s["h"] = torch.empty_like(s["x"])
        if case["i8"]:
            s["q"] = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=DEV)[:, :cols]
            s["scale"] = torch.empty(rows, device=DEV)
        else:
            s["y"] = torch.empty_like(s["x"])
        return s
    s["h"] = g.stream(rows, cols, dt)
    s["dy"] = g.normal(rows, cols, dtype=dt)
    s["dres"] = g.normal(rows, cols, dtype=dt) if case["residual"] else None
    s["dx"] = torch.empty_like(s["dy"])
    s["dgamma"] = torch.empty(cols, device=DEV)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _workspace(s, nbytes):
    """Scratch memory kept with the state, as a program keeps it with its layer."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _run_own(s):
    import paper_2011_11188_amd as mdnn
    case = s["case"]
    kind = case["kind"]
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_gemm_i8_workspace(m, n, k))
        mdnn.mdnn_gemm_i8(m, n, k, s["a"], s["a"].stride(0), s["a_scale"], s["b"], s["b"].stride(0), s["b_scale"],
                          s["bias"], mdnn.ACT_RELU if case["act"] else mdnn.ACT_NONE, s["d"], n, CODE[case["out"]],
                          ws, ws.numel())
        return s["d"]
    rows, cols, code = case["rows"], case["cols"], CODE[case["dtype"]]
    if kind == "quant":
        if case["by"] == "rows":
            mdnn.mdnn_quantize_i8(rows, cols, s["x"], cols, code, s["q"], s["q"].stride(0), s["scale"])
        else:
            ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_quantize_i8_t_workspace(rows, cols))
            mdnn.mdnn_quantize_i8_t(rows, cols, s["x"], cols, code, s["q"], s["q"].stride(0), s["scale"], ws,
                                    ws.numel())
        return {"q": s["q"], "scale": s["scale"]}
    if kind == "norm":
        out = {"h": s["h"]} if case["residual"] else {}
        if case["i8"]:
            mdnn.mdnn_rmsnorm_i8_fwd(rows, cols, s["x"], cols, s.get("res"), cols, s["gamma"], EPS, s.get("h"), cols,
                                     s["q"], s["q"].stride(0), s["scale"], code)
            out.update(q=s["q"], scale=s["scale"])
        else:
            mdnn.mdnn_rmsnorm_fwd(rows, cols, s["x"], cols, s.get("res"), cols, s["gamma"], EPS, s.get("h"), cols,
                                  s["y"], cols, code)
            out["y"] = s["y"]
        return out
    ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_rmsnorm_bwd_workspace(rows, cols))
    mdnn.mdnn_rmsnorm_bwd(rows, cols, s["dy"], cols, s["h"], cols, s["gamma"], EPS, s["dres"], cols, s["dx"], cols,
                          s["dgamma"], code, ws, ws.numel())
    return {"dx": s["dx"], "dgamma": s["dgamma"]}


def _quantize(t):
    """Codes and scales of the rows of an fp32 t; the two quotients of a row are rounded once (from 64 bits)."""
    a = t.abs().amax(1, keepdim=True).clamp(min=A_MIN).double()
    inv = (torch.full_like(a, 127.0) / a).float()
    return (t * inv).round().to(torch.int8), (a / torch.full_like(a, 127.0)).float()[:, 0]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "gemm":
        d = torch.matmul(s["a"].float(), s["b"].float().t())
        d = d * s["a_scale"][:, None] * s["b_scale"]
        if case["bias"]:
            d = d + s["bias"]
        if case["act"]:
            d = d.clamp(min=0)
        return d.to(TORCH[case["out"]])
    dt = TORCH[case["dtype"]]
    if kind == "quant":
        x = s["x"].float()
        q, scale = _quantize(x if case["by"] == "rows" else x.t().contiguous())
        return {"q": q, "scale": scale}
    if kind == "norm":
        h = s["x"].float()
        out = {}
        if case["residual"]:
            h = h + s["res"].float()
            out["h"] = h.to(dt)
        rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        if case["i8"]:
            q, scale = _quantize(h * s["gamma"])
            out.update(q=q, scale=scale * rstd[:, 0])
        else:
            out["y"] = (h * rstd * s["gamma"]).to(dt)
        return out
    h, dy = s["h"].float(), s["dy"].float()
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    xh, g = h * rstd, dy * s["gamma"]
    dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True))
    if case["residual"]:
        dx = dx + s["dres"].float()
    return {"dx": dx.to(dt), "dgamma": (dy * xh).sum(0)}


def run(s):
    if own:
        return _run_own(s)
    return _run_plain(s)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + m * n * BYTES[case["out"]] + 4 * (m + n + (n if case["bias"] else 0)),
                "flops": 2 * m * n * k}
    rows, cols, es = case["rows"], case["cols"], BYTES[case["dtype"]]
    e = rows * cols
    if kind == "quant":
        return {"bytes": e * (es + 1) + 4 * (rows if case["by"] == "rows" else cols), "flops": 3 * e}
    if kind == "norm":
        b = e * es * (3 if case["residual"] else 1) + 4 * cols
        return {"bytes": b + (e + 4 * rows if case["i8"] else e * es), "flops": (6 if case["i8"] else 5) * e}
    return {"bytes": e * es * (4 if case["residual"] else 3) + 8 * cols, "flops": 10 * e}


# --------------------------------------------------------------------------
# the same results in 64 bits
# --------------------------------------------------------------------------

def _f32(v):
    """A value of the definition that is rounded to 32 bits."""
    return v.to(torch.float32).to(torch.float64)


def _exact_codes(t):
    top = torch.clamp(torch.max(torch.abs(t), dim=1).values, min=A_MIN)
    steps = _f32(torch.div(torch.full_like(top, 127.0), top))
    return torch.round(_f32(t * steps.unsqueeze(1))).to(torch.int8), _f32(torch.div(top, torch.full_like(top, 127.0)))


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "gemm":
        acc = s["a"].to(torch.float64) @ s["b"].to(torch.float64).T
        acc.mul_(s["a_scale"].to(torch.float64).unsqueeze(1)).mul_(s["b_scale"].to(torch.float64).unsqueeze(0))
        if s["bias"] is not None:
            acc.add_(s["bias"].to(torch.float64).unsqueeze(0))
        return torch.where(acc < 0, torch.zeros_like(acc), acc) if case["act"] else acc
    if kind == "quant":
        x = s["x"].to(torch.float64)
        codes, scale = _exact_codes(x if case["by"] == "rows" else x.T)
        return {"q": codes, "scale": scale}
    gamma = s["gamma"].to(torch.float64).unsqueeze(0)
    cols = case["cols"]
    if kind == "norm":
        h = s["x"].to(torch.float64)
        out = {}
        if case["residual"]:
            h = h + s["res"].to(torch.float64)
            out["h"] = h
        rms = torch.sqrt(torch.sum(h.square(), dim=1) / cols + EPS)
        if case["i8"]:
            codes, scale = _exact_codes(_f32(_f32(h) * gamma))
            out["q"], out["scale"] = codes, scale / rms
        else:
            out["y"] = gamma * h / rms.unsqueeze(1)
        return out
    # y_c = gamma_c h_c / r with r = sqrt(sum h^2 / n + eps): dy_c / dh_j = gamma_c ([c = j] / r - h_c h_j / (n r^3))
    h, dy = s["h"].to(torch.float64), s["dy"].to(torch.float64)
    r = torch.sqrt(torch.sum(h.square(), dim=1, keepdim=True) / cols + EPS)
    along = torch.sum(dy * gamma * h, dim=1, keepdim=True)
    dx = dy * gamma / r - h * along / (cols * r.pow(3))
    if s["dres"] is not None:
        dx += s["dres"].to(torch.float64)
    return {"dx": dx, "dgamma": torch.sum(dy * h / r, dim=0)}
