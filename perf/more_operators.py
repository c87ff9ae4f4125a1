"""Cases by which dropout, layer norm and the last layer with its cross entropy are measured.

Each case is one pass through one operator:

  dropout      y = residual + keep * s * x, forward, or dx = keep * s * dy, backward (``mdnn_dropout_fwd``,
               ``mdnn_dropout_bwd``).  keep comes from a counter-based generator and is never stored: element (r, c) is
               dropped where its 16 bits are below t = floor(p * 2^16 + 1/2), and s = 2^16 / (2^16 - t).  The bits are
               those of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
               1, 2, 3", 2011) under the key `seed` (64 bits) at the counter (c / 8, r, step, site): 128 bits for eight
               columns, the lowest 16 bits of the first word first;
  norm         h = residual + dropout(x), y = gamma * (h - mean(h)) / sqrt(var(h) + eps) + beta
               (``mdnn_layernorm_fwd``);
  norm_bwd     its gradients with respect to h (plus the one that arrives along the residual), x, gamma and beta
               (``mdnn_layernorm_bwd``);
  xent         a last layer z = x W + bias of many classes and its cross entropy: lse_i = log sum_j exp(z_ij),
               loss_i = lse_i - z_i,label(i), their mean over the rows whose label is not the ignored one
               (``mdnn_linear_xent_fwd``);
  xent_bwd     the mean's gradients, times a loss scale, with respect to x, W and bias, from x, W and lse
               (``mdnn_linear_xent_bwd``).

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
EPS = 1e-5
SITE = 3
IGNORED = -1


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def _drop(name, rows, cols, dtype, p, residual=True, backward=False):
    return {"name": name, "kind": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "p": p,
            "residual": residual and not backward, "backward": backward}


def _norm(name, rows, cols, dtype, p, residual=True):
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _bwd(name, rows, cols, dtype, p, residual=True):
    return {"name": name, "kind": "norm_bwd", "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def _xent(name, m, n, k, dtype, by_class, bias=False, backward=False):
    return {"name": name, "kind": "xent_bwd" if backward else "xent", "m": m, "n": n, "k": k, "dtype": dtype,
            "by_class": by_class, "bias": bias}


def listed():
    return [
        # a small network's hidden activations: latency
        _drop("dropout_64x1024_f32", 64, 1024, "f32", 0.5, residual=False),
        # a large batch's block output on its way into the residual stream
        _drop("dropout_16384x8192_bf16", 16384, 8192, "bf16", 0.1),
        # the gradient of a last batch of odd size
        _drop("dropout_bwd_9999x1531_f16", 9999, 1531, "f16", 0.25, backward=True),
        # one sample between two layers in serving: latency
        _norm("norm_1x4096_f16", 1, 4096, "f16", 0.0),
        # a training step's dropout, residual and norm of a large batch
        _norm("norm_16384x8192_bf16_drop", 16384, 8192, "bf16", 0.1),
        # its gradients at the wide network's batch
        _bwd("norm_bwd_4096x4096_bf16_drop", 4096, 4096, "bf16", 0.1),
        # a last batch of odd size in full precision
        _bwd("norm_bwd_1000x1531_f32", 1000, 1531, "f32", 0.0),
        # one sample's loss under a trained layer: the weights' read is all there is
        _xent("xent_1x32768x4096_f16", 1, 32768, 4096, "f16", False),
        # sizes that divide by nothing in full precision
        _xent("xent_500x10007x777_f32", 500, 10007, 777, "f32", False, bias=True),
        # the loss of a large batch over a large vocabulary, its table stored by classes; the largest
        _xent("xent_8192x131072x4096_bf16", 8192, 131072, 4096, "bf16", True),
        # a training step's last layer
        _xent("xent_bwd_4096x32768x4096_bf16", 4096, 32768, 4096, "bf16", True, backward=True),
        # a small batch, odd sizes, a layer of this library's own form with its bias
        _xent("xent_bwd_1000x5003x1000_f16", 1000, 5003, 1000, "f16", False, bias=True, backward=True),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is spread evenly; half of them multiples of a power of two (as sizes mostly are)."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        q = 8 if v < 128 else 64
        v = max(q, v // q * q) if v >= q else v
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm", "norm_bwd", "norm_bwd", "xent", "xent", "xent_bwd", "xent_bwd"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind.startswith("xent"):
        back = kind == "xent_bwd"
        most = 1 << (34 if dtype == "f32" else 40 if back else 42)
        while True:
            m, n, k = _log(rng, 1, 16384), _log(rng, 1024, 131072), _log(rng, 32, 8192)
            if m * n * k <= most and m * n <= 1 << 30 and n * k <= 1 << 29:
                break
        c = _xent("", m, n, k, dtype, rng.random() < 0.5, rng.random() < 0.3, back)
    else:
        most = 1 << 26 if dtype == "f32" else 1 << 27
        while True:
            rows, cols = _log(rng, 1, 65536), _log(rng, 32, 16384)
            if rows * cols <= most:
                break
        if kind == "dropout":
            c = _drop("", rows, cols, dtype, rng.choice([0.05, 0.1, 0.25, 0.5]), rng.random() < 0.7, rng.random() < 0.4)
        else:
            make = _norm if kind == "norm" else _bwd
            c = make("", rows, cols, dtype, rng.choice([0.0, 0.0, 0.1, 0.3]), rng.random() < 0.7)
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
        """Activations along a residual: a spread of magnitudes over the rows, an offset of its own in each, a few
        columns much larger than the rest, and about one row in 64 that is padding (zeros)."""
        x = torch.randn((rows, cols), generator=self.g, device=DEV) + self.normal(rows, 1)
        x *= torch.exp(torch.randn((rows, 1), generator=self.g, device=DEV))
        x *= torch.where(self.uniform(1, cols) < 0.005, 20.0, 1.0)
        if rows > 1:
            x *= (self.uniform(rows, 1) >= 1.0 / 64).float()
        return x.to(TORCH[dtype])

    def generator(self):
        """The state that dropout draws from: a seed of 64 bits and a step."""
        r = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=self.g, device=DEV)
        r[1] %= 100000
        return r


def prepare(case, seed):
    kind, g = case["kind"], _Rng(seed)
    s, dt = {"case": case}, case["dtype"]
    if kind in ("xent", "xent_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        s["w"] = g.normal(*((n, k) if case["by_class"] else (k, n)), scale=2.0 / math.sqrt(k), dtype=dt)
        s["bias"] = g.normal(n, scale=0.5) if case["bias"] else None
        labels = (g.uniform(m) * n).to(torch.int32).clamp_(max=n - 1)
        # rows that lean towards their label's weights, as a trained layer's inputs do
        lean = s["w"][labels.long()] if case["by_class"] else s["w"][:, labels.long()].t()
        s["x"] = (torch.randn((m, k), generator=g.g, device=DEV) + g.uniform(m, 1) * lean.float()).to(TORCH[dt])
        if m > 1:
            labels[g.uniform(m) < 0.05] = IGNORED  # padding
        s["labels"] = labels
        s["lse"] = torch.empty(m, device=DEV)
        if kind == "xent":
            s["loss"], s["row_loss"] = torch.empty(1, device=DEV), torch.empty(m, device=DEV)
            return s
        w = s["w"].float().t().contiguous() if case["by_class"] else s["w"].float()
        for r in range(0, m, 1024):  # (what the forward pass left)
            z = torch.matmul(s["x"][r:r + 1024].float(), w)
            s["lse"][r:r + 1024] = torch.logsumexp(z if s["bias"] is None else z + s["bias"], 1)
        s["scale"] = torch.full((1,), 65536.0, device=DEV) if dt == "f16" else None
        s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        s["db"] = torch.empty(n, device=DEV) if case["bias"] else None
        return s
    rows, cols = case["rows"], case["cols"]
    s["rng"] = g.generator() if case["p"] > 0 else None
    if kind == "dropout":
        s["x"] = g.normal(rows, cols, dtype=dt)
        s["res"] = g.stream(rows, cols, dt) if case["residual"] else None
        s["y"] = torch.empty_like(s["x"])
        return s
    s["gamma"], s["beta"] = 1.0 + g.normal(cols, scale=0.1), g.normal(cols, scale=0.1)
    if kind == "norm":
        s["x"] = g.normal(rows, cols, dtype=dt) if case["residual"] else g.stream(rows, cols, dt)
        s["res"] = g.stream(rows, cols, dt) if case["residual"] else None
        s["h"] = torch.empty_like(s["x"]) if case["residual"] or case["p"] > 0 else None
        s["y"] = torch.empty_like(s["x"])
        return s
    s["h"] = g.stream(rows, cols, dt)
    s["dy"] = g.normal(rows, cols, dtype=dt)
    s["dres"] = g.normal(rows, cols, dtype=dt) if case["residual"] else None
    s["dx"] = torch.empty_like(s["dy"])
    s["dh"] = torch.empty_like(s["dy"]) if case["p"] > 0 else None
    s["dgamma"], s["dbeta"] = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
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
    kind, code = case["kind"], CODE[case["dtype"]]
    if kind in ("xent", "xent_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        layout, ldw = (mdnn.NT, k) if case["by_class"] else (mdnn.NN, n)
        if kind == "xent":
            ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_linear_xent_fwd_workspace(layout, m, n, k, code))
            mdnn.mdnn_linear_xent_fwd(layout, m, n, k, s["x"], k, s["w"], ldw, code, s["bias"], s["labels"], IGNORED,
                                      s["loss"], s["row_loss"], s["lse"], ws, ws.numel())
            return {"loss": s["loss"], "row_loss": s["row_loss"], "lse": s["lse"]}
        ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_linear_xent_bwd_workspace(layout, m, n, k, code))
        mdnn.mdnn_linear_xent_bwd(layout, m, n, k, s["x"], k, s["w"], ldw, code, s["bias"], s["labels"], IGNORED,
                                  s["lse"], s["scale"], s["dx"], k, s["dw"], ldw, code, s["db"], ws, ws.numel())
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    rows, cols, p, rng = case["rows"], case["cols"], case["p"], s["rng"]
    if kind == "dropout":
        if case["backward"]:
            mdnn.mdnn_dropout_bwd(rows, cols, s["x"], cols, p, rng, SITE, s["y"], cols, code)
        else:
            mdnn.mdnn_dropout_fwd(rows, cols, s["x"], cols, s["res"], cols, p, rng, SITE, s["y"], cols, code)
        return s["y"]
    if kind == "norm":
        mdnn.mdnn_layernorm_fwd(rows, cols, s["x"], cols, s["res"], cols, p, rng, SITE, s["gamma"], s["beta"], EPS,
                                s["h"], cols, s["y"], cols, code)
        return {"h": s["h"], "y": s["y"]}
    ws = s["ws"] if "ws" in s else _workspace(s, mdnn.mdnn_layernorm_bwd_workspace(rows, cols))
    mdnn.mdnn_layernorm_bwd(rows, cols, s["dy"], cols, s["h"], cols, s["gamma"], EPS, s["dres"], cols, p, rng, SITE,
                            s["dx"], cols, s["dh"], cols, s["dgamma"], s["dbeta"], code, ws, ws.numel())
    return {"dx": s["dx"], "dh": s["dh"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


LOW = 0xFFFFFFFF


def _bits(rng, rows, cols):
    """[rows, cols] of 16 bits each: Philox 4x32-10, the 32-bit words held in int64 (products wrap at 64 bits)."""
    a = torch.arange((cols + 7) // 8, device=DEV).expand(rows, -1)
    b = torch.arange(rows, device=DEV)[:, None].expand_as(a)
    c, d = (rng[1] & LOW).expand_as(a), torch.full_like(a, SITE)
    k0, k1 = rng[0] & LOW, (rng[0] >> 32) & LOW
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((v >> 32) & LOW) ^ b ^ k0, v & LOW, ((u >> 32) & LOW) ^ d ^ k1, u & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    w = torch.stack((a, b, c, d), -1)
    return torch.stack((w & 0xFFFF, w >> 16), -1).reshape(rows, -1)[:, :cols]


def _dropped(x, p, rng):
    """keep * s * x in 32 bits."""
    if p == 0.0:
        return x.float()
    t = int(math.floor(p * 65536 + 0.5))
    return torch.where(_bits(rng, *x.shape) >= t, x.float() * (65536.0 / (65536 - t)), 0.0)


def _logits(s):
    w = s["w"].float()
    z = torch.matmul(s["x"].float(), w.t() if s["case"]["by_class"] else w)
    return z if s["bias"] is None else z + s["bias"]


def _run_plain(s):
    case = s["case"]
    kind, dt = case["kind"], TORCH[case["dtype"]]
    if kind == "xent":
        z, counted = _logits(s), s["labels"] != IGNORED
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        at = s["labels"].clamp(min=0).long()[:, None]
        row = torch.where(counted, lse - torch.gather(z, 1, at)[:, 0], 0.0)
        return {"loss": (row.sum() / counted.sum().clamp(min=1)).reshape(1), "row_loss": row, "lse": lse}
    if kind == "xent_bwd":
        counted = s["labels"] != IGNORED
        g = torch.exp(_logits(s) - s["lse"][:, None])
        rows = torch.arange(case["m"], device=DEV)
        g[rows, s["labels"].clamp(min=0).long()] -= 1.0
        a = (1.0 if s["scale"] is None else s["scale"]) / counted.sum().clamp(min=1).float()
        g = torch.where(counted[:, None], g * a, 0.0)
        w, x = s["w"].float(), s["x"].float()
        dx = torch.matmul(g, w if case["by_class"] else w.t())
        dw = torch.matmul(g.t(), x) if case["by_class"] else torch.matmul(x.t(), g)
        return {"dx": dx.to(dt), "dw": dw.to(dt), "db": g.sum(0) if case["bias"] else None}
    p, rng = case["p"], s["rng"]
    if kind == "dropout":
        y = _dropped(s["x"], p, rng)
        return (y if s["res"] is None else y + s["res"].float()).to(dt)
    if kind == "norm":
        h = _dropped(s["x"], p, rng)
        if s["res"] is not None:
            h = h + s["res"].float()
        away = h - h.mean(1, keepdim=True)
        y = away / torch.sqrt((away * away).mean(1, keepdim=True) + EPS) * s["gamma"] + s["beta"]
        return {"h": None if s["h"] is None else h.to(dt), "y": y.to(dt)}
    h, dy = s["h"].float(), s["dy"].float()
    away = h - h.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((away * away).mean(1, keepdim=True) + EPS)
    xh, g = away * rstd, dy * s["gamma"]
    dh = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    if s["dres"] is not None:
        dh = dh + s["dres"].float()
    return {"dx": _dropped(dh, p, rng).to(dt), "dh": None if s["dh"] is None else dh.to(dt),
            "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def run(s):
    if own:
        return _run_own(s)
    return _run_plain(s)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind, es = case["kind"], BYTES[case["dtype"]]
    if kind in ("xent", "xent_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        read = (m * k + n * k) * es + 4 * m + (4 * n if case["bias"] else 0)
        if kind == "xent":
            return {"bytes": read + 8 * m + 4, "flops": 2 * m * n * k}
        # (the logits again, and a product for each of the two gradients)
        return {"bytes": 2 * read, "flops": 6 * m * n * k}
    e, cols = case["rows"] * case["cols"], case["cols"]
    if kind == "dropout":
        return {"bytes": e * es * (3 if case["residual"] else 2), "flops": 2 * e}
    if kind == "norm":
        stored = case["residual"] or case["p"] > 0
        return {"bytes": e * es * (2 + case["residual"] + stored) + 8 * cols, "flops": 9 * e}
    return {"bytes": e * es * (3 + case["residual"] + (case["p"] > 0)) + 12 * cols, "flops": 16 * e}


# --------------------------------------------------------------------------
# the same results in 64 bits
# --------------------------------------------------------------------------

def _product_words(x, m):
    """(high, low) 32-bit words of x * m, from products of 16-bit halves."""
    xl, xh, ml, mh = x % 65536, x // 65536, m % 65536, m // 65536
    low, mid = xl * ml, xl * mh + (xl * ml) // 65536
    mid2 = xh * ml + mid % 65536
    return xh * mh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536


def _exact_kept(case, s):
    """The factor of each element: 0 where it is dropped, 2^16 / (2^16 - t) elsewhere."""
    rows, cols = case["rows"], case["cols"]
    if s["rng"] is None:
        return torch.ones((rows, cols), dtype=torch.float64, device=DEV)
    seed, step = (int(v) % 2 ** 64 for v in s["rng"].tolist())
    blocks = -(-cols // 8)
    ctr = [torch.arange(blocks, device=DEV).repeat(rows), torch.arange(rows, device=DEV).repeat_interleave(blocks),
           torch.full((rows * blocks,), step % 2 ** 32, device=DEV), torch.full((rows * blocks,), SITE, device=DEV)]
    for r in range(10):
        k0 = (seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32
        k1 = (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = _product_words(ctr[0], 0xD2511F53)
        h1, l1 = _product_words(ctr[2], 0xCD9E8D57)
        ctr = [torch.bitwise_xor(torch.bitwise_xor(h1, ctr[1]), k0), l1,
               torch.bitwise_xor(torch.bitwise_xor(h0, ctr[3]), k1), l0]
    t = math.floor(case["p"] * 65536 + 0.5)
    out = torch.empty((rows, blocks, 8), dtype=torch.float64, device=DEV)
    for j in range(8):
        half = ctr[j // 2] // 65536 if j % 2 else ctr[j // 2] % 65536
        out[:, :, j] = (half >= t).to(torch.float64).reshape(rows, blocks)
    return out.reshape(rows, blocks * 8)[:, :cols] * (65536.0 / (65536.0 - t))


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    wide = lambda v: v.to(torch.float64)  # noqa: E731
    if kind in ("xent", "xent_bwd"):
        w = wide(s["w"]).T if case["by_class"] else wide(s["w"])  # [k, n]
        x, labels = wide(s["x"]), s["labels"].tolist()
        real = [i for i, c in enumerate(labels) if c != IGNORED]
        at, to = torch.tensor(real, device=DEV, dtype=torch.long), torch.tensor([labels[i] for i in real], device=DEV,
                                                                                dtype=torch.long)
        z = x @ w
        if s["bias"] is not None:
            z.add_(wide(s["bias"]).unsqueeze(0))
        if kind == "xent":
            lse = torch.logsumexp(z, dim=1)
            row = torch.zeros_like(lse)
            row[at] = lse[at] - z[at, to]
            return {"loss": (row.sum() / max(1, len(real))).reshape(1), "row_loss": row, "lse": lse}
        prob = z.sub_(wide(s["lse"]).unsqueeze(1)).exp_()
        onehot_rows = torch.ones(len(real), dtype=torch.float64, device=DEV)
        prob.index_put_((at, to), -onehot_rows, accumulate=True)
        weight = torch.zeros((case["m"], 1), dtype=torch.float64, device=DEV)
        weight[at] = (1.0 if s["scale"] is None else float(s["scale"])) / max(1, len(real))
        prob.mul_(weight)
        dw = x.T @ prob
        return {"dx": prob @ w.T, "dw": dw.T if case["by_class"] else dw,
                "db": prob.sum(dim=0) if case["bias"] else None}
    kept = _exact_kept(case, s)
    if kind == "dropout":
        y = kept * wide(s["x"])
        return y if s["res"] is None else y + wide(s["res"])
    cols = case["cols"]
    gamma, beta = wide(s["gamma"]).unsqueeze(0), wide(s["beta"]).unsqueeze(0)
    if kind == "norm":
        h = kept * wide(s["x"])
        if s["res"] is not None:
            h = h + wide(s["res"])
        var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
        return {"h": None if s["h"] is None else h, "y": (h - mean) * torch.rsqrt(var + EPS) * gamma + beta}
    # y_c = gamma_c u_c / r + beta_c with u = h - mean(h), r = sqrt(sum u^2 / n + eps):
    # dy_c / dh_j = gamma_c (([c = j] - 1 / n) / r - u_c u_j / (n r^3))
    h, dy = wide(s["h"]), wide(s["dy"])
    u = h - torch.sum(h, dim=1, keepdim=True) / cols
    r = torch.sqrt(torch.sum(u.square(), dim=1, keepdim=True) / cols + EPS)
    g = dy * gamma
    dh = (g - torch.sum(g, dim=1, keepdim=True) / cols) / r - u * torch.sum(g * u, dim=1, keepdim=True) / (cols * r.pow(3))
    if s["dres"] is not None:
        dh += wide(s["dres"])
    return {"dx": kept * dh, "dh": None if s["dh"] is None else dh, "dgamma": torch.sum(dy * u / r, dim=0),
            "dbeta": torch.sum(dy, dim=0)}
