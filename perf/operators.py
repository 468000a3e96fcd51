"""The training side of a replayed MoE layer, as cases that a timer can run: each operator in its plain form and as a user calls it.

  norm     residual addition and root-mean-square norm, with bf16/f32 or e4m3 output, and its gradient
  tokens   token rows sorted by expert, and the gradients of sorting and of the weighted combine
  loss     clipped policy loss with KL and entropy terms on the logits, with the logits' gradient
  linear   both gradients of a block-scaled FP8 linear, dense or one per expert, from the 8-bit activations of its forward pass

`listed()` are the named cases, `draw(rng)` gives others of the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 128
EPS = 1e-6
CLIP_LOW, CLIP_HIGH, KL, ENTROPY, TEMPERATURE = 0.2, 0.28, 0.02, 0.001, 1.0
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# the largest work a drawn case may have, by kind: the largest listed one's
MAX_NORM = 32768 * 7168
MAX_TOKEN_BYTES = 6 * 32768 * 8 * 7168
MAX_LOGITS = 4096 * 131072
MAX_PRODUCTS = 4096 * 5120 * 32768
MAX_WEIGHTS = 1 << 30


def _norm(name, rows, cols, type, backward, extra, fp8=False):
    """extra: forward: there is a residual; backward: a gradient arrives at the sum as well."""
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "type": type, "backward": backward, "extra": extra, "fp8": fp8}


def _tokens(name, T, d, E, k, type, what, load="uniform"):
    return {"name": name, "kind": "tokens", "T": T, "d": d, "E": E, "k": k, "type": type, "what": what, "load": load}


def _loss(name, rows, V, type, gradient, masked=False):
    """masked: a tenth of the vocabulary at -inf.  gradient: "", or its type."""
    return {"name": name, "kind": "loss", "rows": rows, "V": V, "type": type, "gradient": gradient, "masked": masked}


def _linear(name, rows, E, NOUT, K, type, load="uniform"):
    """E == 0: a dense linear.  type: of the weights' gradient."""
    return {"name": name, "kind": "linear", "rows": rows, "E": E, "NOUT": NOUT, "K": K, "type": type, "load": load}


def listed():
    return [
        # one token being decoded: the norm in front of the FP8 layer, where only latency counts
        _norm("norm_decode_1", 1, 4096, "bf16", False, True, fp8=True),
        # the same over a long-context batch
        _norm("norm_longctx_32768", 32768, 7168, "bf16", False, True, fp8=True),
        # the norm's gradient over a micro-batch, with the residual stream's own gradient joining it
        _norm("norm_backward_4096", 4096, 5120, "bf16", True, True),
        # a small decode batch sorted by expert in the layer's widest form
        _tokens("dispatch_16_wide", 16, 7168, 256, 8, "bf16", "dispatch"),
        # a short ragged batch with odd sizes, gradients kept in 32 bits
        _tokens("dispatch_backward_777", 777, 2176, 60, 5, "f32", "dispatch_backward"),
        # the combine's gradient over the long-context batch: the largest traffic
        _tokens("combine_backward_32768", 32768, 7168, 256, 8, "bf16", "combine_backward", "zipf"),
        # scoring the last tokens of a few sequences: log-probabilities alone
        _loss("score_8", 8, 131072, "f32", ""),
        # a ragged micro-batch on an odd vocabulary, part of it masked away
        _loss("loss_333_odd", 333, 50001, "f32", "bf16", masked=True),
        # the policy loss and its gradient over a micro-batch of responses
        _loss("loss_4096", 4096, 131072, "bf16", "bf16"),
        # a dense projection's gradients for a handful of rows, its weights' gradient in 32 bits
        _linear("linear_40", 40, 0, 6144, 4096, "f32"),
        # the experts' down projections under a skewed log: a few hot experts, many cold ones
        _linear("experts_32768_zipf", 32768, 128, 5120, 1536, "bf16", "zipf"),
        # the head that makes the logits: the largest products
        _linear("head_4096", 4096, 0, 32768, 5120, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo=8, hi=56):
    """A multiple of 128 that is one of the widths of hidden layers."""
    return BLOCK * rng.choice([m for m in range(lo, hi + 1) if m != 24])


def draw(rng):
    while True:
        kind, type = rng.choice(["norm", "tokens", "loss", "linear"]), rng.choice(["bf16", "bf16", "f32"])
        if kind == "norm":
            fp8, backward = rng.random() < 0.5, rng.random() < 0.5
            cols = _width(rng) if fp8 or rng.random() < 0.5 else rng.randint(500, 7168) | 1
            case = _norm("", _log_int(rng, 1, 32768), cols, type, backward, rng.random() < 0.7, fp8 and not backward)
            fits = case["rows"] * cols <= MAX_NORM
        elif kind == "tokens":
            E = _log_int(rng, 8, 256)
            case = _tokens("", _log_int(rng, 1, 32768), _width(rng), E, rng.randint(1, 8), type,
                           rng.choice(["dispatch", "dispatch_backward", "combine_backward"]), rng.choice(["uniform", "zipf"]))
            fits = _token_bytes(case) <= MAX_TOKEN_BYTES
        elif kind == "loss":
            case = _loss("", _log_int(rng, 1, 8192), _log_int(rng, 1000, 160000), type, rng.choice(["", "bf16", "bf16", type]), rng.random() < 0.3)
            fits = case["rows"] * case["V"] <= MAX_LOGITS // (2 if type == "f32" else 1)
        else:
            E = rng.choice([0, 0, 0, _log_int(rng, 4, 128), _log_int(rng, 4, 128)])
            case = _linear("", _log_int(rng, 1, 32768), E, _width(rng, 8, 56 if E else 200), _width(rng), type, rng.choice(["uniform", "zipf"]))
            fits = (case["rows"] * case["NOUT"] * case["K"] * (2 if type == "f32" else 1) <= MAX_PRODUCTS
                    and max(E, 1) * case["NOUT"] * case["K"] <= MAX_WEIGHTS)
        if fits and 3072 not in case.values():
            del case["name"]
            return case


# ---------------------------------------------------------------------------------------------- inputs
class _Handle:
    """A context for one layer shape, as a program makes it once."""

    def __init__(self, T=0, d=BLOCK, E=1, k=1):
        import paper_2512_07710_amd as moe
        self.moe, self.ctx = moe, None
        self.ctx = moe.moe_create(T, d, E, k, BLOCK)
        moe.moe_reserve_gradients(self.ctx)

    def __del__(self):
        if self.ctx:
            self.moe.moe_destroy(self.ctx)


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + tag * 7919 + 17) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(shape, g, type, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=type).mul_(std)


def _ids(T, E, k, load, g):
    """k distinct expert ids a token: uniform, or p_e ~ (e+1)^-1.2."""
    e = torch.arange(1, E + 1, device=DEV, dtype=torch.float32)
    logp = -1.2 * torch.log(e) if load == "zipf" else torch.zeros_like(e)
    u = torch.rand((T, E), generator=g, device=DEV).clamp_(1e-20, 1.0 - 1e-7)
    return torch.topk(logp - torch.log(-torch.log(u)), k, dim=1).indices


def _coded(x, blocks):
    """x as e4m3 codes and the scales of its blocks of blocks[0] x 128."""
    rows, cols = x.shape[-2] // blocks, x.shape[-1] // BLOCK
    v = x.view(*x.shape[:-2], rows, blocks, cols, BLOCK)
    s = v.abs().amax(dim=(-3, -1)).div_(448.0).clamp_(min=1e-30)
    return (v / s[..., :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(x.shape), s


def prepare(case, seed):
    new = lambda shape, type: torch.empty(shape, dtype=type, device=DEV)  # noqa: E731
    c = dict(case)
    s = {"case": c, "handle": None}
    f32, type = torch.float32, TYPES[c["type"]]
    if c["kind"] == "norm":
        rows, cols, g = c["rows"], c["cols"], _gen(seed, 1)
        s["gain"] = 1.0 + _normal((cols,), g, f32, 0.2)
        if c["backward"]:
            s["h"] = _normal((rows, cols), g, type, 2.0)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(dim=1) + EPS)
            s["dy"] = _normal((rows, cols), g, type)
            s["dh"] = _normal((rows, cols), g, type) if c["extra"] else None
            s.update(dx=new((rows, cols), type), dgain=new((cols,), f32))
        else:
            s["x"] = _normal((rows, cols), g, type)
            s["residual"] = _normal((rows, cols), g, type, 2.0) if c["extra"] else None
            s["sum"] = new((rows, cols), type) if c["extra"] else None
            s["y"] = None if c["fp8"] else new((rows, cols), type)
            s["q"] = new((rows, cols), torch.uint8) if c["fp8"] else None
            s["scales"] = new((cols // BLOCK, rows), f32) if c["fp8"] else None
            s["rstd"] = new((rows,), f32)
        shape = {}
    elif c["kind"] == "tokens":
        T, d, E, k, g = c["T"], c["d"], c["E"], c["k"], _gen(seed, 2)
        N = T * k
        ids = _ids(T, E, k, c["load"], g)
        perm = torch.argsort(ids.view(-1), stable=True)
        inv = torch.empty_like(perm)
        inv[perm] = torch.arange(N, device=DEV)
        s["inv_perm"], s["topk_idx"] = inv.to(torch.int32), ids.to(torch.int32).contiguous()
        if c["what"] == "combine_backward":
            s["topk_w"] = torch.softmax(_normal((T, k), g, f32), dim=1)
            s["dy"], s["y_perm"] = _normal((T, d), g, type), _normal((N, d), g, f32)
            s.update(dy_perm=new((N, d), type), dw=new((T, k), f32), dlogits=new((T, E), f32))
        elif c["what"] == "dispatch":
            s["x"], s["x_perm"] = _normal((T, d), g, type), new((N, d), type)
        else:
            s["dx_perm"], s["dx"] = _normal((N, d), g, type), new((T, d), type)
        shape = {"T": T, "d": d, "E": E, "k": k}
    elif c["kind"] == "loss":
        rows, V, g = c["rows"], c["V"], _gen(seed, 3)
        logits = _normal((rows, V), g, type, 2.5)
        if c["masked"]:
            logits[:, torch.rand((V,), generator=g, device=DEV) < 0.1] = -math.inf
        s["logits"] = logits
        s["target"] = torch.empty((rows,), dtype=torch.int32, device=DEV)
        logp = torch.empty((rows,), device=DEV)
        for i in range(0, rows, 512):                         # tokens drawn from the policy itself
            part = logits[i:i + 512].float()
            u = torch.empty_like(part).exponential_(generator=g).clamp_(min=1e-30)
            t = torch.argmax(part - torch.log(u), dim=1)
            s["target"][i:i + 512] = t
            logp[i:i + 512] = torch.log_softmax(part, dim=1).gather(1, t[:, None])[:, 0]
        s["old_logp"] = logp + _normal((rows,), g, f32, 0.15)
        s["ref_logp"] = logp + _normal((rows,), g, f32, 0.3)
        s["advantage"] = _normal((rows,), g, f32)
        keep = (torch.rand((rows,), generator=g, device=DEV) > 0.1).float()   # prompt and padding tokens have no weight
        keep[0] = 1.0
        s["weight"] = keep / keep.sum()
        s.update({n: new((rows,), f32) for n in ("logp", "entropy", "row_loss")}, loss=new((1,), f32))
        s["dlogits"] = new((rows, V), TYPES[c["gradient"]]) if c["gradient"] else None
        shape = {}
    else:
        rows, E, NOUT, K, g = c["rows"], c["E"], c["NOUT"], c["K"], _gen(seed, 4)
        s["dy"] = _normal((rows, NOUT), g, torch.bfloat16, 0.01)
        s["xq"] = torch.empty((rows, K), dtype=torch.uint8, device=DEV)
        s["xs"] = torch.empty((K // BLOCK, rows), device=DEV)
        for i in range(0, rows, 8192):
            q, sc = _coded(_normal((min(8192, rows - i), K), g, f32), 1)
            s["xq"][i:i + 8192], s["xs"][:, i:i + 8192] = q, sc.t()
        s["Wq"] = torch.empty((max(E, 1), NOUT, K), dtype=torch.uint8, device=DEV)
        s["ws"] = torch.empty((max(E, 1), NOUT // BLOCK, K // BLOCK), device=DEV)
        for e in range(max(E, 1)):
            s["Wq"][e], s["ws"][e] = _coded(_normal((NOUT, K), g, f32, K ** -0.5), BLOCK)
        s["offsets"], s["bounds"] = None, [0, rows]
        if E:
            ids = _ids(rows, E, 1, c["load"], g)
            s["offsets"] = torch.zeros((E + 1,), dtype=torch.int32, device=DEV)
            s["offsets"][1:] = torch.cumsum(torch.bincount(ids.view(-1), minlength=E), dim=0)
            s["bounds"] = s["offsets"].tolist()               # the plain form's plan
        else:
            s["Wq"], s["ws"] = s["Wq"][0], s["ws"][0]
        s["dx"] = new((rows, K), torch.bfloat16)
        s["dW"] = new((E, NOUT, K) if E else (NOUT, K), type)
        shape = {}
    if own:
        s["handle"] = _Handle(**shape)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _own_norm(s):
    moe, ctx = s["handle"].moe, s["handle"].ctx
    if s["case"]["backward"]:
        moe.moe_add_rmsnorm_backward(ctx, s["dy"], s["h"], s["rstd"], s["gain"], s["dh"], s["dx"], s["dgain"])
        return {"dx": s["dx"], "dgain": s["dgain"]}
    moe.moe_add_rmsnorm(ctx, s["x"], s["residual"], s["gain"], EPS, s["sum"], s["y"], s["q"], s["scales"], s["rstd"])
    codes = None if s["q"] is None else s["q"].view(torch.float8_e4m3fn)
    return {"sum": s["sum"], "y": s["y"], "q": codes, "scales": s["scales"], "rstd": s["rstd"]}


def _plain_norm(s):
    f32, type = torch.float32, TYPES[s["case"]["type"]]
    if s["case"]["backward"]:
        h, r = s["h"].to(f32), s["rstd"][:, None]
        dy = s["dy"].to(f32)
        u = dy * s["gain"]
        dx = r * u - h * (r * r * r) * ((u * h).sum(dim=1, keepdim=True) / h.shape[1])
        if s["dh"] is not None:
            dx = dx + s["dh"].to(f32)
        return {"dx": dx.to(type), "dgain": (dy * h * r).sum(dim=0)}
    h, total = s["x"], None
    if s["residual"] is not None:
        total = h = (h.to(f32) + s["residual"].to(f32)).to(type)
    h = h.to(f32)
    rstd = torch.rsqrt((h * h).sum(dim=1) / h.shape[1] + EPS)
    y = h * rstd[:, None] * s["gain"]
    if not s["case"]["fp8"]:
        return {"sum": total, "y": y.to(type), "q": None, "scales": None, "rstd": rstd}
    v = y.view(y.shape[0], -1, BLOCK)
    scale = v.abs().amax(dim=2) / 448.0
    scale = torch.where(scale == 0, 1.0, scale)
    q = (v / scale[:, :, None]).to(torch.float8_e4m3fn).view(y.shape)
    return {"sum": total, "y": None, "q": q, "scales": scale.t().contiguous(), "rstd": rstd}


def _own_tokens(s):
    moe, ctx, what = s["handle"].moe, s["handle"].ctx, s["case"]["what"]
    if what == "dispatch":
        moe.moe_dispatch(ctx, s["x"], s["inv_perm"], s["x_perm"])
        return {"x_perm": s["x_perm"]}
    if what == "dispatch_backward":
        moe.moe_dispatch_backward(ctx, s["dx_perm"], s["inv_perm"], None, s["dx"])
        return {"dx": s["dx"]}
    moe.moe_combine_backward(ctx, s["dy"], s["y_perm"], s["inv_perm"], s["topk_w"], s["topk_idx"], s["dy_perm"], s["dw"], s["dlogits"])
    return {"dy_perm": s["dy_perm"], "dw": s["dw"], "dlogits": s["dlogits"]}


def _plain_tokens(s):
    c, f32, type = s["case"], torch.float32, TYPES[s["case"]["type"]]
    T, d, k, inv = c["T"], c["d"], c["k"], s["inv_perm"].long()
    if c["what"] == "dispatch":
        rows = torch.empty((T * k, d), dtype=type, device=DEV)
        rows[inv] = s["x"].repeat_interleave(k, dim=0)
        return {"x_perm": rows}
    if c["what"] == "dispatch_backward":
        return {"dx": s["dx_perm"][inv].view(T, k, d).to(f32).sum(dim=1).to(type)}
    dy = s["dy"].to(f32)[:, None, :]
    dw = (s["y_perm"][inv].view(T, k, d) * dy).sum(dim=2)
    rows = torch.empty((T * k, d), dtype=type, device=DEV)
    rows[inv] = (s["topk_w"][:, :, None] * dy).to(type).view(T * k, d)
    w = s["topk_w"]
    dl = w * (dw - (w * dw).sum(dim=1, keepdim=True))
    dlogits = torch.zeros((T, c["E"]), device=DEV).scatter_(1, s["topk_idx"].long(), dl)
    return {"dy_perm": rows, "dw": dw, "dlogits": dlogits}


def _own_loss(s):
    moe, ctx = s["handle"].moe, s["handle"].ctx
    moe.moe_policy_loss(ctx, s["logits"], s["target"], s["old_logp"], s["ref_logp"], s["advantage"], s["weight"], s["logp"], s["entropy"],
                        s["row_loss"], s["loss"], s["dlogits"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL, entropy_coef=ENTROPY,
                        temperature=TEMPERATURE)
    return {n: s[n] for n in ("logp", "entropy", "row_loss", "loss", "dlogits")}


def _plain_loss(s):
    z = s["logits"].to(torch.float32) / TEMPERATURE
    z = z - z.amax(dim=1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    p, logs = e / total, z - torch.log(total)
    entropy = -torch.where(p > 0, p * logs, 0.0).sum(dim=1)
    at = s["target"].long()[:, None]
    logp = logs.gather(1, at)[:, 0]
    A, w, x = s["advantage"], s["weight"], s["ref_logp"] - logp
    ratio = torch.exp(logp - s["old_logp"])
    free, held = ratio * A, torch.minimum(torch.maximum(ratio, ratio.new_tensor(1 - CLIP_LOW)), ratio.new_tensor(1 + CLIP_HIGH)) * A
    kl = torch.exp(x) - x - 1
    row_loss = w * (-torch.minimum(free, held) + KL * kl - ENTROPY * entropy)
    out = {"logp": logp, "entropy": entropy, "row_loss": row_loss, "loss": row_loss.sum()[None], "dlogits": None}
    if s["case"]["gradient"]:
        dlogp = w * (torch.where(free <= held, -free, 0.0) + KL * (1 - torch.exp(x)))
        grad = torch.where(p > 0, p * ((ENTROPY * w)[:, None] * (logs + entropy[:, None]) - dlogp[:, None]), 0.0)
        grad.scatter_add_(1, at, dlogp[:, None])
        out["dlogits"] = (grad / TEMPERATURE).to(TYPES[s["case"]["gradient"]])
    return out


def _own_linear(s):
    moe, ctx = s["handle"].moe, s["handle"].ctx
    moe.moe_linear_fp8_dgrad(ctx, s["dy"], s["Wq"], s["ws"], s["offsets"], s["dx"])
    moe.moe_linear_fp8_wgrad(ctx, s["dy"], s["xq"], s["xs"], s["offsets"], s["dW"])
    return {"dx": s["dx"], "dW": s["dW"]}


def _plain_linear(s):
    c, f32, type = s["case"], torch.float32, TYPES[s["case"]["type"]]
    E, NOUT, K, bounds = max(c["E"], 1), c["NOUT"], c["K"], s["bounds"]
    values = lambda q: q.view(torch.float8_e4m3fn).to(f32)  # noqa: E731
    dy = s["dy"].to(f32)
    x = (values(s["xq"]).view(-1, K // BLOCK, BLOCK) * s["xs"].t()[:, :, None]).view(-1, K)
    Wq, ws = s["Wq"].view(E, NOUT, K), s["ws"].view(E, NOUT // BLOCK, K // BLOCK)
    dx, dW = torch.empty((c["rows"], K), dtype=torch.bfloat16, device=DEV), torch.empty((E, NOUT, K), dtype=type, device=DEV)
    for e in range(E):                                        # one product per expert, as the operator is defined
        at = slice(bounds[e], bounds[e + 1])
        W = (values(Wq[e]).view(NOUT // BLOCK, BLOCK, K // BLOCK, BLOCK) * ws[e][:, None, :, None]).view(NOUT, K)
        dx[at] = torch.matmul(dy[at], W).to(torch.bfloat16)
        dW[e] = torch.matmul(dy[at].t(), x[at]).to(type)
    return {"dx": dx, "dW": dW if c["E"] else dW[0]}


_own = {"norm": _own_norm, "tokens": _own_tokens, "loss": _own_loss, "linear": _own_linear}
_plain = {"norm": _plain_norm, "tokens": _plain_tokens, "loss": _plain_loss, "linear": _plain_linear}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def _token_bytes(c):
    b, T, N = (2 if c["type"] == "bf16" else 4), c["T"], c["T"] * c["k"]
    if c["what"] == "combine_backward":
        return c["d"] * (T * b + N * b + N * 4) + 16 * N + 4 * T * c["E"]
    return c["d"] * b * (T + N) + 4 * N


def work(case):
    c = case
    b = 2 if c["type"] == "bf16" else 4
    if c["kind"] == "norm":
        n = c["rows"] * c["cols"]
        if c["backward"]:
            return {"bytes": n * b * (4 if c["extra"] else 3) + 8 * c["cols"] + 4 * c["rows"], "flops": 10 * n}
        out = n * (1 + 4 / BLOCK) if c["fp8"] else n * b
        return {"bytes": n * b * (3 if c["extra"] else 1) + out + 4 * c["cols"] + 4 * c["rows"], "flops": 6 * n}
    if c["kind"] == "tokens":
        return {"bytes": _token_bytes(c), "flops": (3 if c["what"] == "combine_backward" else 1) * c["T"] * c["k"] * c["d"]}
    if c["kind"] == "loss":
        n, out = c["rows"] * c["V"], {"": 0, "bf16": 2, "f32": 4}[c["gradient"]]
        return {"bytes": n * (b + out) + 32 * c["rows"], "flops": 8 * n}
    E, rows, NOUT, K = max(c["E"], 1), c["rows"], c["NOUT"], c["K"]
    return {"bytes": 2 * rows * NOUT + 3 * rows * K + rows * K // 32 + E * NOUT * K * (1 + b), "flops": 4 * rows * NOUT * K}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    with torch.no_grad():
        return _exact[case["kind"]](case, prepare(case, seed))


def _exact_norm(c, s):
    f64 = torch.float64
    if c["backward"]:
        # the chain rule through the row's mean square, taken column by column of the Jacobian
        h, r, g, dy = s["h"].to(f64), s["rstd"].to(f64), s["gain"].to(f64), s["dy"].to(f64)
        n = h * r[:, None]
        t = dy * g
        along = torch.einsum("rc,rc->r", t, n) / h.shape[1]
        dx = r[:, None] * (t - n * along[:, None])
        return {"dx": dx if s["dh"] is None else dx + s["dh"].to(f64), "dgain": torch.einsum("rc,rc->c", dy, n)}
    h, total = s["x"].to(f64), None
    if s["residual"] is not None:
        total = h + s["residual"].to(f64)
        h = total.to(TYPES[c["type"]]).to(f64)                # the sum is kept in its type, and normalised as it is kept
    rstd = (h.pow(2).mean(dim=1) + EPS).pow(-0.5)
    y = h.mul(rstd[:, None]).mul(s["gain"].to(f64))
    if not c["fp8"]:
        return {"sum": total, "y": y, "q": None, "scales": None, "rstd": rstd}
    groups = y.unflatten(1, (-1, BLOCK))
    scale = groups.abs().max(dim=2).values / 448
    return {"sum": total, "y": None, "q": (groups / scale.unsqueeze(2)).flatten(1), "scales": scale.t().contiguous(), "rstd": rstd}


def _exact_tokens(c, s):
    f64, T, k, d = torch.float64, c["T"], c["k"], c["d"]
    inv = s["inv_perm"].long().view(T, k)
    source = torch.argsort(inv.flatten())                     # the assignment that each sorted row holds
    if c["what"] == "dispatch":
        return {"x_perm": s["x"][source // k].to(f64)}
    if c["what"] == "dispatch_backward":
        dx = torch.zeros((T, d), dtype=f64, device=DEV)
        dx.index_add_(0, source // k, s["dx_perm"].to(f64))
        return {"dx": dx}
    w, dw = s["topk_w"].to(f64), torch.empty((T, k), dtype=f64, device=DEV)
    dy_perm = torch.empty((T * k, d), dtype=torch.float32, device=DEV)
    for t in range(0, T, 2048):                               # (the batch's rows in 64 bits would be large)
        at = inv[t:t + 2048]
        dy = s["dy"][t:t + 2048].to(f64)
        dw[t:t + 2048] = torch.matmul(s["y_perm"][at].to(f64), dy[:, :, None])[:, :, 0]
        dy_perm[at] = (w[t:t + 2048, :, None] * dy[:, None, :]).float()
    softmax = torch.diag_embed(w) - w[:, :, None] * w[:, None, :]
    dlogits = torch.zeros((T, c["E"]), dtype=f64, device=DEV)
    dlogits.scatter_(1, s["topk_idx"].long(), torch.matmul(softmax, dw[:, :, None])[:, :, 0])
    return {"dy_perm": dy_perm, "dw": dw, "dlogits": dlogits}


def _exact_loss(c, s):
    f64, rows = torch.float64, c["rows"]
    out = {n: torch.empty((rows,), dtype=f64, device=DEV) for n in ("logp", "entropy", "row_loss")}
    out["dlogits"] = torch.empty((rows, c["V"]), dtype=f64, device=DEV) if c["gradient"] else None
    for i in range(0, rows, 256):
        at = slice(i, min(i + 256, rows))
        z = s["logits"][at].to(f64) / TEMPERATURE
        logs = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = logs.exp()
        H = -(p * logs).nan_to_num(0.0).sum(dim=1)
        pick = torch.nn.functional.one_hot(s["target"][at].long(), c["V"])
        lp = logs.masked_fill(pick == 0, 0.0).sum(dim=1)
        old, ref, A, w = (s[n][at].to(f64) for n in ("old_logp", "ref_logp", "advantage", "weight"))
        ratio, back = (lp - old).exp(), (ref - lp).exp()
        surrogate = torch.minimum(ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
        out["logp"][at], out["entropy"][at] = lp, H
        out["row_loss"][at] = w * (KL * (torch.expm1(ref - lp) - (ref - lp)) - surrogate - ENTROPY * H)
        if c["gradient"]:
            inside = torch.where(A >= 0, ratio <= 1 + CLIP_HIGH, ratio >= 1 - CLIP_LOW)
            slope = w * (KL * (1 - back) - inside * ratio * A)
            bonus = (p * (logs + H[:, None])).nan_to_num(0.0) * (w * ENTROPY)[:, None]
            out["dlogits"][at] = (slope[:, None] * (pick - p) + bonus) / TEMPERATURE
    out["loss"] = out["row_loss"].sum()[None]
    return out


def _exact_linear(c, s):
    f64, NOUT, K = torch.float64, c["NOUT"], c["K"]
    table = torch.arange(256, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).to(f64)
    dx = torch.zeros((c["rows"], K), dtype=f64, device=DEV)
    dW = torch.zeros((max(c["E"], 1), NOUT, K), dtype=torch.float32 if c["type"] == "bf16" else f64, device=DEV)
    scales = s["xs"].to(f64).repeat_interleave(BLOCK, dim=0)  # [K, rows]
    for e in range(max(c["E"], 1)):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if lo == hi:
            continue
        codes, blocks = s["Wq"].view(-1, NOUT, K)[e], s["ws"].view(-1, NOUT // BLOCK, K // BLOCK)[e]
        W = table[codes.int()] * torch.kron(blocks.to(f64), torch.ones((BLOCK, BLOCK), dtype=f64, device=DEV))
        dy = s["dy"][lo:hi].to(f64)
        dx[lo:hi] = dy @ W
        dW[e] = dy.t() @ (table[s["xq"][lo:hi].int()] * scales[:, lo:hi].t())
    return {"dx": dx, "dW": dW if c["E"] else dW[0]}


_exact = {"norm": _exact_norm, "tokens": _exact_tokens, "loss": _exact_loss, "linear": _exact_linear}
