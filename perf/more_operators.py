"""The two ends of a policy step around a replayed MoE layer, as cases that a timer can run: each operator in its plain form and as a user calls it.

  embed       rows of an embedding table for token ids, with a factor
  embed_grad  its gradient: the rows' gradients summed by token id
  logp        log-probabilities of given tokens, entropy and the most likely tokens of rows of logits
  logp_grad   the logits' gradient from those of the log-probabilities and the entropy
  clip        the global norm of a list of gradients, and the list scaled down to a largest norm

`listed()` are the named cases, `draw(rng)` gives others of the same ranges.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
ALIGN = 256                                                    # elements: where the tensors of a list begin in their buffer
# the largest work a drawn case may have, by kind: the largest listed one's
MAX_TABLE = 131072 * 7168
MAX_LOGITS = 4096 * 131072
MAX_GRADS = 1 << 30


def _embed(name, T, V, d, type, out):
    return {"name": name, "kind": "embed", "T": T, "V": V, "d": d, "type": type, "out": out, "scale": d ** 0.5}


def _embed_grad(name, T, V, d, type, out, load, accumulate=False, padded=False):
    """type: of the rows' gradients, out: of the table's.  padded: a fifth of the ids are -1."""
    return {"name": name, "kind": "embed_grad", "T": T, "V": V, "d": d, "type": type, "out": out, "load": load, "accumulate": accumulate, "padded": padded,
            "scale": d ** 0.5}


def _logp(name, rows, V, type, m, n, temperature=1.0, masked=False):
    """m given tokens and the n most likely ones a row.  masked: a tenth of the vocabulary at -inf."""
    return {"name": name, "kind": "logp", "rows": rows, "V": V, "type": type, "m": m, "n": n, "temperature": temperature, "masked": masked}


def _logp_grad(name, rows, V, type, out, m, entropy, temperature=1.0, masked=False):
    return {"name": name, "kind": "logp_grad", "rows": rows, "V": V, "type": type, "out": out, "m": m, "entropy": entropy, "temperature": temperature,
            "masked": masked}


def _clip(name, n, total, type, clipped):
    """n gradients of `total` elements together, of uneven sizes; type "mixed": every third in 32 bits.  clipped: the norm is above the bound, and the scaled
    gradients go to buffers of their own, so that a pass can be repeated; otherwise it is below, and they stay where they are."""
    return {"name": name, "kind": "clip", "n": n, "total": total, "type": type, "clipped": clipped}


def listed():
    return [
        # one token being decoded: only latency counts
        _embed("embed_decode_1", 1, 131072, 4096, "bf16", "bf16"),
        # a long-context batch: the largest lookup
        _embed("embed_longctx_32768", 32768, 131072, 7168, "bf16", "bf16"),
        # a ragged micro-batch with padding on odd sizes, joining the gradients of earlier micro-batches in 32 bits
        _embed_grad("embed_grad_777_odd", 777, 50001, 2177, "f32", "f32", "zipf", accumulate=True, padded=True),
        # a micro-batch of text whose gradients join those of earlier micro-batches
        _embed_grad("embed_grad_4096_add", 4096, 131072, 5120, "bf16", "f32", "zipf", accumulate=True),
        # the long-context batch: the table's whole gradient is written
        _embed_grad("embed_grad_32768", 32768, 131072, 7168, "bf16", "bf16", "zipf"),
        # a few sequences being decoded: what is logged about each sampled token
        _logp("logp_decode_4", 4, 131072, "f32", 1, 20),
        # a ragged batch on an odd vocabulary, part of it masked away, at a sampling temperature
        _logp("logp_333_odd", 333, 50001, "f32", 2, 5, temperature=0.7, masked=True),
        # a micro-batch of responses scored under a policy
        _logp("logp_4096", 4096, 131072, "bf16", 1, 8),
        # distillation on a teacher's tokens: several given tokens a row, with an entropy term
        _logp_grad("logp_grad_1024", 1024, 131072, "bf16", "bf16", 8, True),
        # a small batch on an odd vocabulary, gradients in 32 bits
        _logp_grad("logp_grad_100_odd", 100, 50001, "f32", "f32", 1, False, masked=True),
        # the small parameters of a few layers, below the bound: norms' gains, routers, biases
        _clip("clip_small_60", 60, 300000, "mixed", False),
        # a model's shard: many gradients, scaled down
        _clip("clip_shard_700", 700, 1 << 30, "mixed", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return 128 * rng.randint(8, 56) if rng.random() < 0.6 else rng.randint(500, 7168) | 1


def draw(rng):
    while True:
        kind, type, out = rng.choice(["embed", "embed_grad", "logp", "logp_grad", "clip"]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "f32"])
        if kind == "embed":
            case = _embed("", _log_int(rng, 1, 32768), _log_int(rng, 1000, 160000), _width(rng), type, out)
            fits = case["V"] * case["d"] <= MAX_TABLE and max(case["T"], 1000) * case["d"] * (BYTES[type] + BYTES[out]) <= 32768 * 7168 * 4
        elif kind == "embed_grad":
            case = _embed_grad("", _log_int(rng, 1, 32768), _log_int(rng, 1000, 160000), _width(rng), type, out, rng.choice(["uniform", "zipf", "zipf"]),
                               rng.random() < 0.5, rng.random() < 0.4)
            fits = case["V"] * case["d"] * BYTES[out] <= MAX_TABLE * 2 and case["T"] * case["d"] * BYTES[type] <= 32768 * 7168 * 2
        elif kind == "logp":
            case = _logp("", _log_int(rng, 1, 8192), _log_int(rng, 1000, 160000), type, rng.randint(1, 8), rng.randint(0, 20), rng.choice([1.0, 0.7]),
                         rng.random() < 0.3)
            fits = case["rows"] * case["V"] * BYTES[type] <= MAX_LOGITS * 2
        elif kind == "logp_grad":
            case = _logp_grad("", _log_int(rng, 1, 8192), _log_int(rng, 1000, 160000), type, out, rng.randint(1, 16), rng.random() < 0.5,
                              rng.choice([1.0, 0.7]), rng.random() < 0.3)
            fits = case["rows"] * case["V"] * (BYTES[type] + BYTES[out]) <= MAX_LOGITS * 2
        else:
            case = _clip("", _log_int(rng, 1, 1500), _log_int(rng, 10000, MAX_GRADS), rng.choice(["bf16", "f32", "mixed"]), rng.random() < 0.5)
            fits = case["n"] * 50 <= case["total"] and case["total"] * (BYTES["f32"] if case["type"] == "f32" else 3) <= (1 << 30) * 3
        if fits:
            del case["name"]
            return case


# ---------------------------------------------------------------------------------------------- inputs
class _Handle:
    """A context, as a program makes it once."""

    def __init__(self):
        import paper_2512_07710_amd as moe
        self.moe, self.ctx = moe, None
        self.ctx = moe.moe_create(0, 128, 1, 1, 128)
        moe.moe_reserve_gradients(self.ctx)

    def __del__(self):
        if self.ctx:
            self.moe.moe_destroy(self.ctx)


def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + tag * 7919 + 29) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(shape, g, type, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=type).mul_(std)


def _text(T, V, load, padded, g):
    """Token ids: uniform, or p_r ~ 1/r over the ranks of the vocabulary, which lie anywhere in it."""
    if load == "zipf":
        share = torch.cumsum(1.0 / torch.arange(1, V + 1, device=DEV, dtype=torch.float64), dim=0)
        u = torch.rand((T,), generator=g, device=DEV, dtype=torch.float64) * share[-1]
        ids = torch.randperm(V, generator=g, device=DEV)[torch.searchsorted(share, u).clamp_(max=V - 1)]
    else:
        ids = torch.randint(0, V, (T,), generator=g, device=DEV)
    if padded:
        ids[torch.rand((T,), generator=g, device=DEV) < 0.2] = -1
    return ids.to(torch.int32)


def _sizes(c):
    """Elements of each gradient of a list: uneven, odd ones among them."""
    rng = random.Random(c["n"] * 7919 + c["total"])
    share = [math.exp(rng.gauss(0, 1.5)) for _ in range(c["n"])]
    return [max(1, int(c["total"] * v / sum(share))) for v in share]


def _types(c):
    return [("f32" if i % 3 == 2 else "bf16") if c["type"] == "mixed" else c["type"] for i in range(c["n"])]


def _list(c):
    """(views, buffers): a list's tensors, in one buffer for each type."""
    sizes, types, views, end = _sizes(c), _types(c), [], {"bf16": 0, "f32": 0}
    starts = []
    for size, type in zip(sizes, types):
        starts.append(end[type])
        end[type] += (size + ALIGN - 1) // ALIGN * ALIGN
    buffers = {t: torch.zeros((n,), dtype=TYPES[t], device=DEV) for t, n in end.items() if n}
    for at, size, type in zip(starts, sizes, types):
        views.append(buffers[type][at:at + size])
    return views, buffers


def prepare(case, seed):
    new = lambda shape, type: torch.empty(shape, dtype=type, device=DEV)  # noqa: E731
    c, f32, i32 = dict(case), torch.float32, torch.int32
    s = {"case": c, "handle": None}
    kind = c["kind"]
    if kind == "embed":
        g = _gen(seed, 1)
        s["ids"] = _text(c["T"], c["V"], "zipf", False, g)
        s["table"] = _normal((c["V"], c["d"]), g, TYPES[c["type"]], 0.02)
        s["y"] = new((c["T"], c["d"]), TYPES[c["out"]])
    elif kind == "embed_grad":
        g = _gen(seed, 2)
        s["ids"] = _text(c["T"], c["V"], c["load"], c["padded"], g)
        s["dy"] = _normal((c["T"], c["d"]), g, TYPES[c["type"]], 0.01)
        shape = (c["V"], c["d"])
        s["dtable"] = _normal(shape, g, TYPES[c["out"]], 0.5) if c["accumulate"] else new(shape, TYPES[c["out"]])
    elif kind in ("logp", "logp_grad"):
        rows, V, m, g = c["rows"], c["V"], c["m"], _gen(seed, 3)
        logits = _normal((rows, V), g, TYPES[c["type"]], 2.5)
        open_ = torch.arange(V, device=DEV)
        if c["masked"]:
            keep = torch.rand((V,), generator=g, device=DEV) >= 0.1
            logits[:, ~keep] = -math.inf
            open_ = open_[keep]
        s["logits"] = logits
        # the sampled token is likely, the others are any that are open; distinct, as a teacher's are
        first = torch.argmax(logits[:, :max(1, V // 50)], dim=1)
        s["ids"] = torch.cat([first[:, None], open_[torch.rand((rows, open_.numel() // 7), generator=g, device=DEV).topk(m, dim=1).indices * 7]], dim=1)
        s["ids"] = s["ids"][:, :m].to(i32).contiguous()
        if kind == "logp":
            n = c["n"]
            s.update(logp=new((rows, m), f32), entropy=new((rows,), f32), top_idx=new((rows, n), i32) if n else None, top_logp=new((rows, n), f32) if n else None)
        else:
            s["dlogp"] = _normal((rows, m), g, f32, 1.0 / rows)
            s["dentropy"] = _normal((rows,), g, f32, 0.01 / rows) if c["entropy"] else None
            if rows > 8:
                s["dlogp"][rows // 8:rows // 4] = 0.0           # prompt and padding tokens have no gradient
                if c["entropy"]:
                    s["dentropy"][rows // 8:rows // 4] = 0.0
            # what the forward call leaves for the gradient: each row's largest logit, the sum of exponentials, the entropy
            s["stats"], s["entropy"] = new((rows, 2), f32), new((rows,), f32)
            for i in range(0, rows, 512):
                part = logits[i:i + 512].to(torch.float64)
                top = part.amax(dim=1, keepdim=True)
                z = (part - top) / c["temperature"]
                e = z.exp()
                total = e.sum(dim=1)
                s["stats"][i:i + 512, 0], s["stats"][i:i + 512, 1] = top[:, 0], total
                s["entropy"][i:i + 512] = total.log() - (e * z.clamp(min=-1e4)).sum(dim=1) / total
            s["dlogits"] = new((rows, V), TYPES[c["out"]])
    else:
        g = _gen(seed, 4)
        s["grads"], s["buffers"] = _list(c)
        for v in s["grads"]:
            v.normal_(generator=g)
        s["outs"], s["out_buffers"] = _list(c) if c["clipped"] else (None, None)
        s["max_norm"] = (0.3 if c["clipped"] else 10.0) * math.sqrt(c["total"])
        s["sum_sq"], s["norm"] = new((1,), torch.float64), new((1,), f32)
    if own:
        s["handle"] = _Handle()
        if kind == "clip":
            moe = s["handle"].moe
            s["list"], s["out_list"] = moe.GradList(s["grads"]), moe.GradList(s["outs"]) if c["clipped"] else None
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _own_embed(s):
    h = s["handle"]
    h.moe.moe_embed(h.ctx, s["ids"], s["table"], s["case"]["scale"], s["y"])
    return {"y": s["y"]}


def _plain_embed(s):
    c, ids = s["case"], s["ids"].long()
    known = (ids >= 0) & (ids < c["V"])
    rows = s["table"][torch.where(known, ids, 0)].to(torch.float32) * c["scale"]
    return {"y": torch.where(known[:, None], rows, 0.0).to(TYPES[c["out"]])}


def _own_embed_grad(s):
    h, c = s["handle"], s["case"]
    h.moe.moe_embed_backward(h.ctx, s["dy"], s["ids"], c["scale"], s["dtable"], c["accumulate"])
    return {"dtable": s["dtable"]}


def _plain_embed_grad(s):
    c, ids = s["case"], s["ids"].long()
    known = (ids >= 0) & (ids < c["V"])
    rows = torch.where(known[:, None], s["dy"].to(torch.float32), 0.0)
    total = torch.zeros((c["V"], c["d"]), device=DEV).index_add_(0, torch.where(known, ids, 0), rows) * c["scale"]
    if not c["accumulate"]:
        return {"dtable": total.to(TYPES[c["out"]])}
    s["dtable"].copy_(s["dtable"].to(torch.float32) + total)    # (joined where it is, as the operator does)
    return {"dtable": s["dtable"]}


def _own_logp(s):
    h = s["handle"]
    h.moe.moe_token_logp(h.ctx, s["logits"], s["ids"], s["logp"], s["entropy"], s["top_idx"], s["top_logp"], temperature=s["case"]["temperature"])
    return {n: s[n] for n in ("logp", "entropy", "top_idx", "top_logp")}


def _plain_logp(s):
    c = s["case"]
    logits = s["logits"].to(torch.float32)
    top = logits.amax(dim=1, keepdim=True)
    z = (logits - top) / c["temperature"]
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total[:, 0] - torch.where(e > 0, e * z, 0.0).sum(dim=1) / total[:, 0]
    out = {"logp": z.gather(1, s["ids"].long()) - log_total, "entropy": entropy, "top_idx": None, "top_logp": None}
    if c["n"]:
        # whole numbers in the order of the logits, equal ones by their place: the largest are the same wherever they are looked for
        bits = (logits + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) - torch.arange(c["V"], device=DEV)
        at = key.topk(c["n"], dim=1).indices
        out["top_idx"], out["top_logp"] = at.to(torch.int32), z.gather(1, at) - log_total
    return out


def _own_logp_grad(s):
    h = s["handle"]
    h.moe.moe_token_logp_backward(h.ctx, s["logits"], s["ids"], s["dlogp"], s["dentropy"], s["stats"], s["entropy"], s["dlogits"],
                                  temperature=s["case"]["temperature"])
    return {"dlogits": s["dlogits"]}


def _plain_logp_grad(s):
    c = s["case"]
    logits, ids = s["logits"].to(torch.float32), s["ids"].long()
    z = (logits - s["stats"][:, :1]) / c["temperature"]
    p = torch.exp(z) / s["stats"][:, 1:]
    d = s["dlogp"]
    grad = -p * d.sum(dim=1, keepdim=True)
    if c["entropy"]:
        logs = z - torch.log(s["stats"][:, 1:])
        grad = grad - torch.where(p > 0, s["dentropy"][:, None] * p * (logs + s["entropy"][:, None]), 0.0)
    grad.scatter_add_(1, ids, d)
    return {"dlogits": (grad / c["temperature"]).to(TYPES[c["out"]])}


def _own_clip(s):
    h = s["handle"]
    h.moe.moe_grad_norm(h.ctx, s["list"], s["sum_sq"], s["norm"])
    h.moe.moe_clip_grads(h.ctx, s["list"], s["sum_sq"], s["max_norm"], s["out_list"])
    return {"sum_sq": s["sum_sq"], "norm": s["norm"], "grads": s["out_buffers"] or s["buffers"]}


def _plain_clip(s):
    sum_sq = torch.stack([g.to(torch.float64).square().sum() for g in s["grads"]]).sum()[None]
    norm = torch.sqrt(sum_sq)
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).to(torch.float32)
    [o.copy_(g.to(torch.float32) * factor) for g, o in zip(s["grads"], s["outs"] or s["grads"])]
    return {"sum_sq": sum_sq, "norm": norm.to(torch.float32), "grads": s["out_buffers"] or s["buffers"]}


_own = {"embed": _own_embed, "embed_grad": _own_embed_grad, "logp": _own_logp, "logp_grad": _own_logp_grad, "clip": _own_clip}
_plain = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "logp": _plain_logp, "logp_grad": _plain_logp_grad, "clip": _plain_clip}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "embed":
        n = c["T"] * c["d"]
        return {"bytes": n * (BYTES[c["type"]] + BYTES[c["out"]]) + 4 * c["T"], "flops": n}
    if c["kind"] == "embed_grad":
        out = BYTES[c["out"]]
        n = c["T"] * c["d"] * (0.8 if c["padded"] else 1)
        if c["accumulate"]:
            # rows that occur: of text, about a rank r for every T/(r ln V) > 1 and some of the others
            ranks = sum(1 - math.exp(-c["T"] / (r * math.log(c["V"]))) for r in range(1, c["V"] + 1)) if c["load"] == "zipf" else None
            rows = ranks if ranks is not None else c["V"] * (1 - math.exp(-c["T"] / c["V"]))
            return {"bytes": n * BYTES[c["type"]] + 2 * rows * c["d"] * out + 4 * c["T"], "flops": n}
        return {"bytes": n * BYTES[c["type"]] + c["V"] * c["d"] * out + 4 * c["T"], "flops": n}
    if c["kind"] == "logp":
        n = c["rows"] * c["V"]
        return {"bytes": n * BYTES[c["type"]] + c["rows"] * (8 * c["m"] + 8 * c["n"] + 4), "flops": 8 * n}
    if c["kind"] == "logp_grad":
        rows = c["rows"] - (c["rows"] // 4 - c["rows"] // 8 if c["rows"] > 8 else 0)     # (those without a gradient are not read)
        return {"bytes": c["V"] * (rows * BYTES[c["type"]] + c["rows"] * BYTES[c["out"]]) + c["rows"] * (8 * c["m"] + 16), "flops": 8 * rows * c["V"]}
    n = sum(size * BYTES[t] for size, t in zip(_sizes(c), _types(c)))
    return {"bytes": n * (2 if c["clipped"] else 1), "flops": 3 * sum(_sizes(c))}


# ---------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    with torch.no_grad():
        return _exact[case["kind"]](case, prepare(case, seed))


def _exact_embed(c, s):
    y = torch.empty((c["T"], c["d"]), dtype=torch.float64, device=DEV)
    for i in range(0, c["T"], 4096):
        at = s["ids"][i:i + 4096].long()
        y[i:i + 4096] = torch.index_select(s["table"], 0, at).double().mul_(c["scale"])
    return {"y": y}


def _exact_embed_grad(c, s):
    # runs of equal ids in the sorted order, their sums as differences of running sums
    order = torch.argsort(s["ids"], stable=True)
    order = order[s["ids"][order] >= 0]
    seen, count = torch.unique_consecutive(s["ids"][order].long(), return_counts=True)
    end = torch.cumsum(count, dim=0)
    out = torch.zeros((c["V"], c["d"]), dtype=torch.float64, device=DEV)
    for i in range(0, c["d"], 512):
        run = torch.cumsum(s["dy"][order, i:i + 512].double(), dim=0)[end - 1]
        run[1:] -= run[:-1].clone()
        out[seen, i:i + 512] = run * c["scale"]
    return {"dtable": out.add_(s["dtable"].double()) if c["accumulate"] else out}


def _exact_logp(c, s):
    f64, rows, n = torch.float64, c["rows"], c["n"]
    out = {"logp": torch.empty((rows, c["m"]), dtype=f64, device=DEV), "entropy": torch.empty((rows,), dtype=f64, device=DEV),
           "top_idx": torch.empty((rows, n), dtype=torch.int32, device=DEV) if n else None, "top_logp": torch.empty((rows, n), dtype=f64, device=DEV) if n else None}
    for i in range(0, rows, 256):
        at = slice(i, min(i + 256, rows))
        logs = torch.log_softmax(s["logits"][at].to(f64) / c["temperature"], dim=1)
        out["logp"][at] = torch.take_along_dim(logs, s["ids"][at].long(), dim=1)
        out["entropy"][at] = -(logs.exp() * logs).nan_to_num(0.0).sum(dim=1)
        if n:
            by = torch.sort(s["logits"][at], dim=1, descending=True, stable=True).indices[:, :n]
            out["top_idx"][at], out["top_logp"][at] = by.int(), torch.take_along_dim(logs, by, dim=1)
    return out


def _exact_logp_grad(c, s):
    f64, rows, V = torch.float64, c["rows"], c["V"]
    out = torch.empty((rows, V), dtype=f64, device=DEV)
    for i in range(0, rows, 256):
        at = slice(i, min(i + 256, rows))
        logs = torch.log_softmax(s["logits"][at].to(f64) / c["temperature"], dim=1)
        p, d = logs.exp(), s["dlogp"][at].to(f64)
        pick = torch.zeros_like(p).scatter_add_(1, s["ids"][at].long(), d)
        grad = pick - p * pick.sum(dim=1, keepdim=True)
        if c["entropy"]:
            plogs = (p * logs).nan_to_num(0.0)
            grad -= s["dentropy"][at].to(f64)[:, None] * (plogs - p * plogs.sum(dim=1, keepdim=True))
        out[at] = grad / c["temperature"]
    return {"dlogits": out}


def _exact_clip(c, s):
    dots = [torch.dot(v, v) for v in (g.double() for g in s["grads"])]
    sum_sq = sum(dots[1:], dots[0])
    factor = min(1.0, s["max_norm"] / math.sqrt(float(sum_sq)))
    return {"sum_sq": sum_sq[None], "norm": sum_sq.sqrt()[None], "grads": {t: b.double() * factor for t, b in s["buffers"].items()}}


_exact = {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "logp": _exact_logp, "logp_grad": _exact_logp_grad, "clip": _exact_clip}
