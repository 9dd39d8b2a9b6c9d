"""Workloads of the operators around a reduced activation: the residual and norm
that consume a tensor-parallel reduction, and the routing, ordering and weighted
reduction of a mixture of experts.

A case is a dict of plain values: ``op`` names the operator and its direction,
the other fields give types, sizes and options.  ``listed()`` are the standing
cases, ``draw(rng)`` gives one more of the same ranges, ``prepare`` builds what a
program holds before the call, ``run`` makes one pass (the operators' plain form
in elementary torch, or with ``own`` the library's calls), ``work`` counts the
bytes and operations a pass cannot do without, and ``exact`` computes the same
outputs in 64 bits.

Ranges: one token (a decode step) to 65536 (a prefill or a training batch), rows
of 64 to 16384 elements, whole and odd, 1 to 16 partial sums, 8 to 1024 experts
with 1 to 16 choices, in fp32, bf16 and fp16, with 8-bit outputs by row or group.
"""
from __future__ import annotations

import math

import torch

own = False   # True: run() calls the library

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-6
E4M3_MAX, LEAST_AMAX = 448.0, 2.0 ** -100
ROUTED_SCALE = 2.5
MOST_BYTES = 1000 << 20   # read and written by a drawn case


def listed():
    return [
        # one decode step's hidden state after a tensor-parallel reduction over 8 ranks,
        # for an 8-bit product with a scale for each token: all launch and call cost
        {"name": "norm_token", "op": "norm", "rows": 1, "hidden": 4096, "nsrc": 8,
         "dtype": "bf16", "residual": True, "out": False, "group": 0, "pad": 0},
        # a prefill's hidden states over 8 ranks; bf16 for the router, 8 bits in groups for
        # the experts
        {"name": "norm_prefill", "op": "norm", "rows": 8192, "hidden": 4096, "nsrc": 8,
         "dtype": "bf16", "residual": True, "out": True, "group": 128, "pad": 0},
        # rows of odd length and stride, fp16, two ranks, no 8-bit output
        {"name": "norm_ragged", "op": "norm", "rows": 1999, "hidden": 5003, "nsrc": 2,
         "dtype": "f16", "residual": True, "out": True, "group": -1, "pad": 5},
        # a training step's backward pass, the residual stream's gradient joining
        {"name": "norm_grad", "op": "norm_grad", "rows": 16384, "hidden": 4096, "dtype": "bf16",
         "dsum": True},
        # a decode batch through a sigmoid router with balance bias and groups of experts
        {"name": "route_tokens", "op": "route", "tokens": 4, "experts": 256, "topk": 8,
         "dtype": "f32", "score": "sigmoid", "bias": True, "groups": 8, "group_topk": 4,
         "renorm": True, "masked": 0.0},
        # the same router over a long prefill, some of whose rows are padding
        {"name": "route_prefill", "op": "route", "tokens": 65536, "experts": 256, "topk": 8,
         "dtype": "f32", "score": "sigmoid", "bias": True, "groups": 8, "group_topk": 4,
         "renorm": True, "masked": 0.05},
        # a softmax router's backward pass; not renormalised, so every logit has a gradient
        {"name": "route_grad", "op": "route_grad", "tokens": 32768, "experts": 128, "topk": 6,
         "dtype": "bf16", "score": "softmax", "renorm": False, "masked": 0.0},
        # a decode batch's rows sent to their experts
        {"name": "dispatch_tokens", "op": "dispatch", "tokens": 61, "hidden": 4096,
         "experts": 256, "topk": 8, "dtype": "bf16", "dropped": 0.0},
        # a prefill's 8-bit rows with their scales, some slots on other ranks' experts
        {"name": "dispatch_prefill", "op": "dispatch", "tokens": 16384, "hidden": 4096,
         "experts": 128, "topk": 8, "dtype": "e4m3", "dropped": 0.1},
        # a decode batch's expert outputs, added to a shared expert's
        {"name": "combine_tokens", "op": "combine", "tokens": 8, "hidden": 4096, "experts": 256,
         "topk": 8, "dtype": "bf16", "base": True, "weights": True, "dropped": 0.0},
        # the same for a prefill
        {"name": "combine_prefill", "op": "combine", "tokens": 12288, "hidden": 4096,
         "experts": 128, "topk": 8, "dtype": "bf16", "base": True, "weights": True,
         "dropped": 0.0},
        # its backward pass in fp32 with rows of odd length
        {"name": "combine_grad", "op": "combine_grad", "tokens": 4096, "hidden": 2501,
         "experts": 64, "topk": 4, "dtype": "f32", "dropped": 0.1},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """A row's elements, log-uniform; half of the draws 4, 5 or 7 times a power of two."""
    n = _log_int(rng, lo, hi)
    if rng.random() < 0.5:
        return n | 1
    return max(lo, max(m << j for m in (4, 5, 7) for j in range(12) if m << j <= n))


def draw(rng):
    op = rng.choices(["norm", "norm_grad", "route", "route_grad", "dispatch", "combine",
                      "combine_grad"], [5, 2, 3, 2, 3, 3, 2])[0]
    case = {"op": op, "dtype": rng.choices(["bf16", "f16", "f32"], [4, 1, 1])[0]}
    if op in ("norm", "norm_grad"):
        case.update(rows=_log_int(rng, 1, 16384), hidden=_length(rng, 64, 16384))
        if op == "norm":
            group = rng.choice([-1, 0, 32, 128])
            case.update(nsrc=rng.choice([1, 1, 2, 3, 4, 8, 8, 16]),
                        residual=rng.random() < 0.7,
                        out=group < 0 or rng.random() < 0.5, group=group,
                        pad=rng.choice([0, 0, 0, 1, 8, 13]))
        else:
            case.update(dsum=rng.random() < 0.7)
        size = "rows"
    elif op in ("route", "route_grad"):
        experts = rng.choice([8, 16, 32, 60, 64, 96, 128, 160, 256, 384, 512, 1000, 1024])
        case.update(tokens=_log_int(rng, 1, 65536), experts=experts,
                    topk=min(experts, rng.choice([1, 2, 4, 6, 8, 8, 10, 16])),
                    score=rng.choice(["softmax", "sigmoid"]), renorm=rng.random() < 0.6,
                    masked=rng.choice([0.0, 0.0, 0.05, 0.3]))
        if op == "route":
            groups = rng.choice([1, 1] + [g for g in (2, 4, 8, 16) if experts % g == 0])
            case.update(bias=rng.random() < 0.5, groups=groups,
                        group_topk=rng.randint(max(1, groups // 2), groups))
        size = "tokens"
    else:
        experts = rng.choice([8, 16, 60, 64, 128, 160, 256, 512])
        case.update(tokens=_log_int(rng, 1, 16384), hidden=_length(rng, 64, 8192),
                    experts=experts, topk=min(experts, rng.choice([1, 2, 4, 6, 8, 8, 10, 16])),
                    dropped=rng.choice([0.0, 0.0, 0.1, 0.8]))
        if op == "dispatch":
            case.update(dtype=rng.choice(["bf16", "e4m3", "f32", "f16"]))
        elif op == "combine":
            case.update(base=rng.random() < 0.5, weights=rng.random() < 0.8)
        size = "tokens"
    while case[size] > 1 and work(case)["bytes"] > MOST_BYTES:
        case[size] = case[size] * 3 // 4
    return case


def work(case):
    op, es = case["op"], SIZE[case["dtype"]]
    if op == "norm":
        n = case["rows"] * case["hidden"]
        b = n * es * (case["nsrc"] + case["residual"] + 1 + case["out"])
        if case["group"] >= 0:
            b += n + 4 * case["rows"] * _groups(case["hidden"], case["group"])
        return {"bytes": b + case["hidden"] * es + 4 * case["rows"],
                "flops": n * (case["nsrc"] + 6)}
    if op == "norm_grad":
        n = case["rows"] * case["hidden"]
        return {"bytes": n * es * (3 + case["dsum"]) + case["hidden"] * (es + 4)
                + 4 * case["rows"], "flops": 10 * n}
    if op in ("route", "route_grad"):
        n, k = case["tokens"] * case["experts"], case["tokens"] * case["topk"]
        if op == "route":
            return {"bytes": n * es + 8 * k + 4 * case["experts"] * case["bias"],
                    "flops": n * 4 + k * 4}
        # what is renormalised, and a sigmoid, needs the chosen logits alone
        dense = case["score"] == "softmax" and not case["renorm"]
        return {"bytes": n * es + (n if dense else k) * es + 8 * k,
                "flops": (n if dense else k) * 6}
    n, k = case["tokens"] * case["hidden"], case["topk"]
    kept = k * (1 - case["dropped"])
    if op == "dispatch":
        scales = 4 * case["tokens"] * _groups(case["hidden"], 128) if case["dtype"] == "e4m3" else 0
        return {"bytes": (n * es + scales) * (1 + kept) + case["tokens"] * k * 8, "flops": 0}
    if op == "combine":
        return {"bytes": n * es * (kept + 1 + case["base"]) + case["tokens"] * k * 8,
                "flops": 2 * n * kept}
    return {"bytes": n * es * (1 + 2 * kept) + case["tokens"] * k * 12, "flops": 3 * n * kept}


def _groups(hidden, group):
    return 1 if group == 0 else -(-hidden // group)


# ------------------------------------------------------------------ inputs --
def _normal(g, shape, scale=1.0):
    return torch.empty(shape, device="cuda").normal_(0, scale, generator=g)


def _activations(g, rows, hidden, dtype, scale=1.0):
    """Values as hidden states have them: a few channels much larger than the others."""
    channel = torch.where(torch.rand(hidden, device="cuda", generator=g) < 0.01, 8.0, 1.0)
    return (_normal(g, (rows, hidden), scale) * channel).to(dtype)


def _strided(x, pad):
    """x as a view of rows pad elements further apart."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _logits(g, case):
    t, e = case["tokens"], case["experts"]
    x = _normal(g, (t, e), 1.5) + _normal(g, (1, e), 0.5)   # some experts are more popular
    if case["masked"]:   # experts switched off for a token, and padding rows
        x.masked_fill_(torch.rand((t, e), device="cuda", generator=g) < case["masked"], -math.inf)
        x.masked_fill_(torch.rand((t, 1), device="cuda", generator=g) < case["masked"], -math.inf)
    return x.to(TORCH[case["dtype"]])


def _ids(g, case):
    """topk distinct experts for each token, some more popular than others, -1 where dropped."""
    t, e, k = case["tokens"], case["experts"], case["topk"]
    x = _normal(g, (t, e)) + _normal(g, (1, e), 0.7)
    ids = x.argsort(1, descending=True)[:, :k].int()
    if case["dropped"]:
        ids.masked_fill_(torch.rand((t, k), device="cuda", generator=g) < case["dropped"], -1)
    return ids


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt, dev = case["op"], TORCH[case["dtype"]], "cuda"
    s = {"case": case}
    if op == "norm":
        r, h = case["rows"], case["hidden"]
        s["srcs"] = [_strided(_activations(g, r, h, dt, 0.5), case["pad"])
                     for _ in range(case["nsrc"])]
        s["residual"] = _activations(g, r, h, dt) if case["residual"] else None
        s["weight"] = (1 + _normal(g, (h,), 0.2)).to(dt)
        s["sum"] = torch.empty((r, h), dtype=dt, device=dev)
        s["rstd"] = torch.empty(r, device=dev)
        s["out"] = torch.empty((r, h), dtype=dt, device=dev) if case["out"] else None
        s["out8"] = s["scale"] = None
        if case["group"] >= 0:
            s["out8"] = torch.empty((r, h), dtype=TORCH["e4m3"], device=dev)
            s["scale"] = torch.empty((r, _groups(h, case["group"])), device=dev)
    elif op == "norm_grad":
        r, h = case["rows"], case["hidden"]
        s["dout"] = _normal(g, (r, h), 0.1).to(dt)
        s["sum"] = _activations(g, r, h, dt)
        s["rstd"] = (s["sum"].float().square().mean(1) + EPS).rsqrt()
        s["weight"] = (1 + _normal(g, (h,), 0.2)).to(dt)
        s["dsum"] = _normal(g, (r, h), 0.1).to(dt) if case["dsum"] else None
        s["dx"] = torch.empty((r, h), dtype=dt, device=dev)
        s["dweight"] = torch.empty(h, device=dev)
    elif op in ("route", "route_grad"):
        t, e, k = case["tokens"], case["experts"], case["topk"]
        s["logits"] = _logits(g, case)
        if op == "route":
            s["bias"] = _normal(g, (e,), 0.1) if case["bias"] else None
            s["ids"] = torch.empty((t, k), dtype=torch.int32, device=dev)
            s["weights"] = torch.empty((t, k), device=dev)
        else:
            top = s["logits"].float().sort(dim=1, descending=True, stable=True)
            s["ids"] = top.indices[:, :k].masked_fill(top.values[:, :k] == -math.inf, -1).int()
            s["dweights"] = _normal(g, (t, k))
            s["dlogits"] = torch.empty((t, e), dtype=dt, device=dev)
    else:
        t, h, k, e = case["tokens"], case["hidden"], case["topk"], case["experts"]
        ids = _ids(g, case)
        if op == "dispatch":
            s["ids"] = ids
            x = _activations(g, t, h, torch.float32)
            s["x"] = x.clamp(-E4M3_MAX, E4M3_MAX).to(dt) if case["dtype"] == "e4m3" else x.to(dt)
            # rows of dropped slots are never written: the program's buffer holds zeros there
            s["out"] = torch.zeros((t * k, h), dtype=dt, device=dev)
            s["scale"] = s["out_scale"] = None
            if case["dtype"] == "e4m3":
                n = _groups(h, 128)
                s["scale"] = torch.rand((t, n), device=dev, generator=g) * 0.1 + 1e-3
                s["out_scale"] = torch.zeros((t * k, n), device=dev)
            s["counts"] = torch.empty(e, dtype=torch.int32, device=dev)
            s["offsets"] = torch.empty(e + 1, dtype=torch.int32, device=dev)
            s["pos"] = torch.empty((t, k), dtype=torch.int32, device=dev)
        else:
            # the rows as a dispatch by expert leaves them
            flat = torch.where(ids < 0, e, ids).flatten()
            pos = torch.empty_like(flat)
            pos[flat.argsort(stable=True)] = torch.arange(t * k, dtype=torch.int32, device=dev)
            s["pos"] = torch.where(ids < 0, -1, pos.view(t, k))
            s["y"] = _normal(g, (t * k, h)).to(dt)
            w = torch.rand((t, k), device=dev, generator=g) + 0.05
            w = w / w.sum(1, keepdim=True)
            if op == "combine":
                s["weights"] = w if case["weights"] else None
                s["base"] = _activations(g, t, h, dt) if case["base"] else None
                s["out"] = torch.empty((t, h), dtype=dt, device=dev)
            else:
                s["weights"] = w
                s["dout"] = _normal(g, (t, h), 0.1).to(dt)
                s["dy"] = torch.zeros((t * k, h), dtype=dt, device=dev)
                s["dweights"] = torch.empty((t, k), device=dev)
    return s


# ------------------------------------------------------------- plain forms --
def _plain_norm(s):
    c = s["case"]
    dt = TORCH[c["dtype"]]
    h = torch.stack(s["srcs"]).float().sum(0)
    if s["residual"] is not None:
        h = h + s["residual"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * s["weight"].float()
    got = {"sum": h.to(dt), "rstd": rstd}
    if c["out"]:
        got["out"] = y.to(dt)
    if c["group"] >= 0:
        n, width = _groups(c["hidden"], c["group"]), c["group"] or c["hidden"]
        pad = n * width - c["hidden"]
        parts = torch.nn.functional.pad(y, (0, pad)).view(c["rows"], n, width)
        scale = parts.abs().amax(2).clamp(min=LEAST_AMAX) / E4M3_MAX
        q = (parts / scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(c["rows"], n * width)
        got["out8"] = q[:, :c["hidden"]].to(TORCH["e4m3"])
        got["scale"] = scale
    return got


def _plain_norm_grad(s):
    h, rstd = s["sum"].float(), s["rstd"][:, None]
    dout = s["dout"].float()
    g = dout * s["weight"].float()
    dx = rstd * (g - h * rstd.square() * (g * h).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["dout"].dtype), "dweight": (dout * h * rstd).sum(0)}


def _best(key, k):
    """The k best of each row, in order, ties to the lowest index."""
    top = (key + 0.0).sort(dim=-1, descending=True, stable=True)
    return top.values[..., :k], top.indices[..., :k]


def _plain_route(s):
    c = s["case"]
    x = s["logits"].float()
    t, e, k = c["tokens"], c["experts"], c["topk"]
    score = 1.0 / (1.0 + torch.exp(-x)) if c["score"] == "sigmoid" else x
    key = score if s["bias"] is None else score + s["bias"]
    key = torch.where(x == -math.inf, -math.inf, key)
    if c["groups"] > 1:
        part = key.view(t, c["groups"], e // c["groups"])
        rank = _best(part, 2)[0].sum(2)
        chosen = torch.zeros_like(rank).scatter_(1, _best(rank, c["group_topk"])[1], 1.0)
        key = torch.where(chosen[:, :, None] > 0, part, -math.inf).view(t, e)
    best, ids = _best(key, k)
    none = best == -math.inf
    if c["score"] == "sigmoid":
        w = score.gather(1, ids).masked_fill(none, 0.0)
        if c["renorm"]:
            total = w.sum(1, keepdim=True)
            w = torch.where(total == 0, 0.0, w / total)
    else:
        top = x.gather(1, ids).masked_fill(none, -math.inf)
        over = top if c["renorm"] else x
        m = over.amax(1, keepdim=True)
        w = torch.exp(top - m) / torch.exp(over - m).sum(1, keepdim=True)
        w = w.masked_fill(none, 0.0)
    return {"ids": ids.int().masked_fill(none, -1), "weights": w * ROUTED_SCALE}


def _plain_route_grad(s):
    c = s["case"]
    x = s["logits"].float()
    ids, none = s["ids"].clamp(min=0).long(), s["ids"] < 0
    dw = (s["dweights"] * ROUTED_SCALE).masked_fill(none, 0.0)
    if c["score"] == "sigmoid":
        p = (1.0 / (1.0 + torch.exp(-x.gather(1, ids)))).masked_fill(none, 0.0)
        dp = dw
        if c["renorm"]:
            total = p.sum(1, keepdim=True)
            inv = torch.where(total == 0, 0.0, 1.0 / total)
            dp = (dw - (dw * p).sum(1, keepdim=True) * inv) * inv
        dtop = dp * p * (1.0 - p)
        dx = torch.zeros_like(x).scatter_add_(1, ids, dtop.masked_fill(none, 0.0))
    elif c["renorm"]:
        top = x.gather(1, ids).masked_fill(none, -math.inf)
        p = torch.exp(top - top.amax(1, keepdim=True)).masked_fill(none, 0.0)
        total = p.sum(1, keepdim=True)
        p = torch.where(total == 0, 0.0, p / total)
        dx = torch.zeros_like(x).scatter_add_(1, ids, p * (dw - (dw * p).sum(1, keepdim=True)))
    else:
        m = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
        total = p.sum(1, keepdim=True)
        p = torch.where(total == 0, 0.0, p / total)
        dp = torch.zeros_like(x).scatter_add_(1, ids, dw)
        dx = p * (dp - (dp * p).sum(1, keepdim=True))
    return {"dlogits": dx.to(s["logits"].dtype)}


def _plain_dispatch(s):
    c = s["case"]
    t, k, e = c["tokens"], c["topk"], c["experts"]
    ids = s["ids"]
    flat = torch.where(ids < 0, e, ids).flatten().long()
    counts = torch.zeros(e + 1, dtype=torch.int32, device=ids.device)
    counts.scatter_add_(0, flat, torch.ones_like(flat, dtype=torch.int32))
    offsets = torch.cat([counts.new_zeros(1), counts[:e].cumsum(0, dtype=torch.int32)])
    row = torch.empty_like(flat)
    row[flat.argsort(stable=True)] = torch.arange(t * k, device=ids.device)
    # dropped slots go to a row past the end
    to = torch.where(ids.flatten() < 0, t * k, row)

    def moved(x):
        bits = x.view(torch.uint8)
        rows = bits.new_zeros((t * k + 1, bits.shape[1]))
        rows[to] = bits.repeat_interleave(k, 0)
        return rows[:t * k].view(x.dtype)

    got = {"counts": counts[:e], "offsets": offsets,
           "pos": torch.where(ids < 0, -1, row.view(t, k).int()), "out": moved(s["x"])}
    if s["scale"] is not None:
        got["out_scale"] = moved(s["scale"])
    return got


def _plain_combine(s):
    pos = s["pos"]
    y = s["y"][pos.clamp(min=0).long()].float()
    if s["weights"] is not None:
        y = y * s["weights"][:, :, None]
    out = y.masked_fill_((pos < 0)[:, :, None], 0.0).sum(1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return {"out": out.to(s["y"].dtype)}


def _plain_combine_grad(s):
    pos, none = s["pos"], s["pos"] < 0
    t, k, h = pos.shape[0], pos.shape[1], s["y"].shape[1]
    dout = s["dout"].float()[:, None, :]
    dweights = (s["y"][pos.clamp(min=0).long()].float() * dout).sum(2).masked_fill(none, 0.0)
    dy = s["y"].new_zeros((t * k + 1, h))
    dy[torch.where(none, t * k, pos).long()] = (dout * s["weights"][:, :, None]).to(dy.dtype)
    return {"dy": dy[:t * k], "dweights": dweights}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "route": _plain_route,
         "route_grad": _plain_route_grad, "dispatch": _plain_dispatch,
         "combine": _plain_combine, "combine_grad": _plain_combine_grad}


# -------------------------------------------------------- the library's calls --
def _own(s):
    import paper_2510_20171_amd as xr
    c = s["case"]
    op = c["op"]
    if op == "norm":
        xr.fold_norm(s["srcs"], s["out"], residual=s["residual"], weight=s["weight"],
                     sum=s["sum"], out8=s["out8"], scale=s["scale"], rstd=s["rstd"],
                     group=max(0, c["group"]), eps=EPS)
        names = ("sum", "rstd") + (("out",) if c["out"] else ()) + (
            ("out8", "scale") if c["group"] >= 0 else ())
    elif op == "norm_grad":
        xr.fold_norm_grad(s["dout"], s["sum"], s["rstd"], s["dx"], weight=s["weight"],
                          dsum=s["dsum"], dweight=s["dweight"])
        names = ("dx", "dweight")
    elif op == "route":
        xr.route(s["logits"], s["ids"], s["weights"], score=c["score"], bias=s["bias"],
                 groups=c["groups"], group_topk=c["group_topk"], group_score=2,
                 renorm=c["renorm"], scale=ROUTED_SCALE)
        names = ("ids", "weights")
    elif op == "route_grad":
        xr.route_grad(s["logits"], s["ids"], s["dweights"], s["dlogits"], score=c["score"],
                      renorm=c["renorm"], scale=ROUTED_SCALE)
        names = ("dlogits",)
    elif op == "dispatch":
        xr.dispatch_plan(s["ids"], s["counts"], s["offsets"], s["pos"])
        xr.dispatch(s["x"], s["pos"], s["out"], scale=s["scale"], out_scale=s["out_scale"])
        names = ("counts", "offsets", "pos", "out") + (
            ("out_scale",) if s["scale"] is not None else ())
    elif op == "combine":
        xr.combine(s["y"], s["pos"], s["out"], weights=s["weights"], base=s["base"])
        names = ("out",)
    else:
        xr.combine_grad(s["dout"], s["y"], s["pos"], s["weights"], s["dy"], s["dweights"])
        names = ("dy", "dweights")
    return {n: s[n] for n in names}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- in 64 bits --
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f = torch.float64
    if op == "norm":
        h = torch.zeros((case["rows"], case["hidden"]), dtype=f, device="cuda")
        for x in s["srcs"] + ([s["residual"]] if case["residual"] else []):
            h += x
        norm = torch.linalg.vector_norm(h, dim=1)
        rstd = (norm * norm / case["hidden"] + EPS) ** -0.5
        y = torch.einsum("rh,r,h->rh", h, rstd, s["weight"].to(f))
        got = {"sum": h, "rstd": rstd}
        if case["out"]:
            got["out"] = y
        if case["group"] >= 0:
            columns = torch.arange(case["hidden"], device="cuda") // (case["group"] or case["hidden"])
            scale = torch.zeros((case["rows"], _groups(case["hidden"], case["group"])), dtype=f,
                                device="cuda")
            scale.scatter_reduce_(1, columns.expand_as(y), y.abs(), "amax")
            scale = torch.maximum(scale, torch.full_like(scale, LEAST_AMAX)) / E4M3_MAX
            got["out8"] = y / scale[:, columns]
            got["scale"] = scale
        return got
    if op == "norm_grad":
        h, dout, w, rstd = (s[n].to(f) for n in ("sum", "dout", "weight", "rstd"))
        n = h * rstd[:, None]
        g = torch.einsum("rh,h->rh", dout, w)
        dx = (g - n * (torch.einsum("rh,rh->r", g, n) / case["hidden"])[:, None]) * rstd[:, None]
        return {"dx": dx + s["dsum"] if case["dsum"] else dx,
                "dweight": torch.einsum("rh,rh->h", dout, n)}
    if op in ("route", "route_grad"):
        x = s["logits"].to(f)
        off = x == -math.inf
        sigmoid = case["score"] == "sigmoid"
        if op == "route":
            key = (x.sigmoid() if sigmoid else x) + (s["bias"] if case["bias"] else 0)
            key[off] = -math.inf
            if case["groups"] > 1:
                part = key.unflatten(1, (case["groups"], -1))
                rank = part.topk(min(2, part.shape[2]), 2).values.sum(2)
                least = rank.sort(dim=1, descending=True, stable=True).indices[:, case["group_topk"]:]
                key = part.scatter(1, least[:, :, None].expand(-1, -1, part.shape[2]),
                                   -math.inf).flatten(1)
            ids = key.sort(dim=1, descending=True, stable=True).indices[:, :case["topk"]]
            none = key.gather(1, ids) == -math.inf
        else:
            ids, none = s["ids"].clamp(min=0).long(), s["ids"] < 0
        # every expert's share of the weight, and the chosen ones' of it
        on = torch.zeros_like(off).scatter_(1, ids, True) & ~off
        if sigmoid:
            share = x.sigmoid() * (on if case["renorm"] else 1)
            total = share.sum(1, keepdim=True) if case["renorm"] else torch.ones_like(x[:, :1])
        else:
            share = torch.where(on if case["renorm"] else ~off, (x - x.amax(1, keepdim=True)).exp(), 0)
            total = share.sum(1, keepdim=True)
        p = torch.where(total == 0, 0, share / total)
        if op == "route":
            return {"ids": None, "weights": p.gather(1, ids).masked_fill(none, 0) * ROUTED_SCALE}
        dw = torch.zeros_like(x).scatter_add_(1, ids, s["dweights"].to(f).masked_fill(none, 0))
        dw = dw * ROUTED_SCALE
        if sigmoid:
            mean = (dw * p).sum(1, keepdim=True) if case["renorm"] else 0
            d = torch.where(on & (total > 0), (dw - mean) / total, 0)
            return {"dlogits": d * x.sigmoid() * (1 - x.sigmoid())}
        return {"dlogits": p * (dw - (dw * p).sum(1, keepdim=True))}
    if op == "dispatch":
        k = case["topk"]
        flat = s["ids"].flatten().cpu().long()
        slots = torch.cat([torch.nonzero(flat == e).flatten() for e in range(case["experts"])])
        token = (slots // k).cuda()

        def moved(x, out):
            out.view(torch.uint8)[:len(token)] = x.view(torch.uint8)[token]
            return out

        got = {"counts": None, "offsets": None, "pos": None, "out": moved(s["x"], s["out"])}
        if s["scale"] is not None:
            got["out_scale"] = moved(s["scale"], s["out_scale"])
        return got
    pos = s["pos"].long()
    at, slot = torch.nonzero(pos >= 0, as_tuple=True)
    rows = pos[at, slot]
    if op == "combine":
        out = torch.zeros((case["tokens"], case["hidden"]), dtype=f, device="cuda")
        if case["base"]:
            out += s["base"]
        y = s["y"][rows].to(f)
        if case["weights"]:
            y *= s["weights"][at, slot][:, None]
        return {"out": out.index_add_(0, at, y)}
    dy = torch.zeros(s["y"].shape, dtype=f, device="cuda")
    dy[rows] = s["weights"][at, slot][:, None].to(f) * s["dout"][at]
    dweights = torch.zeros(pos.shape, dtype=f, device="cuda")
    dweights[at, slot] = torch.einsum("nh,nh->n", s["dout"][at].to(f), s["y"][rows].to(f))
    return {"dy": dy, "dweights": dweights}
