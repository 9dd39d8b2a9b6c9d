"""Workloads of the operators between dispatch and combine: the experts' matrix
products over ragged rows with their gradients, the gated activation between
them, and 4-bit microscaled quantisation of rows and weights.

A case is a dict of plain values: ``op`` names the operator and its direction,
the other fields give types, sizes and options.  ``listed()`` are the standing
cases, ``draw(rng)`` gives one more of the same ranges, ``prepare`` builds what a
program holds before the call, ``run`` makes one pass (the operators' plain form
in elementary torch, or with ``own`` the library's calls), ``work`` counts the
bytes and operations a pass cannot do without, and ``exact`` computes the same
outputs in 64 bits.

Ranges: one token (a decode step) to 4096 tokens with 1 to 8 experts each, which
lie together by expert as dispatch leaves them; 1 to 256 experts, some without a
row; products of 64 to 8192 by 64 to 8192, whole and odd, in fp32, bf16, fp16,
e4m3 with a scale for every 128 elements (weights: 128 x 128), and mx4: 4-bit
e2m1 values, two a byte, with an 8-bit power of two for every 32.
"""
from __future__ import annotations

import math

import torch

own = False   # True: run() calls the library

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "e4m3": torch.float8_e4m3fn, "mx4": torch.uint8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1 + 4 / 128, "mx4": 0.5 + 1 / 32}
E4M3_MAX, LEAST_AMAX = 448.0, 2.0 ** -100
BLOCK = 128           # elements that share a scale of an e4m3 operand
MX = 32               # elements that share a scale of an mx4 operand
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
MOST_BYTES, MOST_FLOPS = 1200 << 20, 500e9   # of a drawn case


def listed():
    return [
        # one decode step's token through its 8 of 64 experts: weights are read once
        {"name": "product_token", "op": "product", "tokens": 1, "topk": 8, "experts": 64, "n": 4096,
         "k": 4096, "dtype": "bf16", "transpose": False, "dropped": 0.0},
        # a decode batch with 4-bit weights; its rows are quantised on the way
        {"name": "product_decode_mx4", "op": "product", "tokens": 61, "topk": 8, "experts": 128,
         "n": 4096, "k": 4096, "dtype": "mx4", "transpose": False, "dropped": 0.0},
        # a prefill's (or a training step's) second product of an expert, rows by expert
        {"name": "product_prefill", "op": "product", "tokens": 4096, "topk": 8, "experts": 64,
         "n": 4096, "k": 2048, "dtype": "bf16", "transpose": False, "dropped": 0.0},
        # its first product with 8-bit rows and weights, some slots on other ranks' experts
        {"name": "product_prefill_e4m3", "op": "product", "tokens": 4096, "topk": 8, "experts": 64,
         "n": 4096, "k": 4096, "dtype": "e4m3", "transpose": False, "dropped": 0.1},
        # the same with 4-bit rows and weights
        {"name": "product_prefill_mx4", "op": "product", "tokens": 4096, "topk": 8, "experts": 64,
         "n": 4096, "k": 4096, "dtype": "mx4", "transpose": False, "dropped": 0.0},
        # a training step's gradient of the rows: the weights as they lie, the other way round
        {"name": "product_dx", "op": "product", "tokens": 4096, "topk": 8, "experts": 64, "n": 2048,
         "k": 4096, "dtype": "bf16", "transpose": True, "dropped": 0.0},
        # and of the weights: each expert's rows are what is summed over
        {"name": "product_dw", "op": "product_grad", "tokens": 4096, "topk": 8, "experts": 64,
         "n": 4096, "k": 2048, "dtype": "bf16", "dropped": 0.0},
        # the same of a small layer of odd sizes in fp32
        {"name": "product_dw_odd", "op": "product_grad", "tokens": 1000, "topk": 2, "experts": 8,
         "n": 515, "k": 1027, "dtype": "f32", "dropped": 0.1},
        # a prefill's gated activation, in 8 bits for the second product
        {"name": "gate_prefill", "op": "gate", "tokens": 4096, "topk": 8, "experts": 64,
         "width": 2048, "dtype": "bf16", "group": 128, "dropped": 0.1},
        # its backward pass, rows of odd length
        {"name": "gate_grad", "op": "gate_grad", "tokens": 2048, "topk": 4, "experts": 60,
         "width": 2501, "dtype": "bf16", "dropped": 0.1},
        # a decode batch's rows to 4 bits and back: all launch and call cost
        {"name": "mx4_rows", "op": "mx4", "rows": 61, "columns": 4096, "dtype": "bf16"},
        # the rows of 32 experts' weights of 2048 x 4096, from the fp32 that training keeps
        {"name": "mx4_weights", "op": "mx4", "rows": 65536, "columns": 4096, "dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """A row's elements, log-uniform; two thirds of the draws 4, 5 or 7 times a power of two."""
    n = _log_int(rng, lo, hi)
    if rng.random() < 0.33:
        return n | 1
    return max(lo, max(m << j for m in (4, 5, 7) for j in range(12) if m << j <= n))


def draw(rng):
    op = rng.choices(["product", "product_grad", "gate", "gate_grad", "mx4"], [6, 3, 2, 2, 2])[0]
    case = {"op": op, "dtype": rng.choices(["bf16", "f16", "f32"], [4, 1, 1])[0]}
    if op == "mx4":
        case.update(rows=_log_int(rng, 1, 65536), columns=_length(rng, 64, 8192))
        size, other = "rows", "columns"
    else:
        experts = rng.choice([1, 8, 16, 60, 64, 128, 256])
        case.update(tokens=_log_int(rng, 1, 4096), experts=experts,
                    topk=min(experts, rng.choice([1, 2, 4, 6, 8, 8])),
                    dropped=rng.choice([0.0, 0.0, 0.1, 0.8]))
        size, other = "tokens", "experts"
        if op in ("gate", "gate_grad"):
            case.update(width=_length(rng, 64, 8192))
            if op == "gate":
                case.update(group=rng.choice([0, 32, 128, 128]))
        else:
            case.update(n=_length(rng, 64, 8192), k=_length(rng, 64, 8192))
            if op == "product":
                case.update(dtype=rng.choices(["bf16", "f16", "f32", "e4m3", "mx4"], [4, 1, 1, 3, 3])[0])
                case.update(transpose=case["dtype"] in ("bf16", "f16", "f32") and rng.random() < 0.4)

    def over():   # fp32 products run at a tenth of the rate
        w = work(case)
        return w["bytes"] > MOST_BYTES or w["flops"] * (4 if case["dtype"] == "f32" else 1) > MOST_FLOPS

    while over():
        if case[size] > 64 or case[other] == 1:
            case[size] = case[size] * 3 // 4
        else:
            case[other] = max(1, case[other] // 2)
            case["topk"] = min(case["topk"], case[other])
    return case


def work(case):
    op = case["op"]
    if op == "mx4":   # the codes and scales written once, besides the rows and the values
        n = case["rows"] * case["columns"]
        return {"bytes": n * (2 * SIZE[case["dtype"]] + SIZE["mx4"]), "flops": 4 * n}
    kept = case["tokens"] * case["topk"] * (1 - case["dropped"])
    es = SIZE[case["dtype"]]
    if op == "gate":
        n = kept * case["width"]
        out = 1 + 4 / case["group"] if case["group"] else es
        return {"bytes": n * (2 * es + out), "flops": 6 * n}
    if op == "gate_grad":
        n = kept * case["width"]
        return {"bytes": 5 * n * es, "flops": 12 * n}
    n, k = case["n"], case["k"]
    flops = 2 * kept * n * k
    if op == "product_grad":
        return {"bytes": kept * (n + k) * es + case["experts"] * n * k * es, "flops": flops}
    used = min(case["experts"], kept)   # about so many experts have a row
    es_rows = SIZE["bf16"] if case["dtype"] == "mx4" else es
    es_out = es if case["dtype"] in ("f32", "bf16", "f16") else 2
    return {"bytes": used * n * k * es + kept * (k * es_rows + n * es_out), "flops": flops}


# ------------------------------------------------------------------ inputs --
def _normal(g, shape, scale=1.0):
    return torch.empty(shape, device="cuda").normal_(0, scale, generator=g)


def _activations(g, rows, columns, scale=1.0):
    """Values as hidden states have them: a few channels much larger than the others."""
    channel = torch.where(torch.rand(columns, device="cuda", generator=g) < 0.01, 8.0, 1.0)
    return _normal(g, (rows, columns), scale) * channel


def _blocks(n, size):
    return -(-n // size)


def _padded(x, columns):
    return torch.nn.functional.pad(x, (0, columns - x.shape[-1]))


def _spread(scale, size, columns):
    """A scale for every `size` elements, for each of `columns`."""
    return scale.repeat_interleave(size, -1)[..., :columns]


def _to_e4m3(x, rows, size):
    """e4m3 values of x (..., r, k) and their scales by `rows` x `size` elements."""
    r, k = x.shape[-2:]
    by = _padded(x, _blocks(k, size) * size).unflatten(-1, (-1, size)).abs().amax(-1)
    if rows > 1:
        by = _padded(by.mT, _blocks(r, rows) * rows).unflatten(-1, (-1, rows)).amax(-1).mT
    scale = by.clamp(min=LEAST_AMAX).contiguous() / E4M3_MAX
    wide = _spread(scale, size, k)
    if rows > 1:
        wide = _spread(wide.mT, rows, r).mT
    return (x / wide).clamp(-E4M3_MAX, E4M3_MAX).to(TORCH["e4m3"]), scale


def _to_mx4(x):
    """Packed e2m1 codes of x (..., k), the first of two in the low half, whole blocks of
    32 with zeros behind the row, and the blocks' exponents, biased by 127."""
    k = _blocks(x.shape[-1], MX) * MX
    part = _padded(x.float(), k).unflatten(-1, (-1, MX))
    most = part.abs().amax(-1, keepdim=True)
    exponent = torch.where(most > 0, torch.frexp(most).exponent - 3, -127).clamp(min=-127)
    q = torch.ldexp(part.double(), -exponent)
    a = q.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5) + 8 * torch.signbit(q).to(torch.uint8)).flatten(-2)
    return code[..., ::2] | code[..., 1::2] << 4, (exponent[..., 0] + 127).to(torch.uint8)


def _plan(g, case, s):
    """Rows by expert as dispatch leaves them: topk experts for each token, some more
    popular than others, some slots dropped, so that rows are left at the end."""
    t, e, k = case["tokens"], case["experts"], case["topk"]
    x = _normal(g, (t, e)) + _normal(g, (1, e), 0.7)
    ids = x.argsort(1, descending=True)[:, :k].flatten()
    if case["dropped"]:
        ids = torch.where(torch.rand(t * k, device="cuda", generator=g) < case["dropped"], e, ids)
    counts = torch.bincount(ids, minlength=e + 1)[:e]
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    s["rows"], s["kept"], s["most"] = t * k, int(counts.sum()), max(1, int(counts.max()))
    # the experts that have rows, and where each row lies among rows of `most` for each of them
    s["used"] = torch.nonzero(counts).flatten()
    at = torch.repeat_interleave(torch.arange(len(s["used"]), device="cuda"), counts[s["used"]])
    first = s["offsets"][:-1].long()[s["used"]]
    s["slot"] = at * s["most"] + torch.arange(s["kept"], device="cuda") - first[at]


def _weights(g, case):
    """The experts' weights in the case's type, made one expert at a time."""
    e, shape, dt = case["experts"], (case["n"], case["k"]), case["dtype"]
    if case.get("transpose"):
        shape = shape[::-1]
    scale = case["k"] ** -0.5
    if dt in ("f32", "bf16", "f16"):
        w = torch.empty((e, *shape), dtype=TORCH[dt], device="cuda")
        for i in range(e):
            w[i] = _normal(g, shape, scale)
        return w, None
    to = (lambda x: _to_e4m3(x, BLOCK, BLOCK)) if dt == "e4m3" else _to_mx4
    parts = [to(_normal(g, shape, scale)) for _ in range(e)]
    w = torch.stack([p[0].view(torch.uint8) for p in parts])
    return w.view(TORCH[dt]), torch.stack([p[1] for p in parts])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt, dev = case["op"], TORCH[case["dtype"]], "cuda"
    s = {"case": case}
    if op == "mx4":
        r, k = case["rows"], case["columns"]
        s["x"] = _activations(g, r, k).to(dt)
        s["x4"] = torch.empty((r, _blocks(k, MX) * MX // 2), dtype=torch.uint8, device=dev)
        s["scale"] = torch.empty((r, _blocks(k, MX)), dtype=torch.uint8, device=dev)
        s["values"] = torch.empty((r, k), dtype=dt, device=dev)
        return s
    _plan(g, case, s)
    r = s["rows"]
    if op in ("gate", "gate_grad"):
        w = case["width"]
        s["x"] = _activations(g, r, 2 * w).to(dt)
        if op == "gate":
            s["out"] = s["out8"] = s["scale"] = None
            if case["group"]:
                s["out8"] = torch.zeros((r, w), dtype=TORCH["e4m3"], device=dev)
                s["scale"] = torch.zeros((r, _blocks(w, case["group"])), device=dev)
            else:
                s["out"] = torch.zeros((r, w), dtype=dt, device=dev)
        else:
            s["dout"] = _normal(g, (r, w), 0.1).to(dt)
            s["dx"] = torch.zeros((r, 2 * w), dtype=dt, device=dev)
        return s
    n, k = case["n"], case["k"]
    if op == "product_grad":
        s["dout"] = _normal(g, (r, n), 0.1).to(dt)
        s["x"] = _activations(g, r, k).to(dt)
        s["dw"] = torch.empty((case["experts"], n, k), dtype=dt, device=dev)
        return s
    s["w"], s["w_scale"] = _weights(g, case)
    x = _activations(g, r, k)
    s["scale"] = s["x4"] = None
    if case["dtype"] == "e4m3":
        s["x"], s["scale"] = _to_e4m3(x, 1, BLOCK)
    elif case["dtype"] == "mx4":
        s["x"] = x.to(torch.bfloat16)
        s["x4"] = torch.empty((r, _blocks(k, MX) * MX // 2), dtype=torch.uint8, device=dev)
        s["scale"] = torch.empty((r, _blocks(k, MX)), dtype=torch.uint8, device=dev)
    else:
        s["x"] = x.to(dt)
    # rows behind the last expert's are never written: the program's buffer holds zeros there
    s["out"] = torch.zeros((r, n), dtype=dt if s["w_scale"] is None else torch.bfloat16, device=dev)
    return s


# ------------------------------------------------------------- plain forms --
def _of_mx4(x4, scale):
    """The values that packed codes and exponents stand for."""
    value = torch.tensor(E2M1 + [-v for v in E2M1], device=x4.device)
    part = torch.stack([value[(x4 & 15).int()], value[(x4 >> 4).int()]], -1).flatten(-2)
    return part * _spread(torch.exp2(scale.double() - 127).float(), MX, part.shape[-1])


def _by_expert(s, rows):
    """Rows as (experts that have some, most rows of one, columns), zeros behind an expert's."""
    out = torch.zeros((len(s["used"]) * s["most"], rows.shape[1]), device=rows.device)
    out[s["slot"]] = rows[:s["kept"]].float()
    return out.view(len(s["used"]), s["most"], rows.shape[1])


def _plain_product(s):
    c = s["case"]
    n, k, dt = c["n"], c["k"], c["dtype"]
    x, w = s["x"], s["w"].view(torch.uint8)[s["used"]].view(s["w"].dtype)
    if dt == "e4m3":
        x = x.float() * _spread(s["scale"], BLOCK, k)
        w = w.float() * _spread(_spread(s["w_scale"][s["used"]], BLOCK, k).mT, BLOCK, n).mT
    elif dt == "mx4":
        x4, scale = _to_mx4(x)
        x, w = _of_mx4(x4, scale), _of_mx4(w, s["w_scale"][s["used"]])
    w = w.float() if c["transpose"] else w.float().mT.contiguous()
    out = torch.zeros_like(s["out"])
    out[:s["kept"]] = torch.bmm(_by_expert(s, x), w).flatten(0, 1)[s["slot"]].to(out.dtype)
    return {"out": out}


def _plain_product_grad(s):
    dw = torch.zeros_like(s["dw"])
    dw[s["used"]] = torch.bmm(_by_expert(s, s["dout"]).mT.contiguous(),
                              _by_expert(s, s["x"])).to(dw.dtype)
    return {"dw": dw}


def _kept(s, rows):
    """Rows behind the last expert's as zeros."""
    return torch.cat([rows, rows.new_zeros((s["rows"] - s["kept"], rows.shape[1]))])


def _plain_gate(s):
    c = s["case"]
    gate, up = s["x"][:s["kept"]].float().chunk(2, 1)
    y = gate / (1.0 + torch.exp(-gate)) * up
    if not c["group"]:
        return {"out": _kept(s, y.to(s["x"].dtype))}
    n = _blocks(c["width"], c["group"])
    parts = _padded(y, n * c["group"]).view(-1, n, c["group"])
    scale = parts.abs().amax(2).clamp(min=LEAST_AMAX) / E4M3_MAX
    q = (parts / scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).flatten(1)[:, :c["width"]]
    return {"out8": _kept(s, q.to(TORCH["e4m3"]).view(torch.uint8)).view(TORCH["e4m3"]),
            "scale": _kept(s, scale)}


def _plain_gate_grad(s):
    gate, up = s["x"][:s["kept"]].float().chunk(2, 1)
    dout = s["dout"][:s["kept"]].float()
    share = 1.0 / (1.0 + torch.exp(-gate))
    dgate = dout * up * share * (1.0 + gate * (1.0 - share))
    return {"dx": _kept(s, torch.cat([dgate, dout * gate * share], 1).to(s["x"].dtype))}


def _plain_mx4(s):
    x4, scale = _to_mx4(s["x"])
    return {"values": _of_mx4(x4, scale)[:, :s["case"]["columns"]].to(s["x"].dtype)}


PLAIN = {"product": _plain_product, "product_grad": _plain_product_grad, "gate": _plain_gate,
         "gate_grad": _plain_gate_grad, "mx4": _plain_mx4}


# -------------------------------------------------------- the library's calls --
def _own(s):
    import paper_2510_20171_amd as xr
    c = s["case"]
    op = c["op"]
    if op == "product":
        x = s["x"]
        if s["x4"] is not None:
            xr.quant_mx4(x, s["x4"], s["scale"])
            x = s["x4"]
        xr.group_product(x, s["w"], s["offsets"], s["out"], scale=s["scale"], w_scale=s["w_scale"],
                         transpose=c["transpose"])
        return {"out": s["out"]}
    if op == "product_grad":
        xr.group_product_grad(s["dout"], s["x"], s["offsets"], s["dw"])
        return {"dw": s["dw"]}
    if op == "gate":
        xr.gate(s["x"], s["out"], out8=s["out8"], scale=s["scale"], group=c["group"] or 128,
                offsets=s["offsets"])
        return {"out8": s["out8"], "scale": s["scale"]} if c["group"] else {"out": s["out"]}
    if op == "gate_grad":
        xr.gate_grad(s["dout"], s["x"], s["dx"], offsets=s["offsets"])
        return {"dx": s["dx"]}
    xr.quant_mx4(s["x"], s["x4"], s["scale"])
    xr.dequant_mx4(s["x4"], s["scale"], s["values"])
    return {"values": s["values"]}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- in 64 bits --
def _exact_mx4(x):
    """The values of x after 4 bits: each block over the power of two that brings its
    largest to [4, 8), rounded to multiples of 1/2 below 2, of 1 below 4, of 2 above, to
    even, up to 6."""
    f, k = torch.float64, x.shape[1]
    out = torch.zeros((x.shape[0], _blocks(k, MX) * MX), dtype=f, device=x.device)
    out[:, :k] = x
    out = out.view(x.shape[0], -1, MX)
    scale = 2.0 ** (torch.frexp(out.abs().max(2, keepdim=True).values)[1] - 3).clamp(min=-127).to(f)
    out /= scale
    step = torch.where(out.abs() < 2, 0.5, torch.where(out.abs() < 4, 1.0, 2.0)).to(f)
    return (((out / step).round() * step).clamp(-6, 6) * scale).view(x.shape[0], -1)[:, :k]


def _exact_weights(s, e):
    """Expert e's weights as n x k."""
    c, f = s["case"], torch.float64
    w = s["w"][e]
    if c["dtype"] == "e4m3":
        at = lambda n: torch.arange(n, device="cuda") // BLOCK
        return w.to(f) * s["w_scale"][e].to(f)[at(c["n"])][:, at(c["k"])]
    if c["dtype"] == "mx4":
        code = torch.empty((c["n"], w.shape[1] * 2), dtype=torch.int32, device="cuda")
        code[:, 0::2], code[:, 1::2] = w % 16, w // 16
        step, low = (code & 7) // 2, (code & 1).to(f)
        size = torch.where(step == 0, low / 2, (1 + low / 2) * 2.0 ** (step - 1))
        scale = 2.0 ** (s["w_scale"][e].to(f) - 127)
        size = (size.unflatten(1, (-1, MX)) * scale[:, :, None]).flatten(1)
        return torch.where(code > 7, -size, size)[:, :c["k"]]
    return w.to(f).t() if c["transpose"] else w.to(f)


def exact(case, seed):
    s = prepare(case, seed)
    op, f = case["op"], torch.float64
    if op == "mx4":
        return {"values": torch.cat([_exact_mx4(x) for x in s["x"].split(8192)])}
    at = s["offsets"].tolist()
    if op in ("gate", "gate_grad"):
        w, end = case["width"], at[-1]
        x = s["x"][:end].to(f)
        gate, up = x[:, :w], x[:, w:]
        if op == "gate_grad":
            dx = torch.zeros(s["dx"].shape, dtype=f, device="cuda")
            dout, p = s["dout"][:end].to(f), torch.sigmoid(gate)
            dx[:end, :w] = dout * up * (p + gate * p * torch.sigmoid(-gate))
            dx[:end, w:] = dout * gate * p
            return {"dx": dx}
        y = torch.zeros((s["rows"], w), dtype=f, device="cuda")
        y[:end] = gate * torch.sigmoid(gate) * up
        if not case["group"]:
            return {"out": y}
        columns = torch.arange(w, device="cuda") // case["group"]
        scale = torch.zeros(s["scale"].shape, dtype=f, device="cuda")
        scale[:end].scatter_reduce_(1, columns.expand(end, w), y[:end].abs(), "amax")
        scale[:end] = scale[:end].clamp(min=LEAST_AMAX) / E4M3_MAX
        y[:end] /= scale[:end][:, columns]
        return {"out8": y, "scale": scale}
    if op == "product_grad":
        dw = torch.zeros(s["dw"].shape, dtype=f, device="cuda")
        for e in range(case["experts"]):
            rows = slice(at[e], at[e + 1])
            dw[e] = torch.mm(s["dout"][rows].to(f).t(), s["x"][rows].to(f))
        return {"dw": dw}
    out = torch.zeros(s["out"].shape, dtype=f, device="cuda")
    for e in range(case["experts"]):
        if at[e] == at[e + 1]:
            continue
        x = s["x"][at[e]:at[e + 1]]
        if case["dtype"] == "mx4":
            x = _exact_mx4(x)
        elif case["dtype"] == "e4m3":
            columns = torch.arange(case["k"], device="cuda") // BLOCK
            x = x.to(f) * s["scale"][at[e]:at[e + 1]].to(f)[:, columns]
        out[at[e]:at[e + 1]] = torch.mm(x.to(f), _exact_weights(s, e).t())
    return {"out": out}
