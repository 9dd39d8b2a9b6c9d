"""A mixture-of-experts layer around libxred: what a rank does between the
reduction of one layer's partial sums and the next.

    python examples/expert_layer.py [--tokens N] [--hidden H] [--experts E] [--topk K]

``serve`` is the inference form with 8-bit expert inputs, for any number of
tokens from one; ``train_step`` the same layer in bf16 with its backward pass,
the library's gradients behind torch.autograd.Function.  The products (router
and experts) are torch's; everything between them is the library's.  Run as a
program, it checks both against the layer written in plain torch and times them.
"""
from __future__ import annotations

import argparse
import sys
import time
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))
import paper_2510_20171_amd as xr  # noqa: E402

GROUP = 128       # elements of an 8-bit row that share a scale
SCALE = 2.5       # of the routed experts' weights


class Layer:
    """Weights of one layer: norm, router with its balance bias, experts (one product each)."""

    def __init__(self, hidden, experts, topk, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda *shape, scale=1.0: torch.empty(shape, device=device).normal_(
            0, scale, generator=g).to(dtype)
        self.hidden, self.experts, self.topk = hidden, experts, topk
        self.norm = (1 + new(hidden, scale=0.1)).to(dtype)
        self.router = new(experts, hidden, scale=hidden ** -0.5)
        self.bias = new(experts, scale=0.01).float()
        self.expert = new(experts, hidden, hidden, scale=hidden ** -0.5)


def products(rows, expert, offsets):
    """Each expert's product with its rows, which lie together; rows past the last stay 0."""
    out = []
    at = offsets.tolist()   # the host needs the sizes: torch has no product over ranges on the GPU
    for e in range(len(expert)):
        out.append(rows[at[e]:at[e + 1]] @ expert[e].t())
    out.append(rows.new_zeros((rows.shape[0] - at[-1], rows.shape[1])))
    return torch.cat(out)


def plan(ids, experts):
    counts = torch.empty(experts, dtype=torch.int32, device=ids.device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=ids.device)
    pos = torch.empty_like(ids)
    xr.dispatch_plan(ids, counts, offsets, pos)
    return counts, offsets, pos


def serve(layer, partial_sums, stream_in):
    """The layer on the ranks' partial sums and the residual stream: the new residual
    stream, to which the experts' outputs are added."""
    tokens, hidden, k, dt = stream_in.shape[0], layer.hidden, layer.topk, stream_in.dtype
    dev = stream_in.device
    h, y = torch.empty_like(stream_in), torch.empty_like(stream_in)
    y8 = torch.empty((tokens, hidden), dtype=torch.float8_e4m3fn, device=dev)
    scale = torch.empty((tokens, -(-hidden // GROUP)), device=dev)
    xr.fold_norm(partial_sums, y, residual=stream_in, weight=layer.norm, sum=h, out8=y8,
                 scale=scale, group=GROUP)
    ids = torch.empty((tokens, k), dtype=torch.int32, device=dev)
    weights = torch.empty((tokens, k), device=dev)
    xr.route(y @ layer.router.t(), ids, weights, score="sigmoid", bias=layer.bias, scale=SCALE)
    _, offsets, pos = plan(ids, layer.experts)
    rows8 = torch.empty((tokens * k, hidden), dtype=torch.float8_e4m3fn, device=dev)
    row_scale = torch.empty((tokens * k, scale.shape[1]), device=dev)
    xr.dispatch(y8, pos, rows8, scale=scale, out_scale=row_scale)
    rows = rows8.float() * row_scale.repeat_interleave(GROUP, 1)[:, :hidden]
    out = torch.empty_like(h)
    xr.combine(products(rows.to(dt), layer.expert, offsets), pos, out, weights=weights, base=h)
    return out


class FoldNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, residual, weight, *partial_sums):
        h, y = torch.empty_like(residual), torch.empty_like(residual)
        rstd = torch.empty(residual.shape[0], device=residual.device)
        xr.fold_norm(partial_sums, y, residual=residual, weight=weight, sum=h, rstd=rstd)
        ctx.save_for_backward(h, rstd, weight)
        return h, y

    @staticmethod
    def backward(ctx, dh, dy):
        h, rstd, weight = ctx.saved_tensors
        dx, dweight = torch.empty_like(h), torch.empty(h.shape[1], device=h.device)
        xr.fold_norm_grad(dy.contiguous(), h, rstd, dx, weight=weight, dsum=dh.contiguous(),
                          dweight=dweight)
        return (dx, dweight.to(weight.dtype)) + (dx,) * (len(ctx.needs_input_grad) - 2)


class Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, bias, topk):
        ids = torch.empty((logits.shape[0], topk), dtype=torch.int32, device=logits.device)
        weights = torch.empty(ids.shape, device=logits.device)
        xr.route(logits, ids, weights, score="sigmoid", bias=bias, scale=SCALE)
        ctx.save_for_backward(logits, ids)
        ctx.mark_non_differentiable(ids)
        return ids, weights

    @staticmethod
    def backward(ctx, _, dweights):
        logits, ids = ctx.saved_tensors
        dlogits = torch.empty_like(logits)
        xr.route_grad(logits, ids, dweights.contiguous(), dlogits, score="sigmoid", scale=SCALE)
        return dlogits, None, None


class Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos):
        out = torch.zeros((pos.numel(), x.shape[1]), dtype=x.dtype, device=x.device)
        xr.dispatch(x, pos, out)
        ctx.save_for_backward(pos)
        return out

    @staticmethod
    def backward(ctx, dout):
        pos, = ctx.saved_tensors
        dx = torch.empty((pos.shape[0], dout.shape[1]), dtype=dout.dtype, device=dout.device)
        xr.combine(dout.contiguous(), pos, dx)
        return dx, None


class Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, pos, weights, base):
        out = torch.empty_like(base)
        xr.combine(y, pos, out, weights=weights, base=base)
        ctx.save_for_backward(y, pos, weights)
        return out

    @staticmethod
    def backward(ctx, dout):
        y, pos, weights = ctx.saved_tensors
        dout = dout.contiguous()
        dy, dweights = torch.zeros_like(y), torch.empty_like(weights)
        xr.combine_grad(dout, y, pos, weights, dy, dweights)
        return dy, None, dweights, dout


def forward(layer, partial_sums, stream_in):
    """The layer in the activations' own type, differentiable."""
    h, y = FoldNorm.apply(stream_in, layer.norm, *partial_sums)
    ids, weights = Route.apply(y @ layer.router.t(), layer.bias, layer.topk)
    _, offsets, pos = plan(ids, layer.experts)
    rows = products(Dispatch.apply(y, pos), layer.expert, offsets)
    return Combine.apply(rows, pos, weights, h)


def train_step(layer, partial_sums, stream_in, dout):
    """Output and the gradients of the input stream, of every weight and (all alike) of
    the partial sums."""
    leaves = [stream_in, layer.norm, layer.router, layer.expert, partial_sums[0]]
    for t in leaves:
        t.requires_grad_(True)
        t.grad = None
    out = forward(layer, partial_sums, stream_in)
    out.backward(dout)
    for t in leaves:
        t.requires_grad_(False)
    return out.detach(), [t.grad for t in leaves]


def plain(layer, partial_sums, stream_in, ids, eight_bits, dtype=torch.float32):
    """The layer in plain torch and `dtype`, with the experts chosen beforehand: rounding
    the router's logits apart from the library may choose others where two are close."""
    c = lambda t: t.to(dtype)
    h = sum(map(c, partial_sums)) + c(stream_in)
    y = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * c(layer.norm)
    s = (y @ c(layer.router).t()).sigmoid().gather(1, ids.long())
    w = SCALE * s / s.sum(1, keepdim=True)
    if eight_bits:
        parts = torch.nn.functional.pad(y, (0, -y.shape[1] % GROUP)).unflatten(1, (-1, GROUP))
        scale = parts.abs().amax(2, keepdim=True).clamp(min=2.0 ** -100) / 448
        y = (c((parts / scale).to(torch.float8_e4m3fn)) * scale).flatten(1)[:, :y.shape[1]]
    out = h
    for e in range(layer.experts):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        out = out.index_add(0, t, (y[t] @ c(layer.expert[e]).t()) * w[t, j][:, None])
    return out


def inputs(layer, tokens, ranks=4, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda scale: torch.empty((tokens, layer.hidden), device="cuda").normal_(
        0, scale, generator=g).to(layer.norm.dtype)
    return [new(0.5) for _ in range(ranks)], new(1.0), new(0.1)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--topk", type=int, default=4)
    a = ap.parse_args()
    layer = Layer(a.hidden, a.experts, a.topk)
    sums, x, dout = inputs(layer, a.tokens)
    logits_of = lambda: Route.apply(FoldNorm.apply(x, layer.norm, *sums)[1] @ layer.router.t(),
                                    layer.bias, a.topk)[0]
    ids = logits_of()
    off = lambda got, want: float((got.float() - want).norm() / want.norm())
    print("serve: off by %.4f of the output" % off(serve(layer, sums, x),
                                                   plain(layer, sums, x, ids, True)))
    out, grads = train_step(layer, sums, x, dout)
    print("train_step: off by %.4f of the output" % off(out, plain(layer, sums, x, ids, False)))
    for name, grad in zip(("stream", "norm", "router", "experts", "partial sums"), grads):
        print("  gradient of the %s: norm %.4g" % (name, float(grad.float().norm())))
    for what, f in (("serve", lambda: serve(layer, sums, x)),
                    ("train_step", lambda: train_step(layer, sums, x, dout))):
        f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        print("%s: %.2f ms a pass, the products included" % (what, (time.perf_counter() - t) * 100))


if __name__ == "__main__":
    main()
