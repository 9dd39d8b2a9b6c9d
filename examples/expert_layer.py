"""A mixture-of-experts layer around libxred: what a rank does between the
reduction of one layer's partial sums and the next.

    python examples/expert_layer.py [--tokens N] [--hidden H] [--experts E] [--topk K]

``serve`` is the inference form with 8-bit expert inputs, for any number of
tokens from one; ``train_step`` the same layer in bf16 with its backward pass,
the library's gradients behind torch.autograd.Function.  The router's product is
torch's; everything else is the library's.  ``GatedLayer`` has experts of two
products with a gated activation between them; ``serve_gated`` runs it with its
weights in 8 or 4 bits.  Run as a program, it checks both forms of the plain layer
against torch and times them all.
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


    def weights(self):
        return [self.expert]

    def apply(self, rows, offsets):
        return Products.apply(rows, self.expert, offsets)


class GatedLayer(Layer):
    """Experts of two products: rows of 2 * width gates and values, of which the gated
    activation makes `width`, and back."""

    def __init__(self, hidden, width, experts, topk, dtype=torch.bfloat16, device="cuda", seed=0):
        super().__init__(hidden, experts, topk, dtype, device, seed)
        g = torch.Generator(device=device).manual_seed(seed + 1)
        new = lambda *shape: torch.empty(shape, device=device).normal_(
            0, shape[-1] ** -0.5, generator=g).to(dtype)
        self.width = width
        self.up, self.down = new(experts, 2 * width, hidden), new(experts, hidden, width)

    def weights(self):
        return [self.up, self.down]

    def apply(self, rows, offsets):
        gated = Gate.apply(Products.apply(rows, self.up, offsets), offsets)
        return Products.apply(gated, self.down, offsets)


class Products(torch.autograd.Function):
    """Each expert's product with its rows, which lie together; rows past the last stay 0."""

    @staticmethod
    def forward(ctx, rows, weight, offsets):
        out = rows.new_zeros((rows.shape[0], weight.shape[1]))
        xr.group_product(rows, weight, offsets, out)
        ctx.save_for_backward(rows, weight, offsets)
        return out

    @staticmethod
    def backward(ctx, dout):
        rows, weight, offsets = ctx.saved_tensors
        dout = dout.contiguous()
        drows, dweight = torch.zeros_like(rows), torch.empty_like(weight)
        xr.group_product(dout, weight, offsets, drows, transpose=True)
        xr.group_product_grad(dout, rows, offsets, dweight)
        return drows, dweight, None


class Gate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, offsets):
        out = x.new_zeros((x.shape[0], x.shape[1] // 2))
        xr.gate(x, out, offsets=offsets)
        ctx.save_for_backward(x, offsets)
        return out

    @staticmethod
    def backward(ctx, dout):
        x, offsets = ctx.saved_tensors
        dx = torch.zeros_like(x)
        xr.gate_grad(dout.contiguous(), x, dx, offsets=offsets)
        return dx, None


def to_e4m3(w):
    """Weights in 8 bits with a scale for every 128 x 128 of them."""
    e, n, k = w.shape
    by = torch.nn.functional.pad(w.float(), (0, -k % GROUP, 0, -n % GROUP)).unflatten(
        2, (-1, GROUP)).unflatten(1, (-1, GROUP))
    scale = by.abs().amax((2, 4), keepdim=True).clamp(min=2.0 ** -100) / 448
    w8 = (by / scale).to(torch.float8_e4m3fn).flatten(3).flatten(1, 2)[:, :n, :k].contiguous()
    return w8, scale[:, :, 0, :, 0].contiguous()


def to_mx4(w):
    """Weights in 4 bits with a power of two for every 32 of a row."""
    e, n, k = w.shape
    w4 = torch.empty((e, n, -(-k // 32) * 16), dtype=torch.uint8, device=w.device)
    scale = torch.empty((e, n, -(-k // 32)), dtype=torch.uint8, device=w.device)
    xr.quant_mx4(w.flatten(0, 1), w4.flatten(0, 1), scale.flatten(0, 1))
    return w4, scale


def plan(ids, experts):
    counts = torch.empty(experts, dtype=torch.int32, device=ids.device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=ids.device)
    pos = torch.empty_like(ids)
    xr.dispatch_plan(ids, counts, offsets, pos)
    return counts, offsets, pos


def routed(layer, y):
    """Weights of the tokens' experts, where the experts' rows begin, and the slots' rows."""
    ids = torch.empty((y.shape[0], layer.topk), dtype=torch.int32, device=y.device)
    weights = torch.empty(ids.shape, device=y.device)
    xr.route(y @ layer.router.t(), ids, weights, score="sigmoid", bias=layer.bias, scale=SCALE)
    _, offsets, pos = plan(ids, layer.experts)
    return weights, offsets, pos


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
    weights, offsets, pos = routed(layer, y)
    rows8 = torch.empty((tokens * k, hidden), dtype=torch.float8_e4m3fn, device=dev)
    row_scale = torch.empty((tokens * k, scale.shape[1]), device=dev)
    xr.dispatch(y8, pos, rows8, scale=scale, out_scale=row_scale)
    rows = rows8.float() * row_scale.repeat_interleave(GROUP, 1)[:, :hidden]
    out = torch.empty_like(h)
    xr.combine(layer.apply(rows.to(dt), offsets), pos, out, weights=weights, base=h)
    return out


def serve_gated(layer, weights4or8, partial_sums, stream_in):
    """A GatedLayer with (up, its scales, down, its scales) from to_e4m3 or to_mx4: rows go
    through both products in as many bits."""
    (up, up_scale), (down, down_scale) = weights4or8
    tokens, hidden, dt, dev = stream_in.shape[0], layer.hidden, stream_in.dtype, stream_in.device
    slots, mx4 = tokens * layer.topk, up.dtype == torch.uint8
    new = lambda rows, columns, dtype: torch.empty((rows, columns), dtype=dtype, device=dev)
    h, y = torch.empty_like(stream_in), torch.empty_like(stream_in)
    inner, outer = new(slots, 2 * layer.width, dt), new(slots, hidden, dt)
    out = torch.empty_like(h)
    if mx4:
        xr.fold_norm(partial_sums, y, residual=stream_in, weight=layer.norm, sum=h)
        weights, offsets, pos = routed(layer, y)
        rows, gated = torch.zeros_like(outer), new(slots, layer.width, dt)
        xr.dispatch(y, pos, rows)
        rows4, scale = to_mx4(rows[None])
        xr.group_product(rows4[0], up, offsets, inner, scale=scale[0], w_scale=up_scale)
        xr.gate(inner, gated, offsets=offsets)
        gated4, scale = to_mx4(gated[None])
        xr.group_product(gated4[0], down, offsets, outer, scale=scale[0], w_scale=down_scale)
    else:
        y8, y_scale = new(tokens, hidden, up.dtype), new(tokens, up_scale.shape[2], torch.float32)
        xr.fold_norm(partial_sums, y, residual=stream_in, weight=layer.norm, sum=h, out8=y8,
                     scale=y_scale, group=GROUP)
        weights, offsets, pos = routed(layer, y)
        rows8, scale = new(slots, hidden, up.dtype), new(slots, up_scale.shape[2], torch.float32)
        xr.dispatch(y8, pos, rows8, scale=y_scale, out_scale=scale)
        xr.group_product(rows8, up, offsets, inner, scale=scale, w_scale=up_scale)
        gated8, scale = new(slots, layer.width, up.dtype), new(slots, down_scale.shape[2], torch.float32)
        xr.gate(inner, out8=gated8, scale=scale, group=GROUP, offsets=offsets)
        xr.group_product(gated8, down, offsets, outer, scale=scale, w_scale=down_scale)
    xr.combine(outer, pos, out, weights=weights, base=h)
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
    rows = layer.apply(Dispatch.apply(y, pos), offsets)
    return Combine.apply(rows, pos, weights, h)


def train_step(layer, partial_sums, stream_in, dout):
    """Output and the gradients of the input stream, of every weight and (all alike) of
    the partial sums."""
    leaves = [stream_in, layer.norm, layer.router, *layer.weights(), partial_sums[0]]
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
    gated = GatedLayer(a.hidden, a.hidden, a.experts, a.topk)
    eight, four = ([to(w) for w in gated.weights()] for to in (to_e4m3, to_mx4))
    for what, f in (("serve", lambda: serve(layer, sums, x)),
                    ("train_step", lambda: train_step(layer, sums, x, dout)),
                    ("serve_gated, e4m3", lambda: serve_gated(gated, eight, sums, x)),
                    ("serve_gated, mx4", lambda: serve_gated(gated, four, sums, x)),
                    ("train_step, gated", lambda: train_step(gated, sums, x, dout))):
        f()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(10):
            f()
        torch.cuda.synchronize()
        print("%s: %.2f ms a pass, the products included" % (what, (time.perf_counter() - t) * 100))


if __name__ == "__main__":
    main()
