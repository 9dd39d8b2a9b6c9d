"""The calls around a reduced activation: fold of partial sums with residual
addition and norm, expert routing, dispatch and combine, with their gradients
(the second half of include/xred.h).

Matrices are 2-D GPU tensors whose rows are contiguous; rows may lie further
apart than their length (a column range of a larger matrix).  Outputs are the
caller's tensors, written in place on the current stream (or ``stream``).

    h, y = torch.empty_like(x), torch.empty_like(x)
    xr.fold_norm(partial_sums, y, residual=x, weight=w, sum=h)   # h = x + sum, y = norm(h)
"""
from __future__ import annotations

import ctypes

from . import _dtype_name, _ptr, _require, _stream
from ._lib import (DTYPE, ELEM_SIZE, INVALID_ARGUMENT, ROUTE_RENORM, SCORE, CombineArgs,
                   CombineGradArgs, DispatchArgs, DispatchPlanArgs, FoldNormArgs,
                   FoldNormGradArgs, RouteArgs, RouteGradArgs, XredError, XredRows, check, load,
                   native, ptr_array)


def _refuse(text):
    raise XredError(INVALID_ARGUMENT, text)


def _matrix(t, rows, columns, es, what, device):
    """t as an xred_rows after checking its shape, element size and device; None: absent."""
    if t is None:
        return XredRows(None, 0)
    if not t.is_cuda or t.device != device:
        _refuse(f"{what} is on {t.device}, not {device}")
    if tuple(t.shape) != (rows, columns):
        _refuse(f"{what} has shape {tuple(t.shape)}, expected {(rows, columns)}")
    if t.element_size() != es:
        _refuse(f"{what} has {t.element_size()}-byte elements, expected {es}")
    if columns > 1 and t.stride(1) != 1:
        _refuse(f"{what}: elements of a row are not contiguous")
    # the distance of one row from the next means nothing for a single row
    return XredRows(t.data_ptr(), t.stride(0) if rows > 1 else columns)


def _shape(t, what):
    if t.dim() != 2:
        _refuse(f"{what} has {t.dim()} dimensions, expected 2")
    if not t.is_cuda:
        _refuse(f"{what} is not in GPU memory")
    return t.shape[0], t.shape[1]


def _vector(t, n, es, what, device):
    _require([t], n, es, what, device)
    return _ptr(t)


def _floats(t, n, what, device):
    if t is not None and _dtype_name(t, None) != "f32":
        _refuse(f"{what} is {t.dtype}, expected float32")
    return _vector(t, n, 4, what, device)


def _slots(t, rows, topk, what, device, dtypes):
    """A contiguous tokens x topk tensor of one of `dtypes`, as a pointer."""
    if _dtype_name(t, None) not in dtypes:
        _refuse(f"{what} is {t.dtype}, expected {' or '.join(dtypes)}")
    if tuple(t.shape) != (rows, topk):
        _refuse(f"{what} has shape {tuple(t.shape)}, expected {(rows, topk)}")
    return _vector(t, rows * topk, 4, what, device)


def _count(n, what):
    """n, which the C ABI takes as 32 bits."""
    if not 0 <= n < 1 << 32:
        _refuse(f"{what} = {n}")
    return n


def _score(name):
    if name not in SCORE:
        _refuse(f"unknown score {name!r}")
    return SCORE[name]


def _weight(t, dtype, n, device):
    """(pointer, dtype code) of a row of weights in dtype or fp32; None: ones."""
    name = dtype if t is None else _dtype_name(t, None)
    if name not in (dtype, "f32"):
        _refuse(f"weight is {name}, expected {dtype} or f32")
    return _vector(t, n, ELEM_SIZE[name], "weight", device), DTYPE[name]


def _workspace(nbytes, like, stream):
    """A workspace from torch's allocator, taken on the stream of the call: kernels
    enqueued before on the stream it is taken on may still use the block, and only
    that stream's later work waits for them."""
    import torch
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=like.device)
    if not isinstance(stream, torch.cuda.Stream):
        handle = int(getattr(stream, "cuda_stream", stream))
        stream = torch.cuda.ExternalStream(handle, device=like.device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=like.device)


def _given(t, device):
    """(pointer, bytes) of a workspace tensor, or of none."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.device != device or not t.is_contiguous():
        _refuse(f"workspace is not a contiguous tensor on {device}")
    return t.data_ptr(), t.numel() * t.element_size()


def fold_norm(srcs, out=None, *, residual=None, weight=None, sum=None, out8=None, scale=None,
              rstd=None, group: int = 0, eps: float = 1e-6, stream=None) -> None:
    """Fold of partial sums, residual addition and RMS norm (xred_fold_norm).

    h = srcs[0] + ... + srcs[P-1] + residual; sum = h, out = h * rstd * weight,
    out8 the same in e4m3 with a scale for each row (group = 0) or group of
    elements; rstd the rows' 1 / sqrt(mean(h^2) + eps).  All but one of out and
    out8 is optional."""
    st = native().fold_norm(srcs, out, residual, weight, sum, out8, scale, rstd, group, eps,
                            stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    if len(srcs) < 1:
        _refuse("no sources")
    rows, hidden = _shape(srcs[0], "srcs[0]")
    dt, dev = _dtype_name(srcs[0], None), srcs[0].device
    es = ELEM_SIZE[dt]
    src = [_matrix(s, rows, hidden, es, f"srcs[{k}]", dev) for k, s in enumerate(srcs)]
    if any(m.stride != src[0].stride for m in src):
        _refuse("srcs have different row distances")
    for what, t in (("residual", residual), ("sum", sum), ("out", out), *(
            (f"srcs[{k}]", s) for k, s in enumerate(srcs))):
        if t is not None and t.dtype != srcs[0].dtype:
            _refuse(f"{what} is {t.dtype}, srcs[0] is {srcs[0].dtype}")
    if out8 is not None and _dtype_name(out8, None) not in ("e4m3", "u8"):
        _refuse(f"out8 is {out8.dtype}, expected float8_e4m3fn or uint8")
    if scale is not None and _dtype_name(scale, None) != "f32":
        _refuse(f"scale is {scale.dtype}, expected float32")
    groups = -(-hidden // group) if _count(group, "group") else 1
    w, wt = _weight(weight, dt, hidden, dev)
    ptrs = ptr_array([m.data or 0 for m in src])
    a = FoldNormArgs(
        ctypes.addressof(ptrs), src[0].stride, len(src), group, rows, hidden,
        _matrix(residual, rows, hidden, es, "residual", dev),
        _matrix(sum, rows, hidden, es, "sum", dev), _matrix(out, rows, hidden, es, "out", dev),
        _matrix(out8, rows, hidden, 1, "out8", dev),
        _matrix(scale, rows, groups, 4, "scale", dev), w, _floats(rstd, rows, "rstd", dev),
        DTYPE[dt], wt, eps)
    check(load().xred_fold_norm(ctypes.byref(a), _stream(srcs[0], stream)))


def fold_norm_grad(dout, sum, rstd, dx, *, weight=None, dsum=None, dweight=None, workspace=None,
                   stream=None) -> None:
    """The gradient of fold_norm's out (xred_fold_norm_grad): dx, the gradient of
    the residual and of every source, and dweight (fp32).  dsum: the gradient
    that reaches fold_norm's sum; workspace: a tensor to use for dweight's
    partial sums instead of one from torch's allocator."""
    st = native().fold_norm_grad(dout, sum, rstd, dx, weight, dsum, dweight, workspace, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, hidden = _shape(sum, "sum")
    if dweight is not None and workspace is None:
        workspace = _workspace(load().xred_fold_norm_grad_workspace(rows, hidden), sum, stream)
    dt, dev = _dtype_name(sum, None), sum.device
    es = ELEM_SIZE[dt]
    for what, t in (("dout", dout), ("dsum", dsum), ("dx", dx)):
        if t is not None and t.dtype != sum.dtype:
            _refuse(f"{what} is {t.dtype}, sum is {sum.dtype}")
    w, wt = _weight(weight, dt, hidden, dev)
    a = FoldNormGradArgs(
        rows, hidden, _matrix(dout, rows, hidden, es, "dout", dev),
        _matrix(sum, rows, hidden, es, "sum", dev), _matrix(dsum, rows, hidden, es, "dsum", dev),
        _matrix(dx, rows, hidden, es, "dx", dev), w, _floats(rstd, rows, "rstd", dev),
        _floats(dweight, hidden, "dweight", dev), *_given(workspace, dev), DTYPE[dt], wt)
    check(load().xred_fold_norm_grad(ctypes.byref(a), _stream(sum, stream)))


def route(logits, ids, weights, *, score: str = "softmax", bias=None, groups: int = 1,
          group_topk: int = 1, group_score: int = 2, renorm: bool = True, scale: float = 1.0,
          stream=None) -> None:
    """Each token's best experts and their weights (xred_route).

    logits: tokens x experts; ids (int32) and weights (fp32): tokens x topk,
    best first, ids -1 and weight 0 where no expert is left.  score: "softmax" or
    "sigmoid"; bias (fp32, one an expert) steers the choice only; with groups > 1
    the group_topk best groups of experts are chosen from, ranked by their best
    key (group_score = 1) or their best two.  The key is the sigmoid, or with softmax
    the logit, plus the bias.  For a softmax router whose bias is added to its
    probabilities p, route log(p / (1 - p)) with score="sigmoid"."""
    st = native().route(logits, ids, weights, score, bias, groups, group_topk, group_score,
                        renorm, scale, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    tokens, experts = _shape(logits, "logits")
    topk = _shape(ids, "ids")[1]
    dt, dev = _dtype_name(logits, None), logits.device
    a = RouteArgs(
        tokens, experts, topk, _count(groups, "groups"), _count(group_topk, "group_topk"),
        _count(group_score, "group_score"), ROUTE_RENORM if renorm else 0,
        _matrix(logits, tokens, experts, ELEM_SIZE[dt], "logits", dev),
        _floats(bias, experts, "bias", dev), _slots(ids, tokens, topk, "ids", dev, ("i32",)),
        _slots(weights, tokens, topk, "weights", dev, ("f32",)), DTYPE[dt], _score(score), scale)
    check(load().xred_route(ctypes.byref(a), _stream(logits, stream)))


def route_grad(logits, ids, dweights, dlogits, *, score: str = "softmax", renorm: bool = True,
               scale: float = 1.0, stream=None) -> None:
    """The gradient of route's weights with respect to the logits (xred_route_grad)."""
    st = native().route_grad(logits, ids, dweights, dlogits, score, renorm, scale, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    tokens, experts = _shape(logits, "logits")
    topk = _shape(ids, "ids")[1]
    dt, dev = _dtype_name(logits, None), logits.device
    if dlogits.dtype != logits.dtype:
        _refuse(f"dlogits is {dlogits.dtype}, logits is {logits.dtype}")
    es = ELEM_SIZE[dt]
    a = RouteGradArgs(
        tokens, experts, topk, ROUTE_RENORM if renorm else 0,
        _matrix(logits, tokens, experts, es, "logits", dev),
        _matrix(dlogits, tokens, experts, es, "dlogits", dev),
        _slots(ids, tokens, topk, "ids", dev, ("i32",)),
        _slots(dweights, tokens, topk, "dweights", dev, ("f32",)), DTYPE[dt], _score(score), scale)
    check(load().xred_route_grad(ctypes.byref(a), _stream(logits, stream)))


def _ints(t, n, what, device):
    if t is not None and _dtype_name(t, None) != "i32":
        _refuse(f"{what} is {t.dtype}, expected int32")
    return _vector(t, n, 4, what, device)


def dispatch_plan(ids, counts, offsets, pos, *, slots=None, workspace=None, stream=None) -> None:
    """The order of routed rows by expert (xred_dispatch_plan), all int32.

    ids: tokens x topk, -1 (or any id that is no expert) drops the slot; counts:
    experts; offsets: experts + 1; pos: tokens x topk, each slot's row or -1;
    slots (optional, tokens * topk): each row's slot.  workspace: a tensor to use
    instead of one from torch's allocator."""
    st = native().dispatch_plan(ids, counts, offsets, pos, slots, workspace, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    tokens, topk = _shape(ids, "ids")
    experts, dev = counts.numel(), ids.device
    need = load().xred_dispatch_plan_workspace(tokens * topk, experts)
    if need and workspace is None:
        workspace = _workspace(need, ids, stream)
    a = DispatchPlanArgs(
        tokens, experts, topk, _slots(ids, tokens, topk, "ids", dev, ("i32",)),
        _ints(counts, experts, "counts", dev), _ints(offsets, experts + 1, "offsets", dev),
        _slots(pos, tokens, topk, "pos", dev, ("i32",)),
        _ints(slots, tokens * topk, "slots", dev), *_given(workspace, dev))
    check(load().xred_dispatch_plan(ctypes.byref(a), _stream(ids, stream)))


def dispatch(x, pos, out, *, scale=None, out_scale=None, stream=None) -> None:
    """Rows to their places: out[pos[t][j]] = x[t] (xred_dispatch), any dtype; scale
    (tokens x columns, fp32) travels along to out_scale."""
    st = native().dispatch(x, pos, out, scale, out_scale, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    tokens, hidden = _shape(x, "x")
    topk, rows = _shape(pos, "pos")[1], _shape(out, "out")[0]
    dt, dev = _dtype_name(x, None), x.device
    if out.dtype != x.dtype:
        _refuse(f"out is {out.dtype}, x is {x.dtype}")
    if (scale is None) != (out_scale is None):
        _refuse("scale and out_scale go together")
    for what, t in (("scale", scale), ("out_scale", out_scale)):
        if t is not None and _dtype_name(t, None) != "f32":
            _refuse(f"{what} is {t.dtype}, expected float32")
    es = ELEM_SIZE[dt]
    columns = _shape(scale, "scale")[1] if scale is not None else 0
    a = DispatchArgs(
        tokens, hidden, rows, columns, topk, DTYPE[dt], _matrix(x, tokens, hidden, es, "x", dev),
        _matrix(out, rows, hidden, es, "out", dev), _matrix(scale, tokens, columns, 4, "scale", dev),
        _matrix(out_scale, rows, columns, 4, "out_scale", dev),
        _slots(pos, tokens, topk, "pos", dev, ("i32",)))
    check(load().xred_dispatch(ctypes.byref(a), _stream(x, stream)))


def combine(y, pos, out, *, weights=None, base=None, stream=None) -> None:
    """The experts' rows back to their tokens (xred_combine):
    out[t] = base[t] + sum over j of weights[t][j] * y[pos[t][j]], in order of j."""
    st = native().combine(y, pos, out, weights, base, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, hidden = _shape(y, "y")
    tokens, topk = _shape(pos, "pos")
    dt, dev = _dtype_name(y, None), y.device
    for what, t in (("out", out), ("base", base)):
        if t is not None and t.dtype != y.dtype:
            _refuse(f"{what} is {t.dtype}, y is {y.dtype}")
    es = ELEM_SIZE[dt]
    a = CombineArgs(
        tokens, hidden, rows, topk, DTYPE[dt], _matrix(y, rows, hidden, es, "y", dev),
        _matrix(base, tokens, hidden, es, "base", dev), _matrix(out, tokens, hidden, es, "out", dev),
        _slots(pos, tokens, topk, "pos", dev, ("i32",)),
        None if weights is None else _slots(weights, tokens, topk, "weights", dev, ("f32",)))
    check(load().xred_combine(ctypes.byref(a), _stream(y, stream)))


def combine_grad(dout, y, pos, weights, dy, dweights=None, *, stream=None) -> None:
    """The gradient of combine (xred_combine_grad): dy, the experts' rows', and
    dweights (fp32, tokens x topk); base's is dout itself."""
    st = native().combine_grad(dout, y, pos, weights, dy, dweights, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, hidden = _shape(dy, "dy")
    tokens, topk = _shape(pos, "pos")
    dt, dev = _dtype_name(dout, None), dout.device
    if y is None and dweights is not None:
        _refuse("dweights needs y")
    for what, t in (("y", y), ("dy", dy)):
        if t is not None and t.dtype != dout.dtype:
            _refuse(f"{what} is {t.dtype}, dout is {dout.dtype}")
    es = ELEM_SIZE[dt]
    a = CombineGradArgs(
        tokens, hidden, rows, topk, DTYPE[dt], _matrix(dout, tokens, hidden, es, "dout", dev),
        _matrix(y, rows, hidden, es, "y", dev), _matrix(dy, rows, hidden, es, "dy", dev),
        _slots(pos, tokens, topk, "pos", dev, ("i32",)),
        _slots(weights, tokens, topk, "weights", dev, ("f32",)),
        None if dweights is None else _slots(dweights, tokens, topk, "dweights", dev, ("f32",)))
    check(load().xred_combine_grad(ctypes.byref(a), _stream(dout, stream)))
