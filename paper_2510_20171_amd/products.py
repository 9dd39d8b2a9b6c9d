"""The calls between dispatch and combine: the experts' products over ragged rows
with their gradients, the gated activation, and 4-bit microscaled values (the last
part of include/xred.h).

Rows lie together by expert, as dispatch_plan's offsets tell on the GPU; matrices are
2-D GPU tensors whose rows are contiguous, experts' weights 3-D ones.  Outputs are the
caller's tensors, written in place on the current stream (or ``stream``).

    xr.group_product(rows, w1, offsets, a)              # a[r] = w1[e] @ rows[r]
    xr.gate(a, h, offsets=offsets)                      # h = silu(a's first half) * its second
    xr.group_product(h, w2, offsets, y)
"""
from __future__ import annotations

import ctypes

from . import _dtype_name, _stream
from ._lib import (DTYPE, ELEM_SIZE, PRODUCT_ADD, PRODUCT_MX4, PRODUCT_TRANSPOSE, DequantMx4Args,
                   GateArgs, GateGradArgs, GroupProductArgs, GroupProductGradArgs, QuantMx4Args,
                   XredRows, check, load, native)
from .layer import _count, _ints, _matrix, _refuse, _shape

PLAIN = ("f32", "bf16", "f16")
BLOCK, MX = 128, 32   # elements that share a scale: e4m3, mx4


def _name(t):
    """The element type of t; "u8" for the byte types that hold packed 4-bit codes or
    exponents."""
    if str(t.dtype) in ("torch.float4_e2m1fn_x2", "torch.float8_e8m0fnu"):
        return "u8"
    return _dtype_name(t, None)


def _typed(t, names, what):
    name = _name(t)
    if name not in names:
        _refuse(f"{what} is {t.dtype}, expected {' or '.join(names)}")
    return name


def _stack(t, shape, names, what, device):
    """An experts x rows x columns tensor as (xred_rows of the first expert, elements from
    one expert to the next)."""
    es = ELEM_SIZE[_typed(t, names, what)]
    if not t.is_cuda or t.device != device:
        _refuse(f"{what} is on {t.device}, not {device}")
    if tuple(t.shape) != tuple(shape):
        _refuse(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.element_size() != es:
        _refuse(f"{what} has {t.element_size()}-byte elements, expected {es}")
    experts, rows, columns = shape
    if columns > 1 and t.stride(2) != 1:
        _refuse(f"{what}: elements of a row are not contiguous")
    stride = t.stride(1) if rows > 1 else columns
    apart = t.stride(0) if experts > 1 else rows * stride
    return XredRows(t.data_ptr(), stride), apart


def _experts(offsets, device):
    if offsets.dim() != 1 or offsets.numel() < 2:
        _refuse(f"offsets has shape {tuple(offsets.shape)}, expected experts + 1")
    return offsets.numel() - 1, _ints(offsets, offsets.numel(), "offsets", device)


def _blocks(k, size):
    return -(-k // size)


def group_product(x, w, offsets, out, *, scale=None, w_scale=None, transpose: bool = False,
                  stream=None) -> None:
    """Each expert's product with its rows (xred_group_product):
    out[r] = w[e] @ x[r] for offsets[e] <= r < offsets[e + 1], other rows untouched.

    x: rows x k; w: experts x n x k, or with ``transpose`` experts x k x n; out: rows x n
    in fp32, bf16 or fp16; offsets: experts + 1 int32 (dispatch_plan's).  x and w are fp32,
    bf16 or fp16 (out the same or fp32); or e4m3 with scale (rows x ceil(k / 128)) and
    w_scale (experts x ceil(n / 128) x ceil(k / 128)) in fp32; or mx4 as quant_mx4 leaves
    it (bytes, k / 2 a row in whole blocks of 32) with scale and w_scale of a byte for
    every 32 elements."""
    st = native().group_product(x, w, offsets, out, scale, w_scale, transpose, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, k = _shape(x, "x")
    n = _shape(out, "out")[1]
    dev, name = x.device, _typed(x, PLAIN + ("e4m3", "u8"), "x")
    experts, off = _experts(offsets, dev)
    mx4, scaled = name == "u8", name in ("e4m3", "u8")
    if scaled != (scale is not None) or scaled != (w_scale is not None):
        _refuse(f"scale and w_scale {'are needed' if scaled else 'are given'} with x in {x.dtype}")
    o = _typed(out, PLAIN if scaled else (name, "f32"), "out")
    w_rows, apart = _stack(w, (experts, k, n) if transpose else (experts, n, k), (name,), "w", dev)
    row_scale, w_scales, w_scale_apart = XredRows(None, 0), XredRows(None, 0), 0
    if scaled:
        kind, ss = ("u8", 1) if mx4 else ("f32", 4)
        parts = _blocks(k, 16 if mx4 else BLOCK)
        _typed(scale, (kind,), "scale")
        row_scale = _matrix(scale, rows, parts, ss, "scale", dev)
        w_scales, w_scale_apart = _stack(
            w_scale, (experts, n if mx4 else _blocks(n, BLOCK), parts), (kind,), "w_scale", dev)
    flags = (PRODUCT_TRANSPOSE if transpose else 0) | (PRODUCT_MX4 if mx4 else 0)
    if mx4 and k % 16:
        _refuse(f"x has rows of {k} bytes, expected whole blocks of 16")
    a = GroupProductArgs(
        rows, n, 2 * k if mx4 else k, experts, flags, DTYPE[name], DTYPE[o],
        _matrix(x, rows, k, ELEM_SIZE[name], "x", dev), row_scale, w_rows, w_scales,
        _matrix(out, rows, n, ELEM_SIZE[o], "out", dev), apart, w_scale_apart, off)
    check(load().xred_group_product(ctypes.byref(a), _stream(x, stream)))


def group_product_grad(dout, x, offsets, dw, *, add: bool = False, stream=None) -> None:
    """The gradient of group_product's weights (xred_group_product_grad):
    dw[e] = sum over the expert's rows of dout[r] x[r]^T, or that added to dw.

    dout: rows x n, x: rows x k, in one of fp32, bf16 and fp16; dw: experts x n x k in
    that type or fp32.  The gradient of x is group_product(dout, w, offsets, dx,
    transpose=True); of transposed weights this call's with dout and x exchanged."""
    st = native().group_product_grad(dout, x, offsets, dw, add, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, n = _shape(dout, "dout")
    k = _shape(x, "x")[1]
    dev, name = dout.device, _typed(dout, PLAIN, "dout")
    experts, off = _experts(offsets, dev)
    if x.dtype != dout.dtype:
        _refuse(f"x is {x.dtype}, dout is {dout.dtype}")
    es = ELEM_SIZE[name]
    to, apart = _stack(dw, (experts, n, k), (name, "f32"), "dw", dev)
    a = GroupProductGradArgs(
        rows, n, k, experts, PRODUCT_ADD if add else 0, DTYPE[name], DTYPE[_name(dw)],
        _matrix(dout, rows, n, es, "dout", dev), _matrix(x, rows, k, es, "x", dev), to, apart, off)
    check(load().xred_group_product_grad(ctypes.byref(a), _stream(dout, stream)))


def _row_count(offsets, device):
    """A pointer to the number of rows that hold something: the last of offsets."""
    if offsets is None:
        return None
    n = offsets.numel()
    if n < 1:
        _refuse("offsets is empty")
    return ctypes.c_void_p(_ints(offsets, n, "offsets", device).value + 4 * (n - 1))


def gate(x, out=None, *, out8=None, scale=None, group: int = 128, offsets=None,
         stream=None) -> None:
    """Gated activation (xred_gate): out = silu(x[:, :width]) * x[:, width:].

    x: rows x 2 width in fp32, bf16 or fp16; out the same type, out8 (e4m3) with scale
    (fp32, rows x ceil(width / group)) the same in 8 bits; at least one of the two.  With
    offsets (int32) only the rows below its last value are worked on."""
    st = native().gate(x, out, out8, scale, group, offsets, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, both = _shape(x, "x")
    if both % 2:
        _refuse(f"x has {both} columns: gates and values are as many")
    width, dev, name = both // 2, x.device, _typed(x, PLAIN, "x")
    if out is not None and out.dtype != x.dtype:
        _refuse(f"out is {out.dtype}, x is {x.dtype}")
    if out8 is not None:
        _typed(out8, ("e4m3", "u8"), "out8")
    if scale is not None:
        _typed(scale, ("f32",), "scale")
    groups = _blocks(width, group) if _count(group, "group") else 1
    es = ELEM_SIZE[name]
    a = GateArgs(
        rows, width, group, DTYPE[name], _matrix(x, rows, both, es, "x", dev),
        _matrix(out, rows, width, es, "out", dev), _matrix(out8, rows, width, 1, "out8", dev),
        _matrix(scale, rows, groups, 4, "scale", dev), _row_count(offsets, dev))
    check(load().xred_gate(ctypes.byref(a), _stream(x, stream)))


def gate_grad(dout, x, dx, *, offsets=None, stream=None) -> None:
    """The gradient of gate's out (xred_gate_grad): dx, rows x 2 width, which may be x."""
    st = native().gate_grad(dout, x, dx, offsets, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, width = _shape(dout, "dout")
    dev, name = dout.device, _typed(dout, PLAIN, "dout")
    for what, t in (("x", x), ("dx", dx)):
        if t.dtype != dout.dtype:
            _refuse(f"{what} is {t.dtype}, dout is {dout.dtype}")
    es = ELEM_SIZE[name]
    a = GateGradArgs(
        rows, width, DTYPE[name], _matrix(dout, rows, width, es, "dout", dev),
        _matrix(x, rows, 2 * width, es, "x", dev), _matrix(dx, rows, 2 * width, es, "dx", dev),
        _row_count(offsets, dev))
    check(load().xred_gate_grad(ctypes.byref(a), _stream(dout, stream)))


def quant_mx4(x, out4, scale, *, stream=None) -> None:
    """Rows to 4-bit microscaled values (xred_quant_mx4).

    x: rows x k in fp32, bf16 or fp16; out4: rows x 16 ceil(k / 32) bytes, two codes
    each; scale: rows x ceil(k / 32) bytes, the exponents by 32 elements."""
    st = native().quant_mx4(x, out4, scale, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, k = _shape(x, "x")
    dev, name = x.device, _typed(x, PLAIN, "x")
    _typed(out4, ("u8",), "out4"), _typed(scale, ("u8",), "scale")
    a = QuantMx4Args(
        rows, k, DTYPE[name], _matrix(x, rows, k, ELEM_SIZE[name], "x", dev),
        _matrix(out4, rows, 16 * _blocks(k, MX), 1, "out4", dev),
        _matrix(scale, rows, _blocks(k, MX), 1, "scale", dev))
    check(load().xred_quant_mx4(ctypes.byref(a), _stream(x, stream)))


def dequant_mx4(x4, scale, out, *, stream=None) -> None:
    """4-bit microscaled rows to fp32, bf16 or fp16 (xred_dequant_mx4)."""
    st = native().dequant_mx4(x4, scale, out, stream)
    if st is not None:   # plain tensors; anything else is checked below
        return check(st)
    rows, k = _shape(out, "out")
    dev, name = out.device, _typed(out, PLAIN, "out")
    _typed(x4, ("u8",), "x4"), _typed(scale, ("u8",), "scale")
    a = DequantMx4Args(
        rows, k, DTYPE[name], _matrix(x4, rows, 16 * _blocks(k, MX), 1, "x4", dev),
        _matrix(scale, rows, _blocks(k, MX), 1, "scale", dev),
        _matrix(out, rows, k, ELEM_SIZE[name], "out", dev))
    check(load().xred_dequant_mx4(ctypes.byref(a), _stream(out, stream)))
