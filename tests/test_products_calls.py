"""Refusals of the calls between dispatch and combine, without a GPU: every bad
argument is rejected before anything is enqueued, by the C ABI and by the Python
binding, and the binding's structures are the header's."""
import ctypes
import re
import subprocess
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")
import paper_2510_20171_amd as xr  # noqa: E402
from paper_2510_20171_amd import _lib  # noqa: E402
from test_layer_calls import ALIAS, INVALID, NONE, UNSUPPORTED, args, at, refused, rows  # noqa: E402

HEADER = Path(__file__).resolve().parents[1] / "include"
PRODUCT = dict(rows=8, n=64, k=64, experts=4, dtype=1, out_dtype=1, x=rows(0), w=rows(1),
               out=rows(2), w_expert=64 * 64, offsets=at(3))
E4M3 = dict(dtype=7, scale=rows(4, 1), w_scale=rows(5, 1), w_scale_expert=1)
MX4 = dict(dtype=11, flags=2, x=rows(0, 32), w=rows(1, 32), scale=rows(4, 2), w_scale=rows(5, 2),
           w_expert=64 * 32, w_scale_expert=128)
PRODUCT_BAD = [
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=11), UNSUPPORTED), (dict(dtype=8), UNSUPPORTED),
    (dict(out_dtype=2), UNSUPPORTED), (dict(out_dtype=7), UNSUPPORTED), (dict(flags=4), INVALID),
    (dict(flags=2), UNSUPPORTED), (dict(experts=0), UNSUPPORTED), (dict(experts=1025), UNSUPPORTED),
    (dict(n=0), UNSUPPORTED), (dict(k=0), UNSUPPORTED), (dict(n=(1 << 20) + 1), UNSUPPORTED),
    (dict(k=(1 << 20) + 1), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(rows=(1 << 31) - 1, n=1 << 20, out=rows(2, 1 << 20)), UNSUPPORTED),
    (dict(x=NONE), INVALID), (dict(w=NONE), INVALID), (dict(out=NONE), INVALID),
    (dict(offsets=None), INVALID), (dict(offsets=at(3, 2)), INVALID), (dict(x=rows(0, 63)), INVALID),
    (dict(w=rows(1, 63)), INVALID), (dict(out=rows(2, 64, 1)), INVALID),
    (dict(w_expert=1 << 62), INVALID), (dict(w_expert=(1 << 64) - 1), INVALID),
    (dict(scale=rows(4)), INVALID), (dict(w_scale=rows(4)), INVALID),
    (dict(out=rows(0)), ALIAS), (dict(out=rows(1, 64, 4 * 64 * 64 * 2 - 2)), ALIAS),
    (dict(out=rows(3)), ALIAS), (dict(flags=1, w=rows(1, 63)), INVALID),
    (dict(E4M3, flags=1), UNSUPPORTED), (dict(E4M3, scale=NONE), INVALID),
    (dict(E4M3, w_scale=NONE), INVALID), (dict(E4M3, out=rows(4)), ALIAS),
    (dict(E4M3, scale=rows(4, 1, 2)), INVALID), (dict(E4M3, k=129, x=rows(0, 129), w=rows(1, 129)), INVALID),
    (dict(MX4, flags=3), UNSUPPORTED), (dict(MX4, dtype=7), UNSUPPORTED), (dict(MX4, scale=NONE), INVALID),
    (dict(MX4, k=65), INVALID), (dict(MX4, scale=rows(4, 1)), INVALID), (dict(MX4, out=rows(5)), ALIAS),
]
GRAD = dict(rows=8, n=64, k=32, experts=4, dtype=1, dw_dtype=0, dout=rows(0), x=rows(1, 32),
            dw=rows(2, 32), dw_expert=64 * 32, offsets=at(3))
GRAD_BAD = [
    (dict(dtype=7), UNSUPPORTED), (dict(dw_dtype=2), UNSUPPORTED), (dict(flags=2), INVALID),
    (dict(experts=0), UNSUPPORTED), (dict(n=0), UNSUPPORTED), (dict(k=(1 << 20) + 1), UNSUPPORTED),
    (dict(n=1 << 20, k=1 << 20, dout=rows(0, 1 << 20), x=rows(1, 1 << 20), experts=1024), UNSUPPORTED),
    (dict(dout=NONE), INVALID), (dict(x=NONE), INVALID), (dict(dw=NONE), INVALID),
    (dict(offsets=None), INVALID), (dict(dw_expert=64 * 32 - 1), INVALID),
    (dict(dw_expert=1 << 62), INVALID), (dict(dw=rows(0, 32)), ALIAS), (dict(dw=rows(3, 32)), ALIAS),
    (dict(dw=rows(2, 32, 2)), INVALID),
]
GATE = dict(rows=8, width=64, group=32, dtype=1, x=rows(0, 128), out=rows(1), out8=rows(2),
            scale=rows(3, 2), count=at(4))
GATE_BAD = [
    (dict(dtype=7), UNSUPPORTED), (dict(width=0), UNSUPPORTED), (dict(width=(1 << 20) + 1), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(rows=1 << 30, width=4096), UNSUPPORTED),
    (dict(group=0), INVALID), (dict(group=48), INVALID), (dict(group=1024), INVALID),
    (dict(x=rows(0, 127)), INVALID), (dict(x=NONE), INVALID), (dict(out=NONE, out8=NONE), INVALID),
    (dict(scale=NONE), INVALID), (dict(out8=NONE), INVALID), (dict(scale=rows(3, 1)), INVALID),
    (dict(out=rows(0)), ALIAS), (dict(out8=rows(1)), ALIAS), (dict(scale=rows(4, 2)), ALIAS),
    (dict(count=at(4, 1)), INVALID), (dict(count=at(1, 8)), ALIAS),
]
GATE_GRAD = dict(rows=8, width=64, dtype=1, dout=rows(0), x=rows(1, 128), dx=rows(2, 128), count=at(4))
GATE_GRAD_BAD = [
    (dict(dtype=9), UNSUPPORTED), (dict(width=0), UNSUPPORTED), (dict(dout=NONE), INVALID),
    (dict(x=NONE), INVALID), (dict(dx=NONE), INVALID), (dict(dx=rows(2, 64)), INVALID),
    (dict(dx=rows(1, 128, 2)), ALIAS), (dict(dx=rows(0, 128)), ALIAS), (dict(dx=rows(1, 256)), ALIAS),
    (dict(dx=rows(4, 128)), ALIAS),
]
QUANT = dict(rows=8, columns=65, dtype=1, x=rows(0, 65), out4=rows(1, 48), scale=rows(2, 3))
QUANT_BAD = [
    (dict(dtype=7), UNSUPPORTED), (dict(columns=0), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(x=NONE), INVALID), (dict(out4=NONE), INVALID), (dict(scale=NONE), INVALID),
    (dict(out4=rows(1, 47)), INVALID), (dict(scale=rows(2, 2)), INVALID), (dict(out4=rows(0, 48)), ALIAS),
    (dict(scale=rows(1, 3)), ALIAS), (dict(x=rows(0, 65, 1)), INVALID),
]
DEQUANT = dict(rows=8, columns=65, dtype=0, x4=rows(0, 48), scale=rows(1, 3), out=rows(2, 65))
DEQUANT_BAD = [
    (dict(dtype=7), UNSUPPORTED), (dict(columns=0), UNSUPPORTED), (dict(x4=NONE), INVALID),
    (dict(scale=NONE), INVALID), (dict(out=NONE), INVALID), (dict(x4=rows(0, 47)), INVALID),
    (dict(out=rows(2, 64)), INVALID), (dict(out=rows(0, 65)), ALIAS), (dict(out=rows(1, 65)), ALIAS),
]
CALLS = [("xred_group_product", _lib.GroupProductArgs, PRODUCT, PRODUCT_BAD),
         ("xred_group_product_grad", _lib.GroupProductGradArgs, GRAD, GRAD_BAD),
         ("xred_gate", _lib.GateArgs, GATE, GATE_BAD),
         ("xred_gate_grad", _lib.GateGradArgs, GATE_GRAD, GATE_GRAD_BAD),
         ("xred_quant_mx4", _lib.QuantMx4Args, QUANT, QUANT_BAD),
         ("xred_dequant_mx4", _lib.DequantMx4Args, DEQUANT, DEQUANT_BAD)]


@pytest.fixture(scope="module")
def L():
    if not _lib.LIB_PATH.exists():
        from paper_2510_20171_amd import build
        build.build()
    return xr.load()


@pytest.mark.parametrize("name,cls,good,bad", CALLS, ids=[c[0] for c in CALLS])
def test_bad_arguments_are_refused(L, name, cls, good, bad):
    f = getattr(L, name)
    assert f(None, None) == INVALID
    for change, status in bad:
        assert f(ctypes.byref(args(cls, good, change)), None) == status, (change, L.xred_last_error())
        assert L.xred_last_error() != b""


@pytest.mark.parametrize("name,cls,good,bad", CALLS, ids=[c[0] for c in CALLS])
def test_good_arguments_reach_the_launch(L, name, cls, good, bad):
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the addresses are not device memory")
    more = [E4M3, MX4, dict(flags=1), dict(out_dtype=0), dict(w_expert=0), dict(experts=1, w_expert=0)]
    for change in more if name == "xred_group_product" else [{}]:
        for dtype in (0, 1, 2) if not change else (None,):
            a = args(cls, good, change)
            if dtype is not None:
                a.dtype = dtype
            assert getattr(L, name)(ctypes.byref(a), None) == 4, (change, L.xred_last_error())


def test_nothing_to_do_succeeds(L):
    for name, cls, good, _ in CALLS:
        empty = dict(rows=0, flags=1) if name == "xred_group_product_grad" else dict(rows=0)
        assert getattr(L, name)(ctypes.byref(args(cls, good, empty)), None) == 0, name


def test_structures_match_the_header(tmp_path):
    names = re.findall(r"typedef struct (xred_\w+_args) \1;", (HEADER / "xred.h").read_text())
    assert set(names) == {c[0] + "_args" for c in CALLS}
    lines, want = [], []
    for call, cls, _, _ in CALLS:
        lines.append(f'printf("%zu\\n", sizeof({call}_args));')
        want.append(ctypes.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({call}_args, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "xred.h"\nint main(void){'
                   + "\n".join(lines) + "}\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", f"-I{HEADER}", str(src), "-o",
                    str(tmp_path / "t")], check=True)
    out = subprocess.run([tmp_path / "t"], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want


class F:
    """The attributes of a GPU tensor the binding reads; every case fails before a call."""

    def __init__(self, *shape, dtype=torch.bfloat16, device="cuda:0", stride=None, cuda=True):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)
        self.is_cuda, self._stride = cuda, stride or torch.empty(shape, device="meta").stride()

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, i):
        return self._stride[i]

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def is_contiguous(self):
        return self._stride == torch.empty(self.shape, device="meta").stride()

    def data_ptr(self):
        return 1 << 40


F32, I32, U8, E4 = torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


def test_cpu_tensors_are_refused():
    x, w, o = torch.zeros(4, 64), torch.zeros(2, 8, 64), torch.zeros(3, dtype=I32)
    b = torch.zeros(4, 32, dtype=U8)
    refused("not in GPU", lambda: xr.group_product(x, w, o, x))
    refused("not in GPU", lambda: xr.group_product_grad(x, x, o, w))
    refused("not in GPU", lambda: xr.gate(x, x))
    refused("not in GPU", lambda: xr.gate_grad(x, x, x))
    refused("not in GPU", lambda: xr.quant_mx4(x, b, b))
    refused("not in GPU", lambda: xr.dequant_mx4(b, b, x))


def test_binding_checks_products():
    x, w, o, y = F(4, 64), F(2, 8, 64), F(3, dtype=I32), F(4, 8)
    refused("dimensions", lambda: xr.group_product(F(64), w, o, y))
    refused("x is torch.int32", lambda: xr.group_product(F(4, 64, dtype=I32), w, o, y))
    refused("w is torch.float32", lambda: xr.group_product(x, F(2, 8, 64, dtype=F32), o, y))
    refused("w has shape (2, 8, 63)", lambda: xr.group_product(x, F(2, 8, 63), o, y))
    refused("expected (2, 64, 8)", lambda: xr.group_product(x, w, o, y, transpose=True))
    refused("w: elements", lambda: xr.group_product(x, F(2, 8, 64, stride=(512, 1, 8)), o, y))
    refused("w is on cuda:1", lambda: xr.group_product(x, F(2, 8, 64, device="cuda:1"), o, y))
    refused("offsets is torch.int64", lambda: xr.group_product(x, w, F(3, dtype=torch.int64), y))
    refused("offsets has shape", lambda: xr.group_product(x, w, F(1, dtype=I32), y))
    refused("offsets[0] is not contiguous", lambda: xr.group_product(x, w, F(3, dtype=I32, stride=(2,)), y))
    refused("out is torch.float16", lambda: xr.group_product(x, w, o, F(4, 8, dtype=torch.float16)))
    refused("out has shape", lambda: xr.group_product(x, w, o, F(5, 8)))
    refused("are given", lambda: xr.group_product(x, w, o, y, scale=F(4, 1, dtype=F32)))
    x8, w8 = F(4, 64, dtype=E4), F(2, 8, 64, dtype=E4)
    s, ws = F(4, 1, dtype=F32), F(2, 1, 1, dtype=F32)
    refused("are needed", lambda: xr.group_product(x8, w8, o, y, scale=s))
    refused("scale has shape", lambda: xr.group_product(x8, w8, o, y, scale=F(4, 2, dtype=F32), w_scale=ws))
    refused("scale is torch.bfloat16", lambda: xr.group_product(x8, w8, o, y, scale=F(4, 1), w_scale=ws))
    refused("w_scale has shape", lambda: xr.group_product(x8, w8, o, y, scale=s, w_scale=F(2, 8, 1, dtype=F32)))
    refused("out is torch.float8", lambda: xr.group_product(x8, w8, o, F(4, 8, dtype=E4), scale=s, w_scale=ws))
    x4, w4 = F(4, 32, dtype=U8), F(2, 8, 32, dtype=U8)
    s, ws = F(4, 2, dtype=U8), F(2, 8, 2, dtype=U8)
    refused("whole blocks", lambda: xr.group_product(
        F(4, 24, dtype=U8), F(2, 8, 24, dtype=U8), o, y, scale=s, w_scale=ws))
    refused("w_scale is torch.float32", lambda: xr.group_product(
        x4, w4, o, y, scale=s, w_scale=F(2, 8, 2, dtype=F32)))
    d, dw = F(4, 8), F(2, 8, 64)
    refused("x is torch.float32", lambda: xr.group_product_grad(d, F(4, 64, dtype=F32), o, dw))
    refused("x has shape", lambda: xr.group_product_grad(d, F(5, 64), o, dw))
    refused("dw has shape", lambda: xr.group_product_grad(d, x, o, F(2, 64, 8)))
    refused("dw is torch.float16", lambda: xr.group_product_grad(d, x, o, F(2, 8, 64, dtype=torch.float16)))
    refused("dout is torch.float8", lambda: xr.group_product_grad(F(4, 8, dtype=E4), x, o, dw))


def test_binding_checks_elements():
    x, y, q, s = F(4, 128), F(4, 64), F(4, 64, dtype=U8), F(4, 1, dtype=F32)
    refused("127 columns", lambda: xr.gate(F(4, 127), y))
    refused("out is torch.float32", lambda: xr.gate(x, F(4, 64, dtype=F32)))
    refused("out has shape", lambda: xr.gate(x, F(4, 128)))
    refused("out8 is", lambda: xr.gate(x, out8=y, scale=s))
    refused("scale has shape", lambda: xr.gate(x, out8=q, scale=s, group=32))
    refused("group = -1", lambda: xr.gate(x, out8=q, scale=s, group=-1))
    refused("offsets is", lambda: xr.gate(x, y, offsets=s))
    refused("offsets is empty", lambda: xr.gate(x, y, offsets=F(0, dtype=I32)))
    refused("dx is", lambda: xr.gate_grad(y, x, F(4, 128, dtype=F32)))
    refused("x has shape", lambda: xr.gate_grad(y, y, x))
    refused("out4 is", lambda: xr.quant_mx4(y, y, q))
    refused("out4 has shape", lambda: xr.quant_mx4(y, F(4, 31, dtype=U8), F(4, 2, dtype=U8)))
    refused("scale has shape", lambda: xr.quant_mx4(y, F(4, 32, dtype=U8), F(4, 1, dtype=U8)))
    refused("out is torch.uint8", lambda: xr.dequant_mx4(F(4, 32, dtype=U8), F(4, 2, dtype=U8), q))
