"""Refusals of the calls around a reduced activation, without a GPU: every bad
argument is rejected before anything is enqueued, by the C ABI and by the
Python binding (whose compiled and plain halves make the same checks)."""
import ctypes
import re
import struct
import subprocess
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")
import paper_2510_20171_amd as xr  # noqa: E402
from paper_2510_20171_amd import _lib  # noqa: E402

INVALID, UNSUPPORTED, ALIAS = 1, 2, 3
A = 0x7F0000000000   # fake device addresses: never dereferenced
MB = 1 << 20


@pytest.fixture(scope="module")
def L():
    if not _lib.LIB_PATH.exists():
        from paper_2510_20171_amd import build
        build.build()
    return xr.load()


def rows(k, stride=64, off=0):
    """The k-th buffer of a call, a MiB from the others."""
    return _lib.XredRows(A + k * MB + off, stride)


def at(k, off=0):
    return A + k * MB + off


NONE = _lib.XredRows(None, 0)
SRCS = (ctypes.c_void_p * 2)(A + 20 * MB, A + 21 * MB)
NULLS = (ctypes.c_void_p * 2)(A, None)
INSIDE = (ctypes.c_void_p * 2)(A + 20 * MB, A + 1 * MB + 128)


def args(cls, good, bad):
    values = {**good, **bad}
    a = cls()
    for k, v in values.items():
        setattr(a, k, v)
    return a


FOLD = dict(srcs=ctypes.addressof(SRCS), src_stride=64, nsrc=2, rows=4, hidden=64, residual=rows(0),
            sum=rows(1), out=rows(2), weight=at(3), dtype=1, weight_dtype=1, eps=1e-6)
FOLD_BAD = [
    (dict(nsrc=0), INVALID), (dict(nsrc=65), INVALID), (dict(srcs=None), INVALID),
    (dict(srcs=ctypes.addressof(NULLS)), INVALID), (dict(dtype=7), UNSUPPORTED),
    (dict(dtype=9), UNSUPPORTED), (dict(dtype=99), UNSUPPORTED), (dict(hidden=0), UNSUPPORTED),
    (dict(hidden=32769, src_stride=1 << 20), UNSUPPORTED), (dict(src_stride=63), INVALID),
    (dict(out=NONE), INVALID), (dict(out8=rows(5)), INVALID), (dict(scale=rows(5)), INVALID),
    (dict(group=48), INVALID), (dict(group=1024), INVALID), (dict(group=16), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(weight_dtype=2), UNSUPPORTED), (dict(weight=at(3, 1)), INVALID),
    (dict(residual=rows(0, 64, 1)), INVALID), (dict(sum=rows(1, 2 ** 62)), INVALID),
    (dict(sum=rows(2)), ALIAS), (dict(sum=rows(0, 64, 2)), ALIAS), (dict(out=rows(3)), ALIAS),
    (dict(sum=rows(0, 128)), ALIAS), (dict(rstd=at(2, 4)), ALIAS), (dict(rstd=at(6, 2)), INVALID),
    (dict(out8=rows(2, 64), scale=rows(7, 1)), ALIAS), (dict(out8=rows(5), scale=rows(5, 1)), ALIAS),
    (dict(out8=rows(5), scale=rows(7, 1), group=32), INVALID),   # two groups a row
    (dict(srcs=ctypes.addressof(INSIDE)), ALIAS),
]
GRAD = dict(rows=4, hidden=64, dout=rows(0), sum=rows(1), dsum=rows(2), dx=rows(3), weight=at(4),
            rstd=at(5), dweight=at(6), workspace=at(7), workspace_bytes=1 << 19, dtype=1,
            weight_dtype=1)
GRAD_BAD = [
    (dict(dtype=3), UNSUPPORTED), (dict(hidden=32769), UNSUPPORTED), (dict(dout=NONE), INVALID),
    (dict(sum=NONE), INVALID), (dict(rstd=None), INVALID), (dict(dx=NONE), INVALID),
    (dict(workspace=None), INVALID), (dict(workspace_bytes=255), INVALID),
    (dict(workspace=at(7, 8)), INVALID), (dict(weight_dtype=2), UNSUPPORTED),
    (dict(dx=rows(1)), ALIAS), (dict(dx=rows(0, 64, 2)), ALIAS), (dict(dweight=at(4)), ALIAS),
    (dict(workspace=at(6)), ALIAS), (dict(workspace=at(0)), ALIAS), (dict(dsum=rows(2, 10)), INVALID),
]
ROUTE = dict(tokens=4, experts=64, topk=8, groups=1, group_topk=1, group_score=1, logits=rows(0),
             bias=at(1), ids=at(2), weights=at(3), dtype=0, score=1, scale=1.0)
ROUTE_BAD = [
    (dict(dtype=8), UNSUPPORTED), (dict(score=2), INVALID), (dict(score=-1), INVALID),
    (dict(flags=2), INVALID), (dict(experts=0), UNSUPPORTED),
    (dict(experts=1025, logits=rows(0, 2048)), UNSUPPORTED), (dict(topk=0), INVALID),
    (dict(topk=65), INVALID), (dict(topk=33), UNSUPPORTED), (dict(groups=0), INVALID),
    (dict(groups=5), INVALID), (dict(experts=1024, groups=128, logits=rows(0, 1024)), INVALID),
    (dict(groups=8, group_topk=0), INVALID), (dict(groups=8, group_topk=9), INVALID),
    (dict(groups=8, group_score=3), INVALID), (dict(logits=NONE), INVALID),
    (dict(logits=rows(0, 63)), INVALID), (dict(logits=rows(0, 64, 2)), INVALID),
    (dict(ids=None), INVALID), (dict(weights=None), INVALID), (dict(weights=at(2)), ALIAS),
    (dict(ids=at(0, 8)), ALIAS), (dict(bias=at(3, 4)), ALIAS), (dict(tokens=2 ** 62), INVALID),
]
RGRAD = dict(tokens=4, experts=64, topk=8, logits=rows(0), dlogits=rows(1), ids=at(2),
             dweights=at(3), dtype=0, score=0, scale=1.0)
RGRAD_BAD = [
    (dict(topk=65), INVALID), (dict(flags=4), INVALID), (dict(dlogits=NONE), INVALID),
    (dict(dlogits=rows(0)), ALIAS), (dict(dlogits=rows(3)), ALIAS), (dict(ids=None), INVALID),
    (dict(dweights=at(3, 1)), INVALID), (dict(score=7), INVALID),
]
PLAN = dict(tokens=4, experts=64, topk=8, ids=at(0), counts=at(1), offsets=at(2), pos=at(3),
            slots=at(4))
PLAN_BAD = [
    (dict(experts=0), UNSUPPORTED), (dict(experts=1025), UNSUPPORTED), (dict(topk=0), UNSUPPORTED),
    (dict(topk=33), UNSUPPORTED), (dict(tokens=1 << 29), UNSUPPORTED), (dict(ids=None), INVALID),
    (dict(counts=None), INVALID), (dict(offsets=None), INVALID), (dict(pos=None), INVALID),
    (dict(pos=at(0)), ALIAS), (dict(slots=at(3, 64)), ALIAS), (dict(offsets=at(1, 252)), ALIAS),
    (dict(tokens=1 << 16), INVALID),   # needs a workspace
    (dict(tokens=1 << 16, ids=at(32), pos=at(64), slots=None, workspace=at(64),
          workspace_bytes=1 << 20), ALIAS),
]
DISPATCH = dict(tokens=4, hidden=64, out_rows=32, scale_columns=2, topk=8, dtype=7, x=rows(0),
                out=rows(1), scale=rows(2, 2), out_scale=rows(3, 2), pos=at(4))
DISPATCH_BAD = [
    (dict(dtype=12), INVALID), (dict(topk=0), UNSUPPORTED), (dict(topk=33), UNSUPPORTED),
    (dict(hidden=0), UNSUPPORTED), (dict(hidden=(1 << 30) + 1), UNSUPPORTED), (dict(x=NONE), INVALID),
    (dict(out=NONE), INVALID), (dict(scale=NONE), INVALID), (dict(out_scale=NONE), INVALID),
    (dict(pos=None), INVALID), (dict(out=rows(0)), ALIAS), (dict(out_scale=rows(2, 2)), ALIAS),
    (dict(out=rows(3)), ALIAS), (dict(out=rows(4, 64, 8)), ALIAS), (dict(scale=rows(2, 1)), INVALID),
    (dict(scale_columns=0), UNSUPPORTED), (dict(x=rows(0, 60)), INVALID),
]
COMBINE = dict(tokens=4, hidden=64, y_rows=32, topk=8, dtype=1, y=rows(0), base=rows(1), out=rows(2),
               pos=at(3), weights=at(4))
COMBINE_BAD = [
    (dict(dtype=7), UNSUPPORTED), (dict(topk=33), UNSUPPORTED), (dict(hidden=0), UNSUPPORTED),
    (dict(y=NONE), INVALID), (dict(out=NONE), INVALID), (dict(pos=None), INVALID),
    (dict(out=rows(0)), ALIAS), (dict(out=rows(1, 64, 2)), ALIAS), (dict(out=rows(4)), ALIAS),
    (dict(base=rows(1, 63)), INVALID), (dict(weights=at(4, 2)), INVALID),
]
CGRAD = dict(tokens=4, hidden=64, y_rows=32, topk=8, dtype=1, dout=rows(0), y=rows(1), dy=rows(2),
             pos=at(3), weights=at(4), dweights=at(5))
CGRAD_BAD = [
    (dict(dtype=3), UNSUPPORTED), (dict(dout=NONE), INVALID), (dict(y=NONE), INVALID),
    (dict(dy=NONE), INVALID), (dict(weights=None), INVALID), (dict(pos=None), INVALID),
    (dict(dy=rows(0)), ALIAS), (dict(dy=rows(1, 64, 2)), ALIAS), (dict(dweights=at(4)), ALIAS),
    (dict(dweights=at(2, 4)), ALIAS), (dict(topk=0), UNSUPPORTED),
]
CALLS = [("xred_fold_norm", _lib.FoldNormArgs, FOLD, FOLD_BAD),
         ("xred_fold_norm_grad", _lib.FoldNormGradArgs, GRAD, GRAD_BAD),
         ("xred_route", _lib.RouteArgs, ROUTE, ROUTE_BAD),
         ("xred_route_grad", _lib.RouteGradArgs, RGRAD, RGRAD_BAD),
         ("xred_dispatch_plan", _lib.DispatchPlanArgs, PLAN, PLAN_BAD),
         ("xred_dispatch", _lib.DispatchArgs, DISPATCH, DISPATCH_BAD),
         ("xred_combine", _lib.CombineArgs, COMBINE, COMBINE_BAD),
         ("xred_combine_grad", _lib.CombineGradArgs, CGRAD, CGRAD_BAD)]


@pytest.mark.parametrize("name,cls,good,bad", CALLS, ids=[c[0] for c in CALLS])
def test_bad_arguments_are_refused(L, name, cls, good, bad):
    f = getattr(L, name)
    assert f(None, None) == INVALID
    for change, status in bad:
        assert f(ctypes.byref(args(cls, good, change)), None) == status, (change, L.xred_last_error())
        assert L.xred_last_error() != b""


@pytest.mark.parametrize("name,cls,good,bad", CALLS, ids=[c[0] for c in CALLS])
def test_good_arguments_reach_the_launch(L, name, cls, good, bad):
    """The base every refusal departs from is accepted: without a GPU it fails only
    at the launch (with one it is not tried, its addresses being made up)."""
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the addresses are not device memory")
    assert getattr(L, name)(ctypes.byref(args(cls, good, {})), None) == 4, L.xred_last_error()


def test_views_of_one_matrix_may_interleave(L):
    """Column ranges of one larger matrix do not overlap though their spans do."""
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the addresses are not device memory")
    wide = dict(sum=rows(0, 192), out=rows(0, 192, 128), residual=rows(0, 192, 256))
    f = lambda **kw: L.xred_fold_norm(ctypes.byref(args(_lib.FoldNormArgs, FOLD, {**wide, **kw})), None)
    assert f() == 4
    assert f(out=rows(0, 192, 126)) == ALIAS        # one element too far left
    assert f(out=rows(0, 192, 130)) == ALIAS        # and right, into the residual
    assert f(sum=rows(0, 192, 256)) == 4            # the residual itself, in place
    assert f(sum=rows(0, 384, 256)) == ALIAS        # its rows at another distance


def test_nothing_to_do_succeeds(L):
    for name, cls, good, _ in CALLS:
        empty = {"rows": 0, "dweight": None} if "norm" in name else {"tokens": 0}
        if name == "xred_fold_norm":
            empty.pop("dweight")
        if name == "xred_dispatch_plan":
            continue   # counts and offsets are still written
        assert getattr(L, name)(ctypes.byref(args(cls, good, empty)), None) == 0, name


def test_workspace_sizes(L):
    assert L.xred_fold_norm_grad_workspace(0, 64) == 0
    for r in (1, 255, 256, 4096, 1 << 20):
        assert 0 < L.xred_fold_norm_grad_workspace(r, 100) <= min(r, 12 * 256) * 400
    assert L.xred_dispatch_plan_workspace(1, 64) == 0
    assert 0 < L.xred_dispatch_plan_workspace(2 ** 31 - 1, 1024) <= 1 << 20


def test_structures_match_the_header(tmp_path):
    """Sizes and offsets of the ctypes structures against the header's, by a C program."""
    text = (Path(__file__).resolve().parents[1] / "include" / "xred.h").read_text()
    pairs = {"xred_rows": _lib.XredRows, "xred_fold_norm_args": _lib.FoldNormArgs,
             "xred_fold_norm_grad_args": _lib.FoldNormGradArgs, "xred_route_args": _lib.RouteArgs,
             "xred_route_grad_args": _lib.RouteGradArgs,
             "xred_dispatch_plan_args": _lib.DispatchPlanArgs,
             "xred_dispatch_args": _lib.DispatchArgs, "xred_combine_args": _lib.CombineArgs,
             "xred_combine_grad_args": _lib.CombineGradArgs}
    assert set(re.findall(r"}\s*(xred_\w+_args);", text)) < set(pairs)
    lines, want = [], []
    for name, cls in pairs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "xred.h"\nint main(void){' + "\n".join(lines) + "}\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror",
                    f"-I{Path(__file__).resolve().parents[1] / 'include'}", str(src), "-o",
                    str(tmp_path / "t")], check=True)
    out = subprocess.run([tmp_path / "t"], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want


def test_host_and_device_name_the_kernels_alike(tmp_path):
    """Every kernel name the host half hands to the runtime exists in the device code:
    a name that differs (an unnamed type in a kernel's parameters) ends the process at
    its first launch."""
    tools = Path("/opt/rocm/llvm/bin")
    if not (tools / "llvm-readelf").exists() or not (tools / "llvm-objcopy").exists():
        pytest.skip("no LLVM tools")
    for section in ("hip_fatbin", "rodata"):
        subprocess.run([tools / "llvm-objcopy", f"--dump-section=.{section}={tmp_path / section}",
                        _lib.LIB_PATH, tmp_path / "copy"], check=True, timeout=100)
    fat, device = (tmp_path / "hip_fatbin").read_bytes(), set()
    start = fat.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while start >= 0:
        n, = struct.unpack_from("<Q", fat, start + 24)
        pos = start + 32
        for _ in range(n):
            off, size, length = struct.unpack_from("<QQQ", fat, pos)
            pos += 24
            if size and b"gfx950" in fat[pos:pos + length]:
                (tmp_path / "co").write_bytes(fat[start + off:start + off + size])
                syms = subprocess.run([tools / "llvm-readelf", "--dyn-syms", "-W", tmp_path / "co"],
                                      check=True, timeout=100, capture_output=True, text=True).stdout
                device |= {line.split()[-1] for line in syms.splitlines() if "FUNC" in line}
            pos += length
        start = fat.find(b"__CLANG_OFFLOAD_BUNDLE__", start + 1)
    host = {m.decode() for m in re.findall(rb"_Z[A-Za-z0-9_$]*kernel[A-Za-z0-9_$]*",
                                           (tmp_path / "rodata").read_bytes())}
    assert len(host) > 1000 and host <= device, sorted(host - device)[:5]


class FakeGpuTensor:
    """The attributes of a GPU tensor the binding reads; every case fails before a call."""

    def __init__(self, *shape, dtype=torch.bfloat16, device="cuda:0", stride=None, cuda=True):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)
        self.is_cuda, self._stride = cuda, stride or (shape[-1], 1)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, i):
        return self._stride[i]

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def is_contiguous(self):
        return self._stride == (self.shape[-1], 1)

    def data_ptr(self):
        return 1 << 40


F = FakeGpuTensor
F32, I32 = torch.float32, torch.int32


def refused(match, call):
    with pytest.raises(xr.XredError) as e:
        call()
    assert e.value.status == INVALID and match in str(e.value), str(e.value)


def test_cpu_tensors_are_refused():
    x = torch.zeros(4, 64)
    ids, w = torch.zeros(4, 2, dtype=I32), torch.zeros(4, 2)
    refused("not in GPU", lambda: xr.fold_norm([x], x.clone()))
    refused("not in GPU", lambda: xr.fold_norm_grad(x, x, w, x))
    refused("not in GPU", lambda: xr.route(x, ids, w))
    refused("not in GPU", lambda: xr.route_grad(x, ids, w, x))
    refused("not in GPU", lambda: xr.dispatch_plan(ids, ids[0], ids[0], ids))
    refused("not in GPU", lambda: xr.dispatch(x, ids, x))
    refused("not in GPU", lambda: xr.combine(x, ids, x))
    refused("not in GPU", lambda: xr.combine_grad(x, x, ids, w, x, w))


def test_binding_checks_matrices():
    refused("no sources", lambda: xr.fold_norm([], F(4, 64)))
    refused("dimensions", lambda: xr.fold_norm([F(256)], F(4, 64)))
    refused("srcs[1] has shape (4, 63)", lambda: xr.fold_norm([F(4, 64), F(4, 63)], F(4, 64)))
    refused("different row distances",
            lambda: xr.fold_norm([F(4, 64), F(4, 64, stride=(80, 1))], F(4, 64)))
    refused("not contiguous", lambda: xr.fold_norm([F(4, 64, stride=(64, 2))], F(4, 64)))
    refused("residual is torch.float16",
            lambda: xr.fold_norm([F(4, 64)], F(4, 64), residual=F(4, 64, dtype=torch.float16)))
    refused("cuda:1", lambda: xr.fold_norm([F(4, 64)], F(4, 64, device="cuda:1")))
    refused("weight is f16",
            lambda: xr.fold_norm([F(4, 64)], F(4, 64), weight=F(64, dtype=torch.float16)))
    refused("out8 is", lambda: xr.fold_norm([F(4, 64)], out8=F(4, 64), scale=F(4, 1, dtype=F32)))
    refused("scale has shape", lambda: xr.fold_norm(
        [F(4, 64)], out8=F(4, 64, dtype=torch.uint8), scale=F(4, 1, dtype=F32), group=32))
    refused("rstd is torch.int32", lambda: xr.fold_norm([F(4, 64)], F(4, 64), rstd=F(4, dtype=I32)))
    refused("dx is torch.float32",
            lambda: xr.fold_norm_grad(F(4, 64), F(4, 64), F(4, dtype=F32), F(4, 64, dtype=F32)))


def test_binding_checks_slots():
    x, ids, w = F(4, 64), F(4, 2, dtype=I32), F(4, 2, dtype=F32)
    refused("unknown score", lambda: xr.route(x, ids, w, score="topk"))
    refused("ids is torch.int64", lambda: xr.route(x, F(4, 2, dtype=torch.int64), w))
    refused("weights has shape", lambda: xr.route(x, ids, F(4, 3, dtype=F32)))
    refused("bias is", lambda: xr.route(x, ids, w, bias=F(64)))
    refused("bias[0] has 63", lambda: xr.route(x, ids, w, bias=F(63, dtype=F32)))
    refused("dlogits is", lambda: xr.route_grad(x, ids, w, F(4, 64, dtype=F32)))
    refused("offsets[0] has 8", lambda: xr.dispatch_plan(ids, F(8, dtype=I32), F(8, dtype=I32), ids))
    refused("pos is", lambda: xr.dispatch_plan(ids, F(8, dtype=I32), F(9, dtype=I32), w))
    refused("out is", lambda: xr.dispatch(x, ids, F(8, 64, dtype=F32)))
    refused("out has shape", lambda: xr.dispatch(x, ids, F(8, 63)))
    refused("go together", lambda: xr.dispatch(x, ids, F(8, 64), scale=F(4, 2, dtype=F32)))
    refused("pos has shape", lambda: xr.dispatch(x, F(5, 2, dtype=I32), F(8, 64)))
    refused("base has shape", lambda: xr.combine(F(8, 64), ids, x, base=F(5, 64)))
    refused("weights is", lambda: xr.combine(F(8, 64), ids, x, weights=ids))
    refused("dweights needs y", lambda: xr.combine_grad(x, None, ids, w, F(8, 64), w))
    refused("y has shape", lambda: xr.combine_grad(x, F(9, 64), ids, w, F(8, 64), w))
