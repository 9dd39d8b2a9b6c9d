"""Launches of the calls around a reduced activation at sizes whose work items
number 2^32 and more: a launch has to have fewer than 2^32 threads, so its
workgroups take the rest of the work in turns.  The grids are read from the launch
trace, without a GPU: the calls get as far as the launch and fail there."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")
ROOT = Path(__file__).resolve().parents[1]

CALLS = """
import ctypes
import paper_2510_20171_amd as xr
from paper_2510_20171_amd import _lib
L = xr.load()
at = lambda k: 1 << 46 | k << 41          # made up, never dereferenced; 2 TiB apart
rows = lambda k, n: _lib.XredRows(at(k), n)

def call(name, cls, **fields):
    a = cls()
    for k, v in fields.items():
        setattr(a, k, v)
    st = getattr(L, name)(ctypes.byref(a), None)
    assert st == 4, (name, fields, st, L.xred_last_error())

srcs = (ctypes.c_void_p * 8)(*(at(10 + k) for k in range(8)))
for hidden, n, dtype in ((8, (1 << 29) + 1, 0), (512, (1 << 26) + 1, 1), (4096, (1 << 22) + 1, 0),
                         (8192, (1 << 23) + 1, 1), (32768, (1 << 22) + 1, 2)):
    for nsrc in (1, 8):
        call("xred_fold_norm", _lib.FoldNormArgs, srcs=ctypes.addressof(srcs), src_stride=hidden,
             nsrc=nsrc, rows=n, hidden=hidden, out=rows(0, hidden), dtype=dtype,
             weight_dtype=dtype, eps=1e-6)
    need = L.xred_fold_norm_grad_workspace(n, hidden)
    call("xred_fold_norm_grad", _lib.FoldNormGradArgs, rows=n, hidden=hidden, dout=rows(0, hidden),
         sum=rows(1, hidden), dx=rows(2, hidden), rstd=at(3), dweight=at(4), workspace=at(5),
         workspace_bytes=need, dtype=dtype, weight_dtype=dtype)
for experts, n in ((8, (1 << 28) + 1), (200, (1 << 28) + 1), (512, (1 << 26) + 1),
                   (1024, (1 << 28) + 1)):
    call("xred_route", _lib.RouteArgs, tokens=n, experts=experts, topk=4, groups=1,
         logits=rows(0, experts), ids=at(1), weights=at(2), dtype=1, score=1, scale=1.0)
    call("xred_route_grad", _lib.RouteGradArgs, tokens=n, experts=experts, topk=4,
         logits=rows(0, experts), dlogits=rows(1, experts), ids=at(2), dweights=at(3), dtype=1,
         score=1, scale=1.0)
call("xred_dispatch_plan", _lib.DispatchPlanArgs, tokens=(1 << 31) - 1, topk=1, experts=64,
     ids=at(0), counts=at(1), offsets=at(2), pos=at(3), workspace=at(4), workspace_bytes=1 << 20)
for hidden, n, k in ((64, (1 << 26) + 1, 1), (64, (1 << 28) + 1, 16), (8192, (1 << 22) + 1, 4),
                     (8192, (1 << 24) + 1, 2), (16384, (1 << 22) + 1, 8)):
    many = dict(tokens=n, hidden=hidden, topk=k, dtype=1, pos=at(4))
    call("xred_dispatch", _lib.DispatchArgs, out_rows=n, x=rows(0, hidden), out=rows(1, hidden),
         **many)
    call("xred_combine", _lib.CombineArgs, y_rows=n, y=rows(0, hidden), out=rows(1, hidden), **many)
    call("xred_combine_grad", _lib.CombineGradArgs, y_rows=n, dout=rows(0, hidden),
         y=rows(1, hidden), dy=rows(2, hidden), weights=at(5), dweights=at(6), **many)
"""


def test_launches_have_fewer_than_2_32_threads():
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the addresses are not device memory")
    r = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, env={**os.environ, "XRED_TRACE": "1"},
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    launches = [line for line in r.stderr.splitlines() if line.startswith("[xred] launch ")]
    assert len(launches) >= 10 + 5 + 8 + 1 + 15
    threads = {}
    for line in launches:
        grid, block = (int(line.split(f" {key}=")[1].split()[0]) for key in ("grid", "block"))
        threads[line] = grid * block
    over = [line for line, n in threads.items() if n >= 1 << 32]
    assert not over, over
    assert max(threads.values()) > 1 << 30    # and the sizes do ask for as many as there may be


@pytest.mark.gpu
def test_more_tokens_than_a_launch_has_lanes_for():
    """2^28 + 5 tokens at 16 lanes each: the last ones are the first workgroups' second turn."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    g = torch.Generator(device="cuda").manual_seed(2)
    n, e = (1 << 28) + 5, 8
    x = torch.empty((n, e), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ids = torch.full((n, 1), 77, dtype=torch.int32, device="cuda")
    w = torch.full((n, 1), 7.0, device="cuda")
    xr.route(x, ids, w)
    most = torch.full((n,), -torch.inf, dtype=x.dtype, device="cuda")
    best = torch.zeros(n, dtype=torch.int32, device="cuda")
    for k in range(e):                     # the first of the largest
        best.masked_fill_(x[:, k] > most, k)
        torch.maximum(most, x[:, k], out=most)
    assert torch.equal(ids[:, 0], best)
    assert bool((w == 1).all())            # the softmax over one
