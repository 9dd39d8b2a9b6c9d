"""The calls between dispatch and combine through the binding's compiled marshalling and
its Python code, on the current stream, another stream and a raw handle; with canaries
around every output; and from several threads.  What the calls compute is compared with
their definitions elsewhere; here every way of making a call has to give the same bytes."""
import threading

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from test_gpu_layer_binding import Job as Layer  # noqa: E402
from test_gpu_layer_binding import Sub, same  # noqa: E402


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


class Job(Layer):
    """One round of every call, as its base class has them."""

    def __init__(self, seed, dtype=torch.bfloat16, rows=700, n=344, k=203, experts=6, shift=0, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.shift, self.pad, self.outs = shift, pad, []
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        cuts = torch.randint(0, rows + 1, (experts - 1,), device="cuda", generator=g).sort().values
        self.offsets = torch.cat([cuts.new_zeros(1), cuts, cuts.new_tensor([rows])]).int()
        self.x, self.w, self.dout = rand(rows, k).to(dtype), rand(experts, n, k).to(dtype), rand(rows, n).to(dtype)
        self.gates, self.dgated = rand(rows, 2 * n).to(dtype), rand(rows, n).to(dtype)
        f32, u8 = torch.float32, torch.uint8
        kb, nb, blocks = -(-k // 128), -(-n // 128), -(-k // 32)
        self.x8 = rand(rows, k).to(torch.float8_e4m3fn)
        self.w8 = rand(experts, n, k).to(torch.float8_e4m3fn)
        self.x8_scale, self.w8_scale = rand(rows, kb), rand(experts, nb, kb)
        self.w4 = torch.randint(0, 256, (experts, n, blocks * 16), device="cuda", generator=g).to(u8)
        self.w4_scale = torch.randint(120, 134, (experts, n, blocks), device="cuda", generator=g).to(u8)
        self.y, self.dx, self.y8, self.y4 = (self.new(dtype, rows, c) for c in (n, k, n, n))
        self.dw = self.new(f32, experts * n, k)
        self.dw = self.dw.unflatten(0, (experts, n))
        self.gated, self.dgates = self.new(dtype, rows, n), self.new(dtype, rows, 2 * n)
        self.gated8, self.gated_scale = self.new(torch.float8_e4m3fn, rows, n), self.new(f32, rows, -(-n // 64))
        self.x4, self.x4_scale = self.new(u8, rows, blocks * 16), self.new(u8, rows, blocks)
        self.values = self.new(dtype, rows, k)

    def run(self, xr, wrap=lambda t: t, stream=None):
        w, kw, at = wrap, {"stream": stream}, wrap(self.offsets)
        xr.group_product(w(self.x), w(self.w), at, w(self.y), **kw)
        xr.group_product(w(self.dout), w(self.w), at, w(self.dx), transpose=True, **kw)
        xr.group_product(w(self.x8), w(self.w8), at, w(self.y8), scale=w(self.x8_scale),
                         w_scale=w(self.w8_scale), **kw)
        xr.group_product_grad(w(self.dout), w(self.x), at, w(self.dw), **kw)
        xr.group_product_grad(w(self.dout), w(self.x), at, w(self.dw), add=True, **kw)
        xr.gate(w(self.gates), w(self.gated), out8=w(self.gated8), scale=w(self.gated_scale), group=64,
                offsets=at, **kw)
        xr.gate_grad(w(self.dgated), w(self.gates), w(self.dgates), offsets=at, **kw)
        xr.quant_mx4(w(self.x), w(self.x4), w(self.x4_scale), **kw)
        xr.dequant_mx4(w(self.x4), w(self.x4_scale), w(self.values), **kw)
        xr.group_product(w(self.x4), w(self.w4), at, w(self.y4), scale=w(self.x4_scale),
                         w_scale=w(self.w4_scale), **kw)
        return self


@pytest.mark.parametrize("which", ["current", "object", "handle"])
def test_same_results(xr, which):
    s = torch.cuda.Stream()
    stream = {"current": None, "object": s, "handle": s.cuda_stream}[which]
    fast, slow = Job(3), Job(3)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        fast.run(xr, stream=stream)
        slow.run(xr, wrap=lambda t: t.as_subclass(Sub), stream=stream)
    torch.cuda.synchronize()
    same(fast, slow)


def test_same_results_without_the_module(xr, monkeypatch):
    fast = Job(4).run(xr)
    assert not isinstance(xr._lib.native(), xr._lib._Declines)
    monkeypatch.setattr(xr._lib, "_native", xr._lib._Declines())
    slow = Job(4).run(xr)
    torch.cuda.synchronize()
    same(fast, slow)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 0), (0, 8), (3, 5)])
def test_bytes_around_the_outputs_are_left_alone(xr, dtype, shift, pad):
    for rows, n, k, experts in ((1, 1, 1, 1), (33, 72, 40, 16), (130, 203, 131, 5), (1500, 3848, 72, 2),
                                (1500, 3845, 71, 2), (40, 264, 512, 64), (600, 2056, 2064, 2)):
        j = Job(rows, dtype, rows, n, k, experts, shift, pad).run(xr)
        torch.cuda.synchronize()
        j.check_bands()


def test_threads_on_their_own_streams(xr):
    """Four threads, each with its own stream, while another changes the CU budget:
    each round's outputs are those of the same round run alone."""
    shapes = [(rows, n, k) for rows in (20, 700, 1400) for n, k in ((344, 203), (1288, 136))]
    want = [Job(100 + r, rows=s[0], n=s[1], k=s[2]).run(xr) for r, s in enumerate(shapes)]
    jobs = [[Job(100 + r, rows=s[0], n=s[1], k=s[2]) for r, s in enumerate(shapes)] for _ in range(4)]
    torch.cuda.synchronize()
    streams, errors = [torch.cuda.Stream() for _ in range(4)], []
    start, stop = threading.Barrier(5), threading.Event()

    def worker(t):
        try:
            start.wait()
            for j in jobs[t]:
                j.run(xr, stream=streams[t])
        except Exception as e:   # raised again below, in the test's thread
            errors.append((t, e))

    def budgets():
        start.wait()
        r = 0
        while not stop.is_set():
            xr.set_max_workgroups((0, 1, 7, 0, 64, 300)[r % 6])
            r += 1

    threads = [threading.Thread(target=worker, args=(t,)) for t in range(4)]
    other = threading.Thread(target=budgets)
    try:
        for t in threads + [other]:
            t.start()
        for t in threads:
            t.join(100)
    finally:
        stop.set()
        other.join(10)
        xr.set_max_workgroups(0)
    assert not errors, errors
    torch.cuda.synchronize()
    for mine in jobs:
        for j, ref in zip(mine, want):
            same(j, ref)
