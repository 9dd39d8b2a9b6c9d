"""The calls around a reduced activation as the other entry points are tested: through
the binding's compiled marshalling and its Python code, on the current stream, another
stream and a raw handle; with canaries around every output; and from several threads.
What the calls compute is compared with their definitions elsewhere; here every way of
making a call has to give the same bytes."""
import threading

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

CANARY = 0x5A


class Sub(torch.Tensor):
    pass


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


class Job:
    """Inputs and outputs of one round of every call.  Outputs lie between bands of
    canaries, `shift` elements off a 16-byte boundary; rows are `pad` elements apart."""

    def __init__(self, seed, dtype=torch.bfloat16, rows=700, hidden=1003, experts=96, topk=8,
                 shift=0, pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden, self.experts = hidden, experts
        self.shift, self.pad, self.outs = shift, pad, []
        rand = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        self.srcs = [rand(rows, hidden).to(dtype) for _ in range(3)]
        self.residual, self.weight = rand(rows, hidden).to(dtype), rand(hidden).to(dtype)
        self.bias, self.logits = 0.1 * rand(experts), rand(rows, experts).to(dtype)
        self.dout, self.dsum = rand(rows, hidden).to(dtype), rand(rows, hidden).to(dtype)
        self.dweights, self.y = rand(rows, topk), rand(rows * topk, hidden).to(dtype)
        f32, i32, u8 = torch.float32, torch.int32, torch.uint8
        self.sum, self.out = self.new(dtype, rows, hidden), self.new(dtype, rows, hidden)
        self.out8, self.scale = self.new(u8, rows, hidden), self.new(f32, rows, -(-hidden // 128))
        self.rstd, self.dweight = self.new(f32, rows), self.new(f32, hidden)
        self.dx, self.dlogits = self.new(dtype, rows, hidden), self.new(dtype, rows, experts)
        self.ids, self.weights = self.new(i32, rows, topk, pad=0), self.new(f32, rows, topk, pad=0)
        self.counts, self.offsets = self.new(i32, experts), self.new(i32, experts + 1)
        self.pos, self.slots = self.new(i32, rows, topk, pad=0), self.new(i32, rows * topk)
        self.moved = self.new(u8, rows * topk, hidden)
        self.moved_scale = self.new(f32, rows * topk, self.scale.shape[1])
        self.back, self.dy = self.new(dtype, rows, hidden), self.new(dtype, rows * topk, hidden)
        self.dw = self.new(f32, rows, topk, pad=0)

    def new(self, dtype, *shape, pad=None):
        pad = self.pad if pad is None else pad
        es = torch.empty(0, dtype=dtype).element_size()
        row = shape[-1] + (pad if len(shape) == 2 else 0)
        n = row * (shape[0] if len(shape) == 2 else 1)
        lead = 4096 + self.shift * es
        store = torch.full((lead + n * es + 4096,), CANARY, dtype=torch.uint8, device="cuda")
        t = store[lead:lead + n * es].view(dtype)
        if len(shape) == 2:
            t = t.view(shape[0], row)[:, :shape[1]]
        self.outs.append((store, t, es, lead, n))
        return t

    def run(self, xr, wrap=lambda t: t, stream=None):
        w, kw = wrap, {"stream": stream}
        xr.fold_norm([w(s) for s in self.srcs], w(self.out), residual=w(self.residual),
                     weight=w(self.weight), sum=w(self.sum), out8=w(self.out8), scale=w(self.scale),
                     rstd=w(self.rstd), group=128, **kw)
        xr.fold_norm_grad(w(self.dout), w(self.sum), w(self.rstd), w(self.dx), weight=w(self.weight),
                          dsum=w(self.dsum), dweight=w(self.dweight), **kw)
        xr.route(w(self.logits), w(self.ids), w(self.weights), score="sigmoid", bias=w(self.bias),
                 groups=8, group_topk=4, scale=2.5, **kw)
        xr.route_grad(w(self.logits), w(self.ids), w(self.dweights), w(self.dlogits),
                      score="sigmoid", scale=2.5, **kw)
        xr.dispatch_plan(w(self.ids), w(self.counts), w(self.offsets), w(self.pos),
                         slots=w(self.slots), **kw)
        xr.dispatch(w(self.out8), w(self.pos), w(self.moved), scale=w(self.scale),
                    out_scale=w(self.moved_scale), **kw)
        xr.combine(w(self.y), w(self.pos), w(self.back), weights=w(self.weights), base=w(self.sum),
                   **kw)
        xr.combine_grad(w(self.dout), w(self.y), w(self.pos), w(self.weights), w(self.dy),
                        w(self.dw), **kw)
        return self

    def stores(self):
        return [store for store, *_ in self.outs]

    def check_bands(self):
        """Every byte outside the outputs' rows is a canary still."""
        for k, (store, t, es, lead, n) in enumerate(self.outs):
            bytes_ = store.clone()
            inside = bytes_[lead:lead + n * es]
            if t.dim() == 2:
                inside = inside.view(t.shape[0], -1)[:, :t.shape[1] * es]
            inside.fill_(CANARY)
            assert bool((bytes_ == CANARY).all()), k


def same(a, b):
    for k, (x, y) in enumerate(zip(a.stores(), b.stores())):
        assert torch.equal(x, y), k


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


def test_plain_tensors_are_taken(xr):
    """Every call with plain tensors is marshalled in compiled code; others are left to
    the Python code."""
    nat, j = xr.native(), Job(5)
    calls = {
        "fold_norm": (j.srcs, j.out, j.residual, j.weight, j.sum, j.out8, j.scale, j.rstd, 128, 1e-6,
                      None),
        "fold_norm_grad": (j.dout, j.sum, j.rstd, j.dx, j.weight, j.dsum, j.dweight, None, None),
        "route": (j.logits, j.ids, j.weights, "sigmoid", j.bias, 8, 4, 2, True, 2.5, None),
        "route_grad": (j.logits, j.ids, j.dweights, j.dlogits, "sigmoid", True, 2.5, None),
        "dispatch_plan": (j.ids, j.counts, j.offsets, j.pos, j.slots, None, None),
        "dispatch": (j.out8, j.pos, j.moved, j.scale, j.moved_scale, None),
        "combine": (j.y, j.pos, j.back, j.weights, j.sum, None),
        "combine_grad": (j.dout, j.y, j.pos, j.weights, j.dy, j.dw, None)}
    for name, args in calls.items():
        assert getattr(nat, name)(*args) == xr.SUCCESS, name
        for k, a in enumerate(args):
            if not isinstance(a, torch.Tensor):
                continue
            for other in (a.as_subclass(Sub), a.cpu(), a[:-1]):
                if (name, k) == ("combine", 0) and other.shape != a.shape:
                    continue    # fewer rows of y are a call of their own
                assert getattr(nat, name)(*args[:k], other, *args[k + 1:]) is None, (name, k)
    torch.cuda.synchronize()
    j.check_bands()
    same(j, Job(5).run(xr))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 0), (0, 8), (3, 5)])
def test_bytes_around_the_outputs_are_left_alone(xr, dtype, shift, pad):
    for rows, hidden, experts, topk in ((1, 1, 8, 1), (33, 72, 16, 4), (130, 1003, 96, 8),
                                        (700, 4096, 256, 16)):
        j = Job(rows, dtype, rows, hidden, experts, topk, shift, pad).run(xr)
        torch.cuda.synchronize()
        j.check_bands()


def test_threads_on_their_own_streams(xr):
    """Four threads, each with its own stream, while another changes the CU budget:
    each round's outputs are those of the same round run alone."""
    rounds = 6
    want = [Job(100 + r, rows=200 + 131 * r) for r in range(rounds)]
    for j in want:
        j.run(xr)
    jobs = [[Job(100 + r, rows=200 + 131 * r) for r in range(rounds)] for _ in range(4)]
    torch.cuda.synchronize()
    streams, errors = [torch.cuda.Stream() for _ in range(4)], []
    start, stop = threading.Barrier(5), threading.Event()

    def worker(t):
        try:
            start.wait()
            for r, j in enumerate(jobs[t]):
                if r % 2:
                    j.run(xr, stream=streams[t])
                else:
                    with torch.cuda.stream(streams[t]):
                        j.run(xr)
        except Exception as e:   # raised again below, in the test's thread
            errors.append((t, e))

    def budgets():
        start.wait()
        k = 0
        while not stop.is_set():
            xr.set_max_workgroups((0, 1, 7, 0, 64, 300)[k % 6])
            k += 1

    threads = [threading.Thread(target=worker, args=(t,)) for t in range(4)]
    knob = threading.Thread(target=budgets)
    prev = xr.set_max_workgroups(0)
    try:
        for th in threads + [knob]:
            th.start()
        for th in threads:
            th.join(timeout=60)
    finally:
        stop.set()
        knob.join(timeout=60)
        xr.set_max_workgroups(prev)
    assert not any(th.is_alive() for th in threads) and not errors, errors
    torch.cuda.synchronize()
    for mine in jobs:
        for a, b in zip(mine, want):
            same(a, b)
