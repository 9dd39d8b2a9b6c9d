"""The workspace that the binding takes for a call on a stream the caller names.

A block that torch's allocator hands out is free for later work of the stream it
is taken on, not for other streams: kernels enqueued on that stream before may
still use it.  So it has to be taken on the stream the call runs on."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")
from paper_2510_20171_amd import layer  # noqa: E402


class FakeStream:
    """The attributes of a torch.cuda.Stream the binding reads."""

    def __init__(self, handle, device=None):
        self.cuda_stream, self.device = handle, device


@pytest.fixture
def allocations(monkeypatch):
    """(bytes, handle of the stream they were taken on) of each allocation; 7 is the
    caller's current stream."""
    current, made = [FakeStream(7)], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        try:
            yield
        finally:
            current.pop()

    def empty(n, dtype, device):
        made.append((n, current[-1].cuda_stream))
        return types.SimpleNamespace(record_stream=lambda stream: None, device=device)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", FakeStream)
    monkeypatch.setattr(torch, "empty", empty)
    return made


LIKE = types.SimpleNamespace(device=torch.device("cuda:0"))


@pytest.mark.parametrize("stream", [1234, FakeStream(1234)], ids=["handle", "object"])
def test_workspace_belongs_to_the_stream_of_the_call(allocations, stream):
    layer._workspace(4096, LIKE, stream)
    assert allocations == [(4096, 1234)]


def test_workspace_belongs_to_the_current_stream_by_default(allocations):
    layer._workspace(4096, LIKE, None)
    assert allocations == [(4096, 7)]


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["object", "handle"])
def test_calls_leave_temporaries_of_the_current_stream_alone(xr, which):
    """The current stream still has to read a temporary, already given back to the
    allocator, of the very size the call asks for.  Neither may see the other."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, hidden, tokens, k, experts = 700, 2048, 6000, 8, 256
    d = torch.randn(rows, hidden, device="cuda", generator=g)
    h = torch.randn(rows, hidden, device="cuda", generator=g)
    rstd = torch.ones(rows, device="cuda")
    dx, dw = torch.empty_like(d), torch.empty(hidden, device="cuda")
    ids = torch.randint(0, experts, (tokens, k), device="cuda", generator=g).int()
    counts = torch.empty(experts, dtype=torch.int32, device="cuda")
    offsets = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
    pos = torch.empty_like(ids)
    calls = ((lambda **kw: xr.fold_norm_grad(d, h, rstd, dx, dweight=dw, **kw), (dx, dw),
              xr.load().xred_fold_norm_grad_workspace(rows, hidden)),
             (lambda **kw: xr.dispatch_plan(ids, counts, offsets, pos, **kw),
              (counts, offsets, pos), xr.load().xred_dispatch_plan_workspace(tokens * k, experts)))
    for call, outs, need in calls:
        assert need > 0
        call()
        want = [t.clone() for t in outs]
        side = torch.cuda.Stream()
        seen = torch.zeros(need, dtype=torch.uint8, device="cuda")
        for t in outs:
            t.zero_()
        temporary = torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)      # some 10 ms of the current stream
        seen.copy_(temporary)              # ... and then a read of the temporary
        del temporary                      # which the allocator has back before that
        call(stream=side if which == "object" else side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        torch.cuda.synchronize()
        assert bool((seen == 0x5A).all())


@pytest.mark.gpu
def test_a_captured_call_on_a_named_stream(xr):
    """Its workspace comes from the graph's memory: replays give the same, whatever is
    allocated and written between them."""
    g = torch.Generator(device="cuda").manual_seed(2)
    tokens, k, experts = 5000, 8, 300
    ids = torch.randint(-1, experts, (tokens, k), device="cuda", generator=g).int()
    outs = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (experts, experts + 1)]
    outs.append(torch.empty_like(ids))
    xr.dispatch_plan(ids, *outs)
    want = [t.clone() for t in outs]
    need = xr.load().xred_dispatch_plan_workspace(tokens * k, experts)
    torch.cuda.synchronize()
    for handle in (False, True):
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            xr.dispatch_plan(ids, *outs, stream=side.cuda_stream if handle else side)
        for n in range(3):
            for t in outs:
                t.fill_(n)
            other = [torch.full((need,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), (handle, n)
            assert all(bool((t == 0x5A).all()) for t in other)
