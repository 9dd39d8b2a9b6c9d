"""The layer of examples/expert_layer.py with experts of two products and the gated
activation between them: norm, routing, dispatch, both products, activation and combine
one after another, as they are used, forward and backward, and with rows and weights of 8
and of 4 bits, against the layer in plain torch (64 bits).

Bounds, of the norm of the whole result.  bf16 rounds each of a path's tensors to 2^-9 of
an element at most, eight of them in a row at most, and the plain layer rounds none:
2^-9 * 8 < 0.016.  Where both sides quantise rows, a value close to the middle of two may go
either way: one in 2^-8 over the step between them, each time by a step.  e4m3's steps are
at most 2^-3 of an element: sqrt(2^-5) * 2^-3 < 0.023.  e2m1's are 2^-1 at most and 2^-2 at
the least where most values are: sqrt(2^-6) * 2^-1 < 0.063.  Both for two products.  e4m3 also
loses up to 7 * 2^-13 of the magnitudes that a sum adds, which are no more than sqrt(k) times
its norm for k of them: 16 times for the 256 here, 0.014, in either product."""
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))
from product_util import of_mx4, quant_mx4, spread  # noqa: E402

BOUND = {"f32": 2e-5, "bf16": 0.016, "e4m3": 0.016 + 2 * (0.023 + 0.014), "mx4": 0.016 + 2 * 0.063}


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import expert_layer
    return expert_layer


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def rounded(x, bits):
    """x as 8 or 4 bits hold it."""
    if bits == "e4m3":
        n = x.shape[1]
        parts = torch.nn.functional.pad(x, (0, -n % 128)).unflatten(1, (-1, 128))
        scale = parts.abs().amax(2, keepdim=True).clamp(min=2.0 ** -100) / 448
        return ((parts / scale).float().to(torch.float8_e4m3fn).double() * scale).flatten(1)[:, :n]
    if bits == "mx4" and len(x):
        return of_mx4(*quant_mx4(x))[:, :x.shape[1]]
    return x


def plain(ex, x, norm, router, up, down, sums, ids, bits=None):
    h = sum(t.double() for t in sums) + x
    y = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * norm
    s = (y @ router.t()).sigmoid().gather(1, ids.long())
    w = ex.SCALE * s / s.sum(1, keepdim=True)
    out, y = h, rounded(y, bits)
    for e in range(len(up)):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        gate, value = (y[t] @ up[e].t()).chunk(2, 1)
        z = rounded(torch.nn.functional.silu(gate) * value, bits)
        out = out.index_add(0, t, (z @ down[e].t()) * w[t, j][:, None])
    return out


def chosen(ex, layer, sums, x):
    _, y = ex.FoldNorm.apply(x, layer.norm, *sums)
    return ex.Route.apply(y @ layer.router.t(), layer.bias, layer.topk)[0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,hidden,width,experts,topk", [(1, 256, 128, 8, 2), (3, 136, 72, 8, 2),
                                                              (260, 256, 200, 16, 4), (401, 199, 101, 5, 3)])
def test_training(ex, dtype, tokens, hidden, width, experts, topk):
    layer = ex.GatedLayer(hidden, width, experts, topk, seed=tokens,
                          dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    sums, x, dout = ex.inputs(layer, tokens, seed=hidden)
    ids = chosen(ex, layer, sums, x)
    out, grads = ex.train_step(layer, sums, x, dout)
    leaves = [t.detach().double().requires_grad_(True)
              for t in (x, layer.norm, layer.router, layer.up, layer.down, sums[0])]
    want = plain(ex, *leaves[:5], [leaves[5]] + sums[1:], ids)
    assert off(out, want.detach()) < BOUND[dtype]
    want.backward(dout.double())
    for name, got, leaf in zip(("stream", "norm", "router", "up", "down", "sums"), grads, leaves):
        assert off(got, leaf.grad) < BOUND[dtype], name


@pytest.mark.parametrize("bits", ["e4m3", "mx4"])
@pytest.mark.parametrize("tokens,hidden,width,experts,topk", [(1, 256, 128, 8, 2), (61, 256, 192, 60, 6),
                                                              (900, 256, 256, 4, 2), (130, 200, 136, 8, 2)])
def test_serving(ex, bits, tokens, hidden, width, experts, topk):
    layer = ex.GatedLayer(hidden, width, experts, topk, seed=tokens)
    held = [(ex.to_e4m3 if bits == "e4m3" else ex.to_mx4)(w) for w in layer.weights()]
    if bits == "e4m3":
        up, down = (w.double() * spread(s, w.shape[1], w.shape[2], 128) for w, s in held)
    else:
        up, down = (of_mx4(w, s)[..., :k] for (w, s), k in zip(held, (hidden, width)))
    sums, x, _ = ex.inputs(layer, tokens, seed=hidden)
    ids = chosen(ex, layer, sums, x)
    want = plain(ex, x.double(), layer.norm.double(), layer.router.double(), up, down, sums, ids, bits)
    got = ex.serve_gated(layer, held, sums, x)
    assert off(got, want) < BOUND[bits]
    # captured: the same from a graph that runs between other work, on other inputs too
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ex.serve_gated(layer, held, sums, x)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        out = ex.serve_gated(layer, held, sums, x)
    for seed in (1, 2, 3):
        _, other, _ = ex.inputs(layer, tokens, seed=seed)
        x.copy_(other)
        eager = ex.serve_gated(layer, held, sums, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_experts_gradients_against_differences(ex):
    """Of sum(d * experts(rows)) along random directions, by central differences in fp32:
    the second derivative's part of a step of 2^-6 is some 2^-12 of the whole, the sums' own
    rounding over that step 2^-23 * 2^6 times some ten."""
    layer = ex.GatedLayer(48, 40, 4, 1, dtype=torch.float32, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.empty(s, device="cuda").normal_(0, 1, generator=g)
    offsets = torch.tensor([0, 7, 7, 40, 50], dtype=torch.int32, device="cuda")
    rows, d = new(52, 48), new(52, 48)
    leaves = [rows, layer.up, layer.down]
    for t in leaves:
        t.requires_grad_(True)
    (layer.apply(rows, offsets)[:50].double() * d[:50]).sum().backward()
    grads = [t.grad for t in leaves]
    for t in leaves:
        t.requires_grad_(False)

    def f():
        return float((layer.apply(rows, offsets)[:50].double() * d[:50]).sum())

    for t, grad in zip(leaves, grads):
        assert (t is not rows) or (grad[50:] == 0).all()
        for _ in range(3):
            way, before = new(*t.shape), t.clone()
            t.copy_(before + way * 2.0 ** -6)
            hi = f()
            t.copy_(before - way * 2.0 ** -6)
            lo = f()
            t.copy_(before)
            want = float((way.double() * grad).sum())
            size = float((way.double() * grad).square().sum().sqrt())
            assert abs((hi - lo) * 2.0 ** 5 - want) <= 0.02 * (abs(want) + size)


def test_backward_in_a_graph(ex):
    """A backward pass captured while another of the same weights was eager before."""
    layer = ex.GatedLayer(128, 72, 8, 2, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.empty(40, 128, device="cuda").normal_(0, 1, generator=g).bfloat16()
    d = torch.empty(40, 128, device="cuda").normal_(0, 1, generator=g).bfloat16()
    offsets = torch.tensor([0, 3, 3, 9, 20, 21, 30, 33, 38], dtype=torch.int32, device="cuda")

    def grads():
        leaves = [t.detach().requires_grad_(True) for t in (x, layer.up, layer.down)]
        gated = ex.Gate.apply(ex.Products.apply(leaves[0], leaves[1], offsets), offsets)
        return torch.autograd.grad(ex.Products.apply(gated, leaves[2], offsets), leaves, d)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            grads()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = grads()
    for seed in (1, 2, 3):
        x.normal_(0, 1, generator=g)
        want = grads()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_program_runs_all_forms(ex, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["expert_layer.py", "--tokens", "33", "--hidden", "256"])
    ex.main()
    said = capsys.readouterr().out
    assert "serve_gated, e4m3" in said and "serve_gated, mx4" in said and "train_step, gated" in said
