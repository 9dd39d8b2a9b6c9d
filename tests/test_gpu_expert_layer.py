"""examples/expert_layer.py: the operators in one layer, as they are used together,
against the layer in plain torch (64 bits) and torch's own gradients of it.

Bounds, of the norm of the whole result: bf16 rounds each of a path's tensors to
2^-9 of an element at most, a handful of them in a row, and the plain layer rounds
none: 2^-9 * 6 < 0.012.  With 8-bit rows both sides quantise, but what lies near
the middle of two e4m3 values may go either way: a step of at most 2^-3 of an
element, for about 2^-8 / 2^-3 of the elements, so sqrt(1/32) * 2^-3 = 0.022
more."""
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
sys.path.insert(0, str(Path(__file__).resolve().parents[1] / "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import expert_layer
    return expert_layer


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def chosen(ex, layer, sums, x):
    _, y = ex.FoldNorm.apply(x, layer.norm, *sums)
    return ex.Route.apply(y @ layer.router.t(), layer.bias, layer.topk)[0]


@pytest.mark.parametrize("tokens,hidden,experts,topk", [(1, 256, 8, 2), (5, 200, 16, 4),
                                                        (300, 512, 16, 4), (1025, 384, 60, 6)])
def test_serving(ex, tokens, hidden, experts, topk):
    layer = ex.Layer(hidden, experts, topk, seed=tokens)
    sums, x, _ = ex.inputs(layer, tokens, seed=hidden)
    want = ex.plain(layer, sums, x, chosen(ex, layer, sums, x), True, torch.float64)
    assert off(ex.serve(layer, sums, x), want) < 0.012 + 0.022


@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-5), (torch.bfloat16, 0.012)])
@pytest.mark.parametrize("tokens,hidden,experts,topk", [(3, 136, 8, 2), (260, 256, 16, 4)])
def test_training(ex, dtype, bound, tokens, hidden, experts, topk):
    """fp32: sums of at most 260 products, some 1e-6, room for a row of them."""
    layer = ex.Layer(hidden, experts, topk, dtype=dtype, seed=tokens)
    sums, x, dout = ex.inputs(layer, tokens, seed=hidden)
    ids = chosen(ex, layer, sums, x)
    out, grads = ex.train_step(layer, sums, x, dout)
    ref = ex.Layer(hidden, experts, topk, dtype=dtype, seed=tokens)
    leaves = []
    for t in (x, ref.norm, ref.router, ref.expert, sums[0]):
        leaves.append(t.detach().double().requires_grad_(True))
    ref.norm, ref.router, ref.expert = leaves[1:4]
    want = ex.plain(ref, [leaves[4]] + sums[1:], leaves[0], ids, False, torch.float64)
    assert off(out, want.detach()) < bound
    want.backward(dout.double())
    for name, got, leaf in zip(("stream", "norm", "router", "experts", "sums"), grads, leaves):
        assert off(got, leaf.grad) < bound, name


def test_program_runs(ex, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["expert_layer.py", "--tokens", "64", "--hidden", "256"])
    ex.main()
    assert "train_step: off by 0.00" in capsys.readouterr().out
