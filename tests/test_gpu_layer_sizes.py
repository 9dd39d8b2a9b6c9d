"""dispatch, combine and combine_grad at numbers of tokens that choose the launches of
large batches: workgroups limited by an LDS reservation, smaller workgroups for few
slots.  Copies and folds are compared bit for bit; dweights, a sum of `hidden`
products, in 64 bits: at most hidden / 256 + 64 additions follow one another, each off
by u = 2^-24 of the magnitudes, doubled for the products' own rounding."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, scale=1.0):
    return torch.empty(shape, device="cuda").normal_(0, scale, generator=g)


def places(g, tokens, topk, dropped=0.1):
    """A random order of all slots, -1 where dropped."""
    pos = torch.randperm(tokens * topk, device="cuda", generator=g).int().view(tokens, topk)
    return pos.masked_fill(torch.rand((tokens, topk), device="cuda", generator=g) < dropped, -1)


def many():
    """More waves of one column tile than 64 workgroups a CU hold."""
    return 4 * 64 * torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("hidden", [24, 25, 1304, 2057])
def test_dispatch_of_many_rows(xr, hidden):
    """On the 16-byte grid and off it, rows of one column tile and of several."""
    tiles = -(-hidden * 2 // 1024)
    tokens, g = many() // tiles + 4567, gen(hidden)
    for topk in (1, 3):
        pos = places(g, tokens, topk)
        x = randn(g, tokens, hidden).bfloat16()
        scale = randn(g, tokens, 3)
        out = torch.full((tokens * topk, hidden), 7.0, device="cuda").bfloat16()
        out_scale = torch.full((tokens * topk, 3), 7.0, device="cuda")
        want, want_scale = out.clone(), out_scale.clone()
        at, slot = torch.nonzero(pos >= 0, as_tuple=True)
        to = pos[at, slot].long()
        want[to], want_scale[to] = x[at], scale[at]
        xr.dispatch(x, pos, out, scale=scale, out_scale=out_scale)
        assert torch.equal(out, want) and torch.equal(out_scale, want_scale)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [24, 25, 1304, 2057])
def test_combine_of_many_rows(xr, dtype, hidden):
    dt = DT[dtype]
    tiles = -(-hidden * (4 if dtype == "f32" else 2) // 1024)
    tokens, g = many() // tiles + 4567, gen(hidden)
    for topk in (2, 5):
        pos = places(g, tokens, topk)
        y, base = randn(g, tokens * topk, hidden).to(dt), randn(g, tokens, hidden).to(dt)
        w = randn(g, tokens, topk)
        want = base.float()
        for j in range(topk):
            term = w[:, j, None] * y[pos[:, j].clamp(min=0).long()].float()
            want = torch.where(pos[:, j, None] >= 0, want + term, want)
        out = torch.empty_like(base)
        xr.combine(y, pos, out, weights=w, base=base)
        assert torch.equal(out, want.to(dt))
        xr.combine(y, pos, base, weights=w, base=base)     # in place
        assert torch.equal(base, out)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [1032, 4096, 5001, 9000])
@pytest.mark.parametrize("topk", [1, 2, 3])
def test_combine_gradient_of_many_tokens(xr, dtype, hidden, topk):
    """More than two tokens a CU: with one or two slots in workgroups of at most 256
    threads, with three in one pass."""
    dt = DT[dtype]
    tokens, g = 2 * (many() // 256) + 77, gen(hidden + topk)
    pos = places(g, tokens, topk)
    dout, w = randn(g, tokens, hidden).to(dt), randn(g, tokens, topk)
    y = randn(g, tokens * topk, hidden).to(dt)
    dy = torch.full((tokens * topk, hidden), 7.0, device="cuda").to(dt)
    dw = torch.full((tokens, topk), torch.nan, device="cuda")
    want = dy.clone()
    at, slot = torch.nonzero(pos >= 0, as_tuple=True)
    to = pos[at, slot].long()
    want[to] = (w[at, slot][:, None] * dout[at].float()).to(dt)
    xr.combine_grad(dout, y, pos, w, dy, dw)
    assert torch.equal(dy, want)
    products = dout[at].double() * y[to].double()
    ref = torch.zeros((tokens, topk), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(ref)
    ref[at, slot], mag[at, slot] = products.sum(1), products.abs().sum(1)
    assert bool(((dw.double() - ref).abs() <= 2 * (hidden / 256 + 64) * U * mag).all())
    assert bool((dw[pos < 0] == 0).all())
    alone = torch.full_like(dy, 7.0)
    xr.combine_grad(dout, None, pos, w, alone)              # without dweights
    assert torch.equal(alone, want)
    over, again = y.clone(), torch.empty_like(dw)
    xr.combine_grad(dout, over, pos, w, over, again)        # over y
    assert torch.equal(again, dw) and torch.equal(over[to], want[to])
