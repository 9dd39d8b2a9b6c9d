"""The experts' products have the same bits wherever their operands lie: on the 16-byte grid
or off it, rows close together or 8 MB apart, under any budget of workgroups.  What they
compute is compared with their definition elsewhere; outputs are fp32, so that no rounding
hides the order of a sum."""
import pytest

torch = pytest.importorskip("torch")
from product_util import (TYPES, check_sum, generator, inside, normal, of_mx4, offsets_of,  # noqa: E402
                          product, quant_mx4)

pytestmark = pytest.mark.gpu

FAR = (1 << 23) + 16   # elements from row to row
# rows of each expert, n, k: sizes of streaming tiles (few rows, few tiles), of 64 x 64 ones,
# and of 128 x 128 and 256 x 256 ones, which alignment and distances choose between
SIZES = {"few rows": ([3, 0, 2], 72, 136), "one row": ([1], 69, 2143), "one expert": ([65], 200, 264),
         "64 x 64": ([100, 0, 300, 21, 90, 60, 131, 5], 1288, 136), "short": ([40, 30], 56, 72),
         "many rows": ([1100, 0, 900], 3848, 72), "long rows": ([1500, 0, 1400], 3848, 328)}


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def far(x):
    """x's rows FAR elements apart."""
    flat = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    rows, n = flat.reshape(-1, flat.shape[-1]).shape
    view = torch.empty(rows * FAR, dtype=flat.dtype, device=x.device).view(rows, FAR)[:, :n]
    view.copy_(flat.reshape(rows, n))
    return view.unflatten(0, x.shape[:-1]).view(x.dtype)


def placed(xr, call, out, operands):
    """call(operands) into out, and again with the operands elsewhere: every time the same."""
    places = [lambda t: inside(t, 16, 16), lambda t: inside(t, 3, 1), lambda t: inside(t, 1)]
    call(operands, out)
    assert torch.isfinite(out).any()

    def again(held, what):
        got = torch.full_like(out, float("nan"))
        call(held, got)
        same = got.nan_to_num(-77.0) == out.nan_to_num(-77.0)
        assert same.all(), (what, int((~same).sum()), float((got - out).abs().nan_to_num(0).max()))

    for i, place in enumerate(places):
        again([place(t) for t in operands], ("place", i))
    for i, t in enumerate(operands):   # at most 12 GiB
        if t.numel() // t.shape[-1] * FAR * t.element_size() <= 12 << 30:
            again(operands[:i] + [far(t)] + operands[i + 1:], ("far", i))
    for most in (5, 64):
        before = xr.set_max_workgroups(most)
        try:
            again(operands, ("budget", most))
        finally:
            xr.set_max_workgroups(before)


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("which", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_product(xr, dtype, which, transpose):
    counts, n, k = SIZES[which]
    g = generator(20)
    x, w = normal(g, sum(counts) + 1, k).to(TYPES[dtype]), normal(g, len(counts), n, k).to(TYPES[dtype])
    held = w.transpose(1, 2).contiguous() if transpose else w
    offsets, out = offsets_of(counts), torch.full((len(x), n), float("nan"), device="cuda")
    placed(xr, lambda t, to: xr.group_product(t[0], t[1], offsets, to, transpose=transpose), out, [x, held])
    want, size = product(x, w, offsets)
    check_sum(out[:-1], want[:-1], size[:-1], k, which)


@pytest.mark.parametrize("which", SIZES)
@pytest.mark.parametrize("dtype", ["e4m3", "mx4"])
def test_scaled_product(xr, dtype, which):
    counts, n, k = SIZES[which]
    g = generator(21)
    rows, experts = sum(counts) + 1, len(counts)
    if dtype == "e4m3":
        x, w = (normal(g, *s, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
                for s in ((rows, k), (experts, n, k)))
        kb = -(-k // 128)
        scale = torch.rand(rows, kb, device="cuda", generator=g) + 0.1
        w_scale = torch.rand(experts, -(-n // 128), kb, device="cuda", generator=g) + 0.1
    else:
        x, scale = quant_mx4(normal(g, rows, k))
        w, w_scale = (t.unflatten(0, (experts, n)) for t in quant_mx4(normal(g, experts * n, k)))
    offsets, out = offsets_of(counts), torch.full((rows, n), float("nan"), device="cuda")
    placed(xr, lambda t, to: xr.group_product(t[0], t[1], offsets, to, scale=t[2], w_scale=t[3]), out,
           [x, w, scale, w_scale])
    if dtype == "mx4":
        want, size = product(of_mx4(x, scale), of_mx4(w, w_scale), offsets)
        check_sum(out[:-1], want[:-1], size[:-1], k, which)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("counts,n,k", [([3, 0, 70], 72, 136), ([300, 0, 129, 64], 640, 520), ([200], 2056, 2064)])
def test_gradient(xr, dtype, counts, n, k):
    g = generator(22)
    dout, x = normal(g, sum(counts), n).to(TYPES[dtype]), normal(g, sum(counts), k).to(TYPES[dtype])
    offsets, out = offsets_of(counts), torch.full((len(counts), n, k), float("nan"), device="cuda")
    placed(xr, lambda t, to: xr.group_product_grad(t[0], t[1], offsets, to), out, [dout, x])
