"""Products of 8 and 4 bits with NaN and infinite values and scales and with scales at both ends
of their range: what they reach becomes so, and nothing else does."""
import pytest

torch = pytest.importorskip("torch")
from product_util import (TYPES, check_sum, generator, inside, normal, of_mx4, offsets_of,  # noqa: E402
                          product, quant_mx4, spread)

pytestmark = pytest.mark.gpu
# rows of each expert, n, k: streaming tiles, 64 x 64, 128 x 128 (off the grid) and 256 x 256
SIZES = {"few": ([3, 0, 2], 72, 256), "64 x 64": ([70, 30], 56, 320), "128 x 128": ([700, 0, 420, 1], 3848, 384),
         "256 x 256": ([700, 0, 420, 1], 3848, 384)}


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def held(which, t):
    return inside(t, 3, 1) if which == "128 x 128" else t


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", SIZES)
def test_mx4(xr, which, out_dtype):
    counts, n, k = SIZES[which]
    g = generator(50)
    rows, experts = sum(counts), len(counts)
    x = normal(g, rows, k)
    x[1, k - 1] = float("nan")            # its block's scale becomes NaN, its codes 0
    x4, scale = quant_mx4(x)
    w4, w_scale = (t.unflatten(0, (experts, n)) for t in quant_mx4(normal(g, experts * n, k)))
    w4, w_scale = w4.contiguous(), w_scale.contiguous()
    assert scale[1, -1] == 255
    w_scale[0, 5, 0] = w_scale[0, 40, 3] = 255
    # a pair of blocks at the ends of the scales' range, whose product is in the middle of it
    scale[2, 1], w_scale[:, :, 1] = 254, 0
    scale[0, 1], scale[3:, 1] = 254, 253
    offsets, out = offsets_of(counts), torch.full((rows, n), -7.0, dtype=TYPES[out_dtype], device="cuda")
    xr.group_product(held(which, x4), held(which, w4), offsets, out, scale=held(which, scale),
                     w_scale=held(which, w_scale))
    want, size = product(of_mx4(x4, scale), of_mx4(w4, w_scale), offsets)
    bad = torch.isnan(want)
    assert bad[1].all() and bad[0, 5] and bad[2, 40] and not bad[2, 6]
    assert torch.equal(torch.isnan(out), bad)
    check_sum(out[~bad], want[~bad], size[~bad], k, which)


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", SIZES)
def test_mx4_results_past_either_end(xr, which, out_dtype):
    """Scales whose product is past binary32: infinities of the result's sign, and zeros."""
    counts, n, k = SIZES[which]
    rows, experts = sum(counts), len(counts)
    x4 = torch.full((rows, k // 2), 0x22, dtype=torch.uint8, device="cuda")        # ones
    w4 = torch.full((experts, n, k // 2), 0x22, dtype=torch.uint8, device="cuda")
    w4[:, 1::2] = 0xAA                                                             # minus ones
    scale = torch.full((rows, k // 32), 254, dtype=torch.uint8, device="cuda")
    w_scale = torch.full((experts, n, k // 32), 254, dtype=torch.uint8, device="cuda")
    scale[1::2] = 0
    w_scale[:, 2:] = 0
    offsets, out = offsets_of(counts), torch.full((rows, n), -7.0, dtype=TYPES[out_dtype], device="cuda")
    xr.group_product(held(which, x4), held(which, w4), offsets, out, scale=held(which, scale),
                     w_scale=held(which, w_scale))
    assert (out[::2, 0] == float("inf")).all() and (out[::2, 1] == -float("inf")).all()
    assert (out[1::2, :2].abs() == k).all() and (out[::2, 2:].abs() == k).all()
    assert (out[1::2, 2:] == 0).all()


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", SIZES)
def test_e4m3(xr, which, out_dtype):
    counts, n, k = SIZES[which]
    g = generator(51)
    rows, experts = sum(counts), len(counts)
    x, w = (normal(g, *s, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
            for s in ((rows, k), (experts, n, k)))
    kb, nb = -(-k // 128), -(-n // 128)
    scale = torch.rand(rows, kb, device="cuda", generator=g) + 0.1
    w_scale = torch.rand(experts, nb, kb, device="cuda", generator=g) + 0.1
    x.view(torch.uint8)[1, k - 1] = 0x7F          # NaN
    w.view(torch.uint8)[0, 6, 3] = 0xFF
    scale[2, kb - 1] = float("inf")
    scale[rows - 1, 0] = float("nan")
    offsets, out = offsets_of(counts), torch.full((rows, n), -7.0, dtype=TYPES[out_dtype], device="cuda")
    xr.group_product(held(which, x), held(which, w), offsets, out, scale=held(which, scale),
                     w_scale=held(which, w_scale))
    want, size = product(x.double() * spread(scale, rows, k), w.double() * spread(w_scale, n, k, 128), offsets)
    fine = torch.isfinite(want)
    assert not fine[1].any() and not fine[2].any() and not fine[rows - 1].any() and not fine[0, 6] and fine[0, 7]
    assert torch.equal(torch.isfinite(out), fine)
    assert torch.isnan(out[1]).all() and torch.isnan(out[0, 6]) and torch.isnan(out[rows - 1]).all()
    check_sum(out[fine], want[fine], size[fine], k + 3 * kb, which, 7 * 2.0 ** -13)
