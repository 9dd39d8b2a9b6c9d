"""4-bit microscaled values: quant_mx4 and dequant_mx4, bit for bit against the
definition in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
from product_util import TYPES, generator, inside, normal, of_mx4, quant_mx4  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def quant(xr, x, pad=0, off=0):
    blocks = -(-x.shape[1] // 32)
    codes = inside(torch.full((len(x), 16 * blocks), 0xA5, dtype=torch.uint8, device="cuda"), pad, off)
    scale = inside(torch.full((len(x), blocks), 0xA5, dtype=torch.uint8, device="cuda"), pad, off)
    xr.quant_mx4(x, codes, scale)
    for t, n in ((codes, 16 * blocks), (scale, blocks)):
        if pad and len(x) > 1:
            assert (t.as_strided((len(x) - 1, n + pad), (n + pad, 1), t.storage_offset())[:, n:] == 255).all()
    return codes, scale


@pytest.mark.parametrize("columns", [1, 7, 8, 9, 31, 32, 33, 63, 64, 100, 256, 511, 512, 513, 1000, 4096])
@pytest.mark.parametrize("dtype", TYPES)
def test_round_trip(xr, dtype, columns):
    g = generator(columns)
    dt = TYPES[dtype]
    for rows, pad, off in ((1, 0, 0), (3, 0, 0), (17, 5, 3), (130, 1, 0)):
        spread = 1.0 if dtype == "f16" else 8.0
        x = (normal(g, rows, columns) * torch.exp2(normal(g, rows, columns) * spread).clamp(max=2.0 ** 10)).to(dt)
        x = inside(x, pad, off)
        codes, scale = quant(xr, x, pad, off)
        want, byte = quant_mx4(x)
        assert torch.equal(codes, want) and torch.equal(scale, byte)
        for to in TYPES.values():
            out = inside(torch.full((rows, columns), 5.0, dtype=to, device="cuda"), pad, off)
            xr.dequant_mx4(codes, scale, out)
            value = of_mx4(codes, scale)[:, :columns]
            assert torch.equal(out, value.to(torch.float32).to(to))
            if pad and rows > 1:
                assert torch.isnan(out.as_strided((rows - 1, columns + pad), (columns + pad, 1),
                                                  out.storage_offset())[:, columns:]).all()


def test_every_border_and_exponent(xr):
    """Each code's value, the middles between neighbours and the next numbers on both
    sides of them, times every power of two that binary32 has."""
    grid = [0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0, 7.75]
    v = torch.tensor(grid)
    v = torch.cat([v, torch.nextafter(v, torch.tensor(9.0)), torch.nextafter(v, torch.tensor(-9.0))])
    v = torch.cat([v, -v])
    top = torch.tensor([4.0, 5.0, 6.0, 7.0, 7.9999995])   # what makes the exponent
    rows = []
    for t in top:
        for i in range(0, len(v), 31):
            part = torch.zeros(32)
            part[0] = t
            part[1:1 + len(v[i:i + 31])] = v[i:i + 31].clamp(-t, t)
            rows.append(part)
    base = torch.stack(rows).double()
    x = torch.cat([(base * 2.0 ** e).float() for e in range(-152, 126)]).cuda()
    codes, scale = quant(xr, x)
    want, byte = quant_mx4(x)
    assert torch.equal(scale, byte) and torch.equal(codes, want)
    out = torch.empty_like(x)
    xr.dequant_mx4(codes, scale, out)
    assert torch.equal(out, of_mx4(codes, scale).float())


def test_zeros_infinities_and_nan(xr):
    x = torch.zeros(6, 96, device="cuda")
    x[1, 40] = float("inf")
    x[2, 31] = float("nan")
    x[3, 64] = -float("inf")
    x[4] = -0.0
    x[5, :32] = 3.4e38
    for dt in TYPES.values():
        y = x.to(dt)
        codes, scale = quant(xr, y)
        want, byte = quant_mx4(y)
        assert torch.equal(scale, byte) and torch.equal(codes, want)
        out = torch.empty_like(y)
        xr.dequant_mx4(codes, scale, out)
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[1, 32:64] = bad[2, :32] = bad[3, 64:] = True
        if dt != torch.float32:
            bad[5, :32] = True   # 3.4e38 is infinite there: past the middle of bf16's last and 2^128
        assert torch.equal(torch.isnan(out), bad)
        assert (out[4] == 0).all()


def test_every_code_and_scale(xr):
    """All 16 codes at all 256 exponents."""
    codes = torch.arange(16, dtype=torch.uint8, device="cuda").repeat(256, 1)   # low halves
    scale = torch.arange(256, dtype=torch.uint8, device="cuda").view(256, 1)
    for dt in TYPES.values():
        out = torch.empty(256, 32, dtype=dt, device="cuda")
        xr.dequant_mx4(codes, scale, out)
        want = of_mx4(codes, scale).float().to(dt)
        assert torch.equal(torch.isnan(out), torch.isnan(want))
        assert torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0))


def test_empty_and_graph(xr):
    e = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    xr.quant_mx4(torch.empty(0, 64, device="cuda"), e(0, 32), e(0, 2))
    xr.dequant_mx4(e(0, 32), e(0, 2), torch.empty(0, 64, device="cuda"))
    g = generator(3)
    x = normal(g, 50, 300).bfloat16()
    codes, scale, out = e(50, 160), e(50, 10), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xr.quant_mx4(x, codes, scale)
        xr.dequant_mx4(codes, scale, out)
    for _ in range(3):
        x.copy_(normal(g, 50, 300))
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, byte = quant_mx4(x)
        assert torch.equal(codes, want) and torch.equal(scale, byte)
        assert torch.equal(out, of_mx4(want, byte)[:, :300].bfloat16())
