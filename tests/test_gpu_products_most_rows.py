"""The calls between dispatch and combine with as many rows as they take, 2^31 - 1, and with more
lanes of work than a launch has threads: the first and last rows, and rows between them, against
the formulas, and nothing behind the last."""
import pytest

torch = pytest.importorskip("torch")
from product_util import SENTINEL, generator, of_mx4, quant_mx4  # noqa: E402

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    torch.cuda.empty_cache()
    yield xr
    torch.cuda.empty_cache()


def places(rows, size=1 << 20):
    """Parts of the rows: the ends, 2^30 and a few between."""
    return [slice(a, min(a + size, rows)) for a in (0, rows // 3, (1 << 30) - size // 2, rows - size)
            if 0 <= a < rows]


def random(g, rows, columns):
    """bf16 whole numbers -8 to 7, over and over: made quickly."""
    part = torch.randint(-8, 8, (1 << 24, columns), device="cuda", generator=g).bfloat16()
    x = torch.empty(rows, columns, dtype=torch.bfloat16, device="cuda")
    for a in range(0, rows, len(part)):
        x[a:a + len(part)] = part[:rows - a]
        x[a:a + 1] = a % 5 + 1.0   # not the same everywhere
    return x


def behind(rows, columns, dtype=torch.bfloat16):
    """rows x columns, and a part behind them that stays as it is."""
    store = torch.full((rows * columns + 64,), SENTINEL if dtype.is_floating_point else 0x5A, dtype=dtype,
                       device="cuda")
    return store[:rows * columns].view(rows, columns), store[rows * columns:]


def test_gate(xr):
    g = generator(60)
    x = random(g, MOST, 2)
    out, rest = behind(MOST, 1)
    xr.gate(x, out)
    for part in places(MOST):
        gate, up = x[part].double().chunk(2, 1)
        want = gate * torch.sigmoid(gate) * up
        assert ((out[part].double() - want).abs() <= want.abs() * 2.0 ** -8 + 1e-30).all()
    assert (rest == SENTINEL).all()


def test_gate_grad(xr):
    g = generator(61)
    rows = MOST
    x, d = random(g, rows, 2), random(g, rows, 1)
    dx, rest = behind(rows, 2)
    xr.gate_grad(d, x, dx)
    for part in places(rows):
        gate, up = x[part].double().chunk(2, 1)
        s, do = torch.sigmoid(gate), d[part].double()
        want = torch.cat([do * up * s * (1 + gate * torch.sigmoid(-gate)), do * gate * s], 1)
        # beside the rounding: some binary32 operations on a sum whose terms can cancel
        assert ((dx[part].double() - want).abs() <= want.abs() * 2.0 ** -8 + 600 * 2.0 ** -20).all()
    assert (rest == SENTINEL).all()


def test_mx4(xr):
    g = generator(62)
    rows = (1 << 30) + 77   # four lanes a row: more than 2^32
    x = random(g, rows, 1)
    codes, codes_rest = behind(rows, 16, torch.uint8)
    scale, scale_rest = behind(rows, 1, torch.uint8)
    xr.quant_mx4(x, codes, scale)
    for part in places(rows):
        want, byte = quant_mx4(x[part])
        assert torch.equal(codes[part], want) and torch.equal(scale[part], byte)
    out, rest = behind(rows, 1)
    xr.dequant_mx4(codes, scale, out)
    for part in places(rows):
        assert torch.equal(out[part], of_mx4(codes[part], scale[part])[:, :1].bfloat16())
    assert (codes_rest == 0x5A).all() and (scale_rest == 0x5A).all() and (rest == SENTINEL).all()


def test_product(xr):
    g = generator(63)
    x = random(g, MOST, 1)
    w = torch.tensor([3.0, 5.0, 7.0], dtype=torch.bfloat16, device="cuda").view(3, 1, 1)
    cut = [0, MOST // 2, MOST // 2, MOST - 9]
    offsets = torch.tensor(cut, dtype=torch.int32, device="cuda")
    out, rest = behind(MOST, 1)
    xr.group_product(x, w, offsets, out)
    for part in places(MOST) + [slice(MOST // 2 - 300, MOST // 2 + 300)]:
        r = torch.arange(part.start, part.stop, device="cuda")[:, None]
        want = torch.where(r < cut[1], 3.0, 7.0) * x[part].float()   # whole numbers below 64: exact
        assert torch.equal(out[part].float(), torch.where(r < cut[3], want, SENTINEL))
    assert (rest == SENTINEL).all()


def test_product_grad(xr):
    """Experts' sums over few rows at either end of 2^31 - 1, and over a million."""
    g = generator(64)
    x, d = random(g, MOST, 1), random(g, MOST, 1)
    dw = torch.full((5, 1, 1), float("nan"), device="cuda")
    offsets = torch.tensor([5, 40, 40, 1 << 20, 1 << 20, 1 << 20], dtype=torch.int32, device="cuda")
    xr.group_product_grad(d, x, offsets, dw)
    for e, (lo, hi) in enumerate(((5, 40), (40, 40), (40, 1 << 20), (0, 0), (0, 0))):
        a, b = d[lo:hi].double(), x[lo:hi].double()
        assert abs(float(dw[e]) - float((a * b).sum())) <= float((a * b).abs().sum()) * (hi - lo + 4) * 2.0 ** -23
    offsets = torch.tensor([MOST - 33] * 5 + [MOST], dtype=torch.int32, device="cuda")
    xr.group_product_grad(d, x, offsets, dw)
    assert (dw[:4] == 0).all() and float(dw[4]) == float((d[MOST - 33:].double() * x[MOST - 33:].double()).sum())
