"""The experts' products where a workgroup takes many tiles in turns: the next tile's first
loads and scales are on their way while the last one's results go out.  Under small budgets of
workgroups every kind of tile follows every other; results are compared with 64 bits, and bit
for bit with a call that has all workgroups."""
import pytest

torch = pytest.importorskip("torch")
from product_util import (E4M3_CUT, SENTINEL, TYPES, check_sum, generator, inside, normal,  # noqa: E402
                          of_mx4, offsets_of, product, quant_mx4, spread)

pytestmark = pytest.mark.gpu

MANY = [700, 0, 420, 1, 64, 129]   # 10 tiles of 256 rows at most, of every length
DECODE = [0, 1, 0, 0, 3, 0, 1, 1, 0, 2] * 6 + [0, 33, 0, 1]
# an expert's last tile of every kind, and enough tiles that those of few rows go side by side
RAGGED = [257, 1, 64, 65, 128, 129, 0, 320, 384, 300, 512, 31, 255, 256, 385, 2] * 2


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def in_turns(xr, call, rows, n, dtype, pad=0, budgets=(8, 3)):
    """What call(out) leaves in rows x n, the same under every budget, with nothing written
    between the rows and around them."""
    def run():
        store = torch.full((rows + 2, n + pad), SENTINEL, dtype=dtype, device="cuda")
        out = store[1:-1, :n]
        call(out)
        torch.cuda.synchronize()
        assert (store[0] == SENTINEL).all() and (store[-1] == SENTINEL).all()
        assert (store[:, n:] == SENTINEL).all()
        return out

    want = run()
    for most in budgets:
        before = xr.set_max_workgroups(most)
        try:
            got = run()
        finally:
            xr.set_max_workgroups(before)
        assert torch.equal(got, want), (most, int((got != want).sum()))
    return want


def plain(xr, g, dt, to, counts, n, k, transpose, pad, off, budgets=(8, 3)):
    rows = sum(counts) + 2
    x, w = normal(g, rows, k).to(dt), normal(g, len(counts), n, k, scale=0.2).to(dt)
    x[rows - 2:] = float("nan")
    w[[e for e, c in enumerate(counts) if c == 0]] = float("nan")
    held = inside(w.transpose(1, 2).contiguous() if transpose else w, pad, off)
    rows_held, offsets = inside(x, pad, off), offsets_of(counts)
    out = in_turns(xr, lambda out: xr.group_product(rows_held, held, offsets, out, transpose=transpose),
                   rows, n, to, pad, budgets)
    check_sum(out, *product(x, w, offsets), k, (n, k, transpose, pad, off))


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 8), (3, 1)])
@pytest.mark.parametrize("out", ["own", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_rows(xr, dtype, out, pad, off, transpose):
    """256 x 256 tiles; off the grid 128 x 128 ones, or 256 x 256 by way of registers."""
    g = generator(40)
    for k in (8, 72, 128, 136, 200, 264, 392, 449):
        plain(xr, g, TYPES[dtype], TYPES[dtype if out == "own" else "f32"], MANY, 3848, k, transpose, pad, off)
    plain(xr, g, TYPES[dtype], TYPES[dtype if out == "own" else "f32"], [700, 500], 6664, 264, transpose, pad, off)


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
def test_many_rows_and_columns_f32(xr, pad, off, transpose):
    g = generator(41)
    for k in (8, 72, 160):
        plain(xr, g, torch.float32, torch.float32, [1300, 801], 26248, k, transpose, pad, off, (40,))


@pytest.mark.parametrize("dtype", TYPES)
def test_tiles_of_few_rows_side_by_side(xr, dtype):
    g = generator(42)
    for k in (72, 264):
        plain(xr, g, TYPES[dtype], TYPES[dtype], RAGGED, 13320, k, False, 0, 0, (100,))


def e4m3(xr, g, to, counts, n, k, pad, budgets):
    rows, experts = sum(counts) + 2, len(counts)
    x, w = (normal(g, *s, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
            for s in ((rows, k), (experts, n, k)))
    kb, nb = -(-k // 128), -(-n // 128)
    scale = torch.rand(rows, kb, device="cuda", generator=g) * 0.02 + 1e-3
    w_scale = torch.rand(experts, nb, kb, device="cuda", generator=g) * 0.02 + 1e-3
    scale[rows - 2:] = float("nan")
    w_scale[[e for e, c in enumerate(counts) if c == 0]] = float("nan")
    held = [inside(t, pad) for t in (x, w, scale, w_scale)]
    offsets = offsets_of(counts)
    out = in_turns(xr, lambda out: xr.group_product(*held[:2], offsets, out, scale=held[2], w_scale=held[3]),
                   rows, n, to, pad, budgets)
    want, size = product(x.double() * spread(scale, rows, k), w.double() * spread(w_scale, n, k, 128), offsets)
    check_sum(out, want, size, k + 3 * kb, (n, k), E4M3_CUT)


def mx4(xr, g, to, counts, n, k, pad, budgets):
    rows, experts = sum(counts) + 2, len(counts)
    x4, scale = quant_mx4(normal(g, rows, k))
    w4, w_scale = (t.unflatten(0, (experts, n)) for t in quant_mx4(normal(g, experts * n, k, scale=0.2)))
    scale[rows - 2:] = 255
    w_scale[[e for e, c in enumerate(counts) if c == 0]] = 255
    held = [inside(t, pad) for t in (x4, w4, scale, w_scale)]
    offsets = offsets_of(counts)
    out = in_turns(xr, lambda out: xr.group_product(*held[:2], offsets, out, scale=held[2], w_scale=held[3]),
                   rows, n, to, pad, budgets)
    check_sum(out, *product(of_mx4(x4, scale), of_mx4(w4, w_scale), offsets), k, (n, k))


@pytest.mark.parametrize("n", [3848, 3845])
@pytest.mark.parametrize("out", TYPES)
def test_many_rows_e4m3(xr, out, n):
    """k of one step to nine, around the groups of scales and the three steps in LDS."""
    g = generator(43)
    for k, pad in ((16, 0), (128, 0), (256, 16), (272, 0), (400, 0), (512, 0), (640, 16), (1040, 0), (1152, 0)):
        e4m3(xr, g, TYPES[out], MANY, n, k, pad, (8, 3))


@pytest.mark.parametrize("n", [3848, 3845])
@pytest.mark.parametrize("out", TYPES)
def test_many_rows_mx4(xr, out, n):
    """k of one step to nine; 608: exponents off the grid of words, so 128 x 128 tiles."""
    g = generator(44)
    for k, pad in ((128, 0), (256, 0), (512, 16), (608, 0), (640, 0), (768, 0), (1280, 16), (2176, 0)):
        mx4(xr, g, TYPES[out], MANY, n, k, pad, (8, 3))


@pytest.mark.parametrize("dtype", ["e4m3", "mx4"])
def test_more_tiles_than_workgroups_scaled(xr, dtype):
    """Eight tiles a CU, so that those of few rows go two or three together, without a budget too."""
    g = generator(45)
    for k in (128, 384, 1152):
        if dtype == "e4m3":
            e4m3(xr, g, torch.bfloat16, RAGGED, 6664, k, 0, (100,))
        else:
            mx4(xr, g, torch.bfloat16, RAGGED, 13320, k, 0, (100,))


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("pad,off", [(0, 0), (3, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows(xr, dtype, pad, off, transpose):
    g = generator(46)
    for n, k in ((136, 64), (264, 136), (161, 200), (136, 520)):
        plain(xr, g, TYPES[dtype], TYPES[dtype], DECODE, n, k, transpose, pad, off)


@pytest.mark.parametrize("dtype", ["e4m3", "mx4"])
def test_few_rows_scaled(xr, dtype):
    g = generator(47)
    for n, k, pad in ((136, 128, 0), (264, 288, 16), (161, 640, 0), (136, 1056, 0)):
        (e4m3 if dtype == "e4m3" else mx4)(xr, g, torch.bfloat16, DECODE, n, k, pad, (8, 3))


@pytest.mark.parametrize("add", [False, True], ids=["set", "add"])
@pytest.mark.parametrize("n,k,pad,off", [(2056, 2064, 0, 0), (2056, 2064, 8, 8), (2051, 2053, 3, 1), (136, 72, 0, 0)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradient(xr, dtype, n, k, pad, off, add):
    """Experts without rows between others: tiles of no step."""
    g = generator(48)
    dt, counts = TYPES[dtype], [0, 200, 0, 64, 1, 0]
    rows, experts = sum(counts) + 2, len(counts)
    dout, x = normal(g, rows, n).to(dt), normal(g, rows, k).to(dt)
    dout[rows - 2:] = x[rows - 2:] = float("nan")
    held, offsets = [inside(t, pad, off) for t in (dout, x)], offsets_of(counts)
    at = offsets.tolist()
    for to in {dt, torch.float32}:
        before = normal(g, experts * n, k).to(to)

        def call(out):
            out.copy_(before if add else torch.full_like(before, float("nan")))
            xr.group_product_grad(*held, offsets, out.unflatten(0, (experts, n)), add=add)

        got = in_turns(xr, call, experts * n, k, to, pad).unflatten(0, (experts, n))
        old = before.double().unflatten(0, (experts, n))
        for e in range(experts):
            a, b = dout[at[e]:at[e + 1]].double(), x[at[e]:at[e + 1]].double()
            want, size = a.t() @ b, a.abs().t() @ b.abs()
            if add:
                want, size = want + old[e], size + old[e].abs()
            check_sum(got[e], want, size, counts[e] + 1, (to, e))
