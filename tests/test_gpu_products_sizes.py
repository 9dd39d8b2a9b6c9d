"""The experts' products at the sizes that choose one way of computing them or another:
many rows (tiles of 256 x 256), few rows of many experts (weights streamed), and operands
past 4 GiB, each with whole and odd sizes, against 64-bit references."""
import pytest

torch = pytest.importorskip("torch")
from product_util import (E4M3_CUT, SENTINEL, TYPES, check_sum, generator, inside, normal,  # noqa: E402
                          of_mx4, offsets_of, product, quant_mx4, spread)

pytestmark = pytest.mark.gpu

MANY = [700, 0, 420, 1]   # rows of four experts: 8 tiles of 256 at most
WIDE_N = (3848, 3845)     # 16 columns of tiles
DECODE = [0, 1, 0, 0, 3, 0, 1, 1, 0, 2] * 6 + [0, 33, 0, 1]


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def run(xr, g, dt, counts, left, n, k, transpose=False, pad=0, off=0, out_dtype=None):
    """As a program holds it: rows of no expert and experts without rows hold NaN."""
    rows = sum(counts) + left
    x = normal(g, rows, k).to(dt)
    x[rows - left:] = float("nan")
    w = normal(g, len(counts), n, k, scale=0.2).to(dt)
    w[[e for e, c in enumerate(counts) if c == 0]] = float("nan")
    held = inside(w.transpose(1, 2).contiguous() if transpose else w, pad, off)
    out = inside(torch.full((rows, n), SENTINEL, dtype=out_dtype or dt, device="cuda"), pad, off)
    offsets = offsets_of(counts)
    xr.group_product(inside(x, pad, off), held, offsets, out, transpose=transpose)
    check_sum(out, *product(x, w, offsets), k, (n, k, transpose, pad, off))
    if pad:
        base = out.as_strided((rows, n + pad), (n + pad, 1), out.storage_offset())
        assert torch.isnan(base[:, n:]).all()


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("n", WIDE_N)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(xr, dtype, n, transpose):
    """k of one step, of two, and around the end of the loop of whole steps."""
    g = generator(1)
    for k in (8, 40, 72, 128, 200, 264, 456, 9, 33, 65, 127, 129, 257, 449):
        run(xr, g, TYPES[dtype], MANY, 3, n, k, transpose)


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("pad,off", [(8, 8), (1, 0), (3, 1), (4, 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_strides(xr, dtype, pad, off, transpose):
    g = generator(2)
    for k in (72, 321):
        run(xr, g, TYPES[dtype], MANY, 2, 3848, k, transpose, pad, off)
    run(xr, g, TYPES[dtype], MANY, 2, 3848, 264, transpose, pad, off, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_tiles_of_few_rows_side_by_side(xr, dtype):
    """Every length of an expert's last tile, enough columns that several go together."""
    g = generator(3)
    counts = [0, 1, 32, 64, 65, 127, 128, 129, 255, 256, 257, 300, 384, 385, 320, 513] * 4
    run(xr, g, TYPES[dtype], counts, 5, 6664, 136)


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("n", [26248, 26245])
def test_many_rows_and_columns_f32(xr, n, transpose):
    """fp32 takes tiles of 256 x 256 where there are a thousand of them."""
    g = generator(13)
    for k, pad, off in ((8, 0, 0), (72, 8, 8), (160, 0, 0), (33, 0, 0), (131, 3, 1)):
        run(xr, g, torch.float32, [1300, 801], 3, n, k, transpose, pad, off)


@pytest.mark.parametrize("n", WIDE_N)
@pytest.mark.parametrize("out_dtype", TYPES)
def test_many_rows_e4m3(xr, out_dtype, n):
    g = generator(4)
    rows = sum(MANY) + 3
    for k, pad in ((16, 0), (128, 0), (272, 16), (400, 0), (640, 0), (1040, 0), (1152, 16), (257, 0)):
        x = normal(g, rows, k, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
        w = normal(g, 4, n, k, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
        kb, nb = -(-k // 128), -(-n // 128)
        scale = torch.rand(rows, kb, device="cuda", generator=g) * 0.02 + 1e-3
        w_scale = torch.rand(4, nb, kb, device="cuda", generator=g) * 0.02 + 1e-3
        scale[rows - 3:] = float("nan")
        w_scale[1] = float("nan")
        x, w, scale, w_scale = (inside(t, pad) for t in (x, w, scale, w_scale))
        offsets = offsets_of(MANY)
        out = torch.full((rows, n), SENTINEL, dtype=TYPES[out_dtype], device="cuda")
        xr.group_product(x, w, offsets, out, scale=scale, w_scale=w_scale)
        want, size = product(x.double() * spread(scale, rows, k),
                             w.double() * spread(w_scale, n, k, 128), offsets)
        check_sum(out, want, size, k + 3 * kb, (n, k), E4M3_CUT)


@pytest.mark.parametrize("n", WIDE_N)
@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
def test_many_rows_mx4(xr, out_dtype, n):
    """Rows that end within a step and at one; exponents on the grid of words and off it;
    NaN exponents behind the rows' ends."""
    g = generator(5)
    rows = sum(MANY) + 3
    for k, pad in ((32, 0), (128, 0), (256, 0), (600, 4), (896, 0), (1280, 16), (1312, 0), (2176, 4)):
        x4, scale = quant_mx4(normal(g, rows, k))
        w4, w_scale = quant_mx4(normal(g, 4 * n, k, scale=0.2))
        w4, w_scale = w4.view(4, n, -1), w_scale.view(4, n, -1)
        scale[rows - 3:] = 255
        w_scale[1] = 255
        x4, w4, scale, w_scale = (inside(t, pad) for t in (x4, w4, scale, w_scale))
        offsets = offsets_of(MANY)
        out = torch.full((rows, n), SENTINEL, dtype=TYPES[out_dtype], device="cuda")
        xr.group_product(x4, w4, offsets, out, scale=scale, w_scale=w_scale)
        want, size = product(of_mx4(x4, scale), of_mx4(w4, w_scale), offsets)
        check_sum(out, want, size, k, (n, k, pad))


@pytest.mark.parametrize("add", [False, True], ids=["set", "add"])
@pytest.mark.parametrize("n,k", [(2056, 2064), (2051, 2053)])
@pytest.mark.parametrize("dtype", TYPES)
def test_many_tiles_of_a_gradient(xr, dtype, n, k, add):
    g = generator(6)
    dt = TYPES[dtype]
    for counts in ([0, 700, 70], [1, 64, 321], [128, 0, 193]):
        rows = sum(counts) + 2
        dout, x = normal(g, rows, n).to(dt), normal(g, rows, k).to(dt)
        dout[rows - 2:] = float("nan")
        x[rows - 2:] = float("nan")
        offsets = offsets_of(counts)
        for to in {dt, torch.float32}:
            dw = normal(g, 3, n, k).to(to)
            before = dw.double()
            if not add:
                dw.fill_(float("nan"))
            xr.group_product_grad(dout, x, offsets, dw, add=add)
            at = offsets.tolist()
            for e in range(3):
                a, b = dout[at[e]:at[e + 1]].double(), x[at[e]:at[e + 1]].double()
                want, size = a.t() @ b, a.abs().t() @ b.abs()
                if add:
                    want, size = want + before[e], size + before[e].abs()
                check_sum(dw[e], want, size, counts[e] + 1, (counts, to, e))


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows(xr, dtype, transpose):
    """k around every place in a group of four steps, n around a tile's end."""
    g = generator(7)
    for k in (64, 65, 72, 96, 127, 128, 129, 191, 192, 193, 256, 257, 264, 320, 1100):
        for n in (64, 136, 161):
            run(xr, g, TYPES[dtype], DECODE, 1, n, k, transpose)
    for pad, off in ((8, 8), (1, 0), (3, 1), (4, 4)):
        run(xr, g, TYPES[dtype], DECODE, 1, 136, 328, transpose, pad, off)
        run(xr, g, TYPES[dtype], DECODE, 1, 130, 327, transpose, pad, off, torch.float32)


@pytest.mark.parametrize("dtype", ["e4m3", "mx4"])
def test_few_rows_scaled(xr, dtype):
    g = generator(8)
    rows, experts = sum(DECODE) + 2, len(DECODE)
    offsets = offsets_of(DECODE)
    empty = [e for e, c in enumerate(DECODE) if c == 0]
    for k in (64, 65, 128, 129, 200, 256, 320, 384, 511, 513, 1000, 1024, 1056, 2080):
        for n, pad in ((64, 0), (136, 16), (161, 3)):
            if dtype == "e4m3":
                x = normal(g, rows, k, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
                w = normal(g, experts, n, k, scale=60.0).clamp(-448, 448).to(torch.float8_e4m3fn)
                kb, nb = -(-k // 128), -(-n // 128)
                scale = torch.rand(rows, kb, device="cuda", generator=g) * 0.02 + 1e-3
                w_scale = torch.rand(experts, nb, kb, device="cuda", generator=g) * 0.02 + 1e-3
                scale[rows - 2:] = float("nan")
                w_scale[empty] = float("nan")
                terms, cut = k + 3 * kb, E4M3_CUT
                wide_x, wide_w = x.double() * spread(scale, rows, k), w.double() * spread(w_scale, n, k, 128)
            else:
                x, scale = quant_mx4(normal(g, rows, k))
                w, w_scale = quant_mx4(normal(g, experts * n, k, scale=0.2))
                w, w_scale = w.view(experts, n, -1), w_scale.view(experts, n, -1)
                scale[rows - 2:] = 255
                w_scale[empty] = 255
                terms, cut = k, 0.0
                wide_x, wide_w = of_mx4(x, scale), of_mx4(w, w_scale)
            out = torch.full((rows, n), SENTINEL, dtype=torch.bfloat16, device="cuda")
            xr.group_product(inside(x, pad), inside(w, pad), offsets, out, scale=inside(scale, pad),
                             w_scale=inside(w_scale, pad))
            check_sum(out, *product(wide_x, wide_w, offsets), terms, (n, k, pad), cut)


def test_more_tiles_than_workgroups(xr):
    """Workgroups go on from tile to tile, some of them of experts far apart."""
    g = generator(9)
    counts = [(e * 7) % 5 // 3 for e in range(256)]
    for n, k in ((2048, 72), (1989, 71)):
        run(xr, g, torch.bfloat16, counts, 0, n, k)
    run(xr, g, torch.bfloat16, [33, 0, 31, 2] * 4, 0, 16000, 328)   # and with few of them


@pytest.mark.parametrize("counts,n", [(MANY, 3848), (MANY, 3845), (DECODE, 136), (DECODE, 161)],
                         ids=["many", "many odd", "few", "few odd"])
def test_infinities_stay_with_their_rows(xr, counts, n):
    g = generator(10)
    rows = sum(counts)
    for k in (72, 200, 201):
        x = normal(g, rows, k).bfloat16()
        w, offsets = normal(g, len(counts), n, k).bfloat16(), offsets_of(counts)
        x[3] = float("inf")
        x[rows - 2, k - 1] = float("nan")
        out = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
        xr.group_product(x, w, offsets, out)
        kept = torch.tensor([r for r in range(rows) if r not in (3, rows - 2)], device="cuda")
        assert not torch.isfinite(out[3]).any() and torch.isnan(out[rows - 2]).all()
        want, size = product(x, w, offsets)
        check_sum(out[kept], want[kept], size[kept], k)


@pytest.mark.parametrize("k", [4096, 4095])
def test_weights_past_4_gib(xr, k):
    g = generator(11)
    experts, n = 135, 4096
    w = torch.empty(experts, n, k, dtype=torch.bfloat16, device="cuda")
    w.normal_(0, 0.02, generator=g)
    for many in (1, 290):   # streamed, and in tiles
        counts = [many] + [0] * (experts - 2) + [many + 1]
        x, offsets = normal(g, sum(counts) + (0 if many == 1 else 17 * experts), k).bfloat16(), offsets_of(counts)
        out = torch.empty(len(x), n, dtype=torch.bfloat16, device="cuda")
        xr.group_product(x, w, offsets, out)
        for lo, hi, e in ((0, many, 0), (many, 2 * many + 1, experts - 1)):
            a, b = x[lo:hi].double(), w[e].double()
            check_sum(out[lo:hi], a @ b.t(), a.abs() @ b.abs().t(), k, (many, e))


def test_rows_past_4_gib(xr):
    g = generator(12)
    rows, k = 530000, 4128
    x = torch.empty(rows, k, dtype=torch.bfloat16, device="cuda")
    x.normal_(0, 1, generator=g)
    counts = [rows - 1000, 990]
    offsets = offsets_of(counts)
    for n in (256, 72):
        w = normal(g, 2, n, k, scale=0.02).bfloat16()
        out = torch.full((rows, n), SENTINEL, dtype=torch.bfloat16, device="cuda")
        xr.group_product(x, w, offsets, out)
        for lo, hi, e in ((0, 300, 0), (rows - 1300, rows - 1000, 0), (rows - 1000, rows - 10, 1)):
            a, b = x[lo:hi].double(), w[e].double()
            check_sum(out[lo:hi], a @ b.t(), a.abs() @ b.abs().t(), k, (lo, n))
        assert (out[rows - 10:] == SENTINEL).all()
        dw = torch.empty(2, n, k, device="cuda")
        xr.group_product_grad(out, x, offsets, dw)
        a, b = out[rows - 1000:rows - 10].double(), x[rows - 1000:rows - 10].double()
        check_sum(dw[1], a.t() @ b, a.abs().t() @ b.abs(), 990)


@pytest.mark.parametrize("far", ["x", "w", "out", "scale"])
def test_rows_far_apart(xr, far):
    """8 MB and more from row to row: few rows, many, and a gradient."""
    g = generator(14)
    apart = (1 << 23) + 16

    def spaced(t, yes):
        if not yes:
            return t
        rows, n = t.shape
        store = torch.empty(rows * apart, dtype=t.dtype, device="cuda")
        view = store.view(rows, apart)[:, :n]
        view.copy_(t)
        return view

    for counts, n, k in (([3, 2], 72, 136), ([30, 35], 72, 136), ([1, 0, 2], 130, 264)):
        rows, experts, offsets = sum(counts), len(counts), offsets_of(counts)
        x, w = normal(g, rows, k).bfloat16(), normal(g, experts * n, k).bfloat16()
        out = spaced(torch.full((rows, n), SENTINEL, dtype=torch.bfloat16, device="cuda"), far == "out")
        w_far = spaced(w, far == "w").unflatten(0, (experts, n)) if experts * n <= 150 else w.view(experts, n, k)
        x_far = spaced(x, far == "x")
        xr.group_product(x_far, w_far, offsets, out)
        check_sum(out, *product(x, w.view(experts, n, k), offsets), k, (far, n))
        dw = torch.empty(experts, n, k, device="cuda")
        d = normal(g, rows, n).bfloat16()
        xr.group_product_grad(spaced(d, far == "out"), x_far, offsets, dw)
        at = offsets.tolist()
        for e in range(experts):
            a, b = d[at[e]:at[e + 1]].double(), x[at[e]:at[e + 1]].double()
            check_sum(dw[e], a.t() @ b, a.abs().t() @ b.abs(), counts[e] + 1)
        x4, scale = quant_mx4(x.float())
        w4, w_scale = quant_mx4(w.float())
        w4, w_scale = w4.view(experts, n, -1), w_scale.view(experts, n, -1)
        out = torch.full((rows, n), SENTINEL, dtype=torch.bfloat16, device="cuda")
        xr.group_product(spaced(x4, far == "x"), w4, offsets, out, scale=spaced(scale, far == "scale"),
                         w_scale=w_scale)
        check_sum(out, *product(of_mx4(x4, scale), of_mx4(w4, w_scale), offsets), k, (far, n))
