"""The experts' products (group_product, group_product_grad) against 64-bit references:
types, both orders of the weights, ragged and odd sizes, rows of no expert, strides and
alignments, graphs, streams and budgets."""
import pytest

torch = pytest.importorskip("torch")
from product_util import (E4M3_CUT, SENTINEL, TYPES, check_sum, generator, inside, normal,  # noqa: E402
                          of_mx4, offsets_of, product, quant_mx4, spread)

pytestmark = pytest.mark.gpu

# rows of each expert, and rows left at the end
COUNTS = {"one row": ([1], 0), "one expert": ([131], 0), "few": ([1, 0, 3, 2, 0, 0, 1], 1),
          "ragged": ([0, 257, 1, 0, 64, 300, 31, 0], 9), "none": ([0, 0, 0], 5),
          "many": ([(7 * e * e) % 23 for e in range(200)], 3), "most": ([3] + [0] * 1022 + [40], 2)}
# n, k: below, at and past what a step, a tile and a vector hold
SIZES = [(1, 1), (64, 64), (128, 64), (129, 65), (72, 200), (256, 512), (515, 1027), (320, 136),
         (37, 7), (100, 2000)]


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def plain_case(g, dt, counts, left, n, k, transpose=False, pad=0, off=0):
    """x, w, offsets, and w as experts x n x k; rows of no expert and experts without rows
    hold NaN."""
    rows = sum(counts) + left
    x = normal(g, rows, k).to(dt)
    x[rows - left:] = float("nan")
    w = normal(g, len(counts), n, k, scale=0.2).to(dt)
    w[[e for e, c in enumerate(counts) if c == 0]] = float("nan")
    held = w.transpose(1, 2).contiguous() if transpose else w
    return inside(x, pad, off), inside(held, pad, off), offsets_of(counts), w


def run_plain(xr, g, dt, counts, left, n, k, transpose=False, pad=0, off=0, wide=False):
    x, w, offsets, flat = plain_case(g, dt, counts, left, n, k, transpose, pad, off)
    out = inside(torch.full((len(x), n), SENTINEL, device="cuda",
                            dtype=torch.float32 if wide else dt), pad, off)
    xr.group_product(x, w, offsets, out, transpose=transpose)
    want, size = product(x, flat, offsets)
    check_sum(out, want, size, k, (counts[:8], n, k, transpose, pad, off))
    if pad:   # between and behind the rows nothing was written
        base = out.as_strided((len(x), n + pad), (n + pad, 1), out.storage_offset())
        assert torch.isnan(base[:, n:]).all()


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("which", COUNTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_product(xr, dtype, which, transpose):
    g = generator(1)
    for n, k in SIZES:
        if which == "most" and n * k > 20000:
            continue
        run_plain(xr, g, TYPES[dtype], *COUNTS[which], n, k, transpose)


@pytest.mark.parametrize("transpose", [False, True], ids=["nk", "kn"])
@pytest.mark.parametrize("pad,off", [(8, 0), (8, 8), (1, 0), (3, 1), (5, 2), (16, 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignments(xr, dtype, pad, off, transpose):
    g = generator(2)
    for n, k in ((64, 128), (136, 72), (129, 65), (260, 200)):
        for counts, left in (([5, 0, 150, 1], 2), ([1, 2, 0], 0)):
            run_plain(xr, g, TYPES[dtype], counts, left, n, k, transpose, pad, off)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_wide_output(xr, dtype):
    g = generator(3)
    for n, k in ((64, 64), (129, 264), (37, 7)):
        run_plain(xr, g, TYPES[dtype], *COUNTS["ragged"], n, k, wide=True)
        run_plain(xr, g, TYPES[dtype], *COUNTS["few"], n, k, wide=True)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_rows_of_one_expert(xr, rows):
    """Around the ends of every tile."""
    g = generator(rows)
    for transpose in (False, True):
        run_plain(xr, g, torch.bfloat16, [rows, rows], 1, 192, 320, transpose)
        run_plain(xr, g, torch.bfloat16, [rows], 0, 257, 96, transpose)


def e4m3(g, *shape):
    x = normal(g, *shape, scale=60.0).clamp(-448, 448)
    return x.to(torch.float8_e4m3fn)


@pytest.mark.parametrize("out_dtype", TYPES)
@pytest.mark.parametrize("which", COUNTS)
def test_product_e4m3(xr, which, out_dtype):
    g = generator(4)
    counts, left = COUNTS[which]
    rows = sum(counts) + left
    for (n, k), pad in zip(SIZES, (0, 0, 0, 0, 8, 16, 1, 0, 3, 16)):
        if which == "most" and n * k > 20000:
            continue
        x, w = inside(e4m3(g, rows, k), pad), inside(e4m3(g, len(counts), n, k), pad)
        kb, nb = -(-k // 128), -(-n // 128)
        scale = torch.rand(rows, kb, device="cuda", generator=g) * 0.02 + 1e-3
        w_scale = torch.rand(len(counts), nb, kb, device="cuda", generator=g) * 0.02 + 1e-3
        scale[rows - left:] = float("nan")
        scale, w_scale = inside(scale, pad), inside(w_scale, pad)
        offsets = offsets_of(counts)
        out = torch.full((rows, n), SENTINEL, dtype=TYPES[out_dtype], device="cuda")
        xr.group_product(x, w, offsets, out, scale=scale, w_scale=w_scale)
        want, size = product(x.double() * spread(scale, rows, k),
                             w.double() * spread(w_scale, n, k, 128), offsets)
        check_sum(out, want, size, k + 3 * kb, (which, n, k), E4M3_CUT)


@pytest.mark.parametrize("out_dtype", TYPES)
@pytest.mark.parametrize("which", COUNTS)
def test_product_mx4(xr, which, out_dtype):
    g = generator(5)
    counts, left = COUNTS[which]
    rows = sum(counts) + left
    for (n, k), pad in zip(SIZES, (0, 0, 0, 0, 8, 16, 1, 0, 3, 16)):
        if which == "most" and n * k > 20000:
            continue
        x4, scale = quant_mx4(normal(g, rows, k))
        w4, w_scale = quant_mx4(normal(g, len(counts) * n, k, scale=0.2))
        w4, w_scale = w4.view(len(counts), n, -1), w_scale.view(len(counts), n, -1)
        scale[rows - left:] = 255
        # exponents of every size that products and sums of binary32 hold
        w_scale += torch.randint(0, 30, w_scale.shape, device="cuda", generator=g).to(torch.uint8)
        w_scale -= 15
        x4, w4, scale, w_scale = (inside(t, pad) for t in (x4, w4, scale, w_scale))
        offsets = offsets_of(counts)
        out = torch.full((rows, n), SENTINEL, dtype=TYPES[out_dtype], device="cuda")
        xr.group_product(x4, w4, offsets, out, scale=scale, w_scale=w_scale)
        want, size = product(of_mx4(x4, scale), of_mx4(w4, w_scale), offsets)
        fits = want.abs() < (65000 if out_dtype == "f16" else float("inf"))
        check_sum(out[fits], want[fits], size[fits], k, (which, n, k))
        assert (out[~fits].abs() >= 64900).all()   # 65000 less a k-th of 2^-23 and half a step


@pytest.mark.parametrize("add", [False, True], ids=["set", "add"])
@pytest.mark.parametrize("which", COUNTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_product_grad(xr, dtype, which, add):
    g = generator(6)
    counts, left = COUNTS[which]
    dt, rows = TYPES[dtype], sum(counts) + left
    for (n, k), (pad, off) in zip(SIZES, ((0, 0), (0, 0), (8, 0), (3, 1), (0, 0), (8, 8), (1, 0),
                                          (0, 0), (0, 0), (5, 0))):
        if which in ("most", "many") and n * k > 20000:
            continue
        dout, x = normal(g, rows, n).to(dt), normal(g, rows, k).to(dt)
        dout[rows - left:] = float("nan")
        x[rows - left:] = float("nan")
        dout, x, offsets = inside(dout, pad, off), inside(x, pad, off), offsets_of(counts)
        for to in {dt, torch.float32}:
            dw = inside(normal(g, len(counts), n, k).to(to), pad, off)
            before = dw.double()
            if not add:
                dw.fill_(float("nan"))
            xr.group_product_grad(dout, x, offsets, dw, add=add)
            at = offsets.tolist()
            for e in range(len(counts)):
                a, b = dout[at[e]:at[e + 1]].double(), x[at[e]:at[e + 1]].double()
                want, size = a.t() @ b, a.abs().t() @ b.abs()
                if add:
                    want, size = want + before[e], size + before[e].abs()
                check_sum(dw[e], want, size, counts[e] + 1, (which, n, k, to, e))


def test_gradients_against_differences(xr):
    """Of sum(out * d) with respect to single weights and inputs, by central differences:
    the function is linear, so steps can be large."""
    g = generator(7)
    counts, n, k = [3, 0, 70, 5], 40, 24
    x, w, offsets, _ = plain_case(g, torch.float32, counts, 0, n, k)
    w = torch.nan_to_num(w)
    d = normal(g, len(x), n)

    def f(x, w):
        out = torch.empty(len(x), n, device="cuda")
        xr.group_product(x, w, offsets, out)
        return float((out.double() * d.double()).sum())

    dx, dw = torch.empty_like(x), torch.empty_like(w)
    xr.group_product(d, w, offsets, dx, transpose=True)
    xr.group_product_grad(d, x, offsets, dw)
    # f sums len(x) * n values of about k terms each, off by (k + 4) 2^-23 of their sizes
    size = float((product(x, w, offsets)[1] * d.double().abs()).sum())
    for t, grad in ((x, dx), (w, dw)):
        for i in torch.randint(0, t.numel(), (12,), generator=torch.Generator().manual_seed(1)).tolist():
            lo, hi = t.clone(), t.clone()
            lo.view(-1)[i] -= 64
            hi.view(-1)[i] += 64
            args = ((lo, w), (hi, w)) if t is x else ((x, lo), (x, hi))
            diff = (f(*args[1]) - f(*args[0])) / 128
            assert abs(diff - float(grad.view(-1)[i])) <= 40 * (k + 4) * 2.0 ** -23 * size / 64 + 1e-5


def test_transposed_gradient_is_the_exchanged_one(xr):
    g = generator(8)
    counts, n, k = [30, 0, 99], 72, 40
    x, d, offsets = normal(g, 129, k), normal(g, 129, n), offsets_of(counts)
    a, b = torch.empty(3, n, k, device="cuda"), torch.empty(3, k, n, device="cuda")
    xr.group_product_grad(d, x, offsets, a)
    xr.group_product_grad(x, d, offsets, b)
    for e, (lo, hi) in enumerate(((0, 30), (30, 30), (30, 129))):
        want, size = d[lo:hi].double().t() @ x[lo:hi].double(), d[lo:hi].double().abs().t() @ x[lo:hi].double().abs()
        check_sum(a[e], want, size, hi - lo)
        check_sum(b[e].t().contiguous(), want, size, hi - lo)


def test_experts_may_share_weights(xr):
    """Experts 0 elements apart, and every second expert of a larger tensor."""
    g = generator(9)
    counts, n, k = [4, 9, 0, 2], 64, 96
    x, offsets = normal(g, 15, k).bfloat16(), offsets_of(counts)
    w = normal(g, 8, n, k).bfloat16()
    for view in (w[:1].expand(4, n, k), w[::2], w[1::2]):
        out = torch.full((15, n), SENTINEL, dtype=torch.bfloat16, device="cuda")
        xr.group_product(x, view, offsets, out)
        check_sum(out, *product(x, view, offsets), k)


def test_offsets_outside_the_rows_are_cut_off(xr):
    """Nothing outside the rows is read or written, whatever the offsets say."""
    g = generator(10)
    n = k = 64
    x, w = normal(g, 40, k).bfloat16(), normal(g, 4, n, k).bfloat16()
    big = torch.full((120, n), SENTINEL, dtype=torch.bfloat16, device="cuda")
    out = big[40:80]
    for bad, cut in (([-5, 10, 20, 30, 99], [0, 10, 20, 30, 40]),
                     ([0, 10, 8, 30, 2 ** 31 - 1], None), ([-9, -5, -1, 41, 50], [0, 0, 0, 40, 40])):
        big.fill_(SENTINEL)
        xr.group_product(x, w, torch.tensor(bad, dtype=torch.int32, device="cuda"), out)
        torch.cuda.synchronize()
        assert (big[:40] == SENTINEL).all() and (big[80:] == SENTINEL).all()
        if cut:
            check_sum(out, *product(x, w, torch.tensor(cut)), k)
        dw = torch.empty(4, n, k, device="cuda")
        xr.group_product_grad(out, x, torch.tensor(bad, dtype=torch.int32, device="cuda"), dw)
        assert torch.isfinite(dw).all()


def test_infinities_stay_with_their_rows(xr):
    """A row of infinities or NaN makes its own row of the output so and no other; the
    steps' zeros past k do not meet them."""
    g = generator(11)
    for dt in TYPES.values():
        for k in (64, 72, 65, 200):
            x, w, offsets = normal(g, 70, k).to(dt), normal(g, 2, 96, k).to(dt), offsets_of([50, 20])
            x[7] = float("inf")
            x[60, k - 1] = float("nan")
            out = torch.empty(70, 96, dtype=dt, device="cuda")
            xr.group_product(x, w, offsets, out)
            rows = torch.tensor([r for r in range(70) if r not in (7, 60)], device="cuda")
            assert not torch.isfinite(out[7]).any() and torch.isnan(out[60]).all()
            want, size = product(x, w, offsets)
            check_sum(out[rows], want[rows], size[rows], k)


def test_results_are_the_same_every_time(xr):
    """Bit for bit: on another stream, under a budget of workgroups, and replayed from a
    graph between other work."""
    g = generator(12)
    counts = [0, 300, 1, 77, 0, 140]
    x, w, offsets, _ = plain_case(g, torch.bfloat16, counts, 2, 320, 448)
    w = torch.nan_to_num(w)
    d = normal(g, len(x), 320).bfloat16()

    def call(stream=None):
        out = torch.zeros(len(x), 320, dtype=torch.bfloat16, device="cuda")
        dw = torch.zeros(6, 320, 448, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        xr.group_product(x, w, offsets, out, stream=stream)
        xr.group_product_grad(d, x, offsets, dw, stream=stream)
        torch.cuda.synchronize()
        return out, dw

    want = call()
    same = lambda got: all(torch.equal(a, b) for a, b in zip(got, want))
    assert same(call()) and same(call(torch.cuda.Stream()))
    for most in (1, 7, 100):
        before = xr.set_max_workgroups(most)
        try:
            assert same(call())
        finally:
            xr.set_max_workgroups(before)
    out, dw = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        xr.group_product(x, w, offsets, out)
        xr.group_product_grad(d, x, offsets, dw)
    for _ in range(3):
        out.zero_()
        dw.zero_()
        call()
        graph.replay()
        torch.cuda.synchronize()
        assert same((out, dw))
    # the counts are read when the graph runs
    offsets.copy_(offsets_of([10, 0, 200, 0, 300, 8]))
    again = call()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again[0][:518], out[:518]) and torch.equal(again[1], dw)
    assert not torch.equal(dw, want[1])
