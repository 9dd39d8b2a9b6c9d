"""dispatch_plan, dispatch, combine and combine_grad against their definitions.

The plan and the copies are exact.  Combine is a left fold with one rounding an
operation, so it is compared bit for bit with the same operations in torch's
binary32, and with 64 bits; dweights, a sum of `hidden` products, with 64 bits:
at most hidden / 256 + 64 additions follow one another in a lane and between
lanes (pieces of 8 included with room), each off by u = 2^-24 of the magnitudes."""
import math

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


def draw_ids(g, tokens, experts, topk, dropped=0.1):
    """Popular experts and others; distinct within a token where that is possible."""
    if topk <= experts:
        x = randn(g, tokens, experts) + randn(g, 1, experts)
        ids = x.argsort(1, descending=True)[:, :topk].int()
    else:
        ids = torch.randint(0, experts, (tokens, topk), device="cuda", generator=g).int()
    ids[torch.rand(ids.shape, device="cuda", generator=g) < dropped] = -1
    return ids.contiguous()


def plan_of(ids, experts):
    flat = ids.flatten().cpu().long()
    valid = (flat >= 0) & (flat < experts)
    counts = torch.bincount(flat[valid], minlength=experts)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    slots = torch.where(valid, flat, experts).argsort(stable=True)[:int(valid.sum())]
    pos = torch.full_like(flat, -1)
    pos[slots] = torch.arange(len(slots))
    return counts, offsets, pos.view(ids.shape), slots


def plan(xr, ids, experts, **kw):
    t, k = ids.shape
    counts = torch.full((experts,), 99, dtype=torch.int32, device="cuda")
    offsets = torch.full((experts + 1,), 99, dtype=torch.int32, device="cuda")
    pos = torch.full((t, k), 99, dtype=torch.int32, device="cuda")
    slots = torch.full((t * k,), -7, dtype=torch.int32, device="cuda")
    xr.dispatch_plan(ids, counts, offsets, pos, slots=slots, **kw)
    return counts, offsets, pos, slots


def check_plan(xr, ids, experts):
    counts, offsets, pos, slots = plan(xr, ids, experts)
    want = plan_of(ids, experts)
    for got, ref, what in ((counts, want[0], "counts"), (offsets, want[1], "offsets"),
                           (pos, want[2], "pos")):
        assert torch.equal(got.cpu().long(), ref), what
    n = len(want[3])
    assert torch.equal(slots[:n].cpu().long(), want[3])
    assert bool((slots[n:] == -7).all()), "slots past the last row were written"


@pytest.mark.parametrize("experts", [1, 2, 31, 64, 65, 256, 257, 1000, 1024])
@pytest.mark.parametrize("tokens,topk", [(1, 1), (1, 32), (63, 1), (65, 8), (1023, 2), (2049, 1),
                                         (2051, 8)])
def test_plan_in_one_workgroup(xr, experts, tokens, topk):
    g = gen(experts + tokens)
    for dropped in (0.0, 0.3):
        check_plan(xr, draw_ids(g, tokens, experts, topk, dropped), experts)


@pytest.mark.parametrize("tokens,topk,experts", [(16385, 1, 64), (5000, 8, 256), (40001, 6, 1000),
                                                 (130001, 8, 128), (300007, 4, 3)])
def test_plan_over_workgroups(xr, tokens, topk, experts):
    g = gen(tokens)
    ids = draw_ids(g, tokens, experts, topk)
    check_plan(xr, ids, experts)
    before = plan(xr, ids, experts)
    prev = xr.set_max_workgroups(3)
    try:
        after = plan(xr, ids, experts)
    finally:
        xr.set_max_workgroups(prev)
    assert all(torch.equal(a, b) for a, b in zip(before, after))


def test_plan_extremes(xr):
    """One expert for all, none at all, ids that are no experts, no tokens."""
    for tokens in (700, 9000):
        ids = torch.full((tokens, 4), 5, dtype=torch.int32, device="cuda")
        check_plan(xr, ids, 8)
        check_plan(xr, torch.full_like(ids, -1), 8)
        ids[::3, 1] = 8
        ids[1::3, 2] = 2 ** 31 - 1
        ids[2::3, 0] = -2 ** 31
        check_plan(xr, ids, 8)
    empty = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    counts, offsets, _, _ = plan(xr, empty, 8)
    assert bool((counts == 0).all()) and bool((offsets == 0).all())


@pytest.mark.parametrize("dtype", [torch.uint8, torch.float8_e4m3fn, torch.bfloat16,
                                   torch.float32, torch.int64])
@pytest.mark.parametrize("hidden", [1, 3, 8, 15, 16, 17, 127, 1000, 2048, 5001])
def test_dispatch_moves_bits(xr, dtype, hidden):
    g = gen(hidden)
    es = torch.empty(0, dtype=dtype).element_size()
    for tokens, topk, experts, pad in ((1, 1, 4, 0), (33, 8, 16, 3), (70, 3, 5, 1)):
        ids = draw_ids(g, tokens, experts, topk)
        _, offsets, pos, _ = plan(xr, ids, experts)
        rows = tokens * topk
        raw = torch.randint(0, 256, (tokens, (hidden + pad) * es), device="cuda", generator=g)
        x = raw.to(torch.uint8).view(dtype)[:, :hidden]
        wide = torch.full((rows, (hidden + pad) * es), 55, dtype=torch.uint8, device="cuda")
        out = wide.view(dtype)[:, :hidden]
        scale = randn(g, tokens, 70)[:, :67]
        out_scale = torch.full((rows, 69), 7.0, device="cuda")
        xr.dispatch(x, pos, out, scale=scale, out_scale=out_scale[:, :67])
        want = torch.full_like(wide, 55)
        want_scale = torch.full_like(out_scale, 7.0)
        for t in range(tokens):
            for j in range(topk):
                r = int(pos[t, j])
                if r >= 0:
                    want[r, :hidden * es] = raw[t, :hidden * es].to(torch.uint8)
                    want_scale[r, :67] = scale[t]
        assert torch.equal(wide, want) and torch.equal(out_scale, want_scale)


def test_places_past_the_rows_are_passed_over(xr):
    """pos beyond out_rows or y_rows is dropped, whatever it holds."""
    g = gen(1)
    x = randn(g, 6, 100)
    pos = torch.tensor([[0, 3], [4, 2 ** 31 - 1], [-1, 2], [5, -2 ** 31], [1, 6], [-5, -1]],
                       dtype=torch.int32, device="cuda")
    out = torch.full((6, 100), 9.0, device="cuda")
    xr.dispatch(x, pos, out[:4])
    assert torch.equal(out[0], x[0]) and torch.equal(out[3], x[0]) and torch.equal(out[2], x[2])
    assert torch.equal(out[1], x[4]) and bool((out[4:] == 9).all())
    got = torch.empty(6, 100, device="cuda")
    xr.combine(out[:4], pos, got)
    want = torch.stack([out[0] + out[3], torch.zeros_like(x[0]), out[2], torch.zeros_like(x[0]),
                        out[1], torch.zeros_like(x[0])])
    assert torch.equal(got, want)
    dy = torch.full((6, 100), 8.0, device="cuda")
    dw = torch.full((6, 2), 8.0, device="cuda")
    w = torch.ones((6, 2), device="cuda")
    xr.combine_grad(x, out[:4], pos, w, dy[:4], dw)
    assert bool((dy[4:] == 8).all()) and torch.equal(dy[:4], torch.stack([x[0], x[4], x[2], x[0]]))
    assert torch.equal(dw == 0, ~((pos >= 0) & (pos < 4)))


def fold(y, pos, weights, base):
    """The definition in torch's binary32, an operation at a time."""
    t, k = pos.shape
    acc = base.float() if base is not None else None
    first = torch.full((t,), base is None, device="cuda")
    acc = acc if acc is not None else torch.zeros((t, y.shape[1]), device="cuda")
    for j in range(k):
        on = pos[:, j] >= 0
        term = y[pos[:, j].clamp(min=0).long()].float()
        if weights is not None:
            term = weights[:, j, None] * term
        new = torch.where(first[:, None], term, acc + term)
        acc = torch.where(on[:, None], new, acc)
        first = first & ~on
    return acc.to(y.dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [1, 7, 8, 9, 511, 512, 513, 1003, 4096, 5001])
def test_combine_bit_for_bit(xr, dtype, hidden):
    g = gen(hidden)
    dt = DT[dtype]
    for n, (tokens, topk, experts) in enumerate(((1, 1, 4), (29, 8, 32), (65, 3, 7), (17, 19, 40),
                                                 (5, 32, 64))):
        ids = draw_ids(g, tokens, experts, topk, 0.2)
        ids[0] = -1 if tokens > 1 else ids[0]      # a token none of whose slots is here
        pos = plan(xr, ids, experts)[2]
        wide = randn(g, tokens * topk, hidden + 2 * (n % 2)).to(dt)
        y = wide[:, n % 2:n % 2 + hidden]
        w = randn(g, tokens, topk)
        for base in (None, randn(g, tokens, hidden + 1).to(dt)[:, 1:]):
            for weights in (None, w):
                out = torch.full((tokens, hidden + 3), 7.0, device="cuda").to(dt)
                xr.combine(y, pos, out[:, :hidden], weights=weights, base=base)
                assert bool((out[:, hidden:].float() == 7).all())
                assert torch.equal(out[:, :hidden], fold(y, pos, weights, base))
        # in place over the base
        over = base.clone()
        xr.combine(y, pos, over, weights=w, base=over)
        assert torch.equal(over, fold(y, pos, w, base))


def test_combine_special_values(xr):
    """Infinities, NaN and -0 pass through; rows of dropped slots, which may hold
    anything, do not."""
    y = torch.randn(6, 40, device="cuda")
    y[0, 0], y[1, 1], y[2] = math.inf, math.nan, -0.0
    y[5] = math.nan
    pos = torch.tensor([[0, 3], [1, 4], [2, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[1.0, 0.5], [0.0, 1.0], [1.0, math.nan], [math.inf, 1.0]], device="cuda")
    out = torch.empty(4, 40, device="cuda")
    xr.combine(y, pos, out, weights=w)
    want = torch.stack([y[0] + 0.5 * y[3], 0.0 * y[1] + y[4], y[2], torch.zeros_like(y[0])])
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.equal(out.nan_to_num(), want.nan_to_num())
    assert bool((1 / out[2] == -math.inf).all()) and bool((1 / out[3] == math.inf).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [1, 7, 8, 9, 500, 513, 2501, 4096, 9000])
def test_combine_gradient(xr, dtype, hidden):
    g = gen(hidden)
    dt = DT[dtype]
    for n, (tokens, topk, experts) in enumerate(((1, 1, 4), (30, 8, 32), (9, 3, 7), (17, 19, 40))):
        pos = plan(xr, draw_ids(g, tokens, experts, topk, 0.2), experts)[2]
        rows = tokens * topk
        dout = randn(g, tokens, hidden + 1).to(dt)[:, n % 2:n % 2 + hidden]
        y = randn(g, rows, hidden).to(dt)
        w = randn(g, tokens, topk)
        wide = torch.full((rows, hidden + 3), 7.0, device="cuda").to(dt)
        dw = torch.full((tokens, topk), math.nan, device="cuda")
        xr.combine_grad(dout, y, pos, w, wide[:, :hidden], dw)
        want = torch.full_like(wide, 7.0)
        at, slot = torch.nonzero(pos >= 0, as_tuple=True)
        to = pos[at, slot].long()
        want[to, :hidden] = (w[at, slot][:, None] * dout[at].float()).to(dt)
        assert torch.equal(wide, want)
        ref = torch.zeros(tokens, topk, device="cuda").double()
        mag = torch.zeros_like(ref)
        products = dout[at].double() * y[to].double()
        ref[at, slot], mag[at, slot] = products.sum(1), products.abs().sum(1)
        err = (dw.double() - ref).abs()
        assert bool((err <= (hidden / 32 + 64) * U * mag + 2 * U * ref.abs()).all())
        assert bool((dw[pos < 0] == 0).all())
        # without dweights y is not needed, and dy may be y
        alone = torch.full_like(wide, 7.0)
        xr.combine_grad(dout, None, pos, w, alone[:, :hidden])
        assert torch.equal(alone, want)
        again = torch.empty_like(dw)
        over = y.clone()
        xr.combine_grad(dout, over, pos, w, over, again)
        assert torch.equal(again, dw) and torch.equal(over[to], wide[to, :hidden])


def test_gradients_against_differences(xr):
    """combine is linear in y, base and weights, so central differences are exact up
    to rounding: of fp32 sums of about 1e3 over steps of 2^-2, below 1e-4 of the
    scale.  The gradient of dispatch is combine without weights."""
    g = gen(5)
    t, k, h, e, s = 7, 3, 60, 5, 0.25
    pos = plan(xr, draw_ids(g, t, e, k, 0.1), e)[2]
    y, base, w, r = randn(g, t * k, h), randn(g, t, h), randn(g, t, k), randn(g, t, h)
    out = torch.empty(t, h, device="cuda")

    def value(y, base, w):
        xr.combine(y, pos, out, weights=w, base=base)
        return float((out.double() * r).sum())

    dy, dw = torch.zeros_like(y), torch.empty_like(w)
    xr.combine_grad(r, y, pos, w, dy, dw)
    for _ in range(3):
        a, b, c = randn(g, t * k, h), randn(g, t, h), randn(g, t, k)
        for up, down, slope, size in (
                ((y + s * a, base, w), (y - s * a, base, w), (dy.double() * a).sum(), a.norm() * dy.norm()),
                ((y, base + s * b, w), (y, base - s * b, w), (r.double() * b).sum(), b.norm() * r.norm()),
                ((y, base, w + s * c), (y, base, w - s * c), (dw.double() * c).sum(), c.norm() * dw.norm())):
            got = (value(*up) - value(*down)) / (2 * s)
            assert abs(got - float(slope)) <= 1e-4 * float(size)
    x, dx = randn(g, t, h), torch.empty(t, h, device="cuda")
    rows = torch.zeros(t * k, h, device="cuda")
    rr = randn(g, t * k, h)
    xr.combine(rr, pos, dx)
    d = randn(g, t, h)
    got = []
    for v in (x + s * d, x - s * d):
        xr.dispatch(v, pos, rows)
        got.append(float((rows.double() * rr).sum()))
    slope = float((dx.double() * d).sum())
    assert abs((got[0] - got[1]) / (2 * s) - slope) <= 1e-4 * float(d.norm() * dx.norm())


def test_round_trip_streams_and_graphs(xr):
    """ids to rows and back, then the same on another stream and in a replayed graph."""
    g = gen(6)
    t, k, h, e = 3000, 8, 768, 64
    ids = draw_ids(g, t, e, k, 0.0)
    x = randn(g, t, h)
    w = torch.full((t, k), 0.125, device="cuda")
    counts = torch.empty(e, dtype=torch.int32, device="cuda")
    offsets = torch.empty(e + 1, dtype=torch.int32, device="cuda")
    pos = torch.empty((t, k), dtype=torch.int32, device="cuda")
    rows, out = torch.empty((t * k, h), device="cuda"), torch.empty_like(x)
    dy, dw = torch.empty_like(rows), torch.empty_like(w)

    def calls(**kw):
        xr.dispatch_plan(ids, counts, offsets, pos, **kw)
        xr.dispatch(x, pos, rows, **kw)
        xr.combine(rows, pos, out, weights=w, **kw)
        xr.combine_grad(x, rows, pos, w, dy, dw, **kw)

    calls()
    assert torch.equal(out, fold(rows, pos, w, None))
    want = [v.clone() for v in (pos, rows, out, dy, dw)]
    side = torch.cuda.Stream()
    for v in (pos, rows, out, dy, dw):
        v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((pos, rows, out, dy, dw), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for n in range(3):
        for v in (pos, rows, out, dy, dw):
            v.fill_(n)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((pos, rows, out, dy, dw), want)), n
    prev = xr.set_max_workgroups(5)
    try:
        calls()
    finally:
        xr.set_max_workgroups(prev)
    assert all(torch.equal(a, b) for a, b in zip((pos, rows, out, dy, dw), want))


def test_rows_past_4_gib(xr):
    """Places whose byte offsets pass 32 bits."""
    g = gen(7)
    h, rows = 8192, 600_000    # 9.2 GiB of bf16 rows
    y = torch.empty((rows, h), dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor([[0, rows - 1], [rows // 2, 300_000 + 7]], dtype=torch.int32, device="cuda")
    x = randn(g, 2, h).bfloat16()
    xr.dispatch(x, pos, y)
    assert torch.equal(y[rows - 1], x[0]) and torch.equal(y[rows // 2], x[1])
    out = torch.empty_like(x)
    w = torch.tensor([[0.5, 0.25], [1.0, 2.0]], device="cuda")
    xr.combine(y, pos, out, weights=w)
    assert torch.equal(out, fold(y, pos, w, None))
    dw = torch.empty_like(w)
    xr.combine_grad(x, y, pos, w, y, dw)
    assert torch.equal(y[rows - 1], (0.25 * x[0].float()).bfloat16())


def test_no_tokens(xr):
    none = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    x, y = torch.empty((0, 64), device="cuda"), torch.ones((5, 64), device="cuda")
    xr.dispatch(x, none, y)
    xr.combine(y, none, x)
    xr.combine_grad(x, y, none, torch.empty((0, 4), device="cuda"), y,
                    torch.empty((0, 4), device="cuda"))
    assert bool((y == 1).all())
    # tokens, but no rows anywhere: every slot is passed over
    pos = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    w, dw = torch.ones((3, 2), device="cuda"), torch.ones((3, 2), device="cuda")
    out = torch.ones((3, 64), device="cuda")
    empty = torch.empty((0, 64), device="cuda")
    xr.combine(empty, pos, out, weights=w)
    assert bool((out == 0).all())
    xr.dispatch(out, pos, empty)
    xr.combine_grad(out, empty, pos, w, empty, dw)
    assert bool((dw == 0).all())
