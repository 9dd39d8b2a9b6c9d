"""fold_norm and fold_norm_grad against their formulas in 64 bits.

The tolerances are error bounds of the formulas in binary32, u = 2^-24: a sum
of n terms is off by at most n u times the sum of their magnitudes, a row's
reductions add at most 64 terms one after another (8 of a piece, 4 pieces, 6
steps over a wave, 16 waves, with room), and an output's rounding adds half a
unit of its type."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, relative, and of the smallest subnormals
ROUND = {torch.float32: (U, 2.0 ** -150), torch.bfloat16: (2.0 ** -9, 2.0 ** -134),
         torch.float16: (2.0 ** -12, 2.0 ** -25), torch.float8_e4m3fn: (2.0 ** -5, 2.0 ** -10)}
ADDS = 64


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


def view(x, pad, offset=0):
    """x as a column range of a larger matrix, `offset` elements off its start."""
    wide = torch.full((x.shape[0], x.shape[1] + pad + offset), 7, device=x.device).to(x.dtype)
    wide[:, offset:offset + x.shape[1]] = x
    return wide[:, offset:offset + x.shape[1]], wide


def near(got, want, err, what):
    """|got - want| <= err plus the rounding of got's type, and NaN where want is NaN.
    (A row with an infinity has no finite error bound, and needs none: its rstd is 0.)"""
    err = err.nan_to_num(nan=0.0)
    rel, least = ROUND[got.dtype]
    got64 = got.double()
    ok = (got64 - want).abs() <= err + rel * (want.abs() + err) * 2 + least
    ok |= (got64 == want) | (got64.isnan() & want.isnan())
    if got.dtype == torch.float16:    # past the largest value: infinity
        ok |= (want.abs() + err >= 65504) & got64.isinf() & (got64.sign() == want.sign())
    bad = ~ok
    assert not bad.any(), (what, int(bad.sum()), got64[bad][:3], want[bad][:3])


class Forward:
    def __init__(self, srcs, residual, weight, eps, group):
        parts = [s.double() for s in srcs] + ([residual.double()] if residual is not None else [])
        self.h = torch.stack(parts).sum(0)
        mag = torch.stack(parts).abs().sum(0)
        self.eh = len(parts) * U * mag                  # error of h
        n = self.h.shape[1]
        self.rstd = 1 / (self.h.square().mean(1) + eps).sqrt()
        # mean of squares: its own additions, and h's errors
        ems = (ADDS + 4) * U * self.h.square().mean(1) + 2 * (self.h.abs() * self.eh).mean(1)
        self.erstd = self.rstd * (0.5 * ems * self.rstd.square() + 4 * U)
        w = weight.double() if weight is not None else torch.ones(n, device="cuda").double()
        self.y = self.h * self.rstd[:, None] * w
        self.ey = (self.eh * self.rstd[:, None] + self.h.abs() * self.erstd[:, None]) * w.abs() \
            + 3 * U * self.y.abs()
        size = group or n
        self.of = torch.arange(n, device="cuda") // size
        self.groups = -(-n // size)
        idx = self.of.expand_as(self.y)
        zero = torch.zeros((self.y.shape[0], self.groups), device="cuda").double()
        self.amax = zero.scatter_reduce(1, idx, self.y.abs(), "amax")
        self.amax = torch.where(zero.scatter_add(1, idx, self.y).isnan(), math.nan, self.amax)
        eamax = zero.scatter_reduce(1, idx, self.ey, "amax") + 2 * U * self.amax
        self.scale = self.amax.clamp(min=2.0 ** -100) / 448
        self.escale = eamax / 448 + 2 * U * self.scale

    def check(self, s, rstd, out, out8, scale):
        near(s, self.h, self.eh, "sum")
        near(rstd, self.rstd, self.erstd, "rstd")
        if out is not None:
            near(out, self.y, self.ey, "out")
        if out8 is not None:
            near(scale, self.scale, self.escale, "scale")
            sc = self.scale[:, self.of]
            q = self.y / sc
            near(out8, q, self.ey / sc + q.abs() * self.escale[:, self.of] / sc + 2 * U * q.abs(),
                 "out8")


def run(xr, srcs, residual, weight, group, *, out=True, eps=1e-5, pad=0):
    r, n = srcs[0].shape
    dt = srcs[0].dtype
    new = lambda dtype, cols: view(torch.full((r, cols), 3, device="cuda").to(dtype), pad)
    s, ws = new(dt, n)
    o, wo = new(dt, n)
    q, wq = new(torch.float8_e4m3fn, n)
    k = -(-n // group) if group > 0 else 1
    sc, wsc = new(torch.float32, k)
    rstd = torch.empty(r, device="cuda")
    use8 = group >= 0
    xr.fold_norm(srcs, o if out else None, residual=residual, weight=weight, sum=s,
                 out8=q if use8 else None, scale=sc if use8 else None, rstd=rstd,
                 group=max(group, 0), eps=eps)
    for wide, cols in ((ws, n), (wo, n), (wq, n), (wsc, k)):
        assert bool((wide[:, cols:].float() == 7).all()), "written past a row's end"
    Forward(srcs, residual, weight, eps, max(group, 0)).check(
        s, rstd, o if out else None, q if use8 else None, sc)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [1, 7, 8, 9, 64, 513, 1000, 2048, 2056, 4097, 8192, 16391,
                                    32768])
def test_lengths(xr, dtype, hidden):
    g = gen(hidden)
    for k, (rows, nsrc) in enumerate(((1, 1), (5, 8), (3, 3), (2, 17))):
        srcs = [randn(g, rows, hidden).to(DT[dtype]) for _ in range(nsrc)]
        res = randn(g, rows, hidden, scale=2).to(DT[dtype]) if k % 2 else None
        w = (1 + randn(g, hidden, scale=0.3)).to(DT[dtype])
        run(xr, srcs, res, w, (-1, 0, 32, 512)[k], out=k != 1)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256, 512])
def test_views_strides_and_groups(xr, dtype, group):
    """Rows at odd elements and distances, a weight in fp32, groups that end short."""
    g = gen(group)
    for hidden, pad, offset in ((705, 3, 1), (4096, 8, 5), (1280, 1, 0)):
        srcs = [view(randn(g, 37, hidden).to(DT[dtype]), pad, offset)[0] for _ in range(2)]
        res = view(randn(g, 37, hidden).to(DT[dtype]), 2, 3)[0]
        run(xr, srcs, res, 1 + randn(g, hidden, scale=0.3), group, pad=5)
        run(xr, srcs[:1], None, None, group, out=False)


@pytest.mark.parametrize("nsrc", [1, 2, 5, 8, 9, 16, 64])
def test_fold_is_in_source_order(xr, nsrc):
    """sum without a residual is allreduce_local's, bit for bit."""
    g = gen(nsrc)
    for dt in DT.values():
        srcs = [randn(g, 19, 1003, scale=10 ** (k % 5 - 2)).to(dt) for k in range(nsrc)]
        s, o, want = (torch.empty_like(srcs[0]) for _ in range(3))
        xr.fold_norm(srcs, o, sum=s)
        xr.allreduce_local(srcs, want)
        assert torch.equal(s, want)


def test_many_rows(xr):
    g = gen(5)
    for rows, hidden in ((70001, 96), (3001, 1536)):
        srcs = [randn(g, rows, hidden).bfloat16() for _ in range(2)]
        run(xr, srcs, srcs[0], 1 + randn(g, hidden, scale=0.1).bfloat16(), 32)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("hidden", [15, 32, 61, 64, 65, 100, 128, 129, 250, 256, 257, 500, 512])
def test_short_rows(xr, dtype, hidden):
    """Several rows a wave, numbers of rows that leave some of its lanes without one."""
    g = gen(hidden + 1)
    dt = DT[dtype]
    for k, rows in enumerate((1, 2, 5, 31, 32, 33, 127, 130)):
        srcs = [randn(g, rows, hidden).to(dt) for _ in range((1, 2, 5, 4)[k % 4])]
        res = view(randn(g, rows, hidden).to(dt), 1, 1)[0] if k % 3 else None
        w = (1 + randn(g, hidden, scale=0.3)).to(dt) if k % 2 else None
        run(xr, srcs, res, w, (32, 128, 512, 0, 64, 256, 128, -1)[k], out=k != 2, pad=k % 5)


def test_special_values(xr):
    """Zero rows, infinities and NaN stay in their rows; subnormal and huge rows."""
    g = gen(9)
    x = randn(g, 12, 640)
    x[1] = 0
    x[2, 5] = math.inf
    x[3, 639] = math.nan
    x[4] *= 1e-30
    x[5] *= 1e15
    x[6, 0] = -math.inf
    x[7] = -0.0
    x[8] *= 2.0 ** -140
    for dt in (torch.float32, torch.bfloat16):
        run(xr, [x.to(dt)], None, 1 + randn(g, 640, scale=0.1), 128)
        run(xr, [x.to(dt)], None, None, 0)


def test_in_place(xr):
    """The residual stream updated in place, and out over a source."""
    g = gen(11)
    srcs = [randn(g, 33, 5001).bfloat16() for _ in range(3)]
    res = randn(g, 33, 5001).bfloat16()
    s, o = torch.empty_like(res), torch.empty_like(res)
    xr.fold_norm(srcs, o, residual=res, sum=s)
    xr.fold_norm(srcs, srcs[1], residual=res, sum=res)
    assert torch.equal(res, s) and torch.equal(srcs[1], o)


def backward(dout, h, rstd, w, dsum):
    """Values and binary32 error bounds of dx and dweight."""
    d, h, r = dout.double(), h.double(), rstd.double()[:, None]
    w = w.double() if w is not None else torch.ones(h.shape[1], device="cuda").double()
    n, g = h * r, d * w
    mean, mag = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dx = r * (g - n * mean)
    err = r * (8 * U * (g.abs() + n.abs() * mag) + n.abs() * mag * (ADDS + 4) * U)
    if dsum is not None:
        dx = dx + dsum.double()
        err = err + 2 * U * dx.abs() + U * dsum.double().abs()
    rows = h.shape[0]
    terms = rows if rows < 256 else 64 + rows // 256 + 1 + 64
    return dx, err, (d * n).sum(0), (terms + 4) * U * (d * n).abs().sum(0)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,hidden", [(1, 1), (1, 7), (4, 64), (3, 4097), (257, 513),
                                         (1000, 2048), (2, 32768), (300, 5001), (5, 16390),
                                         (9000, 72)])
def test_gradient_against_the_formula(xr, dtype, rows, hidden):
    g = gen(rows + hidden)
    dt = DT[dtype]
    for k in range(2):
        h = randn(g, rows, hidden).to(dt)
        rstd = (h.float().square().mean(1) + 1e-5).rsqrt()
        dout = view(randn(g, rows, hidden).to(dt), 3 * k, k)[0]
        w = (1 + randn(g, hidden, scale=0.3)) if k else (1 + randn(g, hidden, scale=0.3)).to(dt)
        dsum = randn(g, rows, hidden).to(dt) if k else None
        dx, wide = view(torch.zeros(rows, hidden, device="cuda").to(dt), 3)
        dw = torch.full((hidden,), math.nan, device="cuda")
        xr.fold_norm_grad(dout, h, rstd, dx, weight=w, dsum=dsum, dweight=dw)
        assert bool((wide[:, hidden:].float() == 7).all())
        vx, ex, vw, ew = backward(dout, h, rstd, w, dsum)
        near(dx, vx, ex, "dx")
        near(dw, vw, ew, "dweight")
        # without dweight, over dout
        over = dout.contiguous()
        xr.fold_norm_grad(over, h, rstd, over, weight=w, dsum=dsum)
        assert torch.equal(over, dx)


@pytest.mark.parametrize("hidden", [9, 64, 100, 128, 200, 256, 512])
@pytest.mark.parametrize("rows", [1, 15, 33, 4099, 30001])
def test_gradient_of_short_rows(xr, rows, hidden):
    """A column of ones for g and n = +-1 by turns: dweight counts rows exactly, and
    dx = rstd (g - n mean(g n)) is +-1 or 0 by the row's own balance."""
    for dt in DT.values():
        sign = torch.ones(rows, hidden, device="cuda")
        sign[1::2] = -1
        d = torch.ones(rows, hidden, device="cuda").to(dt)
        rstd = torch.ones(rows, device="cuda")
        dw = torch.empty(hidden, device="cuda")
        wide = torch.full((rows, hidden + 3), 7.0, device="cuda").to(dt)
        xr.fold_norm_grad(d, sign.to(dt), rstd, wide[:, :hidden], dweight=dw)
        assert bool((wide[:, hidden:] == 7).all())
        assert bool((dw == rows % 2).all())
        # mean(g n) n = 1 up to 1 / hidden's rounding, a part of 2^-24, and the sum's
        assert bool((wide[:, :hidden].float().abs() <= hidden * 2.0 ** -24 + 2.0 ** -23).all())


def test_gradient_against_differences(xr):
    """Derivatives along random directions, by central differences of the kernel's
    own forward pass in fp32: with steps of 2^-6 the third derivative's part is
    below 1e-3 of the scale of a derivative, rounding below that."""
    g = gen(21)
    rows, n, t = 4, 384, 2.0 ** -6
    x, res = randn(g, rows, n), randn(g, rows, n)
    w, r, rs = 1 + randn(g, n, scale=0.2), randn(g, rows, n), randn(g, rows, n)
    rstd = torch.empty(rows, device="cuda")

    def value(x, res, w):
        s, o = torch.empty_like(x), torch.empty_like(x)
        xr.fold_norm([x], o, residual=res, weight=w, sum=s, rstd=rstd, eps=1e-5)
        return float((o.double() * r).sum() + (s.double() * rs).sum()), s

    _, s = value(x, res, w)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    xr.fold_norm_grad(r, s, rstd.clone(), dx, weight=w, dsum=rs, dweight=dw)
    for k in range(4):
        d, dd = randn(g, rows, n), randn(g, n)
        for up, down, slope, size in (
                ((x + t * d, res, w), (x - t * d, res, w), (dx.double() * d).sum(), d.norm() * dx.norm()),
                ((x, res + t * d, w), (x, res - t * d, w), (dx.double() * d).sum(), d.norm() * dx.norm()),
                ((x, res, w + t * dd), (x, res, w - t * dd), (dw.double() * dd).sum(), dd.norm() * dw.norm())):
            got = (value(*up)[0] - value(*down)[0]) / (2 * t)
            assert abs(got - float(slope)) <= 1e-3 * float(size), (k, got, float(slope))


def test_budget_and_repeats_do_not_change_results(xr):
    g = gen(31)
    h = randn(g, 2000, 1000).bfloat16()
    d = randn(g, 2000, 1000).bfloat16()
    rstd = (h.float().square().mean(1) + 1e-5).rsqrt()
    got = []
    for cap in (0, 7, 0):
        prev = xr.set_max_workgroups(cap)
        try:
            o, dx, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(1000, device="cuda")
            xr.fold_norm([h, d], o)
            xr.fold_norm_grad(d, h, rstd, dx, dweight=dw)
            got.append((o, dx, dw))
        finally:
            xr.set_max_workgroups(prev)
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


def test_another_stream_and_a_graph(xr):
    g = gen(41)
    h, d = randn(g, 64, 4096).bfloat16(), randn(g, 64, 4096).bfloat16()
    rstd = torch.empty(64, device="cuda")
    o, dx, dw = torch.empty_like(h), torch.empty_like(h), torch.empty(4096, device="cuda")

    def calls(**kw):
        xr.fold_norm([h, d], o, rstd=rstd, **kw)
        xr.fold_norm_grad(d, h, rstd, dx, dweight=dw, **kw)

    calls()
    want = [t.clone() for t in (o, dx, dw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (o, dx, dw):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((o, dx, dw), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(3):
        for t in (o, dx, dw):
            t.fill_(k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((o, dx, dw), want)), k


def test_no_rows(xr):
    x = torch.empty((0, 64), device="cuda")
    xr.fold_norm([x], torch.empty_like(x), sum=torch.empty_like(x))
    dw = torch.full((64,), 5.0, device="cuda")
    xr.fold_norm_grad(x, x, torch.empty(0, device="cuda"), torch.empty_like(x), dweight=dw)
    assert bool((dw == 0).all())
