"""route and route_grad against their definition.

The choice is exact: keys are computed here in binary32 by torch, operation by
operation as the header defines them, and a stable sort gives the expected ids.
Weights and gradients are compared with their formulas in 64 bits, to error
bounds of binary32 (u = 2^-24; exp is taken as good to 2 units, with the rounding
of its argument, |x - max| u, beside that)."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {torch.float32: (U, 2.0 ** -149), torch.bfloat16: (2.0 ** -9, 2.0 ** -133),
         torch.float16: (2.0 ** -12, 2.0 ** -24)}


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


def in_order(key, k):
    """The k largest, NaN above all, ties to the lowest index (sorted on the CPU)."""
    key = (key.float() + 0.0).cpu()
    rank = torch.where(key.isnan(), torch.tensor(math.inf).double(), key.double())
    big = torch.finfo(torch.float64).max
    rank = torch.where(key == math.inf, torch.tensor(big), rank)   # below NaN
    got = rank.sort(dim=-1, descending=True, stable=True)
    return key.gather(-1, got.indices)[..., :k].cuda(), got.indices[..., :k].cuda()


def choose(x, score, bias, groups, group_topk, group_score, k):
    x = x.float()
    key = 1.0 / (1.0 + torch.exp(-x)) if score == "sigmoid" else x
    if bias is not None:
        key = key + bias
    key = torch.where(x == -math.inf, -math.inf, key)
    if groups > 1:
        t, e = key.shape
        part = key.view(t, groups, e // groups)
        best = in_order(part, group_score)[0]
        rank = best[..., 0] + best[..., 1] if best.shape[-1] == 2 else best[..., 0]
        on = torch.zeros_like(rank).scatter_(1, in_order(rank, group_topk)[1], 1.0)
        key = torch.where(on[:, :, None] > 0, part, -math.inf).reshape(t, e)
    best, ids = in_order(key, k)
    return torch.where(best == -math.inf, -1, ids)


def sigmoid64(x):
    """exp(-x) overflows binary32 below -88.72: the score is 0 there."""
    return torch.where(x < -88.722839, 0.0, x.sigmoid())


def weights64(x, ids, score, renorm):
    """Scores of the chosen before scaling, 0 where none, and their relative error."""
    x = x.double()
    none = ids < 0
    top = x.gather(1, ids.clamp(min=0)).masked_fill(none, -math.inf)
    if score == "sigmoid":
        s = sigmoid64(top)
        rel = torch.full_like(s, 6 * U)
        if renorm:
            total = s.sum(1, keepdim=True)
            s = torch.where(total == 0, 0.0, s / total)
            rel = rel * 2 + 40 * U
    else:
        over = top if renorm else x
        m = over.amax(1, keepdim=True)
        total = (over - m).exp().sum(1, keepdim=True)
        s = (top - m).exp() / total
        rel = (3 + (top - m).abs().nan_to_num(posinf=0)) * U * 2 + (over.shape[1] + 8) * U
    return s.masked_fill(none, 0.0), rel


def near(got, want, err, what):
    rel, least = ROUND[got.dtype]
    g = got.double()
    ok = (g - want).abs() <= err.nan_to_num(nan=0.0) + 2 * rel * want.abs() + least
    ok |= (g == want) | (g.isnan() & want.isnan())
    assert bool(ok.all()), (what, int((~ok).sum()), g[~ok][:3], want[~ok][:3])


def check(xr, x, k, *, score, bias=None, groups=1, group_topk=1, group_score=2, renorm=True,
          scale=1.0):
    t = x.shape[0]
    ids = torch.full((t + 1, k), 77, dtype=torch.int32, device="cuda")
    w = torch.full((t + 1, k), 77.0, device="cuda")
    xr.route(x, ids[:t], w[:t], score=score, bias=bias, groups=groups, group_topk=group_topk,
             group_score=group_score, renorm=renorm, scale=scale)
    assert bool((ids[t] == 77).all()) and bool((w[t] == 77).all())
    want = choose(x, score, bias, groups, group_topk, group_score, k)
    assert torch.equal(ids[:t].long(), want), (ids[:t].long() != want).sum()
    s, rel = weights64(x, want, score, renorm)
    near(w[:t], s * scale, s.abs() * scale * (rel + 2 * U) + 2.0 ** -126, "weights")
    return ids[:t], w[:t]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("experts", [1, 2, 7, 16, 17, 60, 64, 65, 128, 160, 200, 256, 257, 384,
                                     512, 513, 1000, 1024])
def test_sizes(xr, dtype, experts):
    g = gen(experts)
    for n, (tokens, k) in enumerate(((1, 1), (5, 2), (67, 8), (130, 32))):
        x = randn(g, tokens, experts, scale=2).to(DT[dtype])
        bias = randn(g, experts, scale=0.2) if n % 2 else None
        for score in ("softmax", "sigmoid"):
            for renorm in (False, True):
                check(xr, x, min(k, experts), score=score, bias=bias, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("experts,groups", [(8, 2), (24, 8), (64, 64), (64, 16), (96, 4), (160, 5),
                                            (256, 8), (256, 32), (255, 5), (320, 64),
                                            (1000, 8), (1024, 64), (1024, 2), (15, 15)])
def test_groups(xr, experts, groups):
    g = gen(experts * groups)
    for n, dt in enumerate(DT.values()):
        x = randn(g, 41, experts).to(dt)
        for group_topk in {1, (groups + 1) // 2, groups}:
            for group_score in (1, 2):
                for score, bias in (("sigmoid", randn(g, experts, scale=0.1)), ("softmax", None)):
                    check(xr, x, min(experts, 6 + n), score=score, bias=bias, groups=groups,
                          group_topk=group_topk, group_score=group_score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lowest(xr, score):
    """Few distinct values, zeros of both signs, whole rows alike."""
    g = gen(3)
    for experts in (16, 100, 256, 1024):
        x = torch.randint(-1, 2, (300, experts), device="cuda", generator=g).float()
        x = torch.where(torch.rand(x.shape, device="cuda", generator=g) < 0.3, -x * 0.0, x)
        x[0], x[1], x[2] = 0.0, -0.0, 5.0
        check(xr, x, 8, score=score)
        check(xr, x.bfloat16(), 8, score=score, groups=4, group_topk=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masks_infinities_and_nan(xr, score, renorm):
    g = gen(4)
    for experts, groups in ((64, 8), (256, 8), (1000, 10)):
        x = randn(g, 40, experts)
        bias = randn(g, experts, scale=0.1)
        x[0] = -math.inf                       # a padding row
        x[1, :-3] = -math.inf                  # fewer experts than slots
        x[2, 5] = math.nan
        x[3, 9] = -math.nan
        x[4, 7] = math.inf
        x[5, :experts // 2] = -math.inf        # whole groups masked
        x[6] = torch.finfo(torch.float32).min  # the type's lowest value is a number
        x[7] = -300.0                          # sigmoids that underflow to 0
        x[8, 1::2] = torch.finfo(torch.float32).min
        x[9] = -90.0
        x[10, 11:13] = math.nan
        bias[3] = -math.inf                    # an expert switched off for all
        for b in (None, bias):
            check(xr, x, 8, score=score, bias=b, renorm=renorm)
            ids, w = check(xr, x, 8, score=score, bias=b, groups=groups, group_topk=groups // 2,
                           renorm=renorm)
            assert bool((ids[0] == -1).all()) and bool((w[0] == 0).all())


def test_strides(xr):
    g = gen(5)
    wide = randn(g, 50, 300).bfloat16()
    for lo, e in ((0, 256), (3, 256), (1, 128), (7, 61)):
        check(xr, wide[:, lo:lo + e], 6, score="sigmoid")
        check(xr, wide[::2, lo:lo + e], 6, score="softmax", renorm=False)


@pytest.mark.parametrize("experts,groups", [(129, 1), (160, 8), (160, 5), (200, 1), (256, 1), (256, 8),
                                            (256, 16), (256, 32), (255, 5)])
@pytest.mark.parametrize("tokens", [40, 2111])
def test_few_and_many_tokens(xr, tokens, experts, groups):
    """Either number of lanes a token, with masks, ties and infinities among the rows."""
    g = gen(tokens + experts + groups)
    x = randn(g, tokens, experts)
    x[::5] = x[::5].round()                                     # ties
    x[torch.rand(tokens, experts, generator=g, device="cuda") < 0.2] = -math.inf
    x[7] = -math.inf
    x[11, 1:] = -math.inf
    x[13, 3] = math.nan
    x[17, :9] = torch.finfo(torch.float32).min
    x[23, 5] = math.inf
    bias = randn(g, experts, scale=0.1)
    for k in (1, 6, 8, 10, 16, 20):
        for score, b in (("sigmoid", bias), ("softmax", None)):
            check(xr, x, k, score=score, bias=b, groups=groups, group_topk=(groups + 1) // 2,
                  renorm=k != 6)


def test_many_tokens(xr):
    g = gen(6)
    check(xr, randn(g, 70003, 64).bfloat16(), 6, score="softmax", renorm=False)
    check(xr, randn(g, 33333, 256), 8, score="sigmoid", bias=randn(g, 256, scale=0.1), groups=8,
          group_topk=4, scale=2.5)


def gradient64(x, ids, dw, score, renorm, scale):
    """dlogits in 64 bits and a bound on binary32's error."""
    x = x.double()
    on = torch.zeros_like(x)
    valid = ids >= 0
    on.scatter_add_(1, ids.clamp(min=0), valid.double())
    d = torch.zeros_like(x).scatter_add_(1, ids.clamp(min=0), (dw.double() * scale) * valid)
    if score == "sigmoid":
        s = sigmoid64(x)
        ds = s * (1 - s)
        if renorm:
            total = (s * on).sum(1, keepdim=True)
            inv = torch.where(total == 0, 0.0, 1 / total)
            mean = (d * s).sum(1, keepdim=True) * inv
            mag = (d * s).abs().sum(1, keepdim=True) * inv
            out = (d - mean) * inv * ds * on
            # 1 - s cancels: s's error there is u, not relative
            err = (d.abs() + mag) * inv * s * on * (80 * U * (1 - s) + 6 * U)
        else:
            out = d * ds
            err = d.abs() * s * (12 * U * (1 - s) + 6 * U)
        return out, err
    over = torch.where(on > 0, x, -math.inf) if renorm else x
    m = over.amax(1, keepdim=True)
    e = (over - torch.where(m == -math.inf, 0.0, m)).exp()
    total = e.sum(1, keepdim=True)
    p = torch.where(total == 0, 0.0, e / total)
    mean, mag = (p * d).sum(1, keepdim=True), (p * d).abs().sum(1, keepdim=True)
    spread = (over - m).abs().nan_to_num(nan=0.0, posinf=0.0)
    rel = (8 + spread + spread.mul(p).sum(1, keepdim=True) + x.shape[1]) * 2 * U
    return p * (d - mean), p * (d.abs() + mag) * rel + p * mag * 8 * U


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("experts", [1, 7, 60, 64, 128, 129, 256, 300, 512, 1000, 1024])
def test_gradient_against_the_formula(xr, dtype, experts):
    g = gen(experts)
    dt = DT[dtype]
    for tokens, k in ((1, 1), (37, 6), (130, 20)):
        k = min(k, experts)
        x = randn(g, tokens, experts, scale=2).to(dt)
        x[0, : experts // 2] = -math.inf
        dw = randn(g, tokens, k)
        for score in ("softmax", "sigmoid"):
            for renorm in (False, True):
                ids = torch.empty((tokens, k), dtype=torch.int32, device="cuda")
                w = torch.empty((tokens, k), device="cuda")
                xr.route(x, ids, w, score=score, renorm=renorm, scale=2.5)
                if tokens > 30:
                    ids[3] = -1            # a token whose every slot was dropped
                    ids[4, 0] = experts    # out of range: passed over
                wide = torch.full((tokens, experts + 3), 7.0, device="cuda").to(dt)
                xr.route_grad(x, ids, dw, wide[:, :experts], score=score, renorm=renorm, scale=2.5)
                assert bool((wide[:, experts:].float() == 7).all())
                known = torch.where(ids < experts, ids, -1).long()
                want, err = gradient64(x, known, dw, score, renorm, 2.5)
                near(wide[:, :experts], want, err + 2.0 ** -126, (score, renorm, tokens))


@pytest.mark.parametrize("low,high", [(-88.6, -86.0), (-40.0, -20.0), (5.0, 30.0)])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_of_a_saturated_sigmoid(xr, low, high, renorm):
    """Scores that are subnormal, or that leave 1 - s far below s's unit: each element is
    good to a part of itself.  r bounds a score's and its complement's own error: half a
    subnormal unit (2^-150, doubled for the product it comes from) and some units of
    2^-24 for the exponential, the sum and the quotient.  The quotient by the scores' sum
    doubles it, the mean it enters doubles that, and D bounds |dweights * scale|."""
    g = gen(11)
    t, e, k = 33, 40, 8
    x = low + (high - low) * torch.rand(t, e, generator=g, device="cuda")
    dw = randn(g, t, k)
    ids = torch.empty((t, k), dtype=torch.int32, device="cuda")
    w, dx = torch.empty((t, k), device="cuda"), torch.empty_like(x)
    xr.route(x, ids, w, score="sigmoid", renorm=renorm, scale=1.5)
    xr.route_grad(x, ids, dw, dx, score="sigmoid", renorm=renorm, scale=1.5)
    at = ids.long()
    v = x.double().gather(1, at)
    s, rest = torch.sigmoid(v), torch.sigmoid(-v)
    d = 1.5 * dw.double()
    r = 2.0 ** -149 / s.amin(1, True) + 2.0 ** -20
    if renorm:
        s = s / s.sum(1, True)
        d = d - (d * s).sum(1, True)
    want = torch.zeros(t, e, dtype=torch.float64, device="cuda").scatter(1, at, d * s * rest)
    most = 1.5 * dw.double().abs().amax(1, True)
    err = torch.zeros_like(want).scatter(1, at, 8 * r * most * s * rest + 2.0 ** -148)
    assert bool(((dx.double() - want).abs() <= err).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(xr, score, renorm):
    """Central differences of the kernel's own weights, the choice held still by a
    wide gap: with steps of 2^-6 the third derivative's part is below 1e-3."""
    g = gen(8)
    t, e, k, h = 6, 48, 5, 2.0 ** -6
    x = randn(g, t, e)
    top = x.topk(k, 1).indices
    x.scatter_add_(1, top, 3 + torch.arange(k, 0, -1, device="cuda").float().expand(t, k) * 0.4)
    r = randn(g, t, k)
    ids = torch.empty((t, k), dtype=torch.int32, device="cuda")
    w = torch.empty((t, k), device="cuda")

    def value(x):
        xr.route(x, ids, w, score=score, renorm=renorm, scale=1.5)
        return float((w.double() * r).sum()), ids.clone()

    _, chosen = value(x)
    dx = torch.empty_like(x)
    xr.route_grad(x, chosen, r, dx, score=score, renorm=renorm, scale=1.5)
    for _ in range(4):
        d = randn(g, t, e)
        (a, ia), (b, ib) = value(x + h * d), value(x - h * d)
        assert torch.equal(ia, chosen) and torch.equal(ib, chosen)
        slope = float((dx.double() * d).sum())
        assert abs((a - b) / (2 * h) - slope) <= 1e-3 * float(d.norm() * r.norm())


def test_no_tokens_streams_and_graphs(xr):
    g = gen(9)
    empty = torch.empty((0, 64), device="cuda")
    none = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    xr.route(empty, none, torch.empty((0, 4), device="cuda"))
    xr.route_grad(empty, none, torch.empty((0, 4), device="cuda"), empty.clone())
    x, dw = randn(g, 99, 256), randn(g, 99, 8)
    ids = torch.empty((99, 8), dtype=torch.int32, device="cuda")
    w, dx = torch.empty((99, 8), device="cuda"), torch.empty_like(x)

    def calls(**kw):
        xr.route(x, ids, w, score="sigmoid", groups=8, group_topk=3, **kw)
        xr.route_grad(x, ids, dw, dx, score="sigmoid", **kw)

    calls()
    want = [t.clone() for t in (ids, w, dx)]
    side = torch.cuda.Stream()
    for t in (ids, w, dx):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    calls(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((ids, w, dx), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for n in range(3):
        for t in (ids, w, dx):
            t.fill_(n)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((ids, w, dx), want)), n
    prev = xr.set_max_workgroups(3)
    try:
        calls()
    finally:
        xr.set_max_workgroups(prev)
    assert all(torch.equal(a, b) for a, b in zip((ids, w, dx), want))
