"""The gated activation and its gradient against 64-bit references."""
import pytest

torch = pytest.importorskip("torch")
from product_util import SENTINEL, TYPES, generator, inside, normal, offsets_of  # noqa: E402

pytestmark = pytest.mark.gpu
WIDTHS = [1, 5, 7, 8, 9, 31, 32, 64, 100, 255, 256, 512, 513, 1000, 2048]


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def near(got, want, terms, what):
    """`terms` binary32 operations on values of at most the sizes in want's second part
    (exponential and reciprocal good to 2 units in the last place each count as two),
    and one rounding to got's type."""
    value, size = want
    half = torch.finfo(got.dtype).eps / 2
    allowed = value.abs() * half + size * terms * 2.0 ** -23 + torch.finfo(got.dtype).smallest_normal
    over = (got.double() - value).abs() - allowed
    assert not torch.isnan(got).any(), what
    assert over.max() <= 0, (what, float(over.max()))


def forward(x):
    g, u = x.double().chunk(2, 1)
    y = g * torch.sigmoid(g) * u
    # an exponential's argument may be rounded: no, it is -g itself; its error is relative
    return y, y.abs()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_gate(xr, dtype, width):
    g = generator(width)
    dt = TYPES[dtype]
    for rows, live, pad, off in ((1, None, 0, 0), (37, 30, 0, 0), (70, 70, 3, 1), (9, 0, 8, 8)):
        x = (normal(g, rows, 2 * width) * 3).to(dt)
        offsets = None
        if live is not None:
            x[live:] = float("nan")
            offsets = offsets_of([live])
        x = inside(x, pad, off)
        live = rows if live is None else live
        for group in (32, 64, 128, 256, 512):
            y = inside(torch.full((rows, width), SENTINEL, device="cuda", dtype=dt), pad, off)
            groups = -(-width // group)
            q = inside(torch.full((rows, width), 1.0, device="cuda").to(torch.float8_e4m3fn), pad, off)
            s = inside(torch.full((rows, groups), SENTINEL, device="cuda"), pad, off)
            xr.gate(x, y, out8=q, scale=s, group=group, offsets=offsets)
            assert (y[live:] == SENTINEL).all() and (q[live:].float() == 1).all() and (s[live:] == SENTINEL).all()
            if live == 0:
                continue
            want, size = forward(x[:live])
            near(y[:live], (want, size), 8, (rows, width))
            part = torch.nn.functional.pad(want, (0, groups * group - width)).unflatten(1, (groups, group))
            scale = part.abs().amax(2).clamp(min=2.0 ** -100) / 448
            assert ((s[:live].double() - scale).abs() <= scale * 12 * 2.0 ** -23).all()
            # half a step of e4m3 (2^-4 relative, 2^-10 among subnormals) and the quotient's error
            z = want / s[:live].double().repeat_interleave(group, 1)[:, :width]
            off8 = (q[:live].double() - z).abs()
            assert (off8 <= z.abs() * (2.0 ** -4 + 2.0 ** -18) + 2.0 ** -10).all()
            # one output alone gives the same
            y2, q2, s2 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(s)
            xr.gate(x, y2, offsets=offsets)
            xr.gate(x, out8=q2, scale=s2, group=group, offsets=offsets)
            assert torch.equal(y2[:live], y[:live]) and torch.equal(s2[:live], s[:live])
            assert torch.equal(q2[:live].view(torch.uint8), q[:live].view(torch.uint8))


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_gate_grad(xr, dtype, width):
    g = generator(100 + width)
    dt = TYPES[dtype]
    for rows, live, pad, off in ((1, None, 0, 0), (37, 30, 0, 0), (70, 70, 3, 1), (9, 0, 8, 8)):
        x, d = (normal(g, rows, 2 * width) * 3).to(dt), normal(g, rows, width).to(dt)
        offsets = offsets_of([3, 0, live - 3]) if live else None if live is None else offsets_of([0])
        live = rows if live is None else live
        x[live:] = float("nan")
        x, d = inside(x, pad, off), inside(d, pad, off)
        dx = inside(torch.full((rows, 2 * width), SENTINEL, device="cuda", dtype=dt), pad, off)
        xr.gate_grad(d, x, dx, offsets=offsets)
        assert (dx[live:] == SENTINEL).all()
        if live:
            gate, up = x[:live].double().chunk(2, 1)
            do, s, c = d[:live].double(), torch.sigmoid(gate), torch.sigmoid(-gate)
            near(dx[:live, :width], (do * up * s * (1 + gate * c),
                                     (do * up).abs() * s * (1 + gate.abs())), 10, (rows, width))
            near(dx[:live, width:], (do * gate * s, (do * gate * s).abs()), 8, (rows, width))
        # in place
        xr.gate_grad(d, x, x, offsets=offsets)
        assert torch.equal(x[:live], dx[:live])
        assert torch.isnan(x[live:]).all()


def test_gradient_against_differences(xr):
    """By central differences of the forward call in fp32: h^2 / 6 of the third derivative
    (below 1 for |u d| of 4 and less) and the call's rounding over 2 h."""
    g = generator(5)
    x, d = normal(g, 40, 128), normal(g, 40, 64).clamp(-2, 2)
    x[:, 64:].clamp_(-2, 2)
    dx = torch.empty_like(x)
    xr.gate_grad(d, x, dx)
    h = 2.0 ** -6
    for half in (0, 1):
        step = torch.zeros_like(x)
        step[:, 64 * half:64 * half + 64] = h
        hi, lo = torch.empty_like(d), torch.empty_like(d)
        xr.gate(x + step, hi)
        xr.gate(x - step, lo)
        diff = (hi.double() - lo.double()) / (2 * h) * d.double()
        assert (diff - dx[:, 64 * half:64 * half + 64].double()).abs().max() <= 4 * h * h / 6 + 2.0 ** -15


def test_far_gates(xr):
    """Gates whose exponential overflows or vanishes."""
    g = torch.tensor([-200.0, -100.0, -89.0, -88.0, -87.0, -20.0, 0.0, 20.0, 88.0, 100.0, 200.0, -0.0],
                     device="cuda")
    x = torch.cat([g, torch.full_like(g, 2.0)]).view(1, -1)
    y = torch.empty(1, len(g), device="cuda")
    xr.gate(x, y)
    near(y, forward(x), 8, "far")
    dx = torch.empty_like(x)
    xr.gate_grad(torch.ones_like(y), x, dx)
    assert torch.isfinite(dx).all()
    assert (dx[0, 8:11] == 2).all() and (dx[0, :2].abs() < 1e-35).all()


def test_zero_rows_graph_and_budget(xr):
    xr.gate(torch.empty(0, 8, device="cuda"), torch.empty(0, 4, device="cuda"))
    xr.gate_grad(torch.empty(0, 4, device="cuda"), torch.empty(0, 8, device="cuda"),
                 torch.empty(0, 8, device="cuda"))
    g = generator(6)
    x, d, offsets = normal(g, 300, 1400).bfloat16(), normal(g, 300, 700).bfloat16(), offsets_of([100, 150])
    y, dx = torch.zeros(300, 700, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)

    def call():
        xr.gate(x, y, offsets=offsets)
        xr.gate_grad(d, x, dx, offsets=offsets)

    call()
    want = y.clone(), dx.clone()
    before = xr.set_max_workgroups(3)
    try:
        y.zero_(), dx.zero_()
        call()
    finally:
        xr.set_max_workgroups(before)
    assert torch.equal(y, want[0]) and torch.equal(dx, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in (250, 17, 300):
        y.zero_(), dx.zero_()
        offsets[-1] = n
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert (y[n:] == 0).all() and torch.equal(y[:min(n, 250)], want[0][:min(n, 250)])
        assert (dx[n:] == 0).all() and bool((y[n - 1] != 0).any())
