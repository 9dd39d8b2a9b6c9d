"""The gated activation and its gradient where gates, values or gradients are infinite or NaN:
each element's own result and its group's 8-bit scale, and no other."""
import pytest

torch = pytest.importorskip("torch")
from product_util import TYPES, generator, inside, normal  # noqa: E402

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
SPECIAL = [INF, -INF, NAN, 0.0, -0.0, 1.0, -1.0, 30000.0, -30000.0, -20.0]


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def same(got, want, what):
    """The same NaN and infinities, and finite values to 2^-7 (what they are to full accuracy is
    tested elsewhere) or the least normal number of the type."""
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    want = want.float().to(got.dtype).double()
    assert torch.equal(torch.isinf(got), torch.isinf(want)), what
    fine = torch.isfinite(want)
    got, least = got.double(), torch.finfo(got.dtype).smallest_normal
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), what
    assert ((got - want)[fine].abs() <= want[fine].abs() * 2.0 ** -7 + least).all(), what


@pytest.mark.parametrize("dtype", TYPES)
def test_every_pair(xr, dtype):
    """All gates with all values, and for the gradient with all incoming gradients.  A gate of
    -30000 has a share of one that is 0 in binary32, as in the definition's 64 bits."""
    v = torch.tensor(SPECIAL, device="cuda").to(TYPES[dtype])
    g, u, d = (t.flatten() for t in torch.meshgrid(v, v, v, indexing="ij"))
    for columns in (len(g), 125, 8, 1):   # rows of one length and another
        rows = len(g) // columns
        x = inside(torch.cat([g.view(rows, columns), u.view(rows, columns)], 1), 3, 1)
        dout = d.view(rows, columns)
        gate, up = x.double().chunk(2, 1)
        s, c = torch.sigmoid(gate), torch.sigmoid(-gate)
        out, dx = torch.empty_like(dout), torch.empty_like(x)
        xr.gate(x, out)
        same(out, gate * s * up, (dtype, columns))
        xr.gate_grad(dout, x, dx)
        same(dx[:, :columns], dout.double() * up * s * (1 + gate * c), (dtype, columns, "gates"))
        same(dx[:, columns:], dout.double() * gate * s, (dtype, columns, "values"))


@pytest.mark.parametrize("group", [32, 64, 128, 256, 512])
@pytest.mark.parametrize("dtype", TYPES)
def test_scales(xr, dtype, group):
    """A NaN makes its group's scale and codes NaN; an infinity makes the scale infinite, its own
    code NaN and the group's others 0.  Groups beside them are as without either."""
    gen, dt, width = generator(group), TYPES[dtype], 4 * group + 20
    x = normal(gen, 6, 2 * width).to(dt)
    x[0, group + 3] = NAN                 # a gate; then a value; infinities of both; infinity and NaN
    x[1, width + 2 * group + 31] = NAN
    x[2, 3 * group] = INF
    x[2, width + 3 * group] = 1.0
    x[3, width + 4 * group + 19] = -INF
    x[3, 4 * group + 19] = 1.0
    x[4, 0], x[4, width], x[4, 5] = INF, 1.0, NAN
    hit = {(0, 1): NAN, (1, 2): NAN, (2, 3): INF, (3, 4): INF, (4, 0): NAN}
    q, scale = torch.empty(6, width, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, 5, device="cuda")
    xr.gate(x, out8=q, scale=scale, group=group)
    fine = x.clone()
    fine[~torch.isfinite(fine)] = 0.0
    q2, scale2 = torch.empty_like(q), torch.empty_like(scale)
    xr.gate(fine, out8=q2, scale=scale2, group=group)
    q, q2 = q.float(), q2.float()
    for r in range(6):
        for i in range(5):
            part = slice(i * group, min((i + 1) * group, width))
            kind = hit.get((r, i))
            if kind is None:
                assert scale[r, i] == scale2[r, i] and torch.equal(q[r, part], q2[r, part])
            elif kind == INF:
                assert scale[r, i] == INF
                bad = torch.isnan(q[r, part])
                assert bad.sum() == 1 and bad[0 if r == 2 else 19] and (q[r, part][~bad] == 0).all()
            else:
                assert torch.isnan(scale[r, i]) and torch.isnan(q[r, part]).all()
