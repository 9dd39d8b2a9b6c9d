"""A router whose bias and group ranks go by the softmax's probabilities p themselves,
as include/xred.h says to have it: the sigmoid form on log(p / (1 - p)).

sigmoid(log(p / (1 - p))) is p up to the rounding of the logit, |logit| u (u = 2^-24), and
some 6 units of its own: for p above 2^-20 less than 32 u = 2^-19 of p, twice that in a sum of
two.  Rows two of whose keys or group ranks lie closer than 2^-17 are left out."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


def gaps(v):
    return v.sort(dim=1).values.diff(dim=1).amin(1)


@pytest.mark.parametrize("groups,keep", [(1, 1), (8, 3)])
@pytest.mark.parametrize("renorm", [False, True])
def test_bias_on_probabilities(xr, groups, keep, renorm):
    t, e, k = 3000, 64, 6
    g = torch.Generator(device="cuda").manual_seed(groups)
    x = torch.randn(t, e, device="cuda", generator=g, dtype=torch.float64).requires_grad_(True)
    bias = 0.02 * torch.randn(e, device="cuda", generator=g)
    p = x.softmax(1)
    key = p.detach() + bias
    sure = gaps(key) > 2.0 ** -17
    if groups > 1:
        part = key.view(t, groups, -1)
        rank = part.topk(2, 2).values.sum(2)
        sure &= gaps(rank) > 2.0 ** -17
        on = torch.zeros_like(rank).scatter_(1, rank.topk(keep, 1).indices, 1.0)
        key = torch.where(on[:, :, None] > 0, part, -torch.inf).reshape(t, e)
    want = key.topk(k, 1).indices
    assert int(sure.sum()) > t // 2
    z = torch.log(p / (1 - p))
    ids = torch.empty((t, k), dtype=torch.int32, device="cuda")
    w = torch.empty((t, k), device="cuda")
    z32 = z.detach().float()
    xr.route(z32, ids, w, score="sigmoid", bias=bias, groups=groups, group_topk=keep, renorm=renorm)
    assert torch.equal(ids[sure].long(), want[sure])
    s = p.gather(1, ids.long())
    s = s / s.sum(1, keepdim=True) if renorm else s
    assert bool(((w.double() - s).abs() <= 2.0 ** -17 * s).all())
    # the gradient goes on through z
    dw, dz = torch.randn(t, k, device="cuda", generator=g), torch.empty_like(z32)
    xr.route_grad(z32, ids, dw, dz, score="sigmoid", renorm=renorm)
    got, = torch.autograd.grad(z, x, dz.double(), retain_graph=True)
    ref, = torch.autograd.grad(s, x, dw.double())
    assert float((got - ref).norm()) <= 2.0 ** -17 * float(ref.norm())
