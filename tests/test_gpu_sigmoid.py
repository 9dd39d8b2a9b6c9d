"""The router's sigmoids, which replace the division by the hardware's reciprocal and
one Newton step.  The choice of experts bounds with these and orders with the
divided ones, so it is exact only if both are the same for every input."""
import ctypes

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


def test_every_input(xr):
    """All 2^32 logits, and the quotient of every 1 <= d < 2^126."""
    from paper_2510_20171_amd import build
    C = ctypes.CDLL(str(build.CEILING_OUT))
    C.xred_ceiling_sigmoids.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    found = torch.tensor([0, 0, 0, -1], dtype=torch.int64, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert C.xred_ceiling_sigmoids(found.data_ptr(), stream) == 0
    inputs, sigmoids, reciprocals, first = found.tolist()
    assert inputs == 1 << 32
    assert sigmoids == 0, hex(first & 0xFFFFFFFF)
    assert reciprocals == 0, hex(first >> 32 & 0xFFFFFFFF)


@pytest.mark.parametrize("tokens", [64, 5000])
@pytest.mark.parametrize("experts,groups", [(16, 1), (64, 1), (128, 8), (256, 1), (256, 8), (512, 1),
                                            (1000, 10)])
def test_keys_a_unit_apart(xr, tokens, experts, groups):
    """Logits within a few units of 2^-23, where 1 + exp(-x) has a significand of all ones,
    and of others: rows of few different keys, some units apart.  Expected ids as
    the header defines the keys, in torch."""
    g = torch.Generator(device="cuda").manual_seed(experts + tokens)
    near = torch.tensor([0.0, 2.0 ** -23, -2.0 ** -22, 1.0, -1.0, -30.0, 6.0, -80.0], device="cuda")
    at = near[torch.arange(tokens, device="cuda") % len(near), None]
    unit = at.abs().clamp(min=1.0).log2().floor().exp2() * 2.0 ** -23
    x = at + unit * torch.randint(-4, 5, (tokens, experts), device="cuda", generator=g)
    key = 1.0 / (1.0 + torch.exp(-x))
    keep = max(1, groups // 2)
    if groups > 1:
        part = key.view(tokens, groups, -1)
        best = part.sort(dim=2, descending=True, stable=True).values
        chosen = (best[..., 0] + best[..., 1]).sort(dim=1, descending=True, stable=True).indices
        on = torch.zeros((tokens, groups), device="cuda").scatter_(1, chosen[:, :keep], 1.0)
        key = torch.where(on[:, :, None] > 0, part, -torch.inf).view(tokens, experts)
    want = key.sort(dim=1, descending=True, stable=True).indices
    for k in (1, 4, 8, 16):
        ids = torch.empty((tokens, k), dtype=torch.int32, device="cuda")
        xr.route(x, ids, torch.empty((tokens, k), device="cuda"), score="sigmoid", groups=groups,
                 group_topk=keep)
        assert torch.equal(ids.long(), want[:, :k]), k
