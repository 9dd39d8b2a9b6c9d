"""Offsets that are not in order: the experts' products touch nothing outside the rows, and do
no more work than that many rows in order would be, however many tiles the offsets ask for."""
import pytest

torch = pytest.importorskip("torch")
from product_util import SENTINEL, check_sum, generator, normal, offsets_of, product  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def xr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    import paper_2510_20171_amd as xr
    xr.load()
    return xr


# rows, experts, n, k, rows of a tile: streaming, 64 x 64, 256 x 256, and (off the grid) 128 x 128 tiles
@pytest.mark.parametrize("rows,experts,n,k,tile", [(4096, 1023, 64, 64, 32), (4096, 63, 56, 64, 64),
                                                   (16384, 31, 3848, 72, 256), (8192, 31, 3845, 71, 128)])
def test_every_other_expert_claims_all_rows(xr, rows, experts, n, k, tile):
    """Expert e's weights make e; each second expert asks for every row.  As many tiles are
    worked on as rows in order can have, of the first experts."""
    x = torch.ones(rows, k, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(experts, n, k, dtype=torch.bfloat16, device="cuda")
    w[:, :, 0] = (torch.arange(experts, device="cuda") % 251).bfloat16()[:, None]   # exact in bf16
    w[:, :, 1] = (torch.arange(experts, device="cuda") // 251 * 251).bfloat16()[:, None]
    value = w[:, 0, 0].float() + w[:, 0, 1].float()
    big = torch.full((rows + 600, n), SENTINEL, device="cuda")
    out = big[300:300 + rows]
    offsets = torch.tensor([0, rows] * (experts // 2 + 1), dtype=torch.int32, device="cuda")
    xr.group_product(x, w, offsets, out)
    torch.cuda.synchronize()
    assert (big[:300] == SENTINEL).all() and (big[300 + rows:] == SENTINEL).all()
    most = rows // tile + min(rows, experts)             # tiles of rows in order
    last = 2 * ((most - 1) // (rows // tile))            # the last expert that has one of them
    assert last < experts - 1
    seen = out[out != SENTINEL]
    assert seen.numel() == out.numel() and torch.isin(seen, value[:last + 1:2]).all()


def test_calls_after_it_are_right(xr):
    g = generator(30)
    x, w = normal(g, 300, 72).bfloat16(), normal(g, 5, 136, 72).bfloat16()
    out = torch.empty(300, 136, device="cuda")
    for bad in ([300, 0, 300, 0, 300, 0], [5, 4, 3, 2, 1, 0], [-2 ** 31, 2 ** 31 - 1] * 3):
        xr.group_product(x, w, torch.tensor(bad, dtype=torch.int32, device="cuda"), out)
        offsets = offsets_of([100, 0, 31, 160, 9])
        xr.group_product(x, w, offsets, out)
        check_sum(out, *product(x, w, offsets), 72)
