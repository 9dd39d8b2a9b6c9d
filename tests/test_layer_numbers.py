"""Numbers the binding hands to the C ABI as 32-bit fields: what does not fit is refused,
not cut to the bits that do (a group of 2^32 + 32 would pass for one of 32, with a scale
checked for another number of columns)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2510_20171_amd as xr  # noqa: E402
from test_layer_calls import F, F32, I32, INVALID  # noqa: E402


class At(F):
    """A FakeGpuTensor at an address of its own, so that no two overlap."""

    def __init__(self, k, *shape, **kw):
        super().__init__(*shape, **kw)
        self.k = k

    def data_ptr(self):
        return 1 << 46 | self.k << 40


def refused(match, call):
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the addresses are not device memory")
    with pytest.raises(xr.XredError) as e:
        call()
    assert e.value.status == INVALID and match in str(e.value), str(e.value)


@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 8, 2 ** 64 + 8, -1, -2 ** 32 + 8])
@pytest.mark.parametrize("name", ["groups", "group_topk", "group_score"])
def test_route(name, value):
    kw = {"groups": 8, "group_topk": 4, "group_score": 2, name: value}
    refused(name, lambda: xr.route(At(0, 4, 64, dtype=F32), At(1, 4, 2, dtype=I32),
                                   At(2, 4, 2, dtype=F32), stream=0, **kw))


@pytest.mark.parametrize("value", [2 ** 32, 2 ** 32 + 32, -1, -2 ** 32 + 32])
def test_fold_norm(value):
    scale = At(3, 4, 1, dtype=F32, stride=(9, 1))
    refused("group", lambda: xr.fold_norm([At(0, 4, 64)], out8=At(1, 4, 64, dtype=torch.uint8),
                                          scale=scale, group=value, stream=0))
