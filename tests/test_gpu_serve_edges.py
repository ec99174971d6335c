"""The serving operators on the GPU at the edges of their number ranges and
rules: wide strides, NaN, sizes around the forms of the plan."""
import pytest
import torch

import paper_2601_18999_amd as K
from gpu_helpers import note
import serve_reference as R
from test_gpu_serve import BF16, DEV, FP16, FP8, attend
from test_gpu_serve_plan import on_device

pytestmark = pytest.mark.gpu


def slots_apart(cache, stride, storage, at):
    """The cache with its slots `stride` bytes apart, in the storage from byte `at` on."""
    pages, page, heads, dim = cache.shape
    assert stride % 16 == 0 and pages * heads * dim * 2 <= 1 << 20
    view = torch.as_strided(storage, cache.shape, (heads * dim, stride // 2, dim, 1), at // 2)
    return view.copy_(cache)


# the last stride whose rows of one load are within 2^32 bytes, the next one, and the widest
@pytest.mark.parametrize("dim,page,stride", [(64, 8, 613566736), (64, 8, 613566752), (64, 8, (1 << 31) - 16),
                                             (128, 4, 1431655680), (128, 4, 1431655696), (128, 4, (1 << 31) - 16),
                                             (256, 2, (1 << 31) - 16)])
@pytest.mark.parametrize("wide", ["k", "v", "both"])
def test_slots_far_apart(dim, page, stride, wide):
    # few rows (a wave's own tiles) and many (tiles that the waves share), whole tiles and ends
    p = R.Problem([1, 70], [100, 150], [1, 1], [64, 70], heads=2, kv_heads=1, dim=dim, page=page)
    args = p.args()
    storage = torch.empty((page * stride + (4 << 20)) // 2, dtype=BF16, device=DEV)
    note(f"slots {stride} bytes apart, dim={dim} page={page} wide={wide}")
    for i, name in ((1, "k"), (2, "v")):
        if wide in (name, "both"):
            args[i] = slots_apart(args[i], stride, storage, (i - 1) << 20)
    R.check(K.shared_attention(*args, **p.kwargs()), None, p, on_device(p))
