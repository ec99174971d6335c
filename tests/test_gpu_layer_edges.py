"""Edges of the norms, 8-bit products and linear attention on the GPU: sizes at a
launch's limit, arguments at the ends of their ranges, what a call refuses."""
import pytest
import torch

import layer_reference as R
import paper_2601_18999_amd as K
from gpu_helpers import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, F32 = torch.bfloat16, torch.float16, torch.float32


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def test_product_of_more_tokens_than_narrow_tiles_fit_a_launch():
    # 2^29 tokens that are one in memory (tiles of 64 x 64 would be 2^32 threads), each with a scale of its own
    tokens, channels, dim = 1 << 29, 3, 16
    g = torch.Generator().manual_seed(0)
    x, w = (torch.randint(-128, 128, (n, dim), generator=g, dtype=torch.int8).to(DEV) for n in (1, channels))
    ws = (torch.rand(channels, generator=g) + 0.5).to(DEV)
    xs = torch.arange(tokens, device=DEV, dtype=torch.int32).remainder_(509).add_(1).float()
    note(f"product {tokens} x {dim} x {channels}")
    got = K.integer_product(x.expand(tokens, dim), w, ws, x_scale=xs)
    sums = (x.double() @ w.double().t()).float()
    for c in range(channels):
        assert torch.equal(got[:, c], (sums[0, c] * xs * ws[c]).bfloat16())


@pytest.mark.parametrize("eps", [2.0 ** -149, 1e-40, 2.0 ** -127, 2.0 ** -126])
@pytest.mark.parametrize("dim", [64, 300, 1024])
def test_norm_with_the_smallest_eps(dim, eps):
    # rows of zeros, and such whose mean square is subnormal, tiny and usual (powers of two: the sums are exact)
    x = torch.tensor([0.0, 2.0 ** -66, 2.0 ** -64, 2.0 ** -63, 2.0 ** -60, 1.0])[:, None].repeat(1, dim).to(BF16)
    x[:, 1::2] *= -1
    w = torch.full((dim,), 1.5, dtype=BF16)
    note(f"norm dim={dim} eps={eps}")
    eps = float(torch.tensor(eps, dtype=F32))
    for which in ("after", "before"):
        got = K.block_norm(x.to(DEV), **{which: w.to(DEV)}, eps=eps).out
        n, _, mn, _ = R.norm(x, **{which: w}, eps=eps)
        R.check_norm(got, n, mn, BF16)
        assert (got[0] == 0).all()


def test_norm_of_no_column_has_the_scale_0():
    torch.full((5,), float("nan"), device=DEV)  # what the allocator hands out next
    got = K.block_norm(torch.empty((5, 0), dtype=BF16, device=DEV), int8=True)
    assert got.out.shape == (5, 0) and (got.scale == 0).all()
