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


def norm_args():
    return dict(x=z(4, 8), after=z(8), gate=z(4, 8), residual=z(4, 8), before=z(8), out=z(4, 8))


def product_args():
    return dict(x=z(4, 32, dtype=torch.int8), weight=z(8, 32, dtype=torch.int8), weight_scale=z(8, dtype=F32),
                x_scale=z(4, dtype=F32), bias=z(8, dtype=F32), out=z(4, 8))


def linear_args():
    return dict(q=z(3, 4, 64), k=z(3, 2, 64), v=z(3, 2, 64), state=z(5, 2, 64, 64, dtype=F32), log_decay=z(2, dtype=F32),
                read=torch.full((3,), -1, dtype=torch.int32, device=DEV), out=z(3, 4, 64))


def store_args():
    return dict(k=z(3, 2, 64), v=z(3, 2, 64), k_cache=z(4, 16, 2, 64), v_cache=z(4, 16, 2, 64),
                slots=z(3, dtype=torch.int32), k_scale=z(2, dtype=F32), v_scale=z(2, dtype=F32))


def attention_args():
    i32 = torch.int32
    return dict(q=z(3, 4, 64), k_cache=z(4, 16, 2, 64), v_cache=z(4, 16, 2, 64), row_start=None,
                table=z(3, 1, dtype=i32), length=torch.ones(3, dtype=i32, device=DEV), out=z(3, 4, 64),
                k_scale=z(2, dtype=F32), v_scale=z(2, dtype=F32))


CALLS = {"block_norm": norm_args, "integer_product": product_args, "linear_attention": linear_args,
         "cache_store": store_args, "shared_attention": attention_args}
FLOATS = {"block_norm": ["x", "after", "gate", "residual", "before", "out"],
          "integer_product": ["x", "weight_scale", "x_scale", "bias", "out"],
          "linear_attention": ["q", "k", "v", "state", "log_decay", "out"],
          "cache_store": ["k", "v", "k_cache", "v_cache"], "shared_attention": ["q", "k_cache", "v_cache", "out"]}


@pytest.mark.parametrize("what,name", [(c, n) for c in FLOATS for n in FLOATS[c]])
def test_a_tangent_is_refused(what, name):
    # in forward mode the result would need one
    call, args = getattr(K, what), CALLS[what]()
    if what == "integer_product" and name == "x":
        args.update(x=z(4, 32), x_scale=None)
    if what in ("cache_store", "shared_attention"):
        args.update(k_scale=None, v_scale=None)
    with torch.autograd.forward_ad.dual_level():
        call(**args)
        t = args[name]
        dual = dict(args, **{name: torch.autograd.forward_ad.make_dual(t, torch.ones_like(t))})
        with pytest.raises(K.KvrError):
            call(**dual)
        with torch.no_grad(), pytest.raises(K.KvrError):  # (which leaves forward mode on)
            call(**dual)
        with torch.inference_mode():
            call(**args)
    call(**args)


def test_tangents_of_scales_are_refused():
    for what, name in (("cache_store", "k_scale"), ("cache_store", "v_scale"), ("shared_attention", "k_scale"),
                       ("shared_attention", "v_scale")):
        args = CALLS[what]()
        eight = {n: args[n].to(torch.float8_e4m3fn) for n in ("k_cache", "v_cache")}
        with torch.autograd.forward_ad.dual_level():
            dual = torch.autograd.forward_ad.make_dual(args[name], torch.ones_like(args[name]))
            with pytest.raises(K.KvrError):
                getattr(K, what)(**dict(args, **eight, **{name: dual}))


@pytest.mark.parametrize("what,name", [("block_norm", "eps"), ("block_norm", "residual_scale"),
                                       ("linear_attention", "scale"), ("shared_attention", "scale")])
@pytest.mark.parametrize("value", [1e39, -1e300, float("inf"), float("nan")])
def test_numbers_that_32_bits_do_not_hold_are_refused(what, name, value):
    args = CALLS[what]()
    args.update({n: None for n in ("k_scale", "v_scale") if n in args})
    with pytest.raises(K.KvrError):
        getattr(K, what)(**args, **{name: value})


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("new,heads,kv,dim", [([200, 0, 9, 64] * 3, 32, 4, 128), ([40, 77] * 8, 15, 5, 64)])
def test_linear_requests_that_begin_with_nothing_and_are_not_kept(new, heads, kv, dim, dtype):
    # (their query heads are taken side by side, as no state is written)
    none = [-1] * len(new)
    p = R.Linear(new, heads=heads, kv_heads=kv, dim=dim, dtype=dtype, read=none, write=none, spare=1)
    args = p.args()
    note(f"linear unkept {heads}/{kv} {dim}")
    out = K.linear_attention(*args)
    R.check_linear(out, args[3], p)
    assert torch.equal(args[3].cpu(), p.state)
    in_place = K.linear_attention(*args[:6], None, args[7])
    assert torch.equal(in_place, out)
