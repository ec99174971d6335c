"""Norms, 8-bit products and linear attention on the GPU against plain
implementations in 64 bits."""
import numpy as np
import pytest
import torch

import layer_reference as R
import paper_2601_18999_amd as K
from gpu_helpers import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


def on(x):
    return x.to(DEV) if isinstance(x, torch.Tensor) else x


# ---------------------------------------------------------------- norms


def norm_problem(tokens, dim, dtype=BF16, residual=None, gate=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((tokens, dim), generator=g) * torch.exp2(4 * torch.rand((tokens, 1), generator=g) - 2)).to(dtype)
    w = [(1 + 0.3 * torch.randn(dim, generator=g)).to(dtype) for _ in range(2)]
    r = None if residual is None else (3 * torch.randn((tokens, dim), generator=g)).to(residual)
    if gate == "token":
        gate = torch.randn((tokens, dim), generator=g).to(dtype)
    elif gate == "channel":
        gate = torch.randn((1, dim), generator=g).to(dtype).expand(tokens, dim)
    return x, w[0], w[1], r, gate


def run_norm(**kw):
    note("norm " + " ".join(f"{k}={tuple(v.shape) if isinstance(v, torch.Tensor) else v}" for k, v in kw.items()))
    got = K.block_norm(**{k: on(v) for k, v in kw.items()})
    torch.cuda.synchronize()
    return got


def check_norm(got, int8=False, **kw):
    n, r, mn, mr = R.norm(**kw)
    if got.residual is not None:
        R.check_norm(got.residual, r, mr, kw["residual"].dtype)
    if not int8:
        R.check_norm(got.out, n, mn, kw["x"].dtype)
        return
    # the scale is that of the largest magnitude; a value is at most half a step of it off, and its own 32-bit error
    scale, steps = got.scale.double().cpu().numpy(), (R.NORM_STEPS + 4) * R.U32
    top = np.abs(n).max(1)
    at = np.abs(n) == top[:, None]
    assert (np.abs(scale - top / 127) <= steps * mn.max(1) / 127).all(), (scale, top / 127, at.sum())
    off = np.abs(got.out.double().cpu().numpy() * scale[:, None] - n)
    assert (off <= (0.5 * scale + steps * 2 * mn.max(1))[:, None]).all()


@pytest.mark.parametrize("dim", [1, 7, 8, 64, 511, 512, 513, 1024, 1500, 2048, 4096, 5003, 8192, 12345, 16384, 20000,
                                 32768, 65536])
@pytest.mark.parametrize("int8", [False, True], ids=["half", "int8"])
def test_norm_sizes(dim, int8):
    x, after, before, r, gate = norm_problem(5, dim, residual=BF16, gate="token")
    kw = dict(x=x, after=after, before=before, residual=r, residual_scale=0.5, gate=gate, activation="silu")
    check_norm(run_norm(**kw, int8=int8), int8, **kw)


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("res", [None, "same", F32], ids=["none", "same", "fp32"])
@pytest.mark.parametrize("parts", ["", "a", "b", "ab"], ids=["neither", "after", "before", "both"])
@pytest.mark.parametrize("gate,activation", [(None, "none"), ("token", "none"), ("token", "sigmoid"),
                                             ("channel", "silu")])
def test_norm_parts(dtype, res, parts, gate, activation):
    x, after, before, r, gate = norm_problem(6, 328, dtype, dtype if res == "same" else res, gate)
    kw = dict(x=x, after=after if "a" in parts else None, before=before if "b" in parts else None, residual=r,
              residual_scale=-1.25, gate=gate, activation=activation)
    check_norm(run_norm(**kw), **kw)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 257, 4099])
@pytest.mark.parametrize("dim", [96, 3000])
def test_norm_tokens(tokens, dim):
    x, after, before, r, _ = norm_problem(tokens, dim, FP16, F32)
    kw = dict(x=x, after=after, before=before, residual=r)
    check_norm(run_norm(**kw), **kw)


def test_norm_strides_and_places():
    x, after, before, r, gate = norm_problem(9, 203, FP16, F32, "token")
    kw = dict(x=x, before=before, residual=r, gate=gate)
    wide = {k: torch.full((9, 203 + 13), NAN, dtype=v.dtype, device=DEV) for k, v in
            (("x", x), ("residual", r), ("gate", gate))}
    cut = {}
    for k, v in wide.items():
        v[:, 5:208] = on(kw[k])
        cut[k] = v[:, 5:208]
    out = torch.full((9, 300), 7.0, dtype=FP16, device=DEV)
    got = K.block_norm(cut["x"], before=on(before), residual=cut["residual"], gate=cut["gate"], in_place=True,
                       out=out[:, 1:204])
    assert got.out.data_ptr() == out[:, 1:].data_ptr() and got.residual.data_ptr() == cut["residual"].data_ptr()
    check_norm(got, **kw)
    assert (out[:, 0] == 7).all() and (out[:, 204:] == 7).all()
    assert wide["residual"][:, :5].isnan().all() and wide["residual"][:, 208:].isnan().all()
    # the result over x itself
    got = K.block_norm(cut["x"], before=on(before), out=cut["x"])
    check_norm(got, x=x, before=before)
    assert wide["x"][:, :5].isnan().all() and wide["x"][:, 208:].isnan().all()


def test_norm_odd_rows():
    # zeros, an infinity, a NaN, the smallest numbers, all equal
    x = torch.randn((6, 400), generator=torch.Generator().manual_seed(3)).to(BF16)
    x[0] = 0
    x[1, 7] = INF
    x[2, 399] = NAN
    x[3] = 2.0 ** -130
    x[4] = -3
    got = run_norm(x=x, int8=True)
    scale = got.scale.cpu()
    assert scale[0] == 0 and scale[1].isnan() and scale[2].isnan() and scale[3] == 0
    assert (got.out[:4] == 0).all() and (got.out[4] == -127).all() and scale[4] == np.float32(3) / np.float32(127)
    q, s = R.integers(x[5:])
    assert (got.out[5].cpu().numpy() == q[0]).all() and scale[5] == s[0]
    w = torch.ones(400, dtype=BF16)
    out = run_norm(x=x, before=w).out.cpu()
    # x / inf is 0, but inf / inf is NaN; a NaN is everywhere
    assert (out[0] == 0).all() and out[1, 7].isnan() and (out[1, :7] == 0).all() and out[2].isnan().all()
    R.check_norm(out[3:], *[R.norm(x[3:], before=w)[i] for i in (0, 2)], BF16)


def test_norm_of_no_token_and_streams():
    x, after, before, r, _ = norm_problem(0, 64, BF16, BF16)
    got = run_norm(x=x, before=before, residual=r, int8=True)
    assert got.out.shape == (0, 64) and got.scale.shape == (0,) and got.residual.shape == (0, 64)
    x, after, before, r, _ = norm_problem(300, 1000, BF16, BF16)
    kw = dict(x=x, before=before, residual=r)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = {k: on(v) for k, v in kw.items()}
        got = K.block_norm(**y)
    side.synchronize()
    check_norm(got, **kw)


# ---------------------------------------------------------------- products


def product_problem(tokens, dim, channels, dtype="int8", bias=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(-128, 128, (channels, dim), generator=g, dtype=torch.int8)
    ws = torch.rand(channels, generator=g) / dim
    b = torch.randn(channels, generator=g) if bias else None
    if dtype == "int8":
        return torch.randint(-128, 128, (tokens, dim), generator=g, dtype=torch.int8), torch.rand(tokens, generator=g), \
            w, ws, b
    x = torch.randn((tokens, dim), generator=g) * torch.exp2(6 * torch.rand((tokens, 1), generator=g) - 3)
    return x.to(dtype), None, w, ws, b


def check_product(problem, dtype=BF16, **kw):
    x, xs, w, ws, b = problem
    note(f"product {tuple(x.shape)} x {tuple(w.shape)} {x.dtype} -> {dtype}")
    got = K.integer_product(on(x), on(w), on(ws), x_scale=on(xs), bias=on(b), dtype=dtype, **kw)
    torch.cuda.synchronize()
    xq, scale = (x.numpy(), xs.numpy()) if xs is not None else R.integers(x)
    R.check_product(got, *R.product(xq, scale, w.numpy(), ws.numpy(), None if b is None else b.numpy()), dtype)
    return got


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 127, 128, 129, 255, 256, 257, 600])
@pytest.mark.parametrize("channels,dim", [(129, 272), (512, 512), (33, 1040)])
def test_product_tokens(tokens, channels, dim):
    check_product(product_problem(tokens, dim, channels, bias=True))


@pytest.mark.parametrize("dim", [16, 32, 48, 64, 80, 96, 112, 128, 144, 160, 240, 256, 272, 368, 1008, 4096, 5008])
@pytest.mark.parametrize("tokens", [3, 40, 300])
def test_product_dims(dim, tokens):
    check_product(product_problem(tokens, dim, 200))


@pytest.mark.parametrize("channels", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700])
@pytest.mark.parametrize("tokens", [1, 20, 70, 260])
def test_product_channels(channels, tokens):
    check_product(product_problem(tokens, 176, channels))


@pytest.mark.parametrize("out", [BF16, FP16, F32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dtype", ["int8", BF16, FP16], ids=["int8", "bf16", "fp16"])
@pytest.mark.parametrize("tokens", [1, 9, 130, 513])
def test_product_types(dtype, out, tokens):
    check_product(product_problem(tokens, 336, 260, dtype, bias=tokens == 9), out)


@pytest.mark.parametrize("dim", [80, 400])
@pytest.mark.parametrize("tokens,channels", [
    (532, 128), (1000, 60), (150, 1600), (200, 1001), (31, 8192), (100, 8190), (129, 8200), (700, 4000), (250, 16300),
    (1000, 8200), (2040, 8100), (2049, 10000)])
def test_product_by_results(tokens, channels, dim):
    # from one round of the smallest workgroups to several of the largest tiles
    check_product(product_problem(tokens, dim, channels))


@pytest.mark.parametrize("tokens,dim", [(1, 16), (7, 65536), (1, 65536), (2, 32784), (16, 4096), (16, 4112), (17, 64),
                                        (15, 1040), (25, 128), (64, 1024), (65, 1008), (100, 640), (1000, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_product_of_few_tokens(tokens, dim, dtype):
    check_product(product_problem(tokens, dim, 67, dtype, bias=True), F32)


def test_product_of_the_largest_sums():
    # 65,536 times (-128)^2 = 2^30, and both signs
    w = torch.full((40, 65536), -128, dtype=torch.int8)
    w[1::2] = 127
    for tokens in (2, 70):
        x = torch.full((tokens, 65536), -128, dtype=torch.int8)
        x[1::2] = 127
        check_product((x, torch.ones(tokens), w, torch.ones(40), None), F32)


def test_product_strides_and_places():
    x, xs, w, ws, b = product_problem(70, 160, 90, bias=True)
    wide_x = torch.full((70, 208), 99, dtype=torch.int8, device=DEV)
    wide_w = torch.full((90, 176), 99, dtype=torch.int8, device=DEV)
    wide_x[:, 32:192], wide_w[:, :160] = on(x), on(w)
    for dtype in (BF16, F32):
        for tokens in (3, 70):
            out = torch.full((70, 101), 7.0, dtype=dtype, device=DEV)
            K.integer_product(wide_x[:tokens, 32:192], wide_w[:, :160], on(ws), x_scale=on(xs[:tokens]), bias=on(b),
                              out=out[:tokens, 3:93])
            want = R.product(x.numpy()[:tokens], xs.numpy()[:tokens], w.numpy(), ws.numpy(), b.numpy())
            R.check_product(out[:tokens, 3:93], *want, dtype)
            assert (out[:, :3] == 7).all() and (out[:, 93:] == 7).all() and (out[tokens:] == 7).all()
    # 16-bit rows of any stride and place
    x, _, w, ws, b = product_problem(20, 160, 90, FP16)
    wide = torch.full((20, 175), NAN, dtype=FP16, device=DEV)
    wide[:, 5:165] = on(x)
    got = K.integer_product(wide[:, 5:165], on(w), on(ws))
    xq, scale = R.integers(x)
    R.check_product(got, *R.product(xq, scale, w.numpy(), ws.numpy(), None), FP16)


def test_product_of_odd_tokens():
    # zeros, infinities and NaN stay in their rows; a NaN or infinite weight scale in its channel
    x, _, w, ws, _ = product_problem(70, 128, 40, BF16)
    x[0] = 0
    x[1, 3], x[69, 9] = NAN, INF
    ws[5] = NAN
    got = check_product((x, None, w, ws, None), BF16)
    assert (got[0, :5] == 0).all() and got[1].isnan().all() and got[69].isnan().all() and got[:, 5].isnan().all()
    got = check_product((x[:9], None, w, ws, None), BF16)
    assert (got[0, :5] == 0).all() and got[1].isnan().all() and got[2:, :5].isfinite().all()


def test_product_of_no_token():
    assert check_product(product_problem(0, 64, 24)).shape == (0, 24)
    assert check_product(product_problem(0, 64, 24, BF16)).shape == (0, 24)


def test_product_offsets_past_32_bits():
    # a token's and a channel's rows 2^27 bytes apart: the 40th starts behind 2^32
    pool = torch.zeros((41 << 27) + 128, dtype=torch.int8, device=DEV)
    x, xs, w, ws, _ = product_problem(40, 96, 40)
    for tokens, far_w in ((40, False), (40, True), (70, True)):
        if tokens == 70:
            x, xs, w, ws, _ = product_problem(70, 96, 40)
        far = pool.as_strided((40, 96), (1 << 27, 1))
        far.copy_(on(w if far_w else x))
        got = K.integer_product(on(x) if far_w else far, far if far_w else on(w), on(ws), x_scale=on(xs))
        R.check_product(got, *R.product(x.numpy(), xs.numpy(), w.numpy(), ws.numpy(), None), BF16)


# ---------------------------------------------------------------- linear attention


def linear(p, ragged=True, **kw):
    note(f"linear new={p.new[:8]} heads={p.heads}/{p.kv_heads} dim={p.dim} {p.q.dtype}")
    args = p.args(ragged)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = K.linear_attention(*args, status=status, **kw)
    torch.cuda.synchronize()
    return out, args[3], int(status)


def check_linear(p, ragged=True, **kw):
    out, state, bits = linear(p, ragged, **kw)
    assert bits == 0
    R.check_linear(out, state, p)


TYPES = pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
DIMS = pytest.mark.parametrize("dim", [64, 128])


@TYPES
@DIMS
@pytest.mark.parametrize("ragged", [False, True], ids=["one", "ragged"])
@pytest.mark.parametrize("requests", [1, 5, 70])
def test_linear_single_tokens(dtype, dim, ragged, requests):
    check_linear(R.Linear([1] * requests, dim=dim, dtype=dtype), ragged)


@TYPES
@DIMS
def test_linear_ragged_requests(dtype, dim):
    new = [3, 0, 64, 1, 65, 130, 0, 16, 17, 1, 15, 2]
    # some begin with nothing, some share a state, one is not kept
    p = R.Linear(new, heads=6, kv_heads=3, dim=dim, dtype=dtype, read=[-1, 4, 4, 4, -1, 7, 2, 3, 3, 9, 9, -1])
    p.write[5] = -1
    check_linear(p)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 96, 127, 128, 129, 191,
                               192, 193, 255, 256, 257, 511, 512, 513, 700])
@TYPES
def test_linear_lengths(n, dtype):
    check_linear(R.Linear([n], heads=2, kv_heads=2, dim=64 if n % 2 else 128, dtype=dtype))


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (8, 1), (15, 5), (7, 7), (64, 32)])
def test_linear_head_layouts(heads, kv):
    check_linear(R.Linear([1, 40, 100], heads=heads, kv_heads=kv))
    check_linear(R.Linear([1, 1, 1], heads=heads, kv_heads=kv), False)


@pytest.mark.parametrize("decay", [0.0, -INF, -1e30, -200.0, -20.0, -1e-6])
@TYPES
def test_linear_decays(decay, dtype):
    check_linear(R.Linear([150, 1, 64], kv_heads=2, decay=[decay, -0.03], dtype=dtype))


@TYPES
def test_linear_many_requests(dtype):
    # more than go without a plan: singles, drafts and prompts among them
    p = R.Linear([1, 0, 2, 4, 5, 1, 1, 20] * 34, heads=2, kv_heads=1, dtype=dtype, read=[i % 7 for i in range(272)],
                 decay=[-0.1])
    check_linear(p)


@TYPES
@DIMS
@pytest.mark.parametrize("requests", [30, 80])
def test_linear_short_requests(dtype, dim, requests):
    # 240 and 640 states: all that the device takes at once, and more; lengths on both sides of a few
    check_linear(R.Linear([i % 11 for i in range(requests)], heads=8, kv_heads=8, dim=dim, dtype=dtype))


@TYPES
@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in place"])
@pytest.mark.parametrize("new, heads, kv, dim", [
    ([65], 8, 2, 128), ([64], 8, 2, 128), ([200], 8, 2, 64), ([129], 4, 4, 64), ([577], 4, 4, 128),
    ([1153], 16, 4, 128), ([70] * 19, 4, 1, 64), ([129, 0, 300], 6, 2, 128),
    ([1] * 30 + [300] + [2, 0] * 15, 4, 2, 128), ([1, 640, 64, 128], 6, 3, 64)])
def test_linear_a_few_longer_requests(new, heads, kv, dim, in_place, dtype):
    # that are cut finely, as the device would be half empty
    n = len(new)
    slots = dict(read=list(range(n)), write=list(range(n))) if in_place else {}
    check_linear(R.Linear(new, heads=heads, kv_heads=kv, dim=dim, dtype=dtype, **slots))


@TYPES
def test_linear_cut_requests_in_place(dtype):
    # cut ones whose last segment writes what the first begins with, teams of query heads beside each other
    check_linear(R.Linear([700, 300, 0, 5], heads=6, kv_heads=2, dtype=dtype, write=None))
    check_linear(R.Linear([130, 64], heads=8, kv_heads=2, dim=128, dtype=dtype, write=None))
    check_linear(R.Linear([130, 64], heads=8, kv_heads=2, dim=128, dtype=dtype))


@TYPES
def test_linear_long_prompts(dtype):
    check_linear(R.Linear([2500, 0, 1300], heads=2, kv_heads=1, dim=64, dtype=dtype))
    check_linear(R.Linear([1800], heads=1, kv_heads=1, dim=128, dtype=dtype, read=[-1]))


def test_linear_in_place_and_not_kept():
    p = R.Linear([70, 1, 0, 3], write=None)
    check_linear(p)
    p = R.Linear([1, 1, 1], read=[2, 0, -1], write=[2, -1, 1])
    check_linear(p, False)
    # begins with nothing and is not kept: no state is touched
    p = R.Linear([80, 2], read=[-1, -1], write=None)
    check_linear(p)


def test_linear_in_pieces_is_the_whole():
    whole = R.Linear([300], heads=2, kv_heads=2, read=[1], write=[0])
    w = whole.want()
    args = whole.args()
    outs, at = [], 0
    for n in (1, 64, 100, 7, 128):
        cut = [x[at:at + n] for x in args[:3]]
        outs.append(K.linear_attention(*cut, args[3], args[4], whole.i32([1] if at == 0 else [0]), whole.i32([0]),
                                       whole.i32([0, n])))
        at += n
    R.check_linear(torch.cat(outs), args[3], whole, w)


@TYPES
def test_linear_what_is_later_or_another_request_has_no_influence(dtype):
    for new in ([70, 40, 1, 3, 130], [1, 1, 1, 1, 1], [4, 2, 4, 1, 3]):
        p = R.Linear(new, heads=2, kv_heads=1, dtype=dtype)
        want = p.want()
        out, state, _ = linear(p)
        start = p.row_start.tolist()
        for value in (NAN, INF):
            q = R.Linear(new, heads=2, kv_heads=1, dtype=dtype)
            # the last token of request 0, and all of request 3: rows before and of others stay as they were
            q.k[start[1] - 1], q.v[start[1] - 1], q.q[start[1] - 1] = value, value, value
            q.v[start[3]:start[4]] = value
            o, s, _ = linear(q)
            kept = torch.ones(sum(new), dtype=torch.bool)
            kept[start[1] - 1] = False
            kept[start[3]:start[4]] = False
            assert torch.equal(o.cpu()[kept], out.cpu()[kept])
            assert not o.cpu()[~kept].isfinite().all()
            slots = [i for i in range(len(state)) if i not in (p.write[0], p.write[3])]
            assert torch.equal(s[slots], state[slots])
            assert not s[[p.write[0], p.write[3]]].isfinite().all()
        R.check_linear(out, state, p, want)


def test_linear_an_infinite_value_in_the_middle_of_a_prompt():
    # rows before it are as without it; in its column all later ones follow the formula
    p = R.Linear([200], heads=1, kv_heads=1, decay=[-0.01])
    q = R.Linear([200], heads=1, kv_heads=1, decay=[-0.01])
    q.v[90, 0, 5] = INF
    (a, sa, _), (b, sb, _) = linear(p), linear(q)
    assert torch.equal(a[:90], b[:90])
    other = [i for i in range(64) if i != 5]
    w = p.want()
    off = (b[:, :, other].double().cpu().numpy() - w[0][:, :, other])
    assert (np.abs(off) <= (2.0 ** -7 * w[2][:, :, other])).all()
    assert not b[90:, 0, 5].isfinite().any()


def test_linear_strides():
    p = R.Linear([5, 70, 1], heads=6, kv_heads=2)
    args = p.args()
    tokens = sum(p.new)
    fused = torch.full((tokens, 10, 72), NAN, dtype=BF16, device=DEV)
    for part, x in zip(fused[:, :, :64].split([6, 2, 2], 1), args[:3]):
        part.copy_(x)
    q, k, v = fused[:, :, :64].split([6, 2, 2], 1)
    pool = torch.full((len(p.state), 3, 64 * 64 + 4), 5.0, device=DEV)
    state = pool[:, :2, :64 * 64].unflatten(2, (64, 64))
    state.copy_(args[3])
    first = torch.full((6, tokens, 64), NAN, dtype=BF16, device=DEV)
    out = K.linear_attention(q, k, v, state, *args[4:], out=first.transpose(0, 1))
    R.check_linear(out, state, p)
    assert (pool[:, 2] == 5).all() and (pool[:, :, 64 * 64:] == 5).all()


def test_linear_tokens_behind_the_last_request_are_left():
    p = R.Linear([5, 70, 9])
    args = p.args()
    args[5:8] = [p.i32(p.read[:2]), p.i32(p.write[:2]), p.i32([0, 5, 75])]
    out = torch.full_like(args[0], 7.0)
    K.linear_attention(*args, out=out)
    w = p.want()
    assert (out[75:] == 7).all()
    p.new, p.write[2] = p.new[:2], -1
    w = [w[0][:75], p.want()[1], w[2][:75], p.want()[3]]
    R.check_linear(out[:75], args[3], p, w)


# few requests, as many as are planned for, long ones that are cut
@pytest.mark.parametrize("new", [[2, 1, 3], [1] * 300 + [2, 1, 3], [200, 1, 300]], ids=["few", "many", "long"])
@pytest.mark.parametrize("at,by", [(-2, -400), (-3, -1000), (-1, 1), (1, -1)])
def test_linear_invalid_lengths(new, at, by):
    p = R.Linear(new)
    args = p.args()
    rows = p.row_start.clone()
    rows[at] += by
    if at == 1:
        rows[0] = -1
    args[7] = rows.to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = K.linear_attention(*args, status=status)
    assert int(status) == 1 and out.isnan().all() and torch.equal(args[3].cpu(), p.state)


@pytest.mark.parametrize("which", ["read", "write"])
@pytest.mark.parametrize("slot", [-2, 8, 1 << 30])
@pytest.mark.parametrize("new", [[2, 1, 70], [1, 1, 1], [1, 70, 5], [40, 700, 3]])
def test_linear_invalid_slots(which, slot, new):
    p = R.Linear(new)
    want = p.want()
    getattr(p, which)[1] = slot
    for ragged in ([True, False] if new == [1, 1, 1] else [True]):
        out, state, bits = linear(p, ragged)
        a, b = new[0], new[0] + new[1]
        assert bits == 512 and out[a:b].isnan().all()
        touched = [p.write[0], p.write[2]]
        rest = [i for i in range(8) if i not in touched]
        assert torch.equal(state[rest].cpu(), p.state[rest])
        kept = [i for i in range(sum(new)) if not a <= i < b]
        w = [want[0][kept], want[1][touched], want[2][kept], want[3][touched]]
        R.check_linear(out[kept], state[touched], p, w)


def test_linear_empty_batches():
    p = R.Linear([0, 0], read=[0, -1], write=[1, 2])
    out, state, bits = linear(p)  # no token: states are copied, or cleared
    assert bits == 0 and out.shape[0] == 0
    assert torch.equal(state[1].cpu(), p.state[0]) and (state[2] == 0).all()
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    args = p.args()
    out = K.linear_attention(*args[:5], none, none, torch.zeros(1, dtype=torch.int32, device=DEV))
    assert out.shape[0] == 0


def test_linear_the_same_call_gives_the_same_bits():
    p = R.Linear([900, 1, 64], heads=4, kv_heads=2, dim=128)
    a, b = linear(p), linear(p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_linear_states_past_32_bits():
    # slots behind 2^31 values, and 2^32 bytes
    n = (1 << 33) // (8 * 128 * 128 * 4) + 6
    pool = torch.zeros((n, 8, 128, 128), device=DEV)
    p = R.Linear([1, 70], heads=8, kv_heads=8, dim=128, read=[0, 1], write=[2, 3])
    want = p.want()
    args = p.args()
    pool[n - 4:] = args[3][:4]
    out = K.linear_attention(*args[:3], pool, args[4], args[5] + n - 4, args[6] + n - 4, args[7])
    R.check_linear(out, pool[n - 4:], p, [want[0], want[1][:4], want[2], want[3][:4]])


# ---------------------------------------------------------------- refusals of tensors


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def far_rows(rows, *rest, dtype=BF16):
    """So many rows of one row's memory."""
    return z(1, *rest, dtype=dtype).expand(rows, *rest)


I32, I8 = torch.int32, torch.int8
NORMS = {
    "one dimension": lambda: dict(x=z(8)),
    "type": lambda: dict(x=z(4, 8, dtype=F32)),
    "columns": lambda: dict(x=z(8, 4).t()),
    "2^31 rows": lambda: dict(x=far_rows(1 << 31, 8)),
    "eps": lambda: dict(x=z(4, 8), eps=0.0),
    "weight": lambda: dict(x=z(4, 8), before=z(9)),
    "weight's type": lambda: dict(x=z(4, 8), before=z(8, dtype=F32)),
    "weight's place": lambda: dict(x=z(4, 8), before=torch.zeros(8, dtype=BF16)),
    "gate": lambda: dict(x=z(4, 8), gate=z(3, 8)),
    "activation": lambda: dict(x=z(4, 8), gate=z(4, 8), activation="tanh"),
    "residual": lambda: dict(x=z(4, 8), residual=z(4, 8, dtype=FP16)),
    "in place of nothing": lambda: dict(x=z(4, 8), in_place=True),
    "overlapping residual": lambda: dict(x=z(4, 8), residual=far_rows(4, 8), in_place=True),
    "overlapping result": lambda: dict(x=z(4, 8), out=far_rows(4, 8)),
    "result's type": lambda: dict(x=z(4, 8), out=z(4, 8), int8=True),
    "gradient": lambda: dict(x=z(4, 8).requires_grad_()),
}
PRODUCTS = {
    "no scale": lambda: ((z(4, 32, dtype=I8), z(8, 32, dtype=I8), z(8, dtype=F32)), {}),
    "scale of 16 bits": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(8, dtype=F32)), dict(x_scale=z(4, dtype=F32))),
    "weight's type": lambda: ((z(4, 32), z(8, 32), z(8, dtype=F32)), {}),
    "weight's rows": lambda: ((z(4, 32), z(8, 48, dtype=I8), z(8, dtype=F32)), {}),
    "weight_scale": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(7, dtype=F32)), {}),
    "bias": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(8, dtype=F32)), dict(bias=z(8))),
    "dim": lambda: ((z(4, 24), z(8, 24, dtype=I8), z(8, dtype=F32)), {}),
    "stride": lambda: ((z(4, 32), z(8, 40, dtype=I8)[:, :32], z(8, dtype=F32)), {}),
    "2^31 rows": lambda: ((far_rows(1 << 31, 32), z(8, 32, dtype=I8), z(8, dtype=F32)), dict(out=z(1, 8))),
    "result's type": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(8, dtype=F32)), dict(dtype=torch.float64)),
    "overlapping result": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(8, dtype=F32)), dict(out=far_rows(4, 8))),
    "gradient": lambda: ((z(4, 32), z(8, 32, dtype=I8), z(8, dtype=F32).requires_grad_()), {}),
}


def linear_args(**change):
    a = dict(q=z(3, 4, 64), k=z(3, 2, 64), v=z(3, 2, 64), state=z(5, 2, 64, 64, dtype=F32), log_decay=z(2, dtype=F32),
             read=z(3, dtype=I32))
    a.update(change)
    return a


LINEARS = {
    "type": lambda: linear_args(q=z(3, 4, 64, dtype=F32)),
    "2^31 rows": lambda: linear_args(q=far_rows(1 << 31, 4, 64)),
    "keys": lambda: linear_args(k=z(2, 2, 64)),
    "values' heads": lambda: linear_args(v=z(3, 4, 64)),
    "heads": lambda: linear_args(q=z(3, 3, 64)),
    "dim": lambda: linear_args(q=z(3, 4, 32), k=z(3, 2, 32), v=z(3, 2, 32), state=z(5, 2, 32, 32, dtype=F32)),
    "state's type": lambda: linear_args(state=z(5, 2, 64, 64)),
    "state's heads": lambda: linear_args(state=z(5, 3, 64, 64, dtype=F32)),
    "transposed states": lambda: linear_args(state=z(5, 2, 64, 64, dtype=F32).transpose(2, 3)),
    "overlapping slots": lambda: linear_args(state=far_rows(5, 2, 64, 64, dtype=F32)),
    "overlapping states": lambda: linear_args(
        state=z(6, 64, 64, dtype=F32).as_strided((5, 2, 64, 64), (4096, 4096, 64, 1))),
    "log_decay": lambda: linear_args(log_decay=z(4, dtype=F32)),
    "read": lambda: linear_args(read=z(2, dtype=I32)),
    "read's type": lambda: linear_args(read=z(3, dtype=torch.int64)),
    "write": lambda: linear_args(write=z(2, dtype=I32)),
    "row_start": lambda: linear_args(row_start=z(3, dtype=I32)),
    "columns": lambda: linear_args(q=z(3, 64, 4).transpose(1, 2)),
    "result": lambda: linear_args(out=z(3, 4, 64, dtype=FP16)),
    "one head's result for all": lambda: linear_args(out=z(3, 1, 64).expand(3, 4, 64)),
    "one token's result for all": lambda: linear_args(out=far_rows(3, 4, 64)),
    "scale": lambda: linear_args(scale=INF),
    "gradient": lambda: linear_args(state=z(5, 2, 64, 64, dtype=F32).requires_grad_()),
}


@pytest.mark.parametrize("what", NORMS)
def test_norm_refuses(what):
    kw = NORMS[what]()
    with pytest.raises(K.KvrError):
        K.block_norm(kw.pop("x"), **kw)


@pytest.mark.parametrize("what", PRODUCTS)
def test_product_refuses(what):
    args, kw = PRODUCTS[what]()
    with pytest.raises(K.KvrError):
        K.integer_product(*args, **kw)


@pytest.mark.parametrize("what", LINEARS)
def test_linear_refuses(what):
    with pytest.raises(K.KvrError):
        K.linear_attention(**LINEARS[what]())


def test_heads_first_results_and_states():
    # (strides in the other order are no overlap)
    p = R.Linear([70, 1], heads=4, kv_heads=2, dim=64)
    args = list(p.args())
    args[3] = args[3].transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty((4, 71, 64), dtype=BF16, device=DEV).transpose(0, 1)
    K.linear_attention(*args, out=out)
    R.check_linear(out, args[3], p)


def test_two_streams_at_once():
    p = [R.Linear([900, 3, 200], heads=4, kv_heads=2, dim=128, seed=i) for i in range(2)]
    x, xs, w, ws, _ = product_problem(300, 512, 700)
    args, sides = [q.args() for q in p], [torch.cuda.Stream() for _ in p]
    data = [on(t) for t in (x, w, ws, xs)]
    torch.cuda.synchronize()
    got = []
    for a, side in zip(args, sides):
        with torch.cuda.stream(side):
            product = [K.integer_product(*data[:3], x_scale=data[3]) for _ in range(3)]
            got.append((K.linear_attention(*a), product))
    torch.cuda.synchronize()
    for q, a, (out, product) in zip(p, args, got):
        R.check_linear(out, a[3], q)
        for y in product:
            R.check_product(y, *R.product(x.numpy(), xs.numpy(), w.numpy(), ws.numpy(), None), BF16)


# ---------------------------------------------------------------- together


class Chain:
    """A layer of a worker with linear attention, from residual to residual."""

    def __init__(self, new, heads=4, dim=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.dim, self.width = heads, dim, heads * dim
        width = self.width

        def weight(n, k):
            return torch.randint(-127, 128, (n, k), generator=g, dtype=torch.int8), \
                torch.rand(n, generator=g) / (64 * k ** 0.5) + 1e-4

        self.p = R.Linear(new, heads=heads, kv_heads=heads, dim=dim, seed=seed)
        self.residual = torch.randn((sum(new), width), generator=g).to(BF16)
        self.up, self.down = weight(4 * width, width), weight(width, width)
        self.w = [(1 + 0.2 * torch.randn(width, generator=g)).to(BF16) for _ in range(3)]

    def tensors(self):
        a = self.p.args()
        return dict(residual=on(self.residual), up=[on(x) for x in self.up], down=[on(x) for x in self.down],
                    w=[on(x) for x in self.w], state=a[3], decay=a[4], read=a[5], write=a[6], rows=a[7])

    def run(self, t):
        n = K.block_norm(t["residual"], before=t["w"][0], int8=True)
        x = K.integer_product(n.out, *t["up"], x_scale=n.scale)
        q, k, v, gate = (x[:, i * self.width:(i + 1) * self.width] for i in range(4))
        split = [y.unflatten(1, (self.heads, self.dim)) for y in (q, k, v)]
        o = K.linear_attention(*split, t["state"], t["decay"], t["read"], t["write"], t["rows"])
        n = K.block_norm(o.flatten(1), after=t["w"][1], gate=gate, activation="silu", int8=True)
        y = K.integer_product(n.out, *t["down"], x_scale=n.scale)
        n = K.block_norm(y, residual=t["residual"], residual_scale=0.5, before=t["w"][2])
        return n.out, n.residual, t["state"], x, o, y


def test_a_layer_from_residual_to_residual():
    c = Chain([1, 70, 5, 130])
    t = c.tensors()
    out, residual, state, x, o, y = (z.cpu() for z in c.run(t))
    # each step against its definition on what the one before gave
    n = R.norm(c.residual, before=c.w[0])[0]
    xs = np.abs(n).max(1) / 127
    want = R.product(np.rint(n / xs[:, None]), xs, c.up[0].numpy(), c.up[1].numpy(), None)[0]
    # a value next to a border may take the other integer: one step of the scale, times a weight
    step = (xs[:, None] * 127 * c.up[1].numpy()) * 4
    assert (np.abs(x.double().numpy() - want) <= 2.0 ** -8 * np.abs(want) + step).all()
    p = c.p
    p.q, p.k, p.v = (x[:, i * c.width:(i + 1) * c.width].unflatten(1, (c.heads, c.dim)) for i in range(3))
    R.check_linear(o, state, p)
    w = R.norm(y, residual=c.residual, residual_scale=0.5, before=c.w[2])
    R.check_norm(out, w[0], w[2], BF16)
    R.check_norm(residual, w[1], w[3], BF16)


def test_captured_layers_replay():
    chains = [Chain([1, 1, 1], seed=1), Chain([64, 3, 200], seed=2)]
    tensors = [c.tensors() for c in chains]
    eager = [c.run(c.tensors()) for c in chains]
    kept = [t["state"].clone() for t in tensors]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for c, t in zip(chains, tensors):
            c.run(t)  # what is set once a process
    side.synchronize()
    graphs, outs = [], []
    for c, t in zip(chains, tensors):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.run(t))
        graphs.append(g)
    for _ in range(3):
        for t, s in zip(tensors, kept):
            t["state"].copy_(s)
        for g in graphs:
            g.replay()
        again = chains[1].run(chains[1].tensors())  # the program's own work between the replays
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            assert all(torch.equal(a, b) for a, b in zip(o, e))
        assert all(torch.equal(a, b) for a, b in zip(again, eager[1]))


def test_the_example_runs():
    import os
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    try:
        import state_worker
        worst = state_worker.main(DEV)
    finally:
        sys.path.remove(os.path.join(root, "examples"))
    # results are rounded once (2^-8 of themselves), and so are two factors of each of their parts at most; parts
    # that cancel may be some times larger than the largest result
    assert worst < 8 * 2.0 ** -8
