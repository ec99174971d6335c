"""The serving operators on the GPU at the edges of their number ranges and
rules: wide strides, NaN, sizes around the forms of the plan."""
import numpy as np
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


NAN_TYPES = [(BF16, None), (FP16, None), (BF16, FP8)]
NAN_IDS = ["bf16", "fp16", "bf16-fp8"]


def put_nan(cache, table, t, head, element):
    """NaN in one element of a token of the cache."""
    page = cache.shape[1]
    at = (int(table[t // page]), t % page, head, element)
    if cache.dtype == FP8:
        cache.view(torch.uint8)[at] = 0x7f
    else:
        cache[at] = float("nan")


def check_beside_nan(out, lse, p):
    """NaN exactly where the definition has it, in the result and in lse; the rest as everywhere."""
    ref, size, ref_lse = on_device(p)
    out, lse = out.cpu(), lse.cpu()
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    assert torch.equal(torch.isnan(lse), torch.isnan(ref_lse))
    bad, bad_lse = torch.isnan(ref), torch.isnan(ref_lse)
    R.check(out.masked_fill(bad, 0.0), lse.masked_fill(bad_lse, 0.0), p,
            [ref.masked_fill(bad, 0.0), size.masked_fill(bad, 0.0), ref_lse.masked_fill(bad_lse, 0.0)])
    return bad, bad_lse


# single tokens: 32, 40 (one wave has no second tile), 128 and 20,011 keys (split); behind a prefix that is shared by a
# group; 200 rows of one request
@pytest.mark.parametrize("new,own,sizes,prefix", [([1], [32], (), ()), ([1], [40], (), ()), ([1], [128], (), ()),
                                                  ([1], [20011], (), ()), ([1] * 24, [33] * 24, [24], [2100]),
                                                  ([50], [90], (), ())],
                         ids=["32", "40", "128", "20011", "group", "rows"])
@pytest.mark.parametrize("types", NAN_TYPES, ids=NAN_IDS)
@pytest.mark.parametrize("dim", [64, 256])
def test_a_nan_key_makes_result_and_lse_nan(new, own, sizes, prefix, types, dim):
    for t in {0, 31, own[0] - new[0] - 1, own[0] // 2 - 20 if own[0] > 100 else 5}:
        p = R.Problem(new, own, sizes, prefix, heads=8, kv_heads=2, dim=dim, dtype=types[0], cache=types[1])
        put_nan(p.k_cache, p.table[0], t, 1, 7)
        out, lse = attend(p)
        bad, bad_lse = check_beside_nan(out, lse, p)
        assert bad[:new[0], 4:].all() and bad_lse[:new[0], 4:].all() and int(bad_lse.sum()) == 4 * new[0]


def test_a_nan_key_of_a_shared_prefix_reaches_its_whole_group():
    for prefix in (40, 2100):
        p = R.Problem([1] * 24, [33] * 24, [20, 4], [prefix, 50], heads=4, kv_heads=2, dim=128)
        put_nan(p.k_cache, p.prefix_table[0], prefix - 3, 0, 0)
        out, lse = attend(p)
        bad, bad_lse = check_beside_nan(out, lse, p)
        assert bad_lse[:20, :2].all() and int(bad_lse.sum()) == 40


def test_a_nan_query_makes_its_result_and_lse_nan():
    for own in (1, 40, 3000):
        p = R.Problem([1, 1, 30], [own, 9, 60], [2, 1], [70, 5], heads=4, kv_heads=2, dim=128)
        p.q[0, 2, 5] = p.q[11, 0, 0] = float("nan")
        out, lse = attend(p)
        _, bad_lse = check_beside_nan(out, lse, p)
        assert bad_lse[0, 2] and bad_lse[11, 0] and int(bad_lse.sum()) == 2


def test_a_nan_value_leaves_lse():
    for own in (40, 3000):
        p = R.Problem([1, 3], [own, 90], heads=4, kv_heads=2, dim=128)
        put_nan(p.v_cache, p.table[0], 20, 1, 9)
        put_nan(p.v_cache, p.table[1], 50, 0, 100)
        bad, bad_lse = check_beside_nan(*attend(p), p)
        assert bad[0, 2:, 9].all() and bad[1:, :2, 100].all() and int(bad.sum()) == 8 and not bad_lse.any()


@pytest.mark.parametrize("own,heads", [(40, 4), (5000, 4), (300, 80)], ids=["few", "split", "rows"])
@pytest.mark.parametrize("cache", [None, FP8], ids=["16-bit", "8-bit"])
@pytest.mark.parametrize("page", [-1, 1 << 30])
def test_a_page_outside_the_cache_makes_result_and_lse_nan(own, heads, cache, page):
    p = R.Problem([1, 1, 1], [own] * 3, [2, 1], [40, 5], heads=heads, kv_heads=2, dim=128, cache=cache)
    want = on_device(p)
    for at in {0, (own - 1) // 16, own // 32}:
        q = R.Problem([1, 1, 1], [own] * 3, [2, 1], [40, 5], heads=heads, kv_heads=2, dim=128, cache=cache)
        q.table[1, at] = page
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        out, lse = attend(q, status=status)
        assert int(status) == 512
        assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
        for i in (0, 2):
            R.check(out[i:i + 1], lse[i:i + 1], p, [x[i:i + 1] for x in want])


@pytest.mark.parametrize("tokens", [(1 << 31) - 1, (1 << 31) - 256, (1 << 31) - 257, 1 << 30])
def test_tables_with_room_for_the_most_tokens(tokens):
    # an upper bound of 2^31 tokens for a batch of few, which gives back more pages than a block of threads has
    rows = 3000
    rng = np.random.default_rng(11)
    held = np.full(rows, 2, np.int32)
    delta = np.where(np.arange(rows) % 5 == 4, 3, -2).astype(np.int32)
    pool = 2 * rows + 2000
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((rows, 5), -1, np.int32)
    table[:, :2] = order[:2 * rows].reshape(rows, 2)
    ring, state = np.roll(order, -2 * rows), np.array([0, 2000, 0])
    new = int(np.maximum(delta, 0).sum())
    want, bits = R.tables(held, delta, table, ring, state, 1, new, held)
    assert not bits
    on = [torch.from_numpy(x.copy()).to(DEV) for x in (held, delta, table, ring, state)]
    note(f"tables rows={rows} tokens={tokens}")
    r = K.block_tables(*on, 1, tokens, base=on[0])
    got = dict(table=on[2], ring=on[3], held=r.held, state=r.state, row_start=r.row_start, slots=r.slots[:new],
               positions=r.positions[:new])
    for k, v in got.items():
        np.testing.assert_array_equal(v.cpu().numpy(), want[k], err_msg=k)
    for x in (r.slots, r.positions):
        assert x.shape == (tokens,)
        for a in range(new, tokens, 1 << 28):
            assert int((x[a:a + (1 << 28)] != -1).sum()) == 0


@pytest.mark.parametrize("rows", [9, 1500])
@pytest.mark.parametrize("in_place", [False, True])
def test_positions_from_held_itself(rows, in_place):
    # base is held: its values before the call, also where the call updates them
    rng = np.random.default_rng(rows)
    held = rng.integers(0, 9, rows).astype(np.int32)
    delta = rng.integers(0, 4, rows).astype(np.int32)
    table = rng.permutation(rows * 12).astype(np.int32).reshape(rows, 12)
    ring, state = np.arange(rows * 12, dtype=np.int32), np.array([0, rows * 12, 0])
    want, bits = R.tables(held, delta, table, ring, state, 1, int(delta.sum()), held)
    assert not bits
    on = [torch.from_numpy(x.copy()).to(DEV) for x in (held, delta, table, ring, state)]
    r = K.block_tables(*on, 1, int(delta.sum()), base=on[0], in_place=in_place)
    np.testing.assert_array_equal(r.positions.cpu().numpy(), want["positions"])
    np.testing.assert_array_equal(r.held.cpu().numpy(), want["held"])
    np.testing.assert_array_equal(r.slots.cpu().numpy(), want["slots"])


MOST = (1 << 31) - 1024  # tokens of a request or of a prefix


@pytest.mark.parametrize("length,prefix", [((1 << 31) - 1, 5), (MOST + 1, 5), (9, MOST + 1), (9, (1 << 31) - 1)])
def test_lengths_past_the_range_of_keys_are_reported(length, prefix):
    p = R.Problem([1, 1], [9, 9], [2], [5], page=1024)
    p.table = p.table[:, :1].repeat(1, 1 << 21)
    p.prefix_table = p.prefix_table[:, :1].repeat(1, 1 << 21)
    p.length[1], p.prefix_length[0] = length, prefix
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = attend(p, status=status)
    assert int(status) == 1 and torch.isnan(out).all() and torch.isnan(lse).all()


def test_the_most_keys():
    # one page of 1,024 tokens, named 2^21 - 1 times: the attention over that page, and its sum as often
    p = R.Problem([1], [1024], heads=2, kv_heads=1, dim=64, page=1024)
    ref, size, ref_lse = p.expect()
    p.table = p.table[:, :1].repeat(1, (1 << 21) - 1)
    p.length[0] = MOST
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = attend(p, status=status)
    assert int(status) == 0
    # 512 workgroups at most, of four waves, two lanes to a row: 2^31 / 2^12 = 2^19 terms that a lane adds one by one
    # in 32 bits, each rounding at most 2^-24 of the sum; in l and in o
    err = (out.double().cpu() - ref).abs()
    assert (err <= 2 * 2.0 ** -5 * size + 2.0 ** -8 * (ref.abs() + size)).all(), float(err.max())
    assert ((lse.double().cpu() - ref_lse - np.log(2.0 ** 21 - 1)).abs() <= 2.0 ** -5 + 1e-3).all()


def odd_where_one(x):
    """The tensor with a stride of 1 in each dimension of one (but the last): a stride that no element follows."""
    return torch.as_strided(x, x.shape, [1 if n == 1 else s for n, s in zip(x.shape[:-1], x.stride())] + [1])


@pytest.mark.parametrize("cache", [None, FP8], ids=["16-bit", "8-bit"])
@pytest.mark.parametrize("tokens,pages,page,heads", [(1, 20, 16, 4), (9, 1, 1024, 4), (1, 40, 1, 1), (1, 1, 64, 1),
                                                     (7, 40, 1, 2), (5, 30, 16, 1)])
def test_strides_that_nothing_follows(tokens, pages, page, heads, cache):
    # one token, one page, pages of one token, one head: any stride does, in the store and in the attention
    g = torch.Generator().manual_seed(tokens)
    k, v, q = (torch.randn((tokens, heads, 64), generator=g).to(BF16).to(DEV) for _ in range(3))
    caches = [torch.randn((pages, page, heads, 64), generator=g).to(cache or BF16).to(DEV) for _ in range(2)]
    slots = torch.randperm(pages * page, generator=g)[:tokens].int().to(DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    length = torch.tensor([min(pages * page, 30)], dtype=torch.int32, device=DEV)
    start = torch.tensor([0, tokens], dtype=torch.int32, device=DEV)

    def both(f):
        copies = [f(c.view(torch.uint8).clone().view(c.dtype)) for c in caches]
        K.cache_store(f(k), f(v), *copies, slots)
        out = torch.full_like(q, 7.0)
        K.shared_attention(f(q), *copies, start, table, length, out=f(out))
        return out, [c.view(torch.uint8).cpu() for c in copies]

    want, stored = both(lambda x: x)
    got, odd = both(odd_where_one)
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(odd, stored))
    assert torch.isfinite(want).all()


def test_a_call_that_would_need_a_gradient_is_refused():
    p = R.Problem([1, 3], [20, 30], heads=2, kv_heads=2, dim=64, cache=FP8)
    args, kw = p.args(), p.kwargs()
    want = K.shared_attention(*args, **kw)
    k = torch.randn((4, 2, 64), device=DEV).to(BF16)
    slots = torch.arange(4, dtype=torch.int32, device=DEV)
    scales = {n: kw[n] for n in ("k_scale", "v_scale")}

    def attention(name, x):
        return K.shared_attention(*([x] + args[1:] if name == "q" else args), **dict(kw, **{name: x} if name != "q" else {}))

    def store(name, x):
        kv = {"k": k, "v": k}
        if name in kv:
            kv[name] = x
        K.cache_store(kv["k"], kv["v"], args[1], args[2], slots, **dict(scales, **{name: x} if name in scales else {}))

    for call, name, x in ((attention, "q", args[0]), (attention, "v_scale", kw["v_scale"]),
                          (attention, "out", torch.empty_like(args[0])), (store, "k", k), (store, "v", k),
                          (store, "k_scale", kw["k_scale"])):
        x = x.clone().requires_grad_()
        before = [c.view(torch.uint8).clone() for c in args[1:3]]
        with pytest.raises(K.KvrError, match="no gradient") as ei:
            call(name, x)
        assert ei.value.status == K.KVR_EINVAL
        assert all(torch.equal(c.view(torch.uint8), b) for c, b in zip(args[1:3], before))
        for off in (torch.no_grad(), torch.inference_mode()):
            with off:
                call(name, x.detach() if name == "out" else x)
        call(name, x.detach())
    q = args[0].clone().requires_grad_()
    with torch.no_grad():
        K.cache_store(k, k, args[1], args[2], torch.full_like(slots, -1), **scales)
        assert torch.equal(K.shared_attention(q, *args[1:], **kw), K.shared_attention(*args, **kw))
    assert not want.requires_grad


@pytest.mark.parametrize("new,own,sizes,prefix,heads,kv", [
    ([257] * 9, [300] * 9, [9], [3000], 1, 1),          # the most rows a request that share a prefix
    ([129] * 40, [129 + i for i in range(40)], [30, 10], [2000, 900], 1, 1),
    ([33] * 64, [40] * 64, [64], [5000], 2, 2),
    ([1] * 300, [1 + 61 * i % 900 for i in range(300)], [200, 100], [700, 40], 8, 1),
    ([1], [30000], (), (), 64, 1),                      # split into as many items as there are slots
    ([1] * 3 + [700], [9000, 50, 20000, 700], (), (), 4, 4),
    ([2000], [2000], (), (), 16, 1),
], ids=["257", "129", "33", "ones", "split", "mixed", "prompt"])
@pytest.mark.parametrize("dim,cache", [(64, None), (256, None), (256, FP8)], ids=["64", "256", "256-8-bit"])
def test_nothing_is_written_behind_the_workspace(new, own, sizes, prefix, heads, kv, dim, cache, monkeypatch):
    from paper_2601_18999_amd import serve
    p = R.Problem(new, own, sizes, prefix, heads=heads, kv_heads=kv, dim=dim, cache=cache)
    call, buffers = serve.kvr_shared_attention, []

    def guarded(cache, args, ws, nbytes, stream):
        whole = torch.full((nbytes + (64 << 20),), 0xA5, dtype=torch.uint8, device=DEV)
        buffers.append((whole, nbytes))
        call(cache, args, whole.data_ptr(), nbytes, stream)

    monkeypatch.setattr(serve, "kvr_shared_attention", guarded)
    out, lse = attend(p)
    (whole, nbytes), = buffers
    assert bool((whole[nbytes:] == 0xA5).all())
    R.check(out, lse, p, on_device(p))


@pytest.mark.parametrize("in_place", [False, True])
def test_tables_without_rows_change_nothing(in_place):
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    table = torch.zeros((0, 8), dtype=torch.int32, device=DEV)
    for tokens in (0, 5):
        ring, state = K.page_ring(10, DEV)
        state[0], state[2] = 4, 128
        r = K.block_tables(none, none.clone(), table, ring, state, 16, tokens, base=none.clone(), in_place=in_place)
        assert r.held.shape == (0,) and r.row_start.tolist() == [0]
        assert r.slots.tolist() == r.positions.tolist() == [-1] * tokens
        assert r.state.tolist() == [4, 10, 128] and ring.tolist() == list(range(10))
        assert r.held.dtype == r.slots.dtype == r.positions.dtype == r.row_start.dtype == torch.int32
        assert (r.held is none and r.state is state) == in_place
    for page, tokens in ((24, 0), (0, 0), (16, -1)):
        with pytest.raises(K.KvrError):
            K.block_tables(none, none.clone(), table, ring, state, page, tokens)
    with pytest.raises(K.KvrError):
        K.block_tables(none, none.clone(), table[:, :0], ring[:0], state, 16, 0)
    with pytest.raises(K.KvrError):
        K.block_tables(none, torch.zeros(1, dtype=torch.int32, device=DEV), table, ring, state, 16, 0)


def test_attention_without_requests_writes_nothing():
    p = R.Problem([1], [20], [1], [9], heads=4, kv_heads=2, dim=64)
    q, kc, vc, rs, tb, ln, gs, pt, pl = p.args()
    for groups in ((), (gs[:1], pt[:0], pl[:0]), (torch.zeros_like(gs), pt, pl)):
        for tokens in (0, 1):
            out = torch.full_like(q[:tokens], 9.0)
            lse = torch.full((tokens, 4), 9.0, device=DEV)
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            got = K.shared_attention(q[:tokens], kc, vc, rs[:1], tb[:0], ln[:0], *groups, out=out, lse=lse,
                                     status=status)
            assert got is out and (out == 9.0).all() and (lse == 9.0).all() and int(status) == 0
            if not tokens:
                assert K.shared_attention(q[:0], kc, vc, None, tb[:0], ln[:0], *groups).shape == (0, 4, 64)
    for bad in ((q[:, :3], kc, vc, rs[:1], tb[:0], ln[:0]), (q.half(), kc, vc, rs[:1], tb[:0], ln[:0]),
                (q, kc, vc, rs, tb[:0], ln[:0]), (q, kc, vc, rs[:1], tb, ln[:0]), (q, kc, vc, None, tb[:0], ln[:0])):
        with pytest.raises(K.KvrError):
            K.shared_attention(*bad)
    # and a request again
    R.check(K.shared_attention(*p.args(), **p.kwargs()), None, p)


# the last item of the split keys, or a wave's last tile, has keys that only the last rows see
@pytest.mark.parametrize("new,own", [(64, 513), (100, 577), (128, 705), (20, 1025), (32, 65), (9, 2049)])
@pytest.mark.parametrize("dim,cache", [(64, None), (256, None), (128, FP8)], ids=["64", "256", "128-8-bit"])
def test_rows_that_see_nothing_of_an_item(new, own, dim, cache):
    p = R.Problem([new], [own], heads=1, kv_heads=1, dim=dim, cache=cache).spoil()
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("new,own,sizes,prefix", [([1, 1], [40, 9], (), ()), ([1, 1], [9000, 9], (), ()),
                                                  ([1] * 24, [33] * 24, [24], [2100]), ([90, 2], [90, 9], (), ())],
                         ids=["few", "split", "group", "rows"])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_scores_of_minus_infinity(new, own, sizes, prefix, dtype):
    # all of a request's own keys, and all keys of its prefix too or not: 0 and -inf, or the prefix alone
    for whole in ((False, True) if sizes else (True,)):
        p = R.Problem(new, own, sizes, prefix, heads=4, kv_heads=2, dim=64, dtype=dtype)
        p.q[..., 3] = 1.0
        rows = [(p.table[0], own[0])] + ([(p.prefix_table[0], prefix[0])] if whole and sizes else [])
        for row, n in rows:
            for t in range(n):
                p.k_cache[row[t // p.page], t % p.page, 1, 3] = -float("inf")
        ref, size, ref_lse = on_device(p)  # softmax of nothing but -inf is NaN
        nothing = torch.isnan(ref).any(-1)
        hidden = torch.zeros_like(nothing)
        if whole:
            hidden[:sum(new) if sizes else new[0], 2:] = True
            if sizes:
                hidden[1:] = False  # the others have their own tokens
        assert torch.equal(nothing, hidden)
        out, lse = attend(p)
        mask = nothing[..., None]
        R.check(out, lse, p, [ref.masked_fill(mask, 0.0), size.masked_fill(mask, 0.0), ref_lse])
        assert (out[nothing.to(DEV)] == 0).all() and (lse[nothing.to(DEV)] == -float("inf")).all()


def unit_room(p):
    """Units that a call has room for: what decides whether its workgroups plan for themselves."""
    rows = sum(p.new) * p.heads // p.kv_heads
    return (2 if p.sizes else 1) * (rows // 128) + len(p.new) + len(p.sizes)


# every workgroup plans for itself up to 256 units, and up to twice as many units times key heads as the device holds
# workgroups: 1,024, or 512 with heads of 256
@pytest.mark.parametrize("requests,groups,kv,dim,room", [
    (254, 0, 1, 64, 255), (255, 0, 1, 64, 256), (253, 2, 1, 64, 257), (256, 0, 1, 64, 258), (254, 1, 1, 128, 257),
    (127, 127, 1, 64, 254), (126, 127, 2, 64, 253), (127, 1, 8, 64, 128), (128, 0, 8, 128, 129), (126, 1, 8, 128, 127),
    (127, 1, 4, 256, 128), (127, 2, 4, 256, 129), (63, 1, 8, 256, 64), (64, 1, 8, 256, 65)])
@pytest.mark.parametrize("cache", [None, FP8], ids=["16-bit", "8-bit"])
def test_units_around_the_forms_of_the_plan(requests, groups, kv, dim, room, cache):
    sizes = [requests // groups] * (groups - 1) + [requests - requests // groups * (groups - 1)] if groups else []
    p = R.Problem([1] * requests, [1 + 29 * i % 300 for i in range(requests)], sizes,
                  [300 - i % 250 for i in range(groups)], heads=kv, kv_heads=kv, dim=dim, cache=cache)
    assert unit_room(p) == room
    R.check(*attend(p), p, on_device(p))
