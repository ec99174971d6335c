"""The serving operators on the GPU against plain implementations in 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2601_18999_amd as K
from gpu_helpers import note
import serve_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, FP8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def attend(p, **kw):
    note(f"attention new={p.new[:6]} own={p.own[:6]} groups={p.sizes[:6]} prefix={p.prefix[:6]} heads={p.heads}/"
         f"{p.kv_heads} dim={p.dim} page={p.page} {p.q.dtype} {p.k_cache.dtype}")
    lse = torch.full((p.q.shape[0], p.heads), 7.0, device=DEV)
    out = K.shared_attention(*p.args(), **p.kwargs(), lse=lse, **kw)
    torch.cuda.synchronize()
    return out, lse


TYPES = [(BF16, BF16), (FP16, FP16), (BF16, FP8), (FP16, FP8)]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("types", TYPES, ids=["bf16", "fp16", "bf16-fp8", "fp16-fp8"])
@pytest.mark.parametrize("page,first", [(1, True), (16, False), (256, True)])
def test_ragged_requests_of_groups(dim, types, page, first):
    # groups: a shared one of single tokens, an empty one, one without prefix, one of longer prompts; requests without
    # new tokens among them
    p = R.Problem([1, 1, 0, 3, 1, 2, 40, 0, 70], [1, 65, 9, 3, 128, 31, 40, 0, 75], [5, 0, 1, 3], [130, 50, 0, 77],
                  heads=6, kv_heads=2, dim=dim, page=page, dtype=types[0], cache=types[1], heads_first=first).spoil()
    R.check(*attend(p), p)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (8, 1), (40, 1), (15, 5), (8, 8), (200, 1)])
def test_head_layouts(heads, kv):
    p = R.Problem([1, 2, 1], [3, 80, 200], [2, 1], [67, 5], heads=heads, kv_heads=kv, dim=64)
    R.check(*attend(p), p)


@pytest.mark.parametrize("keys", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths_around_the_tiles(keys):
    p = R.Problem([1, min(keys, 33), keys if keys < 200 else 1], [keys] * 3, [1, 2], [keys, keys - 1], dim=64,
                  page=8).spoil()
    R.check(*attend(p), p)


@pytest.mark.parametrize("rows", [31, 32, 33, 64, 65, 127, 128, 129, 300])
def test_row_tiles(rows):
    # one head a key head: as many rows as new tokens
    p = R.Problem([rows, 1], [rows + 10, 5], heads=2, kv_heads=2, dim=64)
    R.check(*attend(p), p)


@pytest.mark.parametrize("types", TYPES, ids=["bf16", "fp16", "bf16-fp8", "fp16-fp8"])
def test_long_keys_are_split(types):
    p = R.Problem([1], [20011], heads=4, kv_heads=1, dim=128, page=16, dtype=types[0], cache=types[1])
    R.check(*attend(p), p)


def test_a_long_prefix_for_many():
    n = 96
    p = R.Problem([1] * n, [1 + i * 7 % 50 for i in range(n)], [n - 1, 1], [4097, 300], heads=8, kv_heads=2, dim=128)
    R.check(*attend(p), p)


def test_a_row_that_sees_nothing_gets_zero():
    # a request of own length 0 cannot have a new token: only padding rows see nothing
    p = R.Problem([0, 2], [0, 2], [1, 1], [0, 0])
    R.check(*attend(p), p)
    p = R.Problem([1, 1], [1, 1], [2], [9])
    p.k_cache[:] = -torch.inf  # every score is infinite or NaN in the definition: no claim but that it returns
    attend(p)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "fp16"])
def test_later_tokens_have_no_influence(value, types):
    # infinities and NaN in the keys and values of later tokens of the same tile
    p = R.Problem([50, 90, 1], [50, 140, 70], [3], [40], heads=4, kv_heads=2, dim=128, dtype=types[0])
    want = p.expect()
    rows = []  # the rows before the spoilt tokens
    for r, at in ((0, 30), (1, 130)):
        for c in (p.k_cache, p.v_cache):
            c[p.table[r, at // p.page], at % p.page] = value
        rows += [(sum(p.new[:r]), sum(p.new[:r]) + at - (p.own[r] - p.new[r]))]
    out, lse = attend(p)
    for a, b in rows + [(140, 141)]:
        R.check(out[a:b], lse[a:b], p, [x[a:b] for x in want])
    a = 30
    assert not torch.isfinite(out[a:50]).all(dim=2).any()


def test_an_infinite_value_is_seen_by_the_rows_behind_it():
    p = R.Problem([40], [40], heads=2, kv_heads=2, dim=64)
    want = p.expect()
    p.v_cache[p.table[0, 20 // p.page], 20 % p.page, 1, 5] = float("inf")
    out, lse = attend(p)
    out = out.cpu()
    assert (out[20:, 1, 5] == float("inf")).all()
    out[20:, 1, 5] = want[0][20:, 1, 5].to(BF16)
    R.check(out, lse, p, want)


def test_large_scores():
    p = R.Problem([5, 1], [300, 40], [2], [100], heads=4, kv_heads=2, dim=64)
    p.scale = 3.0  # scores of tens to hundreds: the maxima move, small p vanish
    ref, size, _ = p.expect()
    out, _ = attend(p)
    # scores of size up to 64 * 4 * 4 * 3 = 3072 products' total: 64 * 2^-24 * 3072 = 1.2e-2
    err = (out.double().cpu() - ref).abs()
    assert (err <= 2.0 ** -8 * (ref.abs() + size) * 1.01 + 1.3e-2 * size + 1e-7).all()


def test_strided_queries_and_results():
    p = R.Problem([3, 40], [20, 40], [2], [50], heads=6, kv_heads=2, dim=128)
    args = p.args()
    wide = torch.full((43, 3, 6, 136), 5.0, dtype=BF16, device=DEV)
    wide[:, 1, :, :128] = args[0]
    out = torch.full((6, 43, 132), 3.0, dtype=BF16, device=DEV)
    args[0] = wide[:, 1, :, :128]
    view = out[..., :128].transpose(0, 1)
    assert K.shared_attention(*args, **p.kwargs(), out=view) is view
    R.check(view, None, p)
    assert (out[..., 128:] == 3.0).all()


def test_no_row_start_is_one_token_each():
    p = R.Problem([1] * 5, [9, 1, 70, 33, 2], [3, 2], [20, 0])
    args = p.args()
    want = K.shared_attention(*args, **p.kwargs())
    args[3] = None
    assert torch.equal(K.shared_attention(*args, **p.kwargs()), want)
    R.check(want, None, p)


def test_tokens_behind_the_last_request_are_not_written():
    p = R.Problem([1, 2], [9, 2])
    args = p.args()
    args[0] = torch.cat([args[0], torch.ones_like(args[0])])
    out = torch.full_like(args[0], 9.0)
    K.shared_attention(*args, **p.kwargs(), out=out)
    R.check(out[:3], None, p)
    assert (out[3:] == 9.0).all()


def test_the_same_call_gives_the_same_bits():
    p = R.Problem([1, 5, 130, 1], [4000, 5, 900, 70], [2, 2], [700, 100], heads=8, kv_heads=2, dim=128)
    args = p.args()
    first = K.shared_attention(*args, **p.kwargs())
    for _ in range(5):
        assert torch.equal(K.shared_attention(*args, **p.kwargs()), first)


def test_another_stream():
    p = R.Problem([1, 30], [400, 30], [2], [500], heads=8, kv_heads=2, dim=128)
    args = p.args()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out = K.shared_attention(*args, **p.kwargs())
    s.synchronize()
    R.check(out, None, p)


INVALID = [("row_start", [0, 2, 1, 4]), ("row_start", [1, 1, 3, 4]), ("row_start", [0, 1, 3, 5]),
           ("length", [0, 5, 5]), ("length", [5, 5, 10000]), ("length", [-1, 5, 5]), ("group_start", [0, 4, 3]),
           ("group_start", [0, 1, 2]), ("group_start", [1, 1, 3]), ("prefix_length", [-1, 5]),
           ("prefix_length", [9999, 5])]


@pytest.mark.parametrize("name,value", INVALID, ids=[f"{n}={v}" for n, v in INVALID])
def test_invalid_lengths_are_reported(name, value):
    p = R.Problem([1, 2, 1], [5, 5, 5], [1, 2], [40, 5])
    setattr(p, name, torch.tensor(value, dtype=torch.int32))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = attend(p, status=status)
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    with pytest.raises(K.KvrError, match="lengths"):
        K.check_status("shared_attention", int(status))


@pytest.mark.parametrize("page", [-1, -5, 1 << 30])
def test_a_page_outside_the_cache_is_reported(page):
    p = R.Problem([1, 1, 1], [40, 40, 40], [2, 1], [40, 5])
    want = p.expect()
    p.table[1, 1] = page
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = attend(p, status=status)
    assert int(status) == 512
    assert torch.isnan(out[1]).all()
    for i in (0, 2):
        R.check(out[i:i + 1], lse[i:i + 1], p, [x[i:i + 1] for x in want])


def test_refusals_on_tensors():
    p = R.Problem([1, 2, 1], [5, 5, 5], [1, 2], [40, 5])
    q, kc, vc, rs, tb, ln, gs, pt, pl = p.args()
    good = [q, kc, vc, rs, tb, ln, gs, pt, pl]
    bad = [(0, q.float()), (0, q[:, :3]), (0, q[..., :32]), (0, q.transpose(1, 2)), (1, kc.half()), (1, kc[:-1]),
           (1, kc.float()), (2, vc[..., ::2]), (3, rs.long()), (3, rs[:-1]), (3, rs.cpu()), (4, tb[:-1]),
           (4, tb.long()), (4, tb.expand(3, 1)[:, :1].flip(0)[:0]), (5, ln[:-1]), (5, ln.float()), (6, None),
           (6, gs[:-1]), (7, pt[:-1]), (8, pl.long())]
    for i, x in bad:
        args = list(good)
        args[i] = x
        with pytest.raises(K.KvrError) as ei:
            K.shared_attention(*args)
        assert ei.value.status == K.KVR_EINVAL, i
    for kw in (dict(scale=0.0), dict(scale=float("nan")), dict(out=q[:2]), dict(out=q.half()), dict(lse=q),
               dict(lse=torch.zeros((2, 4), device=DEV)), dict(k_scale=torch.ones(2, device=DEV)),
               dict(status=torch.zeros(2, dtype=torch.int32, device=DEV))):
        with pytest.raises(K.KvrError):
            K.shared_attention(*good, **kw)


def test_offsets_past_32_bits():
    # a cache of 2.2 million tokens: 2.2e6 * 8 * 128 = 2.3e9 elements, 4.5e9 bytes; its last pages are used
    p = R.Problem([1, 17], [300, 40], [2], [200], heads=8, kv_heads=8, dim=128)
    pages = 2200000 // p.page
    q, kc, vc, rs, tb, ln, gs, pt, pl = p.args()
    used = kc.shape[0]
    big = torch.empty((pages, p.page, 8, 128), dtype=BF16, device=DEV)
    big[-used:] = kc
    vbig = torch.empty_like(big)
    vbig[-used:] = vc
    shift = pages - used
    out = K.shared_attention(q, big, vbig, rs, tb + shift * (tb >= 0).int(), ln, gs, pt + shift * (pt >= 0).int(), pl)
    R.check(out, None, p)
    # and the store: the last slots of the cache
    k = torch.randn((20, 8, 128), device=DEV).bfloat16()
    v = torch.randn((20, 8, 128), device=DEV).bfloat16()
    slots = torch.arange(pages * p.page - 20, pages * p.page, dtype=torch.int32, device=DEV)
    K.cache_store(k, v, big, vbig, slots)
    assert torch.equal(big.view(-1, 8, 128)[-20:], k) and torch.equal(vbig.view(-1, 8, 128)[-20:], v)


# ---------------------------------------------------------------- tables


def _run_tables(held, delta, table, ring, state, page, tokens, base, in_place=False):
    on = [torch.from_numpy(x.copy()).to(DEV) for x in (held, delta, table, ring, state)]
    b = None if base is None else torch.from_numpy(base.copy()).to(DEV)
    note(f"tables rows={len(held)} page={page} tokens={tokens}")
    r = K.block_tables(*on, page, tokens, base=b, in_place=in_place)
    torch.cuda.synchronize()
    if in_place:
        assert r.held is on[0] and r.state is on[4]
    got = dict(table=on[2], ring=on[3], held=r.held, state=r.state, row_start=r.row_start, slots=r.slots,
               positions=r.positions)
    return {k: v.cpu().numpy() for k, v in got.items()}


@pytest.mark.parametrize("rows,page,most", [(1, 1, 5), (1, 16, 700), (7, 4, 9), (64, 16, 200), (1023, 1, 6),
                                            (1025, 2, 3), (3000, 64, 40), (1, 1, 9000), (130, 1024, 3000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables_over_several_steps(rows, page, most, in_place):
    rng = np.random.default_rng(rows * 1000 + page)
    width = R.pages_of(3 * most, page)
    pool = max(4, rows * width * 2 // 3 + 2)
    table = np.full((rows, width), -1, np.int32)
    ring, state = rng.permutation(pool).astype(np.int32), np.array([5, 5 + pool, 0])
    held = np.zeros(rows, np.int32)
    base = rng.integers(0, 1000, rows).astype(np.int32)
    for step in range(6):
        grow = rng.integers(0, most + 1, rows)
        delta = np.where(rng.random(rows) < 0.3, -rng.integers(0, held + 1), grow)
        if step == 3:
            delta = -held  # all end
        delta = np.minimum(delta, width * page - held).astype(np.int32)
        if step % 2:
            delta[rng.random(rows) < 0.5] = 0
        tokens = int(np.maximum(delta, 0).sum()) + step % 3
        want, bits = R.tables(held, delta, table, ring, state, page, tokens, base if step else np.zeros_like(base))
        got = _run_tables(held, delta, table, ring, state, page, tokens, base if step else None, in_place)
        if bits:
            assert got["state"][2] == state[2] | bits
            assert (got["slots"] == -1).all() and (got["held"] == held).all() and (got["table"] == table).all()
            assert (got["ring"] == ring).all() and (got["state"][:2] == state[:2]).all()
            continue
        for k in want:
            np.testing.assert_array_equal(got[k], want[k], err_msg=f"{k} at step {step}")
        held, table, ring, state = (want[k].astype(got[k].dtype) for k in ("held", "table", "ring", "state"))
        live = np.concatenate([table[r, :R.pages_of(int(h), page)] for r, h in enumerate(held)])
        free = [ring[i % pool] for i in range(int(state[0]), int(state[1]))]
        assert sorted(live.tolist() + free) == list(range(pool))


def test_tables_of_many_rows_of_few_tokens():
    rows = 70001
    rng = np.random.default_rng(3)
    held = rng.integers(0, 3, rows).astype(np.int32)
    delta = rng.integers(0, 2, rows).astype(np.int32)
    table = np.full((rows, 4), -1, np.int32)
    order = rng.permutation(4 * rows).astype(np.int32)
    at = 0
    for r in range(rows):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
    ring, state = np.roll(order, -at), np.array([0, 4 * rows - at, 0])
    tokens = int(delta.sum())
    want, bits = R.tables(held, delta, table, ring, state, 1, tokens, held)
    assert not bits
    got = _run_tables(held, delta, table, ring, state, 1, tokens, held)
    for k in want:
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)


REJECTED = [("length", dict(delta=[-6, 1, 1])), ("length", dict(held=[-1, 2, 3])), ("tokens", dict(tokens=2)),
            ("row", dict(delta=[200, 0, 0])), ("ring", dict(state=[0, 1, 0])), ("ring", dict(state=[8, 4, 0])),
            ("ring", dict(state=[0, 40, 0]))]


@pytest.mark.parametrize("name,change", REJECTED, ids=[f"{n}-{list(c)[0]}{i}" for i, (n, c) in enumerate(REJECTED)])
def test_tables_rejected_as_a_whole(name, change):
    base = dict(held=[5, 0, 16], delta=[20, 3, 1], tokens=300, state=[3, 20, 0])
    base.update(change)
    held, delta = (np.array(base[k], np.int32) for k in ("held", "delta"))
    state = np.array(base["state"])
    table = np.arange(24, dtype=np.int32).reshape(3, 8)
    ring = np.arange(24, dtype=np.int32) + 100
    got = _run_tables(held, delta, table, ring, state, 16, base["tokens"], None)
    bit = {"length": 1, "tokens": 1, "row": 256, "ring": 128}[name]
    assert got["state"][2] & bit
    assert (got["state"][:2] == state[:2]).all() and (got["held"] == held).all()
    assert (got["table"] == table).all() and (got["ring"] == ring).all()
    assert (got["slots"] == -1).all() and (got["positions"] == -1).all() and (got["row_start"] == 0).all()
    with pytest.raises(K.KvrError):
        K.check_status("block_tables", int(got["state"][2]))


def test_table_refusals_on_tensors():
    held = torch.zeros(3, dtype=torch.int32, device=DEV)
    table = torch.zeros((3, 8), dtype=torch.int32, device=DEV)
    ring, state = K.page_ring(10, DEV)
    good = [held, held.clone(), table, ring, state, 16, 5]
    K.block_tables(*good)
    for i, x in ((0, held.long()), (0, held[:, None]), (1, held[:2]), (2, table[:2]), (2, table.long()),
                 (2, table.expand(3, 8).T), (3, ring.long()), (3, ring.cpu()), (4, state[:2]), (4, state.int()),
                 (5, 0), (5, 24), (5, 2048), (6, -1), (6, 1 << 31)):
        args = list(good)
        args[i] = x
        with pytest.raises(K.KvrError):
            K.block_tables(*args)


# ---------------------------------------------------------------- store


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("types", TYPES, ids=["bf16", "fp16", "bf16-fp8", "fp16-fp8"])
@pytest.mark.parametrize("heads,page,first,fused", [(1, 1, False, False), (5, 16, True, True), (8, 128, False, True)])
def test_store(dim, types, heads, page, first, fused):
    g = torch.Generator().manual_seed(dim + heads)
    tokens, pages = 77, R.pages_of(300, page)
    both = torch.randn((tokens, 2, heads, dim), generator=g) * 300.0  # with an 8-bit cache some are clamped
    both[3, :, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0])
    both = both.to(types[0]).to(DEV)
    k, v = (both[:, i] if fused else both[:, i].contiguous() for i in range(2))
    shape = (pages, heads, page, dim) if first else (pages, page, heads, dim)
    caches = [(torch.randn(shape, generator=g)).to(types[1]).to(DEV) for _ in range(2)]
    caches = [c.transpose(1, 2) if first else c for c in caches]
    scales = [(torch.rand(heads, generator=g) + 0.5) for _ in range(2)] if types[1] == FP8 else [None, None]
    slots = torch.randperm(pages * page, generator=g)[:tokens].int()
    slots[5::9] = -1
    want = [c.float().cpu().clone() for c in caches]
    for x, y, s in zip((k, v), want, scales):
        z = x.float().cpu()
        if s is not None:
            z = (z * (1.0 / s)[:, None]).clamp(-448, 448).to(FP8).float()
        for t in range(tokens):
            if slots[t] >= 0:
                y[slots[t] // page, slots[t] % page] = z[t]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    note(f"store dim={dim} heads={heads} page={page} {types}")
    K.cache_store(k, v, *caches, slots.to(DEV), k_scale=None if scales[0] is None else scales[0].to(DEV),
                  v_scale=None if scales[1] is None else scales[1].to(DEV), status=status)
    assert int(status) == 0
    for c, y in zip(caches, want):
        assert torch.equal(torch.nan_to_num(c.float().cpu(), nan=9e9), torch.nan_to_num(y, nan=9e9))


def test_store_skips_and_reports_slots_behind_the_cache():
    k = torch.ones((3, 2, 64), dtype=BF16, device=DEV)
    c = torch.zeros((4, 16, 2, 64), dtype=BF16, device=DEV)
    d = torch.zeros_like(c)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    K.cache_store(k, k, c, d, torch.tensor([0, 64, 63], dtype=torch.int32, device=DEV), status=status)
    assert int(status) == 512
    assert float(c.sum()) == float(d.sum()) == 2 * 2 * 64 and float(c[3, 15].sum()) == 128.0


def test_store_refusals_on_tensors():
    k = torch.ones((3, 2, 64), dtype=BF16, device=DEV)
    c = torch.zeros((4, 16, 2, 64), dtype=BF16, device=DEV)
    s = torch.zeros(3, dtype=torch.int32, device=DEV)
    for args in ((k.half(), k.half(), c, c, s), (k, k.half(), c, c, s), (k[:2], k, c, c, s), (k, k, c, c.half(), s),
                 (k, k, c[..., :32], c[..., :32], s), (k, k, c, c, s.long()), (k, k, c, c, s[:2]),
                 (k.float(), k.float(), c.float(), c.float(), s), (k, k, c[0], c[0], s), (k, k, c, c.cpu(), s)):
        with pytest.raises(K.KvrError):
            K.cache_store(*args)


# ---------------------------------------------------------------- together


def test_a_step_in_a_graph():
    """Tables, store and attention of a decoding step, captured and replayed; eager work in between."""
    n, page, pool = 12, 16, 400
    g = torch.Generator(DEV).manual_seed(5)
    held = torch.arange(n, dtype=torch.int32, device=DEV) * 13
    one = torch.ones(n, dtype=torch.int32, device=DEV)
    table = torch.full((n, 16), -1, dtype=torch.int32, device=DEV)
    ring, state = K.page_ring(pool, DEV)
    zero = torch.zeros_like(held)
    K.block_tables(zero, held.clone(), table, ring, state, page, int(held.sum()), in_place=True)
    kc = torch.randn((pool, page, 2, 128), generator=g, device=DEV).bfloat16()
    vc = torch.randn((pool, page, 2, 128), generator=g, device=DEV).bfloat16()
    pt = ring[300:320].reshape(2, 10).clone()
    gs = torch.tensor([0, 9, n], dtype=torch.int32, device=DEV)
    pl = torch.tensor([150, 31], dtype=torch.int32, device=DEV)
    q, k, v = (torch.randn((n, h, 128), generator=g, device=DEV).bfloat16() for h in (8, 2, 2))
    work = [x.clone() for x in (held, table, ring, state, kc, vc)]

    def step(held, table, ring, state, kc, vc):
        t = K.block_tables(held, one, table, ring, state, page, n, in_place=True)
        K.cache_store(k, v, kc, vc, t.slots)
        return K.shared_attention(q, kc, vc, t.row_start, table, held, gs, pt, pl)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(*[x.clone() for x in work])
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*work)
    for x, y in zip(work, (held, table, ring, state, kc, vc)):
        x.copy_(y)
    eager = [x.clone() for x in (held, table, ring, state, kc, vc)]
    for i in range(6):
        q.copy_(torch.randn(q.shape, generator=g, device=DEV))
        k.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        want = step(*eager)
        assert torch.equal(out, want), i
        for x, y in zip(work, eager):
            assert torch.equal(x, y), i


def test_the_worker_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import shared_prefix_worker as W
    # p and the result are rounded to bfloat16 once each, for values up to about 4: 2 * 4 * 2^-8
    assert W.main() <= 2 * 4 * 2.0 ** -8
