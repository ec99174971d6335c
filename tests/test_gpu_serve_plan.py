"""The serving operators on the GPU where their forms change: how the
attention plans, splits and joins, how it addresses pages, and the sizes at
which the table kernels change over."""
import numpy as np
import pytest
import torch

import paper_2601_18999_amd as K
from gpu_helpers import note
import serve_reference as R
from test_gpu_serve import BF16, DEV, FP16, FP8, _run_tables, attend

pytestmark = pytest.mark.gpu


def on_device(p):
    """Problem.expect on the GPU: row tiles of one request and key head at a time, in 64 bits."""
    shape = (sum(p.new), p.heads)
    out, size = (torch.zeros((*shape, p.dim), dtype=torch.float64) for _ in range(2))
    lse = torch.full(shape, -torch.inf, dtype=torch.float64)
    share, at = p.heads // p.kv_heads, 0
    for r, n in enumerate(p.new):
        if not n:
            continue
        k, v, prefix = (x.to(DEV) if isinstance(x, torch.Tensor) else x for x in p.path(r))
        q = p.q[at:at + n].to(DEV).double()
        for h in range(p.kv_heads):
            kh, vh = k[:, h].T.contiguous(), v[:, h].contiguous()
            for a in range(0, n, 1024):
                b = min(n, a + 1024)
                seen = prefix + p.own[r] - n + torch.arange(a, b, device=DEV) + 1
                rows = q[a:b, h * share:(h + 1) * share].reshape(-1, p.dim)
                s = (rows @ kh * p.scale).reshape(b - a, share, -1)
                s = s.masked_fill(torch.arange(k.shape[0], device=DEV) >= seen[:, None, None], -torch.inf)
                w = torch.softmax(s, -1).reshape(rows.shape[0], -1)
                heads = slice(h * share, (h + 1) * share)
                out[at + a:at + b, heads] = (w @ vh).reshape(b - a, share, -1).cpu()
                size[at + a:at + b, heads] = (w @ vh.abs()).reshape(b - a, share, -1).cpu()
                lse[at + a:at + b, heads] = torch.logsumexp(s, -1).cpu()
        at += n
    return out, size, lse


def test_the_two_references_agree():
    p = R.Problem([1, 5, 0, 3], [40, 5, 9, 70], [3, 1], [33, 0], heads=6, kv_heads=2, dim=64)
    for a, b in zip(p.expect(), on_device(p)):
        torch.testing.assert_close(a, b, rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("requests", [62, 63, 64, 65, 256, 257, 1023, 1024, 1025, 2500])
def test_numbers_of_requests(requests):
    # up to 64 units every workgroup plans by itself; up to 256 a small planning workgroup; the lengths stand in
    # LDS up to 1,024 requests
    g = np.random.default_rng(requests)
    own = g.integers(1, 90, requests).tolist()
    p = R.Problem([1] * requests, own, [requests - 1, 1], [70, 3], heads=2, kv_heads=1, dim=64)
    R.check(*attend(p), p, on_device(p))


def test_more_groups_than_requests_in_most():
    g = np.random.default_rng(7)
    sizes = g.integers(0, 3, 1500).tolist()
    n = sum(sizes)
    new = g.integers(0, 4, n).tolist()
    own = [a + int(b) for a, b in zip(new, g.integers(0, 40, n))]
    p = R.Problem(new, own, sizes, g.integers(0, 200, 1500).tolist(), heads=2, kv_heads=2, dim=64, page=8)
    R.check(*attend(p), p, on_device(p))


def test_more_units_than_planning_threads():
    # 9,100 tokens of 16 heads to a key head: 1,138 tiles of 128 rows, and a second request behind them
    p = R.Problem([9100, 3], [9100, 70], heads=16, kv_heads=1, dim=64)
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("heads,new", [(5, 3), (7, 2), (3, 11), (40, 1)])
@pytest.mark.parametrize("prefix", [300, 6000])
def test_requests_that_cross_the_tiles_of_their_group(heads, new, prefix):
    # rows of a request that lie in two tiles of 128 rows of its group's prefix
    n = 40
    p = R.Problem([new] * n, [new + i % 50 for i in range(n)], [n], [prefix], heads=heads, kv_heads=1, dim=64)
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("types", [(BF16, BF16), (FP16, FP16), (BF16, FP8), (FP16, FP8)],
                         ids=["bf16", "fp16", "bf16-fp8", "fp16-fp8"])
@pytest.mark.parametrize("page,first", [(1, True), (16, False), (256, True)])
def test_prefixes_taken_for_a_whole_group(dim, types, page, first):
    # long enough to be shared: with requests that have no new token, and an empty group between
    new = [1, 1, 0, 2, 1, 1, 1, 3, 1, 1, 1, 0, 1]
    own = [a + 37 * i % 150 for i, a in enumerate(new)]
    p = R.Problem(new, own, [10, 0, 3], [5003, 70, 4800], heads=6, kv_heads=2, dim=dim, page=page, dtype=types[0],
                  cache=types[1], heads_first=first).spoil()
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("own,prefix", [(64, 0), (128, 0), (129, 0), (512, 0), (513, 0), (320, 192), (321, 192),
                                        (320, 193), (64, 64)])
@pytest.mark.parametrize("requests", [1, 16, 17, 300])
def test_tables_with_room_for_few_keys(own, prefix, requests):
    # at most eight steps of 64 keys (two where there are more than 32 rows) and a short prefix: nothing to join;
    # one token more, and there may be.  Valid lengths, then one that is not.
    p = R.Problem([1] * requests, [own - 7 * i % own for i in range(requests)], [requests] if prefix else [],
                  [prefix] if prefix else [], heads=2, kv_heads=1, dim=64, page=1)
    R.check(*attend(p), p, on_device(p))
    p.length[-1] = p.table.shape[1] + 1
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = attend(p, status=status)
    assert int(status) == 1 and torch.isnan(out).all() and torch.isnan(lse).all()


def test_own_tokens_of_length_zero_behind_a_shared_prefix():
    # the only own token is the new one, of every request
    p = R.Problem([1] * 40, [1] * 40, [40], [3001], heads=4, kv_heads=1, dim=128)
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [1, 2, 4, 8, 64])
@pytest.mark.parametrize("cache", [None, FP8], ids=["16-bit", "8-bit"])
def test_page_sizes_around_the_rows_of_a_load(dim, page, cache):
    # few rows (one wave's tiles) and many (tiles that the waves share), whole tiles and ends
    p = R.Problem([1, 90], [333, 450], [1, 1], [64, 200], heads=2, kv_heads=1, dim=dim, page=page, cache=cache).spoil()
    R.check(*attend(p), p, on_device(p))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_later_tokens_of_few_rows_have_no_influence(dim, dtype):
    # 8 new tokens, 16 rows: a wave's own tile, its V read key by key where it holds a NaN
    p = R.Problem([8], [50], heads=2, kv_heads=1, dim=dim, dtype=dtype)
    want = on_device(p)
    for c in (p.k_cache, p.v_cache):
        c[p.table[0, 46 // p.page], 46 % p.page] = float("nan")
    out, lse = attend(p)
    R.check(out[:4], lse[:4], p, [x[:4] for x in want])  # tokens 42 .. 45
    assert torch.isnan(out[4:]).all()


def test_scores_that_grow_from_tile_to_tile():
    # every key scores higher than the ones before it: the running maximum moves in every tile, by less and by
    # more than what is scaled at once
    for step in (0.05, 0.4, 3.0):
        p = R.Problem([1, 60], [400, 300], [2], [200], heads=2, kv_heads=1, dim=64)
        p.q[:] = 0
        p.q[..., 0] = 1.0
        p.scale = 1.0
        for rows, n in ((p.table, p.own), (p.prefix_table, p.prefix)):
            for row, m in zip(rows.tolist(), n):
                for t in range(m):
                    p.k_cache[row[t // p.page], t % p.page, 0, 0] = step * t
        # scores of size up to 3 * 400: products' 32-bit errors 64 * 2^-24 * 1200 = 4.6e-3
        ref, size, _ = on_device(p)
        out, _ = attend(p)
        err = (out.double().cpu() - ref).abs()
        assert (err <= 2.0 ** -8 * (ref.abs() + size) * 1.01 + 5e-3 * size + 1e-7).all(), step


def test_a_row_is_the_same_with_and_without_a_group():
    # the prefix shared, or each request's own first tokens: the same attention
    n = 20
    p = R.Problem([1] * n, [5 + i for i in range(n)], [n], [100], heads=4, kv_heads=2, dim=128, page=1)
    q = R.Problem([1] * n, [105 + i for i in range(n)], heads=4, kv_heads=2, dim=128, page=1)
    q.q = p.q
    q.k_cache, q.v_cache = p.k_cache, p.v_cache
    for r in range(n):
        q.table[r, :100] = p.prefix_table[0, :100]
        q.table[r, 100:105 + r] = p.table[r, :5 + r]
    want = on_device(p)
    R.check(*attend(p), p, want)
    R.check(*attend(q), q, want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("cache", [None, FP8], ids=["16-bit", "8-bit"])
def test_keys_and_values_laid_out_differently(dim, cache):
    p = R.Problem([1, 100], [333, 300], [1, 1], [64, 200], heads=4, kv_heads=2, dim=dim, cache=cache)
    args = p.args()
    pages, page, heads, _ = args[2].shape
    v = torch.empty((heads, pages, 2, page, dim), dtype=args[2].dtype, device=DEV)
    v[:, :, 1] = args[2].permute(2, 0, 1, 3)
    args[2] = v[:, :, 1].permute(1, 2, 0, 3)
    assert args[2].stride() != args[1].stride()
    R.check(K.shared_attention(*args, **p.kwargs()), None, p, on_device(p))


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
def test_many_small_weights_beside_a_large_one(dtype):
    # one key with a score 17 above 30,000 others: their weights, 4e-8 each and 1.2e-3 in all, count
    p = R.Problem([1], [30001], heads=1, kv_heads=1, dim=64, dtype=dtype, page=64)
    p.q[:] = 0
    p.q[..., 0] = 1.0
    p.scale = 1.0
    p.k_cache[..., 0] = 0.0
    p.v_cache[:] = 100.0
    first = (p.table[0, 0], 0)
    p.k_cache[first[0], first[1], 0, 0] = 17.0
    p.v_cache[first[0], first[1]] = 0.0
    ref, size, _ = p.expect()
    out, _ = attend(p)
    # p and the result rounded once each; halves have steps of 2^-24 * 2^-7 at the small end: half a step each
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -11
    step = 0.0 if dtype == BF16 else 30000 * 100.0 * 2.0 ** -32
    err = (out.double().cpu() - ref).abs()
    assert (err <= 2.1 * u * ref.abs() + 8e-4 * size + step).all(), (float(err.max()), float(ref.max()))


@pytest.mark.parametrize("rows,tokens", [(1024, 4096), (1025, 100), (1024, 4097), (1, 1), (64, 0), (4096, 5000)])
def test_table_sizes_around_the_forms(rows, tokens):
    rng = np.random.default_rng(rows + tokens)
    held = rng.integers(0, 20, rows).astype(np.int32)
    delta = np.zeros(rows, np.int32)
    for r in rng.integers(0, rows, tokens):
        delta[r] += 1
    drop = (delta == 0) & (rng.random(rows) < 0.5)
    delta[drop] = -rng.integers(0, held[drop] + 1)
    width = int((np.maximum(held, held + delta).max() + 3) // 4 + 1)
    table = np.full((rows, width), -1, np.int32)
    used = [R.pages_of(int(h), 4) for h in held]
    pool = sum(used) + tokens + 3
    order = rng.permutation(pool).astype(np.int32)
    at = 0
    for r, n in enumerate(used):
        table[r, :n] = order[at:at + n]
        at += n
    head = int(rng.integers(0, pool))
    ring = np.roll(order, head - at)
    state = np.array([head, head + pool - at, 0])
    want, bits = R.tables(held, delta, table, ring, state, 4, tokens, held)
    assert not bits
    got = _run_tables(held, delta, table, ring, state, 4, tokens, held)
    for k in want:
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)


def test_one_row_among_many_empty_ones():
    # a wave's tokens whose rows lie far apart: thousands of rows without a token between them
    rows = 70000
    held = np.zeros(rows, np.int32)
    delta = np.zeros(rows, np.int32)
    delta[[0, 5000, 5001, 69999]] = [3, 700, 1, 40]
    delta[30000:30200] = 1
    table = np.full((rows, 11), -1, np.int32)
    ring, state = np.arange(2000, dtype=np.int32), np.array([1990, 3990, 0])
    tokens = int(delta.sum()) + 100
    want, bits = R.tables(held, delta, table, ring, state, 64, tokens, held)
    assert not bits
    got = _run_tables(held, delta, table, ring, state, 64, tokens, None)
    for k in want:
        np.testing.assert_array_equal(got[k], want[k], err_msg=k)
    # and all given back
    t, g = want["table"].astype(np.int32), want["ring"].astype(np.int32)
    back, bits = R.tables(delta, -delta, t, g, want["state"], 64, 0, held)
    got = _run_tables(delta, -delta, t, g, want["state"], 64, 0, None)
    for k in back:
        np.testing.assert_array_equal(got[k], back[k], err_msg=k)
