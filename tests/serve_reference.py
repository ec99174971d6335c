"""Plain implementations of the serving operators, in 64 bits on the CPU, and
small problems for them."""
from __future__ import annotations

import math

import numpy as np
import torch


def pages_of(n: int, page: int) -> int:
    return -(-n // page)


def tables(held, delta, table, ring, state, page, num_tokens, base):
    """The definition, row by row (numpy arrays); None where the batch is not valid."""
    head, tail = int(state[0]), int(state[1])
    rows, width = table.shape
    total = held.astype(np.int64) + delta
    if (held < 0).any() or (total < 0).any():
        return None, 1
    if (np.maximum(held, total) > width * page).any():
        return None, 256
    gain = sum(max(0, pages_of(int(t), page) - pages_of(int(h), page)) for h, t in zip(held, total))
    bits = 1 if np.maximum(delta, 0).astype(np.int64).sum() > num_tokens else 0
    give = sum(max(0, pages_of(int(h), page) - pages_of(int(t), page)) for h, t in zip(held, total))
    if gain > tail - head or tail - head + give > len(ring):
        bits |= 128
    if bits:
        return None, bits
    out_table, out_ring = table.copy(), ring.copy()
    start, slots, places = [0], [], []
    for r in range(rows):
        a, b = pages_of(int(held[r]), page), pages_of(int(total[r]), page)
        for c in range(a, b):
            out_table[r, c] = ring[head % len(ring)]
            head += 1
        for c in range(b, a):
            out_ring[tail % len(ring)] = table[r, c]
            tail += 1
        for t in range(int(held[r]), int(total[r])):
            slots.append(int(out_table[r, t // page]) * page + t % page)
            places.append(int(base[r]) + t)
        start.append(len(slots))
    pad = [-1] * (num_tokens - len(slots))
    return dict(table=out_table, ring=out_ring, held=total, state=np.array([head, tail, state[2]]),
                row_start=np.array(start), slots=np.array(slots + pad, dtype=np.int64),
                positions=np.array(places + pad, dtype=np.int64)), 0


class Problem:
    """Requests in groups with a paged cache.  new, own: tokens of each request (own includes new); sizes and
    prefix: requests and prefix tokens of each group."""

    def __init__(self, new, own, sizes=(), prefix=(), heads=4, kv_heads=2, dim=64, page=16, dtype=torch.bfloat16,
                 cache=None, heads_first=False, seed=0, spare=3, device="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        self.new, self.own, self.sizes, self.prefix = list(new), list(own), list(sizes), list(prefix)
        self.heads, self.kv_heads, self.dim, self.page, self.device = heads, kv_heads, dim, page, device
        cache = cache or dtype
        self.fp8 = cache == torch.float8_e4m3fn
        assert not sizes or sum(sizes) == len(new)
        counts = [pages_of(n, page) for n in self.own + self.prefix]
        pages = sum(counts) + spare
        order = torch.randperm(pages, generator=g)
        width, pwidth = max(counts[:len(new)] + [1]), max(counts[len(new):] + [1])
        self.table = torch.full((len(new), width), -1, dtype=torch.int32)
        self.prefix_table = torch.full((len(self.prefix), pwidth), -1, dtype=torch.int32)
        at = 0
        for i, c in enumerate(counts):
            row = self.table[i] if i < len(new) else self.prefix_table[i - len(new)]
            row[:c] = order[at:at + c].to(torch.int32)
            at += c
        tokens = sum(new)
        self.q = torch.randn((tokens, heads, dim), generator=g).to(dtype)
        shape = (pages, page, kv_heads, dim)
        self.k_cache, self.v_cache = (torch.randn(shape, generator=g).to(cache) for _ in range(2))
        self.k_scale = self.v_scale = None
        if self.fp8:
            self.k_scale, self.v_scale = (torch.rand(kv_heads, generator=g) + 0.5 for _ in range(2))
        self.heads_first = heads_first
        self.row_start = torch.tensor(np.concatenate([[0], np.cumsum(self.new)]), dtype=torch.int32)
        self.length = torch.tensor(self.own, dtype=torch.int32)
        self.group_start = torch.tensor(np.concatenate([[0], np.cumsum(self.sizes)]), dtype=torch.int32)
        self.prefix_length = torch.tensor(self.prefix, dtype=torch.int32)
        self.scale = dim ** -0.5

    def spoil(self, value=float("nan")):
        """Puts the value wherever no token of the problem stands."""
        kept = torch.zeros(self.k_cache.shape[:2], dtype=torch.bool)
        for rows, lens in ((self.table, self.own), (self.prefix_table, self.prefix)):
            for row, n in zip(rows.tolist(), lens):
                for t in range(n):
                    kept[row[t // self.page], t % self.page] = True
        for c in (self.k_cache, self.v_cache):
            if self.fp8:
                c.view(torch.uint8)[~kept] = 0x7f
            else:
                c[~kept] = value
        return self

    def on(self, x):
        return None if x is None else x.to(self.device)

    def cache_on(self, x):
        x = x.to(self.device)
        return x.transpose(1, 2).contiguous().transpose(1, 2) if self.heads_first else x

    def args(self):
        """Arguments of shared_attention on the device."""
        g = bool(self.sizes)
        return [self.on(self.q), self.cache_on(self.k_cache), self.cache_on(self.v_cache), self.on(self.row_start),
                self.on(self.table), self.on(self.length), self.on(self.group_start) if g else None,
                self.on(self.prefix_table) if g else None, self.on(self.prefix_length) if g else None]

    def kwargs(self):
        return dict(scale=self.scale, k_scale=self.on(self.k_scale), v_scale=self.on(self.v_scale))

    def path(self, r):
        """A request's keys and values, [keys, kv_heads, dim] in 64 bits, and its prefix's length."""
        group = int(np.searchsorted(np.cumsum(self.sizes), r, side="right")) if self.sizes else -1
        parts = [(self.table[r], self.own[r])]
        if group >= 0:
            parts.insert(0, (self.prefix_table[group], self.prefix[group]))
        out = []
        for cache, scale in ((self.k_cache, self.k_scale), (self.v_cache, self.v_scale)):
            x = torch.cat([cache[row[:pages_of(n, self.page)].long()].double().reshape(-1, self.kv_heads, self.dim)[:n]
                           for row, n in parts]) if not self.fp8 else torch.cat(
                [cache.view(torch.uint8)[row[:pages_of(n, self.page)].long()].view(cache.dtype).double()
                 .reshape(-1, self.kv_heads, self.dim)[:n] for row, n in parts])
            out.append(x if scale is None else x * scale.double()[:, None])
        return out[0], out[1], parts[0][1] if group >= 0 else 0

    def expect(self):
        """(out, sum p |v|, lse) in 64 bits."""
        shape = (sum(self.new), self.heads)
        out, size = (torch.zeros((*shape, self.dim), dtype=torch.float64) for _ in range(2))
        lse = torch.full(shape, -math.inf, dtype=torch.float64)
        share, at = self.heads // self.kv_heads, 0
        for r, n in enumerate(self.new):
            if not n:
                continue
            k, v, prefix = self.path(r)
            for i in range(n):
                seen = prefix + self.own[r] - n + i + 1
                for h in range(self.heads):
                    s = (k[:seen, h // share] @ self.q[at + i, h].double()) * self.scale
                    lse[at + i, h] = torch.logsumexp(s, 0)
                    p = torch.softmax(s, 0)
                    out[at + i, h] = p @ v[:seen, h // share]
                    size[at + i, h] = p @ v[:seen, h // share].abs()
            at += n
        return out, size, lse


def check(out, lse, problem, want=None):
    """Compares a call's result with the 64-bit one.

    The result is rounded once to its type (relative error u = 2^-8 for
    bfloat16, 2^-11 for IEEE halves), and each p once before the second
    product: at most u * sum p |v|.  Scores carry the 32-bit errors of a sum of
    dim <= 256 products of total size below 40 (256 * 2^-24 * 40 = 6e-4 at
    worst), which move p by the same relative amount; 8e-4 covers it and the
    exponentials."""
    ref, size, ref_lse = want or problem.expect()
    u = 2.0 ** -8 if problem.q.dtype == torch.bfloat16 else 2.0 ** -11
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    bound = u * (ref.abs() + size) * (1 + u) + 8e-4 * size + 1e-7
    over = (got - ref).abs() - bound
    assert (over <= 0).all(), float(over.max())
    if lse is not None:
        got = lse.double().cpu()
        seen = torch.isfinite(ref_lse)
        assert torch.equal(seen, torch.isfinite(got))
        assert ((got - ref_lse)[seen].abs() <= 8e-4).all()
        assert (got[~seen] == -math.inf).all()
