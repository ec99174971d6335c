"""Plain implementations of the norms, the 8-bit products and linear attention,
in 64 bits on the CPU, with what their results may be off by."""
from __future__ import annotations

import numpy as np
import torch

U32 = 2.0 ** -24  # half a step of 32 bits, relative


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def tiny(dtype) -> float:
    """Half the distance of the smallest numbers."""
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def act(z, name):
    return {"none": z, "sigmoid": 1 / (1 + np.exp(-z)), "silu": z / (1 + np.exp(-z))}[name]


def norm(x, after=None, gate=None, activation="none", residual=None, residual_scale=1.0, before=None, eps=1e-6):
    """(n, r, m_n, m_r): the results in 64 bits, and the magnitudes that 32-bit errors are relative to."""
    a = x.double().numpy()
    if after is not None:
        a = a / np.sqrt((a * a).mean(1, keepdims=True) + eps) * after.double().numpy()
    if gate is not None:
        a = a * act(gate.double().numpy(), activation)
    m = np.abs(a)
    if residual is not None:
        r = residual.double().numpy()
        m = np.abs(r) + np.abs(residual_scale * a)
        a = r + residual_scale * a
    n, mn = a, m
    if before is not None:
        by = before.double().numpy() / np.sqrt((a * a).mean(1, keepdims=True) + eps)
        n, mn = a * by, m * np.abs(by)
        # an error of r moves the mean: by at most the mean of 2 |r| m, relative to the mean of r^2
        mn = mn + np.abs(n) * ((np.abs(a) * m).mean(1, keepdims=True) / ((a * a).mean(1, keepdims=True) + eps))
    return n, a, mn, m


# Errors of 32 bits that a row's values gather, in half steps: the sum of squares adds at most 64 values a lane, 6 + 16
# partial sums (of positive numbers: at most that many half steps, of which the root keeps half), and some twenty
# operations stand around it, twice.
NORM_STEPS = 2 * (86 / 2 + 21)


def check_norm(got, want, magnitude, dtype):
    bound = half_step(dtype) * np.abs(want) + tiny(dtype) + NORM_STEPS * U32 * magnitude * 1.01
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= bound).all(), (float((off / bound).max()), np.argwhere(off > bound)[:4].tolist())


def integers(x):
    """x [tokens, dim] in 8-bit integers and its scales, by the definition's 32-bit steps (float32 in and out)."""
    x = x.float().numpy()
    top = np.abs(x).max(1, keepdims=True)
    with np.errstate(all="ignore"):
        by = np.float32(127) / top
        usual = np.isfinite(top) & (top >= 2.0 ** -100)
        q = np.where(usual, np.rint(x * by), 0)
        scale = np.where(usual, top / np.float32(127), np.where(np.isfinite(top), np.float32(0), np.float32(np.nan)))
    return q.astype(np.int64), scale[:, 0]


def product(xq, xs, wq, ws, bias):
    """(result, magnitude) in 64 bits; the sums are exact."""
    sums = xq.astype(np.float64) @ wq.astype(np.float64).T
    p = sums * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
    b = 0.0 if bias is None else bias.astype(np.float64)
    return p + b, np.abs(p) + np.abs(b)


def check_product(got, want, magnitude, dtype):
    # the sum to 32 bits, two products, the bias: four half steps; then the result's
    bound = half_step(dtype) * np.abs(want) + tiny(dtype) + 4 * U32 * magnitude * 1.01
    got = got.double().cpu().numpy()
    assert (np.isnan(got) == np.isnan(want)).all()
    off, bound = np.abs(got - want)[~np.isnan(want)], bound[~np.isnan(want)]
    assert (off <= bound).all(), float((off / bound).max())


class Linear:
    """Requests of `new` tokens over a pool of states."""

    def __init__(self, new, heads=4, kv_heads=2, dim=64, dtype=torch.bfloat16, read=None, write="own", seed=0,
                 decay=None, spare=2, device="cuda:0"):
        g = torch.Generator().manual_seed(seed)
        n, tokens = len(new), sum(new)
        self.new, self.heads, self.kv_heads, self.dim, self.device = list(new), heads, kv_heads, dim, device
        self.q = torch.randn((tokens, heads, dim), generator=g).to(dtype)
        self.k, self.v = (torch.randn((tokens, kv_heads, dim), generator=g).to(dtype) for _ in range(2))
        slots = 2 * n + spare
        self.state = torch.randn((slots, kv_heads, dim, dim), generator=g)
        order = torch.randperm(slots, generator=g).tolist()
        self.read = [order[n + i] for i in range(n)] if read is None else list(read)
        free = [s for s in order if s not in self.read]
        self.write = free[:n] if write == "own" else list(write) if write is not None else None
        if decay is None:
            decay = (-torch.exp2(-1 - 7 * torch.rand(kv_heads, generator=g))).tolist()
            decay[0] = 0.0
        self.log_decay = torch.tensor(decay, dtype=torch.float32)
        self.row_start = torch.tensor(np.concatenate([[0], np.cumsum(self.new)]), dtype=torch.int32)
        self.scale = dim ** -0.5

    def i32(self, x):
        return None if x is None else torch.tensor(x, dtype=torch.int32, device=self.device)

    def args(self, ragged=True):
        """Arguments of linear_attention on the device."""
        on = [x.to(self.device) for x in (self.q, self.k, self.v, self.state, self.log_decay)]
        return on + [self.i32(self.read), self.i32(self.write), self.row_start.to(self.device) if ragged else None]

    def want(self):
        """(out, state, magnitudes of both), token by token in 64 bits."""
        q, k, v = (x.double().numpy() for x in (self.q, self.k, self.v))
        state = self.state.double().numpy()
        out, out_m, state_m = np.zeros(q.shape), np.zeros(q.shape), np.abs(state)
        first, share = state.copy(), self.heads // self.kv_heads
        decay = np.exp(self.log_decay.double().numpy())[:, None, None]
        at = 0
        write = self.read if self.write is None else self.write
        for r, n in enumerate(self.new):
            s = first[self.read[r]].copy() if self.read[r] >= 0 else np.zeros_like(first[0])
            m = np.abs(s)
            for t in range(at, at + n):
                kv = k[t][:, :, None] * v[t][:, None, :]
                s, m = decay * s + kv, decay * m + np.abs(kv)
                qt = q[t].reshape(self.kv_heads, share, self.dim) * self.scale
                out[t] = (qt @ s).reshape(self.heads, self.dim)
                out_m[t] = (np.abs(qt) @ m).reshape(self.heads, self.dim)
            at += n
            if write[r] >= 0:
                state[write[r]], state_m[write[r]] = s, m
        return out, state, out_m, state_m


def linear_steps(n):
    """Half steps of 32 bits that n tokens gather: each term of a state passes at most n products with a decay (or
    with powers of it, whose own error is that many steps at most) and n sums, each result a sum over 128 more."""
    return 3 * n + 160


def check_linear(out, state, p, want=None):
    w_out, w_state, m_out, m_state = want or p.want()
    n = max(p.new + [1])
    dtype = p.q.dtype
    # The scores, and the states that queries meet, are rounded to the matrix units' operands: to bfloat16 (once), or,
    # for float16, to pairs of bfloat16 (2^-8 * 2^-8, for each of the two factors).  What a chunk adds to a state has
    # one factor in such pairs, float16 both.
    pair = 2.0 ** -16
    operands = 2.0 ** -8 if dtype == torch.bfloat16 else 2 * pair
    bound = half_step(dtype) * np.abs(w_out) * 1.01 + tiny(dtype) + (operands + 2 * pair + linear_steps(n) * U32) * m_out
    off = np.abs(out.double().cpu().numpy() - w_out)
    assert (off <= bound).all(), (float((off / bound).max()), np.argwhere(off > bound)[:4].tolist())
    bound = (2 * pair + linear_steps(n) * U32) * m_state
    off = np.abs(state.double().cpu().numpy() - w_state)
    assert (off <= bound).all(), (float((off / bound).max()), np.argwhere(off > bound)[:4].tolist())
