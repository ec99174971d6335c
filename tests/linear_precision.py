"""How exact linear attention is, from what its operands hold: bounds without a
half step of the results' type to hide in, and the chunked form on the CPU with
a chosen number of parts of its operands."""
from __future__ import annotations

import numpy as np
import torch

import layer_reference as R

PAIR = 2.0 ** -16  # a number as its leading 8 bits and the rest, rounded to 8: off by at most that of itself


def problem(new, heads, kv_heads, dim, dtype, **kw):
    """Like layer_reference.Linear, but nothing cancels: all values are positive (so a result's magnitude is itself)."""
    p = R.Linear(new, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, **kw)
    p.q, p.k, p.v, p.state = (x.abs() for x in (p.q, p.k, p.v, p.state))
    return p


def state_steps(n):
    """Half steps of 32 bits of a state of n tokens.  Its terms are a key times a value times a power of the decay, as
    three exact products for the matrix units, which may round each sum to a whole step: 2 * 3 n.  The powers' exponents
    are rounded: |log_decay| n half steps, and 32 for the exponentials and the products with them."""
    return 7 * n + 32


def result_steps(n):
    """And of a result: the state's, a sum over 128 elements of a state's two parts, one over 64 tokens' two parts, and
    one over 128 elements of a score, each to a whole step."""
    return state_steps(n) + 2 * (256 + 128 + 128) + 16


def bounds(p, want):
    w_out, w_state, m_out, m_state = want
    n = max(p.new + [1])
    # Scores and the states as operands of results are pairs.  Half-precision tokens are pairs too, exactly, of which
    # the product of the two second parts (each below 2^-7 of its number) is left out: in scores and in results, and
    # of the three parts of a weighed value that of the last.
    halves = p.q.dtype == torch.float16
    out = (PAIR * 1.01 + (2 * 2.0 ** -14 if halves else 0.0) + result_steps(n) * R.U32) * m_out
    state = ((2.0 ** -22 if halves else 0.0) + state_steps(n) * R.U32) * m_state
    return out, state


def outside(out, state, p, want):
    """Shares of the results and of the states' values that no number within the bounds is rounded to."""
    dtype = p.q.dtype
    by_out, by_state = bounds(p, want)
    got = out.double().cpu().numpy()
    # (rounding keeps the order)
    lo, hi = (torch.from_numpy(want[0] + s * by_out).to(dtype).double().numpy() for s in (-1, 1))
    off = np.abs(state.double().cpu().numpy() - want[1])
    return float(((got < lo) | (got > hi)).mean()), float((off > by_state).mean())


def check(out, state, p, want=None):
    shares = outside(out, state, p, want or p.want())
    assert shares == (0.0, 0.0), shares


# ---------------------------------------------------------------- the chunked form


def leading(x):
    return (x.contiguous().view(torch.int32) & -65536).view(torch.float32)


def in_parts(x, n):
    """x (32 bits) as the sum of n numbers of 8 bits; the second of two is rounded, the others are cut off."""
    parts = []
    for k in range(n):
        parts.append((x.bfloat16().float() if n == 2 and k == 1 else leading(x)))
        x = x - parts[-1]
    return sum(parts[1:], parts[0])


def chunked(p, operands=2, weighed=3):
    """(out, state) of the chunked form in 32 bits, one request after the other: scores and states as operands in so
    many parts, weighed values in so many."""
    q, k, v = (x.float() for x in (p.q, p.k, p.v))
    state, first, out = p.state.clone(), p.state, torch.zeros_like(q)
    share, at = p.heads // p.kv_heads, 0
    i = torch.arange(64)
    write = p.read if p.write is None else p.write
    for r, n in enumerate(p.new):
        for h in range(p.kv_heads):
            g = p.log_decay[h]
            s = first[p.read[r], h].clone() if p.read[r] >= 0 else torch.zeros_like(first[0, 0])
            for t in range(at, at + n, 64):
                m = min(64, at + n - t)
                kc, vc = k[t:t + m, h], v[t:t + m, h]
                apart = i[:m, None] - i[:m]
                decay = torch.where(apart >= 0, torch.exp(g * apart.clamp(min=0)), 0.0) * p.scale
                for j in range(h * share, h * share + share):
                    qc = q[t:t + m, j]
                    weights = in_parts((qc @ kc.t().contiguous()) * decay, operands)
                    o = (qc @ in_parts(s, operands)) * (torch.exp(g * (i[:m, None] + 1)) * p.scale)
                    out[t:t + m, j] = o + weights @ vc
                left = torch.exp(g * (m - 1 - i[:m, None]))
                s = torch.exp(g * m) * s + kc.t().contiguous() @ in_parts(vc * left, weighed)
            if write[r] >= 0:
                state[write[r], h] = s
        at += n
    return out.to(p.q.dtype), state
