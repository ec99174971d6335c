"""The precision bounds of linear attention on the CPU: what the operands hold
passes them, and a part less does not."""
import pytest
import torch

import layer_reference as R
import linear_precision as P

LAYOUTS = [([9], 2, 2, 64), ([65], 4, 2, 64), ([129], 8, 2, 128), ([513], 2, 2, 128), ([700], 2, 2, 64),
           ([1153], 4, 1, 128), ([1, 40, 100], 15, 5, 64), ([1300, 0, 700], 2, 1, 64)]


@pytest.mark.parametrize("new,heads,kv,dim", LAYOUTS, ids=[str(x[0]) for x in LAYOUTS])
def test_a_part_less_is_outside_the_bounds(new, heads, kv, dim):
    p = P.problem(new, heads, kv, dim, torch.bfloat16)
    want = p.want()
    P.check(*P.chunked(p), p, want)
    out, state = P.chunked(p, operands=1)
    few, kept = P.outside(out, state, p, want)
    assert few > 0.25 and kept == 0.0, (few, kept)
    if new == [9]:  # (the errors of a second part that is rounded cancel over more tokens)
        out, state = P.chunked(p, weighed=2)
        assert P.outside(out, state, p, want)[1] > 0.0


def test_bounds_of_single_tokens_hold_32_bits():
    p = P.problem([1] * 5, 4, 2, 64, torch.float16)
    w = p.want()
    P.check(torch.from_numpy(w[0]).half(), torch.from_numpy(w[1]), p, w)
