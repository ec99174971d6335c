"""Linear attention on the GPU for batches that a plan lists and in which requests
of a few tokens take the recurrent form: singles and drafts among prompts."""
import pytest
import torch

import linear_precision as P
import paper_2601_18999_amd as K
from gpu_helpers import note
from paper_2601_18999_amd import layer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16 = torch.bfloat16, torch.float16

# more than 512 states (a request's key head), and more than 256 requests or one that is cut; the last fits the device
# at once, so that all of its requests take the chunked form
BATCHES = {
    "300 of 0 to 20, 2 key heads": ([i % 21 for i in range(300)], 4, 2, 64),
    "300 of 0 to 20, 8 key heads": ([(7 * i) % 21 for i in range(300)], 8, 8, 64),
    "300 of 0 to 20, heads of 128": ([(5 * i) % 21 for i in range(300)], 4, 2, 128),
    "70, one cut, heads of 64": ([1, 4, 2, 1, 0, 8, 9] * 5 + [1500] + [1, 3, 1, 10] * 8 + [1, 2], 8, 8, 64),
    "70, one cut, heads of 128": ([1, 4, 2, 1, 0, 8, 9] * 5 + [1500] + [1, 3, 1, 10] * 8 + [1, 2], 16, 8, 128),
    "70, two cut": ([600] + [1, 8, 9, 64, 65] * 13 + [2, 0, 1, 777], 8, 8, 64),
    "300 singles but one": ([1] * 150 + [70] + [1] * 149, 6, 3, 64),
    "300 of a few": ([1 + i % 8 for i in range(300)], 4, 2, 64),
    "17 x 32, one cut": ([1, 1, 5, 700] + [1, 2, 9] * 4 + [30], 32, 32, 64),
    "16 x 32, one cut": ([1, 1, 5, 700] + [1, 2, 9] * 4, 32, 32, 64),
}


def batch(what, dtype, in_place, **kw):
    new, heads, kv, dim = BATCHES[what]
    n = len(new)
    assert layer._linear_bytes(0, sum(new), n, heads, kv, dim, True) > 0 and (n * kv > 512 or what[:2] == "16")
    if in_place:
        kw.update(read=list(range(n)), write=list(range(n)))
    return P.problem(new, heads, kv, dim, dtype, **kw)


def run(p):
    args = p.args()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full_like(args[0], float("nan"))
    assert K.linear_attention(*args, out=out, status=status) is out
    torch.cuda.synchronize()
    return out, args[3], int(status)


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("in_place", [False, True], ids=["apart", "in place"])
@pytest.mark.parametrize("what", BATCHES)
def test_batches(what, in_place, dtype):
    p = batch(what, dtype, in_place)
    note(f"linear {what} {dtype} in_place={in_place}")
    out, state, bits = run(p)
    assert bits == 0
    P.check(out, state, p)


@pytest.mark.parametrize("what", ["300 of 0 to 20, 2 key heads", "70, one cut, heads of 128"])
def test_batches_that_share_states_or_do_not_keep_them(what):
    new = BATCHES[what][0]
    p = batch(what, BF16, False, read=[(i * 5) % 9 - 1 for i in range(len(new))])
    p.write = [-1 if i % 3 == 1 else s for i, s in enumerate(p.write)]
    note(f"linear shared {what}")
    out, state, bits = run(p)
    assert bits == 0
    P.check(out, state, p)


@pytest.mark.parametrize("what", ["300 of 0 to 20, 2 key heads", "70, one cut, heads of 64"])
@pytest.mark.parametrize("which", ["read", "write"])
def test_a_slot_outside_the_pool_among_many(what, which):
    # of a single, a draft, a prompt and the cut one: their results are NaN, the others as they were
    p = batch(what, BF16, False)
    note(f"linear bad slots {what}")
    good, kept, _ = run(p)
    new, bad = p.new, [1, 2, 6, 35, 20]
    for i in bad:
        getattr(p, which)[i] = len(p.state) + i
    out, state, bits = run(p)
    at = p.row_start.tolist()
    mine = torch.zeros(sum(new), dtype=torch.bool)
    for i in bad:
        mine[at[i]:at[i + 1]] = True
    assert bits == 512 and out.cpu()[mine].isnan().all() and torch.equal(out.cpu()[~mine], good.cpu()[~mine])
    left = [s for i, s in enumerate(batch(what, BF16, False).write) if i in bad]
    rest = [s for s in range(len(state)) if s not in left]
    assert torch.equal(state[rest], kept[rest]) and torch.equal(state[left].cpu(), p.state[left])


def test_a_batch_captured_and_replayed():
    p = batch("70, one cut, heads of 128", BF16, True)
    args = p.args()
    first = args[3].clone()
    want, kept, _ = run(p)
    out = torch.empty_like(args[0])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        K.linear_attention(*args, out=out)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.linear_attention(*args, out=out)
    note("linear batch replayed")
    for _ in range(3):
        args[3].copy_(first)
        out.fill_(0)
        g.replay()
        again, _, _ = run(p)  # the program's own work between the replays
        assert torch.equal(out, want) and torch.equal(args[3], kept) and torch.equal(again, want)
