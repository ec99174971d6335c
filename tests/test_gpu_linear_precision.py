"""Linear attention on the GPU to the precision of its operands: scores and
states in 16 bits, weighed values in 24, for both types of tokens."""
import pytest
import torch

import layer_reference as R
import linear_precision as P
import paper_2601_18999_amd as K
from gpu_helpers import note

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
SIGNS = pytest.mark.parametrize("make", [P.problem, R.Linear], ids=["positive", "signed"])

# (new tokens, query heads, key heads, head size): one chunk and several, cut ones, teams of query heads, both head sizes
LAYOUTS = [([1], 2, 2, 64), ([5], 4, 2, 128), ([9], 2, 2, 64), ([9], 2, 2, 128), ([65], 4, 2, 64), ([65], 8, 2, 128),
           ([129], 4, 4, 64), ([200], 8, 1, 128), ([513], 2, 2, 128), ([700], 2, 2, 64), ([1153], 16, 4, 128),
           ([1800], 1, 1, 128), ([2500, 0, 1300], 2, 1, 64), ([1, 40, 100], 15, 5, 64), ([1, 1, 1], 3, 3, 128),
           ([70] * 19, 4, 1, 64), ([3, 0, 64, 1, 65, 130, 0, 16, 17], 6, 3, 128)]


def run(p, **kw):
    note(f"linear new={p.new[:8]} heads={p.heads}/{p.kv_heads} dim={p.dim} {p.q.dtype}")
    args = p.args()
    out = K.linear_attention(*args, **kw)
    torch.cuda.synchronize()
    return out, args[3]


@TYPES
@SIGNS
@pytest.mark.parametrize("new,heads,kv,dim", LAYOUTS, ids=[f"{x[0][0]}x{len(x[0])}-{x[1]}/{x[2]}-{x[3]}" for x in LAYOUTS])
def test_precision(new, heads, kv, dim, make, dtype):
    p = make(new, heads, kv, dim, dtype)
    P.check(*run(p), p)


@TYPES
@pytest.mark.parametrize("new,heads,kv", [([300], 512, 512), ([70, 5], 1024, 1024), ([130, 1, 64], 300, 300),
                                          ([90], 640, 1), ([1, 1], 257, 257)])
def test_precision_of_many_heads(new, heads, kv, dtype):
    # more key heads than compute units, and many query heads beside each other
    p = P.problem(new, heads, kv, 64, dtype)
    P.check(*run(p), p)


@TYPES
@pytest.mark.parametrize("dim", [64, 128])
def test_precision_in_place_and_in_slices(dim, dtype):
    p = P.problem([5, 70, 1, 300], 6, 2, dim, dtype, read=[0, 1, -1, 3], write=[0, 1, 2, 3])
    want = p.want()
    args = p.args()
    fused = torch.full((sum(p.new), 10, dim + 8), float("nan"), dtype=dtype, device=DEV)
    parts = fused[:, :, :dim].split([6, 2, 2], 1)
    for part, x in zip(parts, args[:3]):
        part.copy_(x)
    pool = torch.full((len(p.state), 3, dim * dim + 4), 5.0, device=DEV)
    state = pool[:, :2, :dim * dim].unflatten(2, (dim, dim))
    state.copy_(args[3])
    note(f"linear slices dim={dim} {dtype}")
    out = K.linear_attention(*parts, state, *args[4:])
    P.check(out, state, p, want)
    assert (pool[:, 2] == 5).all() and (pool[:, :, dim * dim:] == 5).all()


@TYPES
def test_precision_in_pieces(dtype):
    whole = P.problem([300], 4, 2, 128, dtype, read=[1], write=[0])
    want, args = whole.want(), whole.args()
    outs, at = [], 0
    for n in (1, 64, 100, 7, 128):
        cut = [x[at:at + n] for x in args[:3]]
        outs.append(K.linear_attention(*cut, args[3], args[4], whole.i32([1] if at == 0 else [0]), whole.i32([0]),
                                       whole.i32([0, n])))
        at += n
    P.check(torch.cat(outs), args[3], whole, want)


@TYPES
@pytest.mark.parametrize("dim", [64, 128])
def test_an_infinite_value_leaves_the_other_columns_their_bits(dim, dtype):
    p, q = (R.Linear([200], heads=2, kv_heads=1, dim=dim, dtype=dtype, decay=[-0.01]) for _ in range(2))
    q.v[90, 0, 5] = float("inf")
    (a, sa), (b, sb) = run(p), run(q)
    other = [i for i in range(dim) if i != 5]
    assert torch.equal(a[:90], b[:90]) and torch.equal(a[:, :, other], b[:, :, other])
    assert torch.equal(sa[:, :, :, other], sb[:, :, :, other])
    assert not b[90:, :, 5].isfinite().any() and not sb[p.write[0], 0, :, 5].isfinite().any()
    P.check(a, sa, p)
