"""A worker that answers the queries routed to it, on one GPU.

    python examples/shared_prefix_worker.py

Routes a stream of grouped queries over two simulated workers, takes one
worker's running batch, and does with its tokens what an engine does in one
attention layer: pages for the groups' shared prefixes and for the requests'
own tokens (block_tables), their keys and values into the paged cache
(cache_store), attention of the prompts and then of one answered token after
the other (shared_attention), and the pages back at the end.  The layer is a
toy: queries, keys and values are random projections of random embeddings of
the token ids and positions.  Results are compared with dense attention.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_18999_amd as K  # noqa: E402
from workload import generate, small_spec  # noqa: E402

HEADS, KV_HEADS, DIM, PAGE, POOL = 16, 4, 128, 16, 4096
ANSWER = 4  # tokens of an answer (the paper's default)


def batches(min_prefix: int = 8, most: int = 24):
    """Routes a stream and returns worker 0's last queries as groups: (prefix, [own tokens])."""
    stream = generate(small_spec(n=300, groups=6, prefix_len=(40, 400), suffix_len=(5, 90), vocab=997))
    sim = K.Simulator(1, 2, 20000, stream.max_len)
    route = sim.run(stream)["route"][0]
    sim.close()
    mine = np.nonzero(route == 0)[0][-most:]
    queries = sorted(stream.tokens[int(stream.offsets[j]):int(stream.offsets[j + 1])].tolist() for j in mine)
    groups = []  # queries that share at least min_prefix tokens, neighbours in this order
    for q in queries:
        same = 0
        if groups:
            p = groups[-1][0]
            while same < min(len(p), len(q) - 1) and p[same] == q[same]:
                same += 1
        if same >= min_prefix:
            groups[-1] = (groups[-1][0][:same], groups[-1][1] + [q])
        else:
            groups.append((q[:-1], [q]))
    return [(p if len(qs) > 1 else [], [q[len(p) if len(qs) > 1 else 0:] for q in qs]) for p, qs in groups]


class Layer:
    """Random embeddings and projections, and the dense attention to compare with."""

    def __init__(self, device):
        gen = torch.Generator(device).manual_seed(1)
        shape = (1000, HEADS + 2 * KV_HEADS, DIM)
        self.embed = torch.randn(shape, generator=gen, device=device)
        self.place = torch.randn((1024, *shape[1:]), generator=gen, device=device)

    def __call__(self, tokens, positions):
        x = (self.embed[tokens.long()] + 0.5 * self.place[positions.long() % 1024]).bfloat16()
        return x.split([HEADS, KV_HEADS, KV_HEADS], 1)

    def dense(self, tokens):
        """Attention of a whole path, in 32 bits."""
        t = torch.tensor(tokens, device=self.embed.device)
        q, k, v = (x.float().transpose(0, 1) for x in self(t, torch.arange(len(t), device=t.device)))
        k, v = (x.repeat_interleave(HEADS // KV_HEADS, 0).contiguous() for x in (k, v))
        s = torch.matmul(q.contiguous(), k.transpose(1, 2).contiguous()) * DIM ** -0.5
        s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -torch.inf)
        return torch.matmul(torch.softmax(s, -1), v).transpose(0, 1)


def main(device: str = "cuda:0") -> float:
    groups = batches()
    requests = [(g, own) for g, (_, members) in enumerate(groups) for own in members]
    n = len(requests)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=device)

    layer = Layer(device)
    ring, state = K.page_ring(POOL // PAGE, device)
    k_cache = torch.zeros((POOL // PAGE, PAGE, KV_HEADS, DIM), dtype=torch.bfloat16, device=device)
    v_cache = torch.zeros_like(k_cache)

    # the groups' prefixes: pages once for each group
    prefix_length = i32([len(p) for p, _ in groups])
    prefix_table = torch.full((len(groups), 512 // PAGE), -1, dtype=torch.int32, device=device)
    held_prefix = torch.zeros_like(prefix_length)
    total = sum(len(p) for p, _ in groups)
    t = K.block_tables(held_prefix, prefix_length, prefix_table, ring, state, PAGE, total, in_place=True)
    _, k, v = layer(i32(sum((p for p, _ in groups), [])), t.positions)
    K.cache_store(k, v, k_cache, v_cache, t.slots)
    group_start = i32(np.cumsum([0] + [len(m) for _, m in groups]).tolist())
    base = i32([len(groups[g][0]) for g, _ in requests])

    # the prompts' own tokens, then the answers token by token
    held = torch.zeros(n, dtype=torch.int32, device=device)
    table = torch.full((n, 1024 // PAGE), -1, dtype=torch.int32, device=device)
    paths = [list(groups[g][0]) + list(own) for g, own in requests]
    new = [own for _, own in requests]
    worst = 0.0
    for step in range(1 + ANSWER):
        t = K.block_tables(held, i32([len(x) for x in new]), table, ring, state, PAGE, sum(map(len, new)), base=base,
                           in_place=True)
        q, k, v = layer(i32(sum(new, [])), t.positions)
        K.cache_store(k, v, k_cache, v_cache, t.slots)
        out = K.shared_attention(q, k_cache, v_cache, t.row_start, table, held, group_start, prefix_table,
                                 prefix_length)
        at = 0
        for path, x in zip(paths, new):
            want = layer.dense(path)[-len(x):]
            worst = max(worst, float((out[at:at + len(x)].float() - want).abs().max()))
            at += len(x)
        # a toy answer: the last result's largest element names the next token
        last = torch.tensor(np.cumsum([len(x) for x in new]) - 1, device=device)
        new = [[int(x)] for x in out[last].flatten(1).float().argmax(1) % 997]
        if step < ANSWER:
            for path, x in zip(paths, new):
                path += x

    # the requests end: their pages and the prefixes' go back to the ring
    K.block_tables(held, -held, table, ring, state, PAGE, 0, in_place=True)
    K.block_tables(held_prefix, -held_prefix, prefix_table, ring, state, PAGE, 0, in_place=True)
    head, tail, bits = state.tolist()
    K.check_status("block_tables", bits)
    assert tail - head == POOL // PAGE and sorted(ring.tolist()) == list(range(POOL // PAGE))
    print(f"{n} requests in {len(groups)} groups, {total} shared tokens, {head} pages used; largest difference from "
          f"dense attention {worst:.4f}")
    return worst


if __name__ == "__main__":
    main()
