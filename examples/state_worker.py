"""A worker whose layer keeps a state in the place of a cache, on one GPU.

    python examples/state_worker.py

Takes the groups of routed queries of shared_prefix_worker.py and answers them
through a layer of linear attention, from residual to residual: a norm whose
result leaves in 8-bit integers (block_norm), the projections (integer_product),
linear attention over a pool of states (linear_attention), the norm of its
result with a gate, the projection back and the residual.  A group's prefix
goes through the layer once and leaves its state in a slot, with which all of
the group's requests begin; a request's own state then stays in its slot, token
by token.  The layer is a toy (random weights and embeddings).  Results are
compared with linear attention over each whole path, in 64 bits.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2601_18999_amd as K  # noqa: E402
from shared_prefix_worker import batches  # noqa: E402

HEADS, DIM = 8, 128
WIDTH = HEADS * DIM
ANSWER = 4  # tokens of an answer (the paper's default)


class Layer:
    def __init__(self, device):
        gen = torch.Generator(device).manual_seed(1)

        def weight(channels, width):  # 8-bit, with a scale for each channel
            w = torch.randn((channels, width), generator=gen, device=device) * width ** -0.5
            scale = w.abs().amax(1) / 127
            return (w / scale[:, None]).round().to(torch.int8), scale

        self.embed = torch.randn((1000, WIDTH), generator=gen, device=device).bfloat16()
        self.up, self.down = weight(4 * WIDTH, WIDTH), weight(WIDTH, WIDTH)
        self.before, self.after = torch.ones((2, WIDTH), dtype=torch.bfloat16, device=device)
        self.log_decay = -torch.exp2(-2.0 - torch.arange(HEADS, device=device, dtype=torch.float32) / 2)

    def projections(self, tokens):
        """(residual, queries, keys, values, gate) of the tokens."""
        residual = self.embed[tokens.long()]
        n = K.block_norm(residual, before=self.before, int8=True)
        x = K.integer_product(n.out, *self.up, x_scale=n.scale)
        q, k, v, gate = x.split(WIDTH, 1)
        return residual, *(y.unflatten(1, (HEADS, DIM)) for y in (q, k, v)), gate

    def __call__(self, tokens, pool, read, write, row_start):
        residual, q, k, v, gate = self.projections(tokens)
        o = K.linear_attention(q, k, v, pool, self.log_decay, read, write, row_start)
        n = K.block_norm(o.flatten(1), after=self.after, gate=gate, activation="silu", int8=True)
        y = K.integer_product(n.out, *self.down, x_scale=n.scale)
        return o, K.block_norm(y, residual=residual, before=self.before)

    def whole(self, tokens):
        """Linear attention over a whole path from nothing, in 64 bits."""
        t = torch.tensor(tokens, device=self.embed.device)
        q, k, v = (x.double().transpose(0, 1).contiguous() for x in self.projections(t)[1:4])
        i = torch.arange(len(t), device=t.device)
        decay = torch.exp(self.log_decay.double()[:, None, None] * (i[:, None] - i).clamp(min=0)).tril()
        score = torch.matmul(q, k.transpose(1, 2).contiguous()) * decay * DIM ** -0.5
        return torch.matmul(score, v).transpose(0, 1)


def main(device: str = "cuda:0") -> float:
    groups = batches()
    requests = [(g, own) for g, (_, members) in enumerate(groups) for own in members]
    n, layer = len(requests), Layer(device)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=device)

    def starts(lists):
        return i32(np.cumsum([0] + [len(x) for x in lists]).tolist())

    # the prefixes, from nothing, into the first slots; the requests' slots stand behind these
    pool = torch.empty((len(groups) + n, HEADS, DIM, DIM), device=device)
    prefixes = [p for p, _ in groups]
    slots = torch.arange(len(groups), dtype=torch.int32, device=device)
    layer(i32(sum(prefixes, [])), pool, torch.full_like(slots, -1), slots, starts(prefixes))

    read = i32([g for g, _ in requests])
    mine = torch.arange(len(groups), len(groups) + n, dtype=torch.int32, device=device)
    paths = [list(groups[g][0]) + list(own) for g, own in requests]
    new = [list(own) for _, own in requests]
    worst = 0.0
    for step in range(1 + ANSWER):
        single = all(len(x) == 1 for x in new)
        o, out = layer(i32(sum(new, [])), pool, read, mine, None if single else starts(new))
        read = mine
        at = 0
        for path, x in zip(paths, new):
            want = layer.whole(path)[-len(x):]
            worst = max(worst, float((o[at:at + len(x)].double() - want).abs().max() / want.abs().max()))
            at += len(x)
        # a toy answer: the last result's largest element names the next token
        last = torch.tensor(np.cumsum([len(x) for x in new]) - 1, device=device)
        new = [[int(x)] for x in out.out[last].float().argmax(1) % 997]
        if step < ANSWER:
            for path, x in zip(paths, new):
                path += x
    print(f"{n} requests in {len(groups)} groups, {sum(map(len, prefixes))} shared tokens; largest difference from whole "
          f"paths {worst:.5f} of the largest result")
    return worst


if __name__ == "__main__":
    main()
