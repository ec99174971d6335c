"""More serving operators whose speed is measured: what stands around a worker's attention in a layer, and the
attention of layers that keep a state in the place of a cache.

``run`` computes an operator in its plain form (elementary torch operations, 32-bit arithmetic, one rounding at the
end) or, where ``own`` is true, by the call that a user of this package makes.

  norm     a = x, normalised and weighted (`after`), gated; r = residual + c a; n = r, normalised and weighted
           (`before`).  Each part can be left out.  Out: n, and r where there is a residual.
  product  out[t][n] = sx[t] sw[n] sum_k xq[t][k] wq[n][k] + bias[n] over 8-bit integers.  Tokens of 16 bits are
           brought to integers first: sx = max |x| / 127, xq = x * (127 / max |x|) rounded.
  project  the two one behind the other, as a layer has them: the norm's result in 8-bit integers with a scale for
           each token goes into the product.  Out: the product and r.
  linear   S_t = e^g S_(t-1) + k_t v_t^T, out_t = scale q_t S_t for each new token of ragged requests, g of each key
           head; the state before a request's first token stands in a slot of a pool (or is 0), the state behind its
           last one goes to another slot (or nowhere).

Sizes and lengths follow from the case alone; values, slots and decays follow from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4, "int8": 1}
EPS = 1e-6

# residual, gate: "" = none; gate "token": a value for each token and channel, "channel": the same for all tokens;
# sliced: x (or q, k and v) are slices of wider rows
NORM = {"op": "norm", "tokens": 64, "dim": 4096, "dtype": "bf16", "residual": "bf16", "after": False, "gate": "",
        "activation": "none", "before": True, "sliced": False}
PRODUCT = {"op": "product", "tokens": 64, "dim": 4096, "channels": 4096, "dtype": "int8", "out": "bf16", "bias": False}
PROJECT = {"op": "project", "tokens": 64, "dim": 4096, "channels": 6144, "dtype": "bf16", "residual": "bf16",
           "after": False, "gate": "", "activation": "none", "before": True, "sliced": False, "out": "bf16",
           "bias": False}
# groups: that many states are read by the requests in turn, 0: every request begins with nothing, -1: each reads a
# state of its own
LINEAR = {"op": "linear", "requests": 64, "groups": -1, "new_lo": 1, "new_hi": 1, "heads": 32, "kv_heads": 32,
          "dim": 128, "dtype": "bf16", "sliced": True, "unkept": 0.0}


def _case(base, **kw):
    c = dict(base)
    for k, v in kw.items():
        if k != "name" and k not in c:
            raise KeyError(k)
        c[k] = v
    return c


def listed():
    return [
        # between two blocks of a layer, for the next tokens of eight requests: latency
        _case(NORM, name="norm_answer", tokens=8),
        # the same for a long prompt, with everything: the block's result normalised and gated, a 32-bit residual
        _case(NORM, name="norm_prompt", tokens=9216, residual="fp32", after=True, gate="token", activation="silu"),
        # odd sizes: rows that fill no vector, one gate for all tokens, x a slice
        _case(NORM, name="norm_odd", tokens=777, dim=5003, dtype="fp16", residual="fp16", after=True, gate="channel",
              activation="sigmoid", sliced=True),
        # projections to queries, keys and values (64 heads in all, of 128) for the next tokens of eight requests
        _case(PRODUCT, name="product_answer", tokens=8, channels=8192, dtype="bf16"),
        # a burst of the long-prompt workload answers: 256 tokens
        _case(PRODUCT, name="product_burst", tokens=256, channels=16384),
        # its longest prompt into a layer's wide middle, tokens of 16 bits
        _case(PRODUCT, name="product_prompt", tokens=9216, channels=16384, dtype="bf16"),
        # odd sizes, a bias, 32-bit results
        _case(PRODUCT, name="product_odd", tokens=333, dim=5008, channels=1001, out="fp32", bias=True),
        # residual, norm and projection of a mid-sized prompt
        _case(PROJECT, name="project_prompt", tokens=2048, channels=8192),
        # one token of each of 64 requests: 64 states of 2 MB, each read and written
        _case(LINEAR, name="linear_answer"),
        # the long-prompt workload's prompts: 16 requests of 128 to 1,024 tokens behind the states of three prefixes
        _case(LINEAR, name="linear_prompt", requests=16, groups=3, new_lo=128, new_hi=1024),
        # its longest prompt on a worker that has nothing of it
        _case(LINEAR, name="linear_cold", requests=1, groups=0, new_lo=9216, new_hi=9216),
        # odd everything: three query heads to a key head, narrow heads, requests of 0 to 77 tokens, some not kept
        _case(LINEAR, name="linear_odd", requests=33, groups=7, new_lo=0, new_hi=77, heads=15, kv_heads=5, dim=64,
              dtype="fp16", sliced=False, unkept=0.2),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _range(rng, lo, hi):
    a, b = sorted((_log(rng, max(1, lo), hi), _log(rng, max(1, lo), hi)))
    return (0 if lo == 0 and rng.random() < 0.25 else a), b


def _draw_norm(rng, base=NORM):
    dim = _log(rng, 64, 16384)
    c = _case(base, tokens=_log(rng, 1, 16384), dim=rng.choice([dim, -(-dim // 64) * 64]),
              dtype=rng.choice(["bf16", "fp16"]), after=rng.random() < 0.5, gate=rng.choice(["", "token", "channel"]),
              before=rng.random() < 0.75, sliced=rng.random() < 0.3)
    c["activation"] = rng.choice(["none", "sigmoid", "silu"]) if c["gate"] else "none"
    c["residual"] = rng.choice(["", c["dtype"], "fp32"])
    return c


def _draw_product(rng, base=PRODUCT):
    c = _case(base, tokens=_log(rng, 1, 16384), dim=16 * _log(rng, 4, 1024), channels=_log(rng, 64, 16384),
              dtype=rng.choice(["int8", "bf16", "fp16"]), bias=rng.random() < 0.3)
    if rng.random() < 0.5:
        c["channels"] = -(-c["channels"] // 64) * 64
    c["out"] = rng.choice(["bf16", "fp16", "fp32"]) if c["dtype"] == "int8" else c["dtype"]
    return c


def _draw_project(rng):
    c = _draw_norm(rng, _draw_product(rng, PROJECT))
    c["dim"] = -(-c["dim"] // 16) * 16
    c["out"] = c["dtype"]
    return c


def _draw_linear(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 16, 32])
    c = _case(LINEAR, heads=kv * rng.choice([1, 1, 2, 3, 4]), kv_heads=kv, dim=rng.choice([64, 128]),
              dtype=rng.choice(["bf16", "bf16", "fp16"]), sliced=rng.random() < 0.5, unkept=rng.choice([0.0, 0.2]))
    if rng.random() < 0.5:
        c["requests"] = _log(rng, 1, 256)
        c["new_lo"], c["new_hi"] = rng.choice([(1, 1), (1, 1), (0, 3), (4, 4)])
    else:
        c["requests"] = _log(rng, 1, 32)
        c["new_lo"], c["new_hi"] = _range(rng, 0, 9216)
    c["groups"] = rng.choice([-1, 0, _log(rng, 1, c["requests"])])
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 400.0)


def _plain_gb(c):
    """GB that the plain form of a linear case holds: padded tokens, scores and states."""
    if c["op"] != "linear":
        return 0.0
    chunk, count = _chunks(c)
    rows = c["requests"] * chunk * count * 4e-9
    return rows * (3 * c["heads"] + 2 * c["kv_heads"]) * c["dim"] + \
        rows * 2 * c["heads"] * chunk + 3 * c["requests"] * count * c["kv_heads"] * c["dim"] ** 2 * 4e-9


def draw(rng):
    most = max(_cost(c) for c in listed())
    make = rng.choice([_draw_norm, _draw_product, _draw_project, _draw_linear, _draw_linear])
    while True:
        c = make(rng)
        if (c["op"] != "linear" or sum(_new(c))) and _cost(c) <= most and _plain_gb(c) <= 30.0:
            return c


# ---------------------------------------------------------------- lengths, inputs


def _new(c):
    """New tokens of each request, the same for every seed."""
    lo, hi = c["new_lo"], c["new_hi"]
    return [lo + (((i + 1) * 2654435761 + 40503) % (1 << 32) * (hi - lo + 1) >> 32) for i in range(c["requests"])]


def _chunks(c):
    """Tokens of a chunk of the plain form, and chunks of the longest request."""
    most = max(max(_new(c)), 1)
    chunk = min(64, most)
    return chunk, -(-most // chunk)


def _ahead(counts):
    out = [0]
    for v in counts:
        out.append(out[-1] + v)
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _randn(gen, shape, dtype="fp32"):
    return torch.randn(shape, generator=gen, device=DEV, dtype=DTYPES[dtype])


def _rows(gen, rows, dim, dtype, sliced=False):
    """[rows, dim] of hidden values: some channels are larger than the others; a slice of wider rows if asked."""
    x = _randn(gen, (rows, dim + 64 if sliced else dim), dtype)[:, :dim]
    return x.mul_((torch.rand(dim, generator=gen, device=DEV) < 0.01).to(x.dtype) * 9 + 1)


def _weights(gen, dim, dtype):
    return (1.0 + 0.2 * _randn(gen, (dim,))).to(DTYPES[dtype])


def _prepare_norm(c, gen):
    t, d, kind = c["tokens"], c["dim"], c["dtype"]
    gate = None
    if c["gate"]:
        gate = _randn(gen, (t if c["gate"] == "token" else 1, d), kind).expand(t, d)
    return {"x": _rows(gen, t, d, kind, c["sliced"]), "after": _weights(gen, d, kind) if c["after"] else None,
            "gate": gate, "activation": c["activation"],
            "residual": _rows(gen, t, d, c["residual"]) if c["residual"] else None, "residual_scale": 0.70703125,
            "before": _weights(gen, d, kind) if c["before"] else None}


def _prepare_product(c, gen, tokens=True):
    k, n = c["dim"], c["channels"]
    s = {"weight": (_randn(gen, (n, k)) * 32.0).round_().clamp_(-127, 127).to(torch.int8),
         "weight_scale": (torch.rand(n, generator=gen, device=DEV) + 0.5) / (32.0 * math.sqrt(k)),
         "bias": _randn(gen, (n,)) if c["bias"] else None, "out": DTYPES[c["out"]]}
    if tokens:
        s["x"] = _rows(gen, c["tokens"], k, c["dtype"] if c["dtype"] != "int8" else "fp32")
        s["x_scale"] = None
        if c["dtype"] == "int8":
            s["x_scale"] = s["x"].abs().amax(1) / 127.0
            s["x"] = (s["x"] / s["x_scale"][:, None]).round_().to(torch.int8)
    return s


def _prepare_project(c, gen):
    return dict(_prepare_norm(c, gen), **_prepare_product(c, gen, False))


def _prepare_linear(c, gen):
    n, heads, kv, d, groups = c["requests"], c["heads"], c["kv_heads"], c["dim"], c["groups"]
    new = _new(c)
    tokens = sum(new)
    sizes = (heads, kv, kv)
    if c["sliced"]:
        q, k, v = _randn(gen, (tokens, heads + 2 * kv, d), c["dtype"]).split(sizes, 1)
    else:
        q, k, v = (_randn(gen, (tokens, h, d), c["dtype"]) for h in sizes)
    before = n if groups < 0 else groups
    slots = torch.randperm(before + n + 1, generator=gen, device=DEV).to(torch.int32)
    of = torch.arange(n, device=DEV)
    write = slots[before:before + n].clone()
    if c["unkept"]:
        write[torch.rand(n, generator=gen, device=DEV) < c["unkept"]] = -1
    # decays of heads that look back over a few to some hundreds of tokens; the first forgets nothing
    log_decay = -torch.exp2(-1.0 - 8.0 * torch.rand(kv, generator=gen, device=DEV))
    log_decay[0] = 0.0
    return {"q": q, "k": k, "v": v, "state": _randn(gen, (before + n + 1, kv, d, d)), "log_decay": log_decay,
            "read": slots[of % groups if groups > 0 else of] if groups else torch.full_like(write, -1),
            "write": write, "row_start": _i32(_ahead(new)) if new != [1] * n else None, "scale": d ** -0.5,
            "chunk": _chunks(c)}


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(int(seed) & 0x7FFFFFFF)
    make = {"norm": _prepare_norm, "product": _prepare_product, "project": _prepare_project,
            "linear": _prepare_linear}[case["op"]]
    return dict(make(case, gen), op=case["op"])


# ---------------------------------------------------------------- the plain forms


def _normalised(a, weight):
    return a * torch.rsqrt(a.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _norm32(s):
    """n and r in 32 bits."""
    a = s["x"].float()
    if s["after"] is not None:
        a = _normalised(a, s["after"])
    if s["gate"] is not None:
        g = s["gate"].float()
        if s["activation"] != "none":
            g = (g if s["activation"] == "silu" else 1.0) / (1.0 + torch.exp(-g))
        a = a * g
    if s["residual"] is not None:
        a = s["residual"].float() + s["residual_scale"] * a
    return a if s["before"] is None else _normalised(a, s["before"]), a


def _with_residual(s, out, r):
    return [out] if s["residual"] is None else [out, r.to(s["residual"].dtype)]


def _plain_norm(s):
    n, r = _norm32(s)
    return _with_residual(s, n.to(s["x"].dtype), r)


def _integers(x):
    """x in 8-bit integers, as floats, and the scale of each row."""
    top = x.abs().amax(1, keepdim=True)
    return (x * (127.0 / top)).round(), top / 127.0


def _multiplied(s, xq, scale):
    out = torch.matmul(xq, s["weight"].float().t()) * scale * s["weight_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    return out.to(s["out"])


def _plain_product(s):
    if s["x_scale"] is not None:
        return [_multiplied(s, s["x"].float(), s["x_scale"][:, None])]
    return [_multiplied(s, *_integers(s["x"].float()))]


def _plain_project(s):
    n, r = _norm32(s)
    return _with_residual(s, _multiplied(s, *_integers(n)), r)


def _plain_linear(s):
    q, k, v, g = s["q"], s["k"], s["v"], s["log_decay"]
    (tokens, heads, d), kv = q.shape, k.shape[1]
    n, (chunk, count), share = s["read"].numel(), s["chunk"], heads // kv
    rs = torch.arange(n + 1, device=DEV) if s["row_start"] is None else s["row_start"].long()
    new = rs[1:] - rs[:-1]
    # token i of chunk c of each request, 0 behind its last
    at = torch.arange(chunk * count, device=DEV)
    there = at < new[:, None]
    place = (rs[:-1, None] + at).clamp(max=tokens - 1)

    def chunked(x):
        x = torch.where(there[:, :, None, None], x[place].float(), 0.0)
        return x.view(n, count, chunk, kv, -1, d).permute(0, 3, 1, 4, 2, 5)  # [n, kv, count, share, chunk, d]

    qs = chunked(q).reshape(n, kv, count, share * chunk, d)
    ks, vs = chunked(k)[:, :, :, 0].contiguous(), chunked(v)[:, :, :, 0].contiguous()
    i = torch.arange(chunk, device=DEV)
    # within a chunk
    apart = i[:, None] - i
    decay = torch.where(apart >= 0, torch.exp(g[:, None, None] * apart.clamp(min=0)), 0.0)[:, None, None]
    score = torch.matmul(qs, ks.transpose(3, 4).contiguous()).view(n, kv, count, share, chunk, chunk).mul_(decay)
    out = torch.matmul(score.view(n, kv, count, share * chunk, chunk), vs).view(n, kv, count, share, chunk, d)
    # what each chunk adds to the state, the states before the chunks, and what they add to the results
    full = (new[:, None] - torch.arange(count, device=DEV) * chunk).clamp(0, chunk)  # [n, count] tokens
    left = (full[:, :, None] - 1 - i).clamp(min=0)[:, None]
    weight = torch.exp(g[:, None, None] * left)
    added = torch.matmul((ks * weight[..., None]).transpose(3, 4).contiguous(), vs)
    c = torch.arange(count, device=DEV)
    back = c[:, None] - 1 - c
    step = torch.where(back >= 0, torch.exp(g[:, None, None] * (chunk * back).clamp(min=0)), 0.0)
    start = torch.where((s["read"] >= 0)[:, None, None, None], s["state"][s["read"].long().clamp(min=0)], 0.0)
    before = torch.matmul(step, added.view(n, kv, count, d * d)).view(n, kv, count, d, d)
    before = before + torch.exp(g[:, None] * (chunk * c))[..., None, None] * start[:, :, None]
    reach = torch.exp(g[:, None] * (i + 1))[:, None, None, :, None]
    out = out + torch.matmul(qs, before).view(n, kv, count, share, chunk, d) * reach
    out = (out * s["scale"]).permute(0, 2, 4, 1, 3, 5).reshape(n, count * chunk, heads, d)
    # the state behind each request's last token
    last = ((new - 1) // chunk).clamp(min=0)
    pick = torch.arange(n, device=DEV)
    end = torch.exp(g * full[pick, last][:, None])[..., None, None] * before[pick, :, last] + added[pick, :, last]
    state, kept = s["state"], s["write"] >= 0
    state[s["write"][kept].long()] = end[kept]
    t = torch.arange(tokens, device=DEV)
    row = torch.searchsorted(rs, t, right=True) - 1
    return [out[row, t - rs[row]].to(q.dtype), state]


def _own_norm(K, s, int8=False):
    return K.block_norm(s["x"], after=s["after"], gate=s["gate"], activation=s["activation"], residual=s["residual"],
                        residual_scale=s["residual_scale"], before=s["before"], eps=EPS, int8=int8)


def _own_block_norm(K, s):
    r = _own_norm(K, s)
    return [r.out] if s["residual"] is None else [r.out, r.residual]


def _own_product(K, s):
    return [K.integer_product(s["x"], s["weight"], s["weight_scale"], x_scale=s["x_scale"], bias=s["bias"],
                              dtype=s["out"])]


def _own_project(K, s):
    r = _own_norm(K, s, int8=True)
    out = K.integer_product(r.out, s["weight"], s["weight_scale"], x_scale=r.scale, bias=s["bias"], dtype=s["out"])
    return [out] if s["residual"] is None else [out, r.residual]


def _own_linear(K, s):
    out = K.linear_attention(s["q"], s["k"], s["v"], s["state"], s["log_decay"], s["read"], s["write"], s["row_start"],
                             scale=s["scale"])
    return [out, s["state"]]


PLAIN = {"norm": _plain_norm, "product": _plain_product, "project": _plain_project, "linear": _plain_linear}
OWN = {"norm": _own_block_norm, "product": _own_product, "project": _own_project, "linear": _own_linear}


def run(state):
    if own:
        import paper_2601_18999_amd as K
        return OWN[state["op"]](K, state)
    return PLAIN[state["op"]](state)


# ---------------------------------------------------------------- the work, and the definition in 64 bits


def _norm_bytes(c):
    t, d, size = c["tokens"], c["dim"], SIZES[c["dtype"]]
    b = t * d * size + d * size * (c["after"] + c["before"])
    b += {"": 0, "channel": d * size, "token": t * d * size}[c["gate"]]
    return b + (2 * t * d * SIZES[c["residual"]] if c["residual"] else 0)


def work(case):
    """Bytes: every input and output once.  Flops: the products; of linear attention the recurrent form's, which are
    the fewest: dim * dim products and sums for each token's key and value, and as many for each of its queries."""
    c = case
    if c["op"] == "norm":
        out = c["tokens"] * c["dim"] * SIZES[c["dtype"]]
        return {"bytes": float(_norm_bytes(c) + out), "flops": 12.0 * c["tokens"] * c["dim"]}
    if c["op"] in ("product", "project"):
        m, k, n = c["tokens"], c["dim"], c["channels"]
        b = n * (k + 4 + 4 * c["bias"]) + m * n * SIZES[c["out"]]
        if c["op"] == "project":
            b += _norm_bytes(c)
        else:
            b += m * k * SIZES[c["dtype"]] + (4 * m if c["dtype"] == "int8" else 0)
        return {"bytes": float(b), "flops": 2.0 * m * n * k}
    n, tokens, kv, heads, d = c["requests"], sum(_new(c)), c["kv_heads"], c["heads"], c["dim"]
    states = (n if c["groups"] < 0 else min(c["groups"], n)) + n * (1.0 - c["unkept"])
    b = 4.0 * tokens * (heads + kv) * d + 4.0 * states * kv * d * d + 12 * n
    return {"bytes": b, "flops": 2.0 * tokens * (heads + kv) * d * d}


def _exact_rows(s):
    """n and r in 64 bits."""
    a = s["x"].double()
    d = a.shape[1]
    if s["after"] is not None:
        a = a / ((a * a).sum(1, keepdim=True) / d + EPS).sqrt() * s["after"].double()
    if s["gate"] is not None:
        g = s["gate"].double()
        a = a * {"none": g, "sigmoid": torch.sigmoid(g), "silu": g * torch.sigmoid(g)}[s["activation"]]
    if s["residual"] is not None:
        a = a * s["residual_scale"] + s["residual"].double()
    n = a
    if s["before"] is not None:
        n = a / ((a * a).sum(1, keepdim=True) / d + EPS).sqrt() * s["before"].double()
    return n, a


def _exact_norm(c, s):
    return [x for x in _exact_rows(s)][:1 if s["residual"] is None else 2]


def _exact_scaled(s, q, scale):
    out = (q @ s["weight"].double().t().contiguous()) * (scale[:, None] * s["weight_scale"].double())
    return out if s["bias"] is None else out + s["bias"].double()


def _exact_integers(x):
    scale = x.abs().max(1).values / 127.0
    return torch.round(x / scale[:, None]), scale


def _exact_product(c, s):
    if s["x_scale"] is not None:
        return [_exact_scaled(s, s["x"].double(), s["x_scale"].double())]
    return [_exact_scaled(s, *_exact_integers(s["x"].double()))]


def _exact_project(c, s):
    n, r = _exact_rows(s)
    out = _exact_scaled(s, *_exact_integers(n))
    return [out] if s["residual"] is None else [out, r]


def _exact_linear(c, s):
    """All pairs of a request's tokens, head by head."""
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    state, share, at = s["state"].double(), c["heads"] // c["kv_heads"], 0
    first = state.clone()
    read, write = s["read"].tolist(), s["write"].tolist()
    g = s["log_decay"].double().tolist()
    for r, n in enumerate(_new(c)):
        to = torch.arange(at, at + n, device=DEV)
        for h in range(c["kv_heads"]):
            k, v = s["k"][to, h].double(), s["v"][to, h].double()
            s0 = first[read[r], h] if read[r] >= 0 else torch.zeros_like(first[0, 0])
            p = torch.exp(((to[:, None] - to) * g[h]).clamp(max=0.0)).tril()
            ahead = torch.exp((to - at + 1) * g[h])[:, None]
            for i in range(h * share, h * share + share):
                q = s["q"][to, i].double() * s["scale"]
                out[to, i] = ((q @ k.t().contiguous()) * p) @ v + ahead * (q @ s0)
            if write[r] >= 0:
                left = torch.exp((at + n - 1 - to) * g[h])[:, None]
                state[write[r], h] = math.exp(n * g[h]) * s0 + (k * left).t().contiguous() @ v
        at += n
    return [out, state]


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "project": _exact_project,
            "linear": _exact_linear}[case["op"]](case, s)
