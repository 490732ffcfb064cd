"""Operators that verify drafted tokens against the paged primary cache: what they compute, and cases to time them on.

A program drafts a small tree of continuations per sequence (node 0 is the last accepted token, every other node names
its parent), runs all nodes through the model in one pass and keeps the branch that the model agrees with.  Beside the
matrix products that pass consists of

- "rope":   rotary positions of queries or keys; its gradient is the same rotation backwards;
- "append": the same on a step's queries and keys, with the keys and values written into the cache's pages;
- "attend": every node attends to the cached positions and to its ancestors among the drafted nodes;
- "sample": a token per row of logits by temperature, top-k, top-p and min-p, from a given uniform number;
- "accept": the walk along the sampled tokens, and the accepted nodes' cache rows moved together in every layer.

The cache is the library's: [layers][2][pages][kv heads][16][head dim].  Shapes are those of the package's own presets.
"""
from __future__ import annotations

import math

import torch

own = False
PAGE = 16
#        layers, query heads, kv heads, head dim, vocabulary, type: the package's presets
MODELS = {"tiny": (4, 4, 4, 64, 4096, "fp32"), "1b": (16, 16, 8, 128, 32000, "bf16"), "8b": (32, 32, 8, 128, 128256, "bf16"),
          "moe": (16, 16, 4, 128, 32000, "bf16")}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed() -> list[dict]:
    return [
        # queries of long prompts into the 8B-shaped model: neighbouring elements form the pairs, the whole head turns
        {"name": "rope-prompt-8b", "kind": "rope", "model": "8b", "rows": 8192, "far": 0, "rot": 128, "interleaved": True},
        # the gradient of a training batch's queries: half of the head turns, frequencies and size set for long contexts
        {"name": "rope-gradient-1b", "kind": "rope", "model": "1b", "rows": 16 * 2048, "far": 120000, "rot": 64, "interleaved": False,
         "scaled": True, "inverse": True},
        # one user's next token, the smallest append: latency is all there is
        {"name": "append-one-1b", "kind": "append", "model": "1b", "batch": 1, "nodes": 1, "ctx": 2048},
        # full trees of a busy server
        {"name": "append-trees-8b", "kind": "append", "model": "8b", "batch": 32, "nodes": 64, "ctx": 4096, "ragged": True, "scaled": True},
        # the smallest attention: two short fp32 sequences, five nodes each
        {"name": "attend-tiny-fp32", "kind": "attend", "model": "tiny", "batch": 2, "nodes": 5, "ctx": 64},
        # a batch behind prompts of 2048, every sequence at its own length with its own number of nodes
        {"name": "attend-1b-ragged", "kind": "attend", "model": "1b", "batch": 16, "nodes": 16, "ctx": 2048, "ragged": True},
        # long documents, full trees: 256 query rows share every key
        {"name": "attend-8b-long", "kind": "attend", "model": "8b", "batch": 4, "nodes": 64, "ctx": 32768},
        # one user's next token, nucleus sampling
        {"name": "sample-one-1b", "kind": "sample", "rows": 1, "vocab": 32000, "filters": "p"},
        # the nodes of a few trees, all filters at once, each row with settings of its own
        {"name": "sample-trees-8b", "kind": "sample", "rows": 256, "vocab": 128256, "filters": "kpm"},
        # a busy server without filters: temperature alone, every token may come
        {"name": "sample-plain-8b", "kind": "sample", "rows": 64, "vocab": 128256, "filters": ""},
        # one short fp32 tree
        {"name": "accept-tiny-fp32", "kind": "accept", "model": "tiny", "batch": 1, "nodes": 5, "ctx": 64, "agree": 2},
        # full trees of a batch, five drafted tokens agreed on: rows move in 32 layers
        {"name": "accept-8b", "kind": "accept", "model": "8b", "batch": 8, "nodes": 64, "ctx": 2048, "agree": 5},
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng) -> dict:
    kind = rng.choice(["rope", "append", "attend", "attend", "sample", "sample", "accept"])
    model = rng.choice(["tiny", "1b", "8b", "moe"])
    case = {"kind": kind, "model": model}
    if kind == "rope":
        case.update(rows=_log_int(rng, 1, 8192), far=rng.choice([0, rng.randint(1, 500000)]), interleaved=rng.random() < 0.5,
                    scaled=rng.random() < 0.5, inverse=rng.random() < 0.5, rot=2 * rng.randint(1, MODELS[model][3] // 2))
    elif kind == "sample":
        case = {"kind": kind, "vocab": rng.choice([4096, 32000, 128256, _log_int(rng, 2, 131072)]), "filters": rng.choice(["", "k", "p", "m", "kp", "kpm"]),
                "type": rng.choice(["fp32", "fp32", "bf16"])}
        case["rows"] = _log_int(rng, 1, min(512, (128256 * 256) // case["vocab"]))
    else:
        case["nodes"] = rng.choice([1, rng.randint(2, 64), _log_int(rng, 2, 64)])
        batch = 32 if kind == "append" else 16
        case["batch"] = _log_int(rng, 1, batch)
        slots = {"append": 65536, "attend": 65536, "accept": 8192}[kind]
        case["ctx"] = _log_int(rng, 1, min(32768, slots // case["batch"]))
        case["ragged"] = rng.random() < 0.5
        if kind == "append":
            case.update(interleaved=rng.random() < 0.5, scaled=rng.random() < 0.5)
        if kind == "accept":
            case["agree"] = rng.randint(0, min(8, case["nodes"] - 1))
    return case


# ---- inputs -----------------------------------------------------------------------------------------------------


def _frequencies(rot: int, scaled: bool) -> tuple[list[float], float]:
    """Angles per position of the rot/2 pairs, and the factor on the rotated values.  Scaled: contexts sixteen times as
    long as the trained 8192, slow pairs slowed by all of it, fast pairs kept, a ramp over the pairs between."""
    base, pairs = 10000.0, rot // 2
    plain = [base ** (-2.0 * i / rot) for i in range(pairs)]
    if not scaled:
        return plain, 1.0
    factor, trained = 16.0, 8192

    def pair_of(turns):  # the pair that makes so many turns over the trained length
        return rot * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))

    lo, hi = max(math.floor(pair_of(32)), 0), min(math.ceil(pair_of(1)), pairs - 1)
    out = []
    for i, f in enumerate(plain):
        slow = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
        out.append(f / factor * slow + f * (1.0 - slow))
    return out, 0.1 * math.log(factor) + 1.0


def _lengths(case: dict) -> list[int]:
    B, hi = case["batch"], case["ctx"]
    if not case.get("ragged"):
        return [hi - 1] * B
    lo = max(1, hi // 16)  # spread over the contexts, in no particular order
    return [lo + (hi - lo) * ((i * 37 + 11) % B) // max(1, B - 1) - 1 for i in range(B)]


def _node_counts(case: dict) -> list[int]:
    B, N = case["batch"], case["nodes"]
    return [N if not case.get("ragged") else max(1, N - (i * 5) % (N // 2 + 1)) for i in range(B)]


def _cache(case: dict, layers: int, gen, lens, filled: bool):
    """A pool and its page table.  The pages that hold the nodes stand together at the pool's end, so that they can be
    looked at in place; those of the cached positions are scattered."""
    _, _, nkv, dh, _, kind = MODELS[case["model"]]
    B, N = case["batch"], case["nodes"]
    fresh = (N + PAGE - 2) // PAGE + 1
    old = max(lens) // PAGE
    pool = torch.empty(layers, 2, B * (old + fresh), nkv, PAGE, dh, dtype=TYPES[kind], device="cuda")
    pool.normal_(0.0, 1.0, generator=gen) if filled else pool.zero_()
    scattered = torch.randperm(B * old, generator=gen, device="cuda").view(B, old)
    table = torch.empty(B, old + fresh, dtype=torch.int64, device="cuda")
    start = torch.tensor(lens, device="cuda")[:, None] // PAGE
    col = torch.arange(old + fresh, device="cuda")[None, :]
    new = B * old + torch.arange(B, device="cuda")[:, None] * fresh
    table[:] = torch.where(col < start, torch.nn.functional.pad(scattered, (0, fresh)), new + (col - start).clamp(0, fresh - 1))
    return pool, table.to(torch.int32).contiguous(), B * old


def _random_parents(B: int, N: int, gen) -> torch.Tensor:
    i = torch.arange(N, device="cuda", dtype=torch.float32)
    u = torch.rand(B, N, generator=gen, device="cuda") ** 0.7
    p = torch.minimum((u * i).floor(), i - 1).to(torch.int32)
    p[:, 0] = -1
    return p


def prepare(case: dict, seed: int) -> dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]

    def randn(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=gen)

    if kind == "sample":
        R, V = case["rows"], case["vocab"]
        # a bulk of unlikely tokens and a few dozen likely ones a row
        z = randn(R, V) * 2.0
        few = min(V, 48)
        at = torch.randint(0, V, (R, few), generator=gen, device="cuda")
        boost = torch.empty(R, few, device="cuda").exponential_(0.5, generator=gen)
        z.scatter_add_(1, at, boost * 2.0)
        pick = torch.randint(0, 4, (4, R), generator=gen, device="cuda")
        s = {"kind": kind, "logits": z.to(TYPES[case.get("type", "fp32")]), "u": torch.rand(R, generator=gen, device="cuda"),
             "temperature": torch.tensor([0.6, 0.8, 1.0, 1.3], device="cuda")[pick[0]],
             "top_k": torch.tensor([0, 20, 50, 400], dtype=torch.int32, device="cuda")[pick[1]] if "k" in case["filters"] else None,
             "top_p": torch.tensor([0.7, 0.9, 0.95, 1.0], device="cuda")[pick[2]] if "p" in case["filters"] else None,
             "min_p": torch.tensor([0.0, 0.02, 0.05, 0.1], device="cuda")[pick[3]] if "m" in case["filters"] else None}
        return s

    layers, nq, nkv, dh, vocab, dt = MODELS[case["model"]]
    dt = TYPES[dt]
    if kind == "rope":
        f, scale = _frequencies(case["rot"], case.get("scaled", False))
        R = case["rows"]
        pos = torch.randint(0, case["far"] + 1, (R,), generator=gen, device="cuda") + torch.arange(R, device="cuda") % 2048
        return {"kind": kind, "x": randn(R, nq, dh, dtype=dt), "positions": pos.to(torch.int32), "frequencies": torch.tensor(f, dtype=torch.float64, device="cuda"),
                "scale": scale, "interleaved": case["interleaved"], "inverse": case.get("inverse", False)}

    B, N, lens, counts = case["batch"], case["nodes"], _lengths(case), _node_counts(case)
    s = {"kind": kind, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "counts": torch.tensor(counts, dtype=torch.int32, device="cuda"),
         "parents": _random_parents(B, N, gen), "status": torch.zeros(2, dtype=torch.int32, device="cuda")}
    if kind == "append":
        f, scale = _frequencies(dh, case.get("scaled", False))
        qkv = randn(B, N, (nq + 2 * nkv) * dh, dtype=dt)  # as one projection leaves them
        q, k, v = qkv.split([nq * dh, nkv * dh, nkv * dh], dim=-1)
        pool, table, first = _cache(case, 1, gen, lens, filled=False)
        depth = torch.randint(0, 12, (B, N), generator=gen, device="cuda").clamp(max=torch.arange(N, device="cuda"))
        s.update(q=q.unflatten(-1, (nq, dh)), k=k.unflatten(-1, (nkv, dh)), v=v.unflatten(-1, (nkv, dh)), cache=pool[0], table=table,
                 fresh=pool[0][:, first:], out=torch.zeros(B, N, nq, dh, dtype=dt, device="cuda"),
                 positions=(s["lens"][:, None] + depth).to(torch.int32), frequencies=torch.tensor(f, dtype=torch.float64, device="cuda"),
                 scale=scale, interleaved=case.get("interleaved", False))
    elif kind == "attend":
        pool, table, _ = _cache(case, 1, gen, lens, filled=True)
        # queries whose scores have a standard deviation of two: some keys stand out, none takes all
        s.update(q=(randn(B, N, nq, dh) * 2.0).to(dt), cache=pool[0], table=table, out=torch.zeros(B, N, nq, dh, dtype=dt, device="cuda"))
    else:
        pool, table, first = _cache(case, layers, gen, lens, filled=True)
        # distinct tokens per tree; the chain of `agree` nodes is what the model samples, the others hang where they may
        tokens = torch.rand(B, vocab, generator=gen, device="cuda").argsort(dim=1)[:, :N].contiguous()
        parents, sampled = s["parents"], torch.full((B, N), vocab, device="cuda")  # `vocab`: no node's token
        n = s["counts"].long()[:, None]
        agree = torch.clamp(n - 1, max=case["agree"])
        rank = torch.rand(B, N, generator=gen, device="cuda")
        rank[:, 0] = -1.0
        rank = torch.where(torch.arange(N, device="cuda")[None, :] < n, rank, 2.0)
        chain = rank.argsort(dim=1)[:, : case["agree"] + 1]  # the root and `agree` random nodes ...
        on = torch.arange(case["agree"] + 1, device="cuda")[None, :] <= agree
        chain = torch.where(on, chain, N).sort(dim=1).values  # ... in rising order
        above, below, both = chain[:, :-1].clamp(max=N - 1), chain[:, 1:].clamp(max=N - 1), chain[:, 1:] < N
        rows = torch.arange(B, device="cuda")[:, None].expand_as(below)
        parents[rows[both], below[both]] = above[both].to(torch.int32)
        sampled[rows[both], above[both]] = tokens[rows[both], below[both]]
        s.update(pool=pool, fresh=pool[:, :, first:], table=table, tokens=tokens.to(torch.int32), sampled=sampled.to(torch.int32), parents=parents)
    return s


# ---- the plain forms --------------------------------------------------------------------------------------------


def _rotate(x, positions, frequencies, scale, interleaved, inverse):
    """x [..., heads, dim], positions [...]: pairs (i, i + rot/2), or neighbours, turned by position * frequency."""
    rot = 2 * frequencies.numel()
    angle = positions.double()[..., None] * frequencies
    cos, sin = (angle.cos() * scale).float()[..., None, :], (angle.sin() * scale).float()[..., None, :]
    if inverse:
        sin = -sin
    turned, rest = x[..., :rot].float(), x[..., rot:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., : rot // 2], turned[..., rot // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((turned.to(x.dtype), rest), dim=-1)


def _slots(table, positions):
    """Page and slot of logical positions [B, n]."""
    return table.long().gather(1, positions // PAGE), positions % PAGE


def _append(s):
    q = _rotate(s["q"], s["positions"], s["frequencies"], s["scale"], s["interleaved"], False)
    k = _rotate(s["k"], s["positions"], s["frequencies"], s["scale"], s["interleaved"], False)
    B, N = s["positions"].shape
    node = torch.arange(N, device="cuda")[None, :]
    on = node < s["counts"][:, None]
    page, slot = _slots(s["table"], s["lens"].long()[:, None] + node.expand(B, N))
    page, slot = page[on], slot[on]
    s["cache"][0][page, :, slot] = k[on]
    s["cache"][1][page, :, slot] = s["v"][on]
    s["out"][on] = q[on]
    return s["out"], s["fresh"]


def _ancestors(parents):
    """[B, N, N]: whether the second node is the first or stands above it."""
    N = parents.shape[1]
    step = torch.arange(N, device="cuda") == parents[..., None]
    seen = step | torch.eye(N, dtype=torch.bool, device="cuda")
    for _ in range(max(1, (N - 1).bit_length())):  # paths of twice the length each time
        seen = torch.bmm(seen.float(), seen.float()) > 0
    return seen


def _attend(s):
    q, lens, counts = s["q"].float(), s["lens"].long(), s["counts"].long()
    B, N, nq, dh = q.shape
    nkv = s["cache"].shape[2]
    T = s["table"].shape[1] * PAGE
    page, slot = _slots(s["table"], torch.arange(T, device="cuda")[None, :].expand(B, T))
    key = torch.arange(T, device="cuda")[None, :] - lens[:, None]  # number among the nodes, negative for cached positions
    node = key.clamp(0, N - 1)
    sees = _ancestors(s["parents"]).gather(2, node[:, None, :].expand(B, N, T))
    sees = (key < 0)[:, None, :] | (sees & ((key >= 0) & (key < counts[:, None]))[:, None, :])
    any_key = (key < counts[:, None])[..., None, None]
    k = s["cache"][0][page, :, slot].float()                      # [B, T, nkv, dh]
    v = torch.where(any_key, s["cache"][1][page, :, slot].float(), 0.0)
    rows = q.view(B, N, nkv, nq // nkv, dh).permute(0, 2, 3, 1, 4).reshape(B, nkv, -1, dh)
    score = torch.matmul(rows, k.permute(0, 2, 3, 1)) * dh ** -0.5
    score = score.view(B, nkv, nq // nkv, N, T).masked_fill_(~sees[:, None, None], -math.inf)
    score = (score - score.amax(dim=-1, keepdim=True)).exp_()
    score = (score / score.sum(dim=-1, keepdim=True)).view(B, nkv, -1, T)
    o = torch.matmul(score, v.permute(0, 2, 1, 3)).view(B, nkv, nq // nkv, N, dh).permute(0, 3, 1, 2, 4).reshape(B, N, nq, dh)
    on = torch.arange(N, device="cuda")[None, :] < counts[:, None]
    s["out"][on] = o.to(s["out"].dtype)[on]
    return s["out"]


def _sample(s):
    # in 64 bits: which token a number falls on hangs on the last bits of sums over the vocabulary
    z = s["logits"].double()
    R, V = z.shape
    zs, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = ((zs - zs[:, :1]) / s["temperature"].double()[:, None]).exp()
    keep = torch.ones(R, V, dtype=torch.bool, device="cuda")
    rank = torch.arange(V, device="cuda")[None, :]
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        mass = (w * keep).cumsum(dim=1)
        keep &= (mass - w * keep < p * mass[:, -1:]) | (p >= 1)
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    keep[:, 0] = True
    kept = torch.zeros_like(w).scatter_(1, order, w * keep)
    mass = kept.cumsum(dim=1)
    total = mass[:, -1:]
    token = (mass <= s["u"].double()[:, None] * total).sum(dim=1, keepdim=True)
    return token[:, 0].to(torch.int32), (kept.gather(1, token) / total).log()[:, 0].float()


def _accept(s):
    tokens, parents, sampled, counts, lens = s["tokens"], s["parents"].long(), s["sampled"], s["counts"].long(), s["lens"].long()
    B, N = tokens.shape
    node = torch.arange(N, device="cuda")
    up = parents.clamp(min=0)
    agreed = (tokens == sampled.gather(1, up)) & (parents >= 0) & (node < counts[:, None])
    # of the agreed children of one node the first
    sibling = agreed[:, None, :] & agreed[:, :, None] & (parents[:, None, :] == parents[:, :, None]) & (node[None, :] < node[:, None])
    agreed &= ~sibling.any(dim=2)
    agreed[:, 0] = True
    on = ~(_ancestors(s["parents"]) & ~agreed[:, None, :]).any(dim=2) & (_ancestors(s["parents"])[:, :, 0])
    count = on.sum(dim=1)
    path = torch.where(on, node, N).sort(dim=1).values
    last = path.gather(1, count[:, None] - 1)
    follows = sampled.gather(1, last)[:, 0]
    # the rows of the accepted nodes, together behind the cached positions
    place = torch.arange(N, device="cuda")[None, :].expand(B, N)
    moves = place < count[:, None]
    page_to, slot_to = _slots(s["table"], lens[:, None] + place)
    page_from, slot_from = _slots(s["table"], lens[:, None] + path.clamp(max=N - 1))
    s["pool"][:, :, page_to[moves], :, slot_to[moves]] = s["pool"][:, :, page_from[moves], :, slot_from[moves]]
    return torch.where(path < N, path, -1).to(torch.int32), count.to(torch.int32), follows, (lens + count).to(torch.int32), s["fresh"]


def run(s):
    kind = s["kind"]
    if own:
        from paper_2608_12385_b200 import binding
        if kind == "rope":
            return binding.op_rope(s["x"], s["positions"], s["frequencies"], scale=s["scale"], interleaved=s["interleaved"], inverse=s["inverse"])
        if kind == "append":
            out = binding.op_rope_append(s["q"], s["k"], s["v"], s["positions"], s["frequencies"], s["cache"], s["table"], s["lens"],
                                         counts=s["counts"], scale=s["scale"], interleaved=s["interleaved"], out=s["out"], status=s["status"])
            return out, s["fresh"]
        if kind == "attend":
            return binding.op_attn_tree(s["q"], s["cache"], s["table"], s["lens"], s["parents"], counts=s["counts"], out=s["out"], status=s["status"])
        if kind == "sample":
            return binding.op_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        got = binding.op_tree_accept(s["tokens"], s["parents"], s["sampled"], s["pool"], s["table"], s["lens"], counts=s["counts"], status=s["status"])
        return (*got, s["fresh"])
    if kind == "rope":
        return _rotate(s["x"], s["positions"], s["frequencies"], s["scale"], s["interleaved"], s["inverse"])
    return {"append": _append, "attend": _attend, "sample": _sample, "accept": _accept}[kind](s)


# ---- what a pass cannot do without, and the same values in 64 bits ----------------------------------------------


def work(case: dict) -> dict:
    kind = case["kind"]
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (2 if case.get("type") == "bf16" else 4) + case["rows"] * 28, "flops": 4 * n}
    layers, nq, nkv, dh, _, dt = MODELS[case["model"]]
    e = 4 if dt == "fp32" else 2
    if kind == "rope":
        return {"bytes": 2 * case["rows"] * nq * dh * e + 4 * case["rows"] + 4 * case["rot"], "flops": 3 * case["rows"] * nq * case["rot"]}
    B, lens, counts = case["batch"], _lengths(case), _node_counts(case)
    n = sum(counts)
    if kind == "append":
        return {"bytes": n * (2 * (nq + 2 * nkv) * dh * e + 4) + 12 * B, "flops": 3 * n * (nq + nkv) * dh}
    if kind == "attend":
        keys = sum(t + c for t, c in zip(lens, counts))
        return {"bytes": 2 * keys * nkv * dh * e + n * (2 * nq * dh * e + 4) + 4 * (keys // PAGE) + 8 * B,
                "flops": sum(4 * c * nq * dh * (t + 1) for t, c in zip(lens, counts))}
    moved = sum(min(case["agree"], c - 1) for c in counts)
    return {"bytes": layers * 2 * moved * nkv * dh * e * 2 + 16 * n + 20 * B, "flops": n}


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(s)
    if kind == "rope":
        return _exact_turn(s["x"].double(), s["positions"], s)
    lens, counts = s["lens"].tolist(), s["counts"].tolist()
    if kind == "append":
        q, k = _exact_turn(s["q"].double(), s["positions"], s), _exact_turn(s["k"].double(), s["positions"], s)
        out, cache = s["out"].double(), s["cache"].double()
        for b, (t, n) in enumerate(zip(lens, counts)):
            out[b, :n] = q[b, :n]
            at = torch.arange(t, t + n, device="cuda")
            page = s["table"][b].long()[at // PAGE]
            cache[0, page, :, at % PAGE] = k[b, :n]
            cache[1, page, :, at % PAGE] = s["v"][b, :n].double()
        return out, cache[:, cache.shape[1] - s["fresh"].shape[1]:]
    if kind == "attend":
        nkv, dh, out = s["cache"].shape[2], s["cache"].shape[4], s["out"].double()
        for b, (t, n) in enumerate(zip(lens, counts)):
            parents = s["parents"][b].tolist()
            sees = torch.zeros(n, t + n, dtype=torch.bool)
            sees[:, :t] = True
            for i in range(n):
                j = i
                while j >= 0:
                    sees[i, t + j] = True
                    j = parents[j]
            bias = torch.zeros(n, t + n, dtype=torch.float64).masked_fill(~sees, -math.inf).cuda()
            at = torch.arange(t + n, device="cuda")
            page = s["table"][b].long()[at // PAGE]
            for h in range(nkv):
                k, v = (s["cache"][w, page, h, at % PAGE].double() for w in (0, 1))
                q = s["q"][b, :n].double().unflatten(1, (nkv, -1))[:, h]  # [n, group, dh]
                p = torch.softmax(torch.einsum("ngd,td->gnt", q, k) / math.sqrt(dh) + bias, dim=-1)
                out[b, :n].unflatten(1, (nkv, -1))[:, h] = torch.einsum("gnt,td->ngd", p, v)
        return out
    pool, path, follows = s["pool"].double(), torch.full(s["tokens"].shape, -1, dtype=torch.int32), []
    taken = []
    for b, (t, n) in enumerate(zip(lens, counts)):
        tokens, parents, sampled = (s[w][b].tolist() for w in ("tokens", "parents", "sampled"))
        walk = [0]
        while True:
            found = [c for c in range(n) if parents[c] == walk[-1] and tokens[c] == sampled[walk[-1]]]
            if not found:
                break
            walk.append(found[0])
        path[b, : len(walk)] = torch.tensor(walk, dtype=torch.int32)
        follows.append(sampled[walk[-1]])
        taken.append(len(walk))
        old = s["pool"]
        for j, c in enumerate(walk):
            to, frm = t + j, t + c
            pool[:, :, int(s["table"][b, to // PAGE]), :, to % PAGE] = old[:, :, int(s["table"][b, frm // PAGE]), :, frm % PAGE].double()
    fresh = pool[:, :, pool.shape[2] - s["fresh"].shape[2]:]
    whole = [torch.tensor(x, dtype=torch.int32) for x in (taken, follows, [t + c for t, c in zip(lens, taken)])]
    return path, *whole, fresh


def _exact_turn(x, positions, s):
    pairs = s["frequencies"].numel()
    angle = positions.double()[..., None, None] * s["frequencies"] * (-1.0 if s.get("inverse") else 1.0)
    first = torch.arange(pairs, device="cuda") * (2 if s["interleaved"] else 1)
    second = first + (1 if s["interleaved"] else pairs)
    turned = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(angle, s["scale"]), angle)
    out = x.clone()
    out[..., first], out[..., second] = turned.real, turned.imag
    return out


def _exact_sample(s):
    """Row by row: candidates taken in falling order, then the number counted off in the order of the token ids."""
    import numpy as np
    z = s["logits"].double().cpu().numpy()
    named = {k: None if s[k] is None else s[k].double().cpu().numpy() for k in ("u", "temperature", "top_k", "top_p", "min_p")}
    tokens, logs = [], []
    for r in range(z.shape[0]):
        row = z[r]
        order = np.argsort(-row, kind="stable")
        w = np.exp((row[order] - row[order[0]]) / named["temperature"][r])
        n = len(w)
        if named["top_k"] is not None and named["top_k"][r] > 0:
            n = min(n, int(named["top_k"][r]))
        if named["top_p"] is not None and named["top_p"][r] < 1:
            run_ = np.cumsum(w[:n])
            n = min(n, int(np.searchsorted(run_, named["top_p"][r] * run_[-1], side="left")) + 1)
        if named["min_p"] is not None:
            n = max(1, min(n, int((w >= named["min_p"][r]).sum())))
        at = np.argsort(order[:n])
        run_ = np.cumsum(w[:n][at])
        k = min(n - 1, int(np.searchsorted(run_, named["u"][r] * run_[-1], side="right")))
        tokens.append(int(order[:n][at[k]]))
        logs.append(math.log(w[:n][at[k]] / run_[-1]))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)
