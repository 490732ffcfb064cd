"""Plain 64-bit forms of the operators for sampled and drafted tokens, on the CPU, one value after the other where that is the
clearest way to write them."""
from __future__ import annotations

import math

import numpy as np
import torch


def rotate(x: torch.Tensor, positions: torch.Tensor, freq: torch.Tensor, scale: float, interleaved: bool, inverse: bool) -> torch.Tensor:
    """x [..., heads, dim] float64, positions [...]."""
    pairs = freq.numel()
    y = x.clone()
    angle = positions.double()[..., None] * freq.double()
    if inverse:
        angle = -angle
    c, s = scale * torch.cos(angle), scale * torch.sin(angle)
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        y[..., a] = x[..., a] * c[..., None, i] - x[..., b] * s[..., None, i]
        y[..., b] = x[..., a] * s[..., None, i] + x[..., b] * c[..., None, i]
    return y


def tree_sees(parents, n: int) -> torch.Tensor:
    sees = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = int(parents[j])
    return sees


def cache_rows(plane: torch.Tensor, table, t0: int, t1: int) -> torch.Tensor:
    """Positions t0..t1-1 of one sequence: [t, kv heads, dim] of a plane [pages, kv heads, 16, dim]."""
    at = torch.arange(t0, t1)
    return plane[torch.as_tensor(table).long()[at // 16], :, at % 16]


def tree_attention(q, cache, table, lens, parents, counts, scale: float):
    """q [B, N, nq, D]; returns (out, bound factors): out float64 [B, N, nq, D] (zeros where a node does not count), the sum of
    p |v| of every output element, and per (B, N, nq) the largest sum |q_d k_d| * scale over visible keys."""
    B, N, nq, D = q.shape
    nkv = cache.shape[2]
    G = nq // nkv
    out, pv, qk = torch.zeros(B, N, nq, D, dtype=torch.float64), torch.zeros(B, N, nq, D, dtype=torch.float64), torch.zeros(B, N, nq, dtype=torch.float64)
    for b in range(B):
        t, n = int(lens[b]), int(counts[b])
        if n == 0:
            continue
        k = cache_rows(cache[0].double(), table[b], 0, t + n)
        v = cache_rows(cache[1].double(), table[b], 0, t + n)
        sees = torch.cat([torch.ones(n, t, dtype=torch.bool), tree_sees(parents[b], n)], dim=1)
        for i in range(n):
            on = sees[i]
            for h in range(nq):
                kk, vv, qq = k[on][:, h // G], v[on][:, h // G], q[b, i, h].double()
                p = torch.softmax((kk * qq).sum(-1) * scale, dim=0)
                out[b, i, h] = (p[:, None] * vv).sum(0)
                pv[b, i, h] = (p[:, None] * vv.abs()).sum(0)
                qk[b, i, h] = (kk * qq).abs().sum(-1).max() * scale
    return out, pv, qk


def sample_row(z: np.ndarray, u: float, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row in 64 bits: (token, log-probability, margin).  margin: how far, in shares of the remaining mass, the nearest
    decision (a border of top-p or min-p, the running sum that u falls on) is from going the other way."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    top = z.max()
    if top == -np.inf:
        return -1, -np.inf, 1.0
    if not temperature > 0:
        return int(np.argmax(z)), 0.0, 1.0
    order = np.argsort(-z, kind="stable")
    if top == np.inf:
        w = (z[order] == np.inf).astype(np.float64)
    else:
        with np.errstate(invalid="ignore"):
            w = np.exp((z[order] - top) / float(temperature))
        w[z[order] == -np.inf] = 0.0
    n, margin = len(w), 1.0
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        sums = np.cumsum(w[:n])
        total = sums[-1]
        margin = min(margin, float(np.min(np.abs(sums - top_p * total)) / total))
        n = min(n, 1 + int((sums < top_p * total).sum()))  # the mass before a token is below top_p of the whole
    if min_p > 0:
        margin = min(margin, float(np.min(np.abs(w - min_p))))
        n = max(1, min(n, int((w >= min_p).sum())))
    ids = np.sort(order[:n])
    place = np.empty(len(w), dtype=np.int64)
    place[order] = np.arange(len(w))
    kept = w[place[ids]]
    sums = np.cumsum(kept)
    total = sums[-1]
    margin = min(margin, float(np.min(np.abs(sums[:-1] - u * total)) / total) if n > 1 else 1.0)
    at = int(np.searchsorted(sums, u * total, side="right"))
    at = min(at, int(np.max(np.nonzero(kept > 0))))
    return int(ids[at]), math.log(kept[at] / total), margin


def accept(tokens, parents, sampled, n: int):
    """(path, token sampled at its end) of one sequence with n nodes."""
    if n == 0:
        return [], -1
    path = [0]
    while True:
        cur = path[-1]
        nxt = [c for c in range(n) if int(parents[c]) == cur and int(tokens[c]) == int(sampled[cur])]
        if not nxt:
            return path, int(sampled[cur])
        path.append(nxt[0])
