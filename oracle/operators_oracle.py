"""The operators on a caller's tensors written out plainly in 64 bits (NumPy only, no code of the library): attention of tree rows over a
cache, drawing of tokens, moves of cached rows.  Test infrastructure."""
from __future__ import annotations

import numpy as np

WEIGHT_ONE = 2.0 ** 38


def tree_masks(parent):
    """[n] parents of rows 1 .. n -> n + 1 masks as Python integers."""
    masks = [1]
    for i, p in enumerate(parent, start=1):
        masks.append(masks[p] | 1 << i if 0 <= p < i and masks[p] else 0)
    return masks


def tree_attention(q, k, v, cached, masks, rows, scale):
    """q [B,T,H,d], k / v [B,Hkv,cap,d] (float64), masks [B][T], rows [B] -> out, and per output the sum of p |v| and the largest
    sum |q_i k_i| scale among the keys seen (what rounding errors are relative to).  Rows beyond rows[b] are NaN."""
    B, T, H, d = q.shape
    G, cap = H // k.shape[1], k.shape[2]
    out = np.full(q.shape, np.nan)
    mag, dots = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(B):
        fits = 0 <= cached[b] <= cap - rows[b]
        for t in range(rows[b]):
            seen = list(range(cached[b])) + [cached[b] + i for i in range(rows[b]) if masks[b][t] >> i & 1] if fits else []
            for h in range(H):
                out[b, t, h] = 0.0
                if not seen:
                    continue
                K, V = k[b, h // G, seen], v[b, h // G, seen]
                s = K @ q[b, t, h] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, t, h], mag[b, t, h] = p @ V, p @ np.abs(V)
                dots[b, t, h] = (np.abs(K) @ np.abs(q[b, t, h])).max() * abs(scale)
    return out, mag, dots


def sample_row(x, temperature, top_k, top_p, min_p, u):
    """One row of logits (float64 copies of the stored values) -> (token, logprob)."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, -np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(x == top, 0.0, np.where(x == -np.inf, -np.inf, (x - top) / temperature))
    w = np.where(x == -np.inf, 0, np.rint(np.exp(z) * WEIGHT_ONE)).astype(np.int64)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if top_k > 0:
        order = order[:top_k]
    total = int(w[order].sum())
    keep = []
    before = 0
    for i in order:
        if keep and ((top_p < 1 and not before < top_p * float(total)) or w[i] < min_p * WEIGHT_ONE):
            break
        keep.append(int(i))
        before += int(w[i])
    index = np.sort(keep)
    sums = np.cumsum(w[index])
    Z = int(sums[-1])
    at = u * float(Z) if u == u else 0.0
    target = min(max(int(at), 0), Z - 1) if at < Z else Z - 1
    token = int(index[np.searchsorted(sums, target, side="right")])
    return token, float(z[token] - np.log(Z / WEIGHT_ONE))


def fork(cache, src, length):
    """cache [layers, sequences, heads, rows, ..] as it is afterwards."""
    new = cache.copy()
    for b, a in enumerate(src):
        if 0 <= a < len(length):
            n = min(max(int(length[a]), 0), cache.shape[3])
            new[:, b, :, :n] = cache[:, a, :, :n]
    return new


def compact(cache, first, path, count):
    new = cache.copy()
    cap = cache.shape[3]
    for b in range(len(first)):
        for i in range(min(int(count[b]), path.shape[1])):
            to, of = int(first[b]) + i, int(first[b]) + int(path[b, i])
            if 0 <= to < cap and 0 <= of < cap:
                new[:, b, :, to] = cache[:, b, :, of]
    return new
