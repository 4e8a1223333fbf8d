"""Plain fp64 CPU restatement of the operators around the cache: norms of queries and keys with the rotation, a cache held in
8 bits, and eviction by attention weight.  numpy, loops over episodes and heads, nothing shared with the GPU path."""
from __future__ import annotations

import numpy as np

PAGE = 64


def rms_norm(x, w, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else w)


def rotate(x, positions, theta):
    """x [tokens, heads, D], half-split pairs."""
    half = x.shape[-1] // 2
    angle = np.asarray(positions, dtype=np.float64)[:, None, None] * theta ** (-np.arange(half) / half)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], axis=-1)


def nearest_code(x):
    """The nearest number with 4 exponent and 3 fraction bits (bias 7), ties to even, at most 448."""
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def scale_for(x):
    """The least power of two in 2^-120 .. 2^120 with |x| <= 448 of it, for every finite x."""
    top = np.abs(x[np.isfinite(x)]).max(initial=0.0)
    e = -120
    while top > 448.0 * 2.0 ** e and e < 120:
        e += 1
    return 2.0 ** e


def append8(codes, scales, new, cache_lens, new_offsets, table, clear):
    """codes [pages, Hkv, 64, D] and scales [pages, Hkv] as they are after `new` [tokens, Hkv, D]: (codes, scales)."""
    codes, scales = codes.copy(), scales.copy()
    for b, L in enumerate(cache_lens):
        n = new_offsets[b + 1] - new_offsets[b]
        for p in range(L // PAGE, (L + n + PAGE - 1) // PAGE if n else L // PAGE):
            page, lo, hi = table[b][p], max(L, p * PAGE), min(L + n, (p + 1) * PAGE)
            first, last = lo - p * PAGE, hi - p * PAGE
            for g in range(codes.shape[1]):
                x = new[new_offsets[b] + lo - L:new_offsets[b] + hi - L, g]
                s = scale_for(x)
                if first and scales[page, g] > s:
                    s = scales[page, g]
                if first:
                    codes[page, g, :first] = nearest_code(codes[page, g, :first] * (scales[page, g] / s))
                codes[page, g, first:last] = nearest_code(x / s)
                if clear:
                    codes[page, g, last:] = 0.0
                scales[page, g] = s
    return codes, scales


def attention(q, k, v, L, scale):
    """q [n, Hq, D] over k, v [L + n, Hkv, D], causal: out, log-sum-exp, and sum p |v| (what errors of p are measured by)."""
    n, hq, _ = q.shape
    G = hq // k.shape[1]
    out, lse, size = np.zeros_like(q), np.zeros((n, hq)), np.zeros_like(q)
    for h in range(hq):
        s = q[:, h] @ k[:, h // G].T * scale
        s[np.arange(L + n)[None] > L + np.arange(n)[:, None]] = -np.inf
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        lse[:, h] = top[:, 0] + np.log(p.sum(1))
        p /= p.sum(1, keepdims=True)
        with np.errstate(invalid="ignore"):
            out[:, h], size[:, h] = p @ v[:, h // G], p @ np.abs(v[:, h // G])
    return out, lse, size


def key_weights(q, k, lse, L, decay, weights, scale):
    """q [n, Hq, D], k [L + n, Hkv, D], lse [n, Hq], weights [Hkv, L]: [Hkv, L + n]."""
    n, hq, _ = q.shape
    G = hq // k.shape[1]
    out = np.zeros((k.shape[1], L + n))
    out[:, :L] = decay * weights[:, :L]
    for h in range(hq):
        p = np.exp(q[:, h] @ k[:, h // G].T * scale - lse[:, h:h + 1])
        p[np.arange(L + n)[None] > L + np.arange(n)[:, None]] = 0.0
        out[h // G] += p.sum(0)
    return out


def select_keys(weights, num_keys, budget, sinks, recent):
    """[Hkv, min(budget, num_keys)] slots, ascending."""
    rows = []
    for w in weights:
        if budget >= num_keys:
            rows.append(list(range(num_keys)))
            continue
        rank = [-np.inf if np.isnan(x) else x for x in w[:num_keys].tolist()]
        best = sorted(range(sinks, num_keys - recent), key=lambda j: (-rank[j], j))[:budget - sinks - recent]
        rows.append(sorted(list(range(sinks)) + best + list(range(num_keys - recent, num_keys))))
    return np.array(rows, dtype=np.int64).reshape(len(weights), -1)
