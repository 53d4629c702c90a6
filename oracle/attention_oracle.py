"""CPU oracle for the attention layer's operators: causal attention of a packed batch with its
log-sum-exp, the 4-bit KV cache, decode attention over it, and eviction by accumulated weight.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy in 64 bits, one function per
definition in include/uniprefill.h, no code shared with the kernels.
"""
from __future__ import annotations

import math

import numpy as np

Q4_GROUP = 64


def causal_attention(q, k, v, cu_seqlens, cu_seqlens_k=None, *, scale=None, gather=None):
    """out [T, Hq, D], lse [Hq, T] and two bounds for tests: the attention of |v| and the largest
    scale * sum |q_d k_d| of every row.  q [T, Hq, D]; k, v [Tk, Hkv, D] packed by cu_seqlens_k
    (default cu_seqlens), or a cache addressed through gather(r, n) -> rows of sequence r's n keys."""
    cu = np.asarray(cu_seqlens, np.int64)
    ck = cu if cu_seqlens_k is None else np.asarray(cu_seqlens_k, np.int64)
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else float(np.float32(scale))
    out, absv = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, top = np.full((Hq, T), -np.inf), np.zeros((Hq, T))
    for r in range(len(cu) - 1):
        n, m = int(cu[r + 1] - cu[r]), int(ck[r + 1] - ck[r])
        if n == 0:
            continue
        rows = np.arange(ck[r], ck[r + 1]) if gather is None else gather(r, m)
        hidden = np.arange(m)[None, :] > (m - n + np.arange(n))[:, None]
        for h in range(Hq):
            K, V = k[rows, h * Hkv // Hq].astype(np.float64), v[rows, h * Hkv // Hq].astype(np.float64)
            Q = q[cu[r]:cu[r + 1], h].astype(np.float64)
            x = Q @ K.T * scale
            x[hidden] = -np.inf
            mx = x.max(axis=1)
            w = np.exp(x - mx[:, None])
            total = w.sum(axis=1)
            w /= total[:, None]
            sl = slice(int(cu[r]), int(cu[r + 1]))
            out[sl, h], absv[sl, h] = w @ V, w @ np.abs(V)
            lse[h, sl] = mx + np.log(total)
            a = np.abs(Q) @ np.abs(K).T * scale
            a[hidden] = 0.0
            top[h, sl] = a.max(axis=1)
    return out, lse, absv, top


def _bf16_bits(x):
    """The float32 bit patterns of bf16 neighbours: (bits of x truncated towards zero)."""
    return np.asarray(x, np.float32).view(np.uint32) & np.uint32(0xFFFF0000)


def bf16_floor(x):
    """Largest bf16 value not above x (float32 or exact in it)."""
    x = np.asarray(x, np.float32)
    b = _bf16_bits(x)
    t = b.view(np.float32)
    lower = np.where(t > x, b + np.uint32(0x10000), b)      # a negative number: one step away from zero
    return lower.astype(np.uint32).view(np.float32).astype(np.float64)


def bf16_ceil_nonneg(x):
    """Smallest bf16 value not below x >= 0 (float64)."""
    b = _bf16_bits(np.asarray(x, np.float64).astype(np.float32))
    t = b.view(np.float32).astype(np.float64)
    return np.where(t < x, (b + np.uint32(0x10000)).view(np.float32).astype(np.float64), t)


def q4_quantise(x):
    """x [n, H, D] -> codes uint8 [n, H, D], lowest and step float64 [n, H, D // 64]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[0], x.shape[1], x.shape[2] // Q4_GROUP, Q4_GROUP)
    lo = bf16_floor(g.min(axis=-1))
    step = bf16_ceil_nonneg((g.max(axis=-1) - lo) / 15.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        t = (g - lo[..., None]) / step[..., None]
    code = np.where(step[..., None] > 0, np.rint(np.where(step[..., None] > 0, t, 0.0)), 0.0)
    return np.clip(code, 0, 15).astype(np.uint8).reshape(x.shape), lo, step


def q4_values(code, lo, step):
    """What codes and pairs stand for, float64 [n, H, D]."""
    g = code.reshape(code.shape[0], code.shape[1], code.shape[2] // Q4_GROUP, Q4_GROUP).astype(np.float64)
    return (lo[..., None] + step[..., None] * g).reshape(code.shape)


def q4_pack(code, lo, step):
    """Rows of the cache, uint8 [n, H * D / 2 + H * D / 64 * 4]."""
    n = code.shape[0]
    flat = code.reshape(n, -1)
    body = flat[:, 0::2] | (flat[:, 1::2] << 4)
    hi = lambda a: (np.asarray(a, np.float32).view(np.uint32) >> 16).astype(np.uint16).reshape(n, -1)
    pairs = np.stack([hi(lo), hi(step)], axis=2).reshape(n, -1)
    return np.concatenate([body, pairs.view(np.uint8).reshape(n, -1)], axis=1)


def q4_unpack(rows, heads, D):
    """codes, lowest, step of rows of the cache."""
    rows = np.asarray(rows)
    n, half = rows.shape[0], heads * D // 2
    code = np.stack([rows[:, :half] & 15, rows[:, :half] >> 4], axis=2).reshape(n, heads, D)
    words = np.ascontiguousarray(rows[:, half:half + heads * (D // Q4_GROUP) * 4]).view(np.uint16).astype(np.uint32) << 16
    pair = words.view(np.float32).astype(np.float64).reshape(n, heads, D // Q4_GROUP, 2)
    return code, pair[..., 0], pair[..., 1]


def page_rows(table_row, n, page):
    """Cache rows of a sequence's first n tokens (Eq. 16's indexing)."""
    i = np.arange(n)
    return np.asarray(table_row, np.int64)[i // page] * page + i % page


def decode_attention_q4(q, k_rows, v_rows, heads, *, scale=None):
    """One query token [Hq, D] over n cached tokens given as rows of the 4-bit caches: out [Hq, D], lse [Hq],
    the mean weight of every token [n], and for tests the weights [Hq, n], the attention of
    step * |code - 8|, that of 31 * step + |lowest|, and the largest scale * sum |q| (31 step + |lowest|)."""
    Hq, D = q.shape
    n = k_rows.shape[0]
    scale = 1.0 / math.sqrt(D) if scale is None else float(np.float32(scale))
    kc, kl, ks = q4_unpack(k_rows, heads, D)
    vc, vl, vs = q4_unpack(v_rows, heads, D)
    K, V = q4_values(kc, kl, ks), q4_values(vc, vl, vs)
    spread = np.repeat(31 * ks + np.abs(kl), Q4_GROUP, axis=2)
    near = np.repeat(vs, Q4_GROUP, axis=2) * np.abs(vc.astype(np.float64) - 8)
    far = np.repeat(31 * vs + np.abs(vl), Q4_GROUP, axis=2)
    out, a_near, a_far = np.zeros((Hq, D)), np.zeros((Hq, D)), np.zeros((Hq, D))
    lse, top, W = np.full(Hq, -np.inf), np.zeros(Hq), np.zeros((Hq, n))
    for h in range(Hq if n else 0):
        g = h * heads // Hq
        x = K[:, g] @ q[h].astype(np.float64) * scale
        w = np.exp(x - x.max())
        lse[h] = x.max() + np.log(w.sum())
        W[h] = w / w.sum()
        out[h], a_near[h], a_far[h] = W[h] @ V[:, g], W[h] @ near[:, g], W[h] @ far[:, g]
        top[h] = (spread[:, g] @ np.abs(q[h].astype(np.float64))).max() * scale
    return out, lse, W.mean(axis=0), W, a_near, a_far, top


def evict_tokens(mass, n, budget, n_sink, n_recent):
    """Ascending indices of the tokens that stay: all if n <= budget, else the first n_sink, the last
    n_recent, and of the others the largest masses up to the budget, equal ones by the lower index."""
    if n <= budget:
        return np.arange(n)
    free = list(range(n_sink, n - n_recent))
    free.sort(key=lambda i: (-float(mass[i]), i))
    return np.array(sorted(list(range(n_sink)) + list(range(n - n_recent, n)) + free[:budget - n_sink - n_recent]), dtype=np.int64)
