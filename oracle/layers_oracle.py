"""CPU oracle for the operators of the layers between two drops: windowed attention, linear attention with a decay,
norm and rotation of heads, pages for new tokens.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy in 64 bits, one function per
definition in include/uniprefill.h, no code shared with the kernels.
"""
from __future__ import annotations

import math

import numpy as np


def visible(first, n, keys, window, n_sink):
    """[n, keys] truth values: which keys the tokens at positions first .. first + n - 1 see."""
    p, i = first + np.arange(n)[:, None], np.arange(keys)[None, :]
    return (i <= p) & ((i > p - window) | (i < n_sink))


def window_attention(q, k, v, cu_seqlens, cu_seqlens_k, window, n_sink, *, scale=None, gather=None):
    """out [T, Hq, D], lse [Hq, T] and two bounds for tests: the attention of |v| and the largest scale * sum |q_d k_d| of
    every row.  Arguments as in attention_oracle.causal_attention; a row that sees no key gets zeros and -inf."""
    cu, ck = np.asarray(cu_seqlens, np.int64), np.asarray(cu_seqlens_k, np.int64)
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else float(np.float32(scale))
    out, absv = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, top = np.full((Hq, T), -np.inf), np.zeros((Hq, T))
    for r in range(len(cu) - 1):
        n, m = int(cu[r + 1] - cu[r]), int(ck[r + 1] - ck[r])
        if n == 0 or m == 0:
            continue
        see = visible(m - n, n, m, window, n_sink)
        used = np.flatnonzero(see.any(axis=0))      # (keys that no token sees may hold anything)
        see = see[:, used]
        rows = (np.arange(ck[r], ck[r + 1]) if gather is None else gather(r, m))[used]
        sl = slice(int(cu[r]), int(cu[r + 1]))
        for h in range(Hq):
            K, V = k[rows, h * Hkv // Hq].astype(np.float64), v[rows, h * Hkv // Hq].astype(np.float64)
            Q = q[sl, h].astype(np.float64)
            x = np.where(see, Q @ K.T * scale, -np.inf)
            mx = x.max(axis=1)
            w = np.exp(x - mx[:, None])
            total = w.sum(axis=1)
            w /= total[:, None]
            out[sl, h], absv[sl, h] = w @ V, w @ np.abs(V)
            lse[h, sl] = mx + np.log(total)
            top[h, sl] = np.where(see, np.abs(Q) @ np.abs(K).T * scale, 0.0).max(axis=1)
    return out, lse, absv, top


def linear_attention(q, k, v, cu_seqlens, log_decay, states=None, state_in=None, state_out=None, *, scale=None):
    """out [T, Hq, D], the pool of states afterwards, and for tests the same two computed of the absolute values of everything.
    Token after token, as the definition has it."""
    cu = np.asarray(cu_seqlens, np.int64)
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else float(np.float32(scale))
    out, bound = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    pool = None if states is None else np.array(states, np.float64)
    pool_bound = None if pool is None else np.zeros_like(pool)
    num = 0 if pool is None else pool.shape[0]
    lam = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0))
    for r in range(len(cu) - 1):
        source = -1 if state_in is None else int(state_in[r])
        for h in range(Hkv):
            S = states[source, h].astype(np.float64) if 0 <= source < num else np.zeros((D, D))
            A = np.abs(S)
            for t in range(int(cu[r]), int(cu[r + 1])):
                S = lam[h] * S + np.outer(k[t, h], v[t, h])
                A = lam[h] * A + np.outer(np.abs(k[t, h]), np.abs(v[t, h]))
                for g in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                    out[t, g], bound[t, g] = scale * (q[t, g] @ S), scale * (np.abs(q[t, g]) @ A)
            to = -1 if state_out is None else int(state_out[r])
            if 0 <= to < num:
                pool[to, h], pool_bound[to, h] = S, A
    return out, pool, bound, pool_bound



def linear_attention_in_chunks(q, k, v, cu_seqlens, log_decay, states=None, state_in=None, state_out=None, *, scale=None, chunk=64):
    """linear_attention for long sequences: the same sums, `chunk` tokens at a time as matrix products."""
    cu = np.asarray(cu_seqlens, np.int64)
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else float(np.float32(scale))
    out, bound = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    pool = None if states is None else np.array(states, np.float64)
    pool_bound = None if pool is None else np.zeros_like(pool)
    num = 0 if pool is None else pool.shape[0]
    for r in range(len(cu) - 1):
        source, to = (-1 if x is None else int(x[r]) for x in (state_in, state_out))
        for h in range(Hkv):
            ld = min(float(log_decay[h]), 0.0)
            S = states[source, h].astype(np.float64) if 0 <= source < num else np.zeros((D, D))
            A = np.abs(S)
            for lo in range(int(cu[r]), int(cu[r + 1]), chunk):
                hi = min(lo + chunk, int(cu[r + 1]))
                i = np.arange(hi - lo)
                age = (i[:, None] - i)
                w = np.where(age >= 0, np.exp(ld * np.maximum(age, 0)), 0.0)
                before, after = np.exp(ld * (i + 1.0))[:, None], np.exp(ld * (hi - lo - 1.0 - i))[:, None]
                K, V = k[lo:hi, h].astype(np.float64), v[lo:hi, h].astype(np.float64)
                for g in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                    Q = q[lo:hi, g].astype(np.float64)
                    out[lo:hi, g] = scale * ((Q @ K.T * w) @ V + before * (Q @ S))
                    bound[lo:hi, g] = scale * ((np.abs(Q) @ np.abs(K).T * w) @ np.abs(V) + before * (np.abs(Q) @ A))
                last = math.exp(ld * (hi - lo))
                S = last * S + (K * after).T @ V
                A = last * A + (np.abs(K) * after).T @ np.abs(V)
            if 0 <= to < num:
                pool[to, h], pool_bound[to, h] = S, A
    return out, pool, bound, pool_bound


def norm_rotate(x, weight, eps, pos, inv_freq, rot_dim, pairs):
    """Rows x [T, H, D] normalised (eps > 0) and turned; and |a| + |b| of every element's pair before the turn, for tests."""
    y = np.asarray(x, np.float64)
    if eps > 0:
        y = y / np.sqrt((y * y).mean(axis=-1, keepdims=True) + float(np.float32(eps)))
        y = y if weight is None else y * weight
    out, size = y.copy(), np.abs(y)
    if rot_dim:
        first, second = (slice(0, rot_dim, 2), slice(1, rot_dim, 2)) if pairs else (slice(0, rot_dim // 2), slice(rot_dim // 2, rot_dim))
        angle = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
        c, s = np.cos(angle), np.sin(angle)
        out[..., first] = y[..., first] * c - y[..., second] * s
        out[..., second] = y[..., second] * c + y[..., first] * s
        size[..., first] = size[..., second] = np.abs(y[..., first]) + np.abs(y[..., second])
    return out, size


def append_pages(kv_len, num_new, page, table, free_pages, num_free, capacity, dropped=None):
    """dict of what uniprefill_append_pages (dropped: _append_pages_dropped) writes, a request at a time."""
    table, free = np.array(table, np.int64), [int(x) for x in free_pages[:max(0, num_free)]]
    new_len, cu, cu_k, pos, slots, served, going = [], [0], [0], [], [], 0, True
    for r in range(len(kv_len)):
        n, add = max(0, int(kv_len[r])), max(0, int(num_new[r]))
        have = -(-n // page)
        need = -(-(n + add) // page) - have
        going = going and need <= len(free) and have + need <= table.shape[1] and len(pos) + add <= capacity and n + add < 2 ** 31
        if not going:
            add = 0
        else:
            served += 1
            for j in range(need):
                table[r, have + j] = free.pop()
        for p in range(n, n + add):
            pos.append(min(p + (0 if dropped is None else max(0, int(dropped[r]))), 2 ** 31 - 1))
            slots.append(int(table[r, p // page]) * page + p % page)
        new_len.append(n + add)
        cu.append(cu[-1] + add)
        cu_k.append(cu_k[-1] + n + add)
    pad = capacity - len(pos)
    return {"table": table, "free_left": len(free), "new_len": new_len, "cu": cu, "cu_k": [min(x, 2 ** 31 - 1) for x in cu_k],
            "pos": pos + [0] * pad, "slots": slots + [-1] * pad, "served": served}
