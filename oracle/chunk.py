"""Oracle of a chunk of new tokens over the paged cache (test infrastructure).

Plain numpy in 64 bits, written from the definitions: pages and slots from the
lengths, per-head RMS norms with the rotation by position, and the attention of
the new tokens over the cache.  Nothing here shares code with the CUDA library.
"""
import numpy as np

PAGE = 16
ERR_LEN, ERR_POOL, ERR_CAP = 0x4, 0x80, 0x200


def pages_of(n):
    return -(-int(n) // PAGE)


def slots(new_len, seq_len, page_table, free, top, max_tokens):
    """Returns (dict of the call's outputs, error bits)."""
    S, max_pages = page_table.shape
    new_len, seq_len = [int(x) for x in new_len], [int(x) for x in seq_len]
    table = page_table.copy()
    got = dict(chunk_cu=np.zeros(S + 1, np.int32), slot=np.full(max_tokens, -1, np.int32),
               pos=np.zeros(max_tokens, np.int32), seq_len=np.array(seq_len, np.int32), free_top=int(top),
               page_table=table)
    cap = max_pages * PAGE
    if any(n < 0 or l < 0 or n + l > cap for n, l in zip(new_len, seq_len)):
        return got, ERR_LEN
    if sum(new_len) > max_tokens:
        return got, ERR_CAP
    need = [pages_of(l + n) - pages_of(l) for n, l in zip(new_len, seq_len)]
    if top < 0 or top > len(free) or sum(need) > top:
        return got, ERR_POOL
    at, t = top - sum(need), 0
    for s in range(S):
        for i in range(need[s]):
            table[s, pages_of(seq_len[s]) + i] = free[at]
            at += 1
        for p in range(seq_len[s], seq_len[s] + new_len[s]):
            got["slot"][t] = table[s, p // PAGE] * PAGE + p % PAGE
            got["pos"][t] = p
            t += 1
        got["chunk_cu"][s + 1] = t
        got["seq_len"][s] += new_len[s]
    got["free_top"] = top - sum(need)
    return got, 0


def norm_rope(x, weight, cos, sin, eps):
    """x [T, H, D] -> (rotated norms, size of the values they are made of: a
    rounding of the normed values moves the result by as much of it)."""
    D = x.shape[-1]
    x = x.astype(np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if weight is not None:
        n = n * weight.astype(np.float64)
    a, b = n[..., : D // 2], n[..., D // 2:]
    c, s = cos[:, None].astype(np.float64), sin[:, None].astype(np.float64)
    y = np.concatenate((a * c - b * s, b * c + a * s), -1)
    size = np.concatenate((np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)), -1)
    return y, size


def attn(q, k_cache, v_cache, page_table, chunk_cu, seq_len, full_len=None, scale=None):
    """q [T, H_q, D], caches [pages, 16, H_kv, D], all float; returns out, lse,
    the weighted sum of |v| and the largest sum of |q_i k_i| scale of a row."""
    T, H_q, D = q.shape
    H_kv = k_cache.shape[2]
    G = H_q // H_kv
    scale = 1.0 / np.sqrt(D) if not scale else scale
    out = np.zeros((T, H_q, D))
    size = np.zeros((T, H_q, D))
    lse = np.full((T, H_q), -np.inf)
    reach = np.zeros((T, H_q))
    for s in range(len(seq_len)):
        t0, t1, L = int(chunk_cu[s]), int(chunk_cu[s + 1]), int(seq_len[s])
        if t1 == t0 or L == 0:
            continue
        slot = [int(page_table[s, j // PAGE]) * PAGE + j % PAGE for j in range(L)]
        K = k_cache.reshape(-1, H_kv, D)[slot].astype(np.float64)
        V = v_cache.reshape(-1, H_kv, D)[slot].astype(np.float64)
        for i in range(t1 - t0):
            lim = L - (t1 - t0) + i + 1
            if full_len is not None:
                lim = max(lim, int(full_len[s]))
            lim = min(max(lim, 0), L)
            if lim == 0:
                continue
            for g in range(H_kv):
                x = q[t0 + i, g * G: (g + 1) * G].astype(np.float64)
                sc = x @ K[:lim, g].T * scale
                top = sc.max(-1, keepdims=True)
                p = np.exp(sc - top)
                tot = p.sum(-1, keepdims=True)
                out[t0 + i, g * G: (g + 1) * G] = p @ V[:lim, g] / tot
                size[t0 + i, g * G: (g + 1) * G] = p @ np.abs(V[:lim, g]) / tot
                lse[t0 + i, g * G: (g + 1) * G] = (top + np.log(tot))[:, 0]
                reach[t0 + i, g * G: (g + 1) * G] = (np.abs(x) @ np.abs(K[:lim, g]).T).max(-1) * abs(scale)
    return out, lse, size, reach
