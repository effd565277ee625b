"""Plain float64 statement of attention over a shared prefix and own caches, of the attention
weight the own entries got, and of the eviction by it. numpy only, one row at a time."""
import numpy as np


def seen(own_len, visible, S, b, i):
    """Own entries position (b, i) sees; -1 for padding, which sees nothing at all."""
    n = min(max(int(own_len[b]), 0), S)
    if visible is None:
        return n
    v = int(visible[b, i])
    return -1 if v < 0 else min(n, v)


def attend(q, k_prefix, v_prefix, k_own, v_own, own_len, visible, scale):
    """out, lse, and for tolerances sum_t p_t |v_t| and the largest sum_d |q_d k_td| of each row."""
    B, L, Hq, D = q.shape
    Hkv = (k_prefix if k_prefix is not None else k_own).shape[-2]
    P = 0 if k_prefix is None else k_prefix.shape[0]
    S = 0 if k_own is None else k_own.shape[1]
    out = np.zeros((B, L, Hq, D))
    mass = np.zeros((B, L, Hq, D))
    big = np.zeros((B, L, Hq))
    lse = np.full((B, L, Hq), -np.inf)
    for b in range(B):
        for i in range(L):
            n = seen(own_len, visible, S, b, i)
            if n < 0 or P + n == 0:
                continue
            for hq in range(Hq):
                h = hq // (Hq // Hkv)
                parts_k = ([k_prefix[:, h]] if P else []) + ([k_own[b, :n, h]] if n else [])
                parts_v = ([v_prefix[:, h]] if P else []) + ([v_own[b, :n, h]] if n else [])
                k, v = np.concatenate(parts_k), np.concatenate(parts_v)
                s = scale * (k @ q[b, i, hq])
                m = s.max()
                e = np.exp(s - m)
                p = e / e.sum()
                out[b, i, hq] = p @ v
                mass[b, i, hq] = p @ np.abs(v)
                big[b, i, hq] = scale * (np.abs(k) @ np.abs(q[b, i, hq])).max()
                lse[b, i, hq] = m + np.log(e.sum())
    return out, lse, mass, big


def weights(q, lse, k_own, own_len, visible, scale, acc_in, decay):
    """acc_out, and for tolerances the largest sum_d |q_d k_td| of any pair."""
    B, L, Hq, _ = q.shape
    S, Hkv = k_own.shape[1:3]
    acc = np.zeros((B, Hkv, S))
    big = 0.0
    for b in range(B):
        n_all = seen(own_len, None, S, b, 0)
        if acc_in is not None:
            acc[b, :, :n_all] = decay * acc_in[b, :, :n_all]
        for i in range(L):
            n = seen(own_len, visible, S, b, i)
            for hq in range(Hq):
                if n <= 0 or lse[b, i, hq] == -np.inf:
                    continue
                h = hq // (Hq // Hkv)
                s = scale * (k_own[b, :n, h] @ q[b, i, hq])
                acc[b, h, :n] += np.exp(s - lse[b, i, hq])
                big = max(big, scale * (np.abs(k_own[b, :n, h]) @ np.abs(q[b, i, hq])).max())
    return acc, big


def evict(k_own, v_own, acc, own_len, keep, recent):
    """k, v [B, keep, Hkv, D], acc [B, Hkv, keep], own_len, kept as the call leaves them."""
    B, S, Hkv, D = k_own.shape
    k, v = np.zeros((B, keep, Hkv, D)), np.zeros((B, keep, Hkv, D))
    acc_to = np.zeros((B, Hkv, keep))
    kept = np.full((B, Hkv, keep), -1, dtype=np.int32)
    new_len = np.zeros(B, dtype=np.int32)
    for b in range(B):
        n = min(max(int(own_len[b]), 0), S)
        new_len[b] = min(n, keep)
        for h in range(Hkv):
            if n <= keep:
                ids = list(range(n))
            else:
                old = n - recent
                # larger weights first, ties by index, NaN behind every number
                key = [(np.isnan(w), -w if not np.isnan(w) else 0.0, t)
                       for t, w in enumerate(acc[b, h, :old])]
                ids = sorted(t for _, _, t in sorted(key)[:keep - recent]) + list(range(old, n))
            for j, t in enumerate(ids):
                kept[b, h, j] = t
                k[b, j, h], v[b, j, h], acc_to[b, h, j] = k_own[b, t, h], v_own[b, t, h], acc[b, h, t]
    return k, v, acc_to, new_len, kept
