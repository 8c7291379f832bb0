"""Float64 oracle of the batched serving calls: row maps of a step, norm and rotation,
attention over a shared context and own suffixes, block means, block selection.  Plain
loops over rows, numpy only; shares no code with the library."""

import numpy as np


def batch_plan(past, new, T_c):
    """(row_off, row_seq, row_pos) of a step."""
    off, seq, pos = [0], [], []
    for b, (p, n) in enumerate(zip(past, new)):
        for i in range(int(n)):
            seq.append(b)
            pos.append(T_c + int(p) + i)
        off.append(off[-1] + int(n))
    return np.array(off), np.array(seq, dtype=np.int64), np.array(pos, dtype=np.int64)


def norm_rope(x, positions, inv_freq=None, weight=None, eps=1e-6, interleaved=False):
    """x [n][heads][d]: y_i = x_i / sqrt(mean x^2 + eps) * w_i, then the rotation of the pairs
    (i, i + r/2), or (2i, 2i + 1), by positions * inv_freq."""
    y = np.array(x, dtype=np.float64)
    n, heads, d = y.shape
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    half = 0 if inv_freq is None else len(inv_freq)
    out = y.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(positions, np.float64) * float(inv_freq[i])
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        out[:, :, a] = y[:, :, a] * c - y[:, :, b] * s
        out[:, :, b] = y[:, :, b] * c + y[:, :, a] * s
    return out


def _row(q, K, V, scale):
    """(O, lse, sum_j p_j |V_j - O|) of one row over its keys; the empty sum for no key."""
    if not len(K):
        return np.zeros(V.shape[1]), -np.inf, np.zeros(V.shape[1])
    s = scale * (K @ q)
    m = s.max()
    e = np.exp(s - m)
    z = e.sum()
    p = e / z
    o = p @ V
    return o, m + np.log(z), p @ np.abs(V - o)


def batch_attn(q, row_seq, row_pos, k_cache, v_cache, k_suffix, v_suffix, softmax_scale=None,
               blocks=None, block=None):
    """q [n][H][d]; k_cache [H_kv][T_c][d]; k_suffix [B][H_kv][S][d].  Returns O, lse and the
    spread sum_j p_j |V_j - O| that rounded probabilities act on.  With blocks
    [n][H_kv][m] the context keys of a row and KV head are those of its listed blocks
    (entries outside the blocks dropped, repeats counted again)."""
    n, H, d = q.shape
    H_kv, T_c = k_cache.shape[:2]
    G = H // H_kv
    scale = 1.0 / np.sqrt(d) if softmax_scale is None else softmax_scale
    O, lse, spread = np.zeros((n, H, d)), np.zeros((n, H)), np.zeros((n, H, d))
    for t in range(n):
        b, m = int(row_seq[t]), int(row_pos[t]) - T_c + 1
        for g in range(H_kv):
            if blocks is None:
                K, V = k_cache[g], v_cache[g]
            else:
                nb = -(-T_c // block)
                at = [np.arange(j * block, min(T_c, (j + 1) * block))
                      for j in blocks[t, g] if 0 <= j < nb]
                at = np.concatenate(at) if at else np.zeros(0, dtype=np.int64)
                K, V = k_cache[g][at], v_cache[g][at]
            K = np.concatenate([K, k_suffix[b, g, :m]])
            V = np.concatenate([V, v_suffix[b, g, :m]])
            for h in range(g * G, (g + 1) * G):
                O[t, h], lse[t, h], spread[t, h] = _row(q[t, h], K, V, scale)
    return O, lse, spread


def block_means(k, block):
    """k [H_kv][T][d] -> [H_kv][ceil(T / block)][d] float64 means."""
    T = k.shape[1]
    return np.stack([k[:, i:min(T, i + block)].astype(np.float64).mean(1)
                     for i in range(0, T, block)], 1)


def block_select(q, means, n_sel):
    """q [n][H][d], means [H_kv][nb][d] -> [n][H_kv][n_sel]: the largest float32-rounded
    products of the summed group queries, ties to the lower block, ascending."""
    n, H, d = q.shape
    H_kv = means.shape[0]
    G = H // H_kv
    out = np.zeros((n, H_kv, n_sel), dtype=np.int32)
    for g in range(H_kv):
        s = (q[:, g * G:(g + 1) * G].astype(np.float64).sum(1) @ means[g].astype(np.float64).T)
        s = s.astype(np.float32)
        s = np.where(np.isnan(s), -np.inf, s)
        for t in range(n):
            out[t, g] = np.sort(np.argsort(-s[t], kind="stable")[:n_sel])
    return out


def round_bf16(x):
    """float64 values rounded to the nearest bf16 (ties to even), as float64."""
    m, e = np.frexp(np.asarray(x, np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)
