"""Definitions of the sampling phase's operators in float64 numpy: rotary positions with several axes, the append to a paged cache, and
the attention of new tokens over their pages.  Test infrastructure: no tiling, no online softmax, no code of the library."""
import numpy as np


def rope(x, positions, inv_freq, pair_axis, layout, sign=1.0):
    """x [T, H, D]: pair i of token t turned by sign * positions[pair_axis[i], t] * inv_freq[i] (inv_freq as given, in fp32)."""
    y = np.array(x, dtype=np.float64)
    n = len(pair_axis)
    for i in range(n):
        a, b = (i, i + n) if layout == "halves" else (2 * i, 2 * i + 1)
        angle = sign * positions[pair_axis[i]].astype(np.float64) * np.float64(inv_freq[i])
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        x0, x1 = x[:, :, a].astype(np.float64), x[:, :, b].astype(np.float64)
        y[:, :, a], y[:, :, b] = x0 * c - x1 * s, x1 * c + x0 * s
    return y


def new_rows(seq_lens, cu_new, tokens):
    """(packed row, sequence, position) of every new token, position < 0 where the sequence is said to be shorter than its new tokens."""
    out = []
    for b in range(len(seq_lens)):
        for t in range(max(0, int(cu_new[b])), min(int(cu_new[b + 1]), tokens)):
            out.append((t, b, int(seq_lens[b]) - int(cu_new[b + 1]) + t))
    return out


def page_of(page_table, b, pos, page_size, num_pages):
    """The page of token `pos` of sequence b, or -1: it has none."""
    if pos < 0 or pos // page_size >= page_table.shape[1]:
        return -1
    page = int(page_table[b, pos // page_size])
    return page if 0 <= page < num_pages else -1


def append(cache, x, page_table, seq_lens, cu_new):
    """cache [pages, Hkv, page_size, D] with the new tokens' rows x [T, Hkv, D] in place."""
    out = np.array(cache, dtype=np.float64)
    pages, page_size = cache.shape[0], cache.shape[2]
    for t, b, pos in new_rows(seq_lens, cu_new, x.shape[0]):
        page = page_of(page_table, b, pos, page_size, pages)
        if page >= 0:
            out[page, :, pos % page_size] = x[t]
    return out


def paged_attention(q, k_cache, v_cache, page_table, seq_lens, cu_new, scale):
    """out [T, Hq, D], lse [Hq, T] and, for error bounds, mass [T, Hq, D] = sum_j w_j |v_j|, reach [T, Hq] = max_j scale sum_d |q_d k_jd|
    and the number of keys [T].  Rows of no sequence: NaN everywhere."""
    T, Hq, D = q.shape
    pages, Hkv, page_size, _ = k_cache.shape
    out, mass = np.full((T, Hq, D), np.nan), np.full((T, Hq, D), np.nan)
    lse, reach, keys = np.full((Hq, T), np.nan), np.full((T, Hq), np.nan), np.zeros(T, dtype=np.int64)
    gathered = {}
    for t, b, pos in new_rows(seq_lens, cu_new, T):
        n = min(pos, page_table.shape[1] * page_size) + 1   # one key behind the table has no page
        if n <= 0:
            out[t], mass[t], lse[:, t], reach[t] = 0.0, 0.0, -np.inf, 0.0
            continue
        keys[t] = n
        if b not in gathered:
            last = min(int(seq_lens[b]), page_table.shape[1] * page_size + 1)
            where = [page_of(page_table, b, j, page_size, pages) for j in range(last)]
            k, v = np.full((last, Hkv, D), np.nan), np.full((last, Hkv, D), np.nan)
            for j, p in enumerate(where):
                if p >= 0:
                    k[j], v[j] = k_cache[p, :, j % page_size], v_cache[p, :, j % page_size]
            gathered[b] = k, v
        k, v = gathered[b]
        for h in range(Hq):
            c = h // (Hq // Hkv)
            kk, vv, qq = k[:n, c], v[:n, c], q[t, h].astype(np.float64)
            s = scale * (kk @ qq)
            top = s.max()
            if np.isnan(top):
                continue
            l = np.exp(s - top).sum()
            w = np.exp(s - top) / l
            lse[h, t] = top + np.log(l)
            out[t, h], mass[t, h], reach[t, h] = w @ vv, w @ np.abs(vv), scale * (np.abs(kk) @ np.abs(qq)).max()
    return out, lse, mass, reach, keys
