"""Plain 64-bit forms of the calls around the paged cache: norm and rotation of heads, append, attention of a chunk.

Written from the definitions, head by head and row by row; shares no code with the GPU path.  Every function also returns,
where a test needs one, the size of the terms that were added up, from which rounding bounds follow.
"""
import numpy as np


def norm_rope(x, position, cos_sin, norm="none", eps=1e-6, weight=None, bias=None, interleaved=False):
    """x [T, heads, D] float64 -> (y, size): size bounds the terms that each element of y was summed from."""
    if norm == "rms" and bias is not None:
        raise ValueError("an RMS norm has no bias")
    x = np.array(x, dtype=np.float64)
    size = np.abs(x)
    if norm == "layer":
        mean = x.mean(-1, keepdims=True)
        size = np.abs(x) + np.abs(mean)
        x = x - mean
    if norm != "none":
        inv = 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
        x = x * inv * weight
        size = size * inv * np.abs(weight)
        if bias is not None:
            x = x + bias
            size = size + np.abs(bias)
    if cos_sin is None:
        return x, size
    rot = cos_sin.shape[1]
    half = rot // 2
    y, ysize = x.copy(), size.copy()
    for t, p in enumerate(position):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = float(cos_sin[p, i]), float(cos_sin[p, half + i])
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
            ysize[t, :, a] = ysize[t, :, b] = size[t, :, a] + size[t, :, b]
    return y, ysize


def cache_rows(row_begin, kv_len):
    """(row of the call, stream, cache row) of every new row."""
    out = []
    for s in range(len(kv_len)):
        n = int(row_begin[s + 1]) - int(row_begin[s])
        for i in range(n):
            out.append((int(row_begin[s]) + i, s, int(kv_len[s]) - n + i))
    return out


def paged_attn(q, k_pages, v_pages, block_table, row_begin, kv_len, scale, masks=None):
    """q [T, H, D], pages [n_pages, H_kv, page, D] float64 -> (out, size) [T, H, D]; rows of no stream are NaN, size is
    sum_j p_j |v_j| of each element."""
    T, H, D = q.shape
    _, H_kv, page, _ = k_pages.shape
    out, size = np.full((T, H, D), np.nan), np.full((T, H, D), np.nan)
    for s in range(len(kv_len)):
        r0, n, kv = int(row_begin[s]), int(row_begin[s + 1]) - int(row_begin[s]), int(kv_len[s])
        if n == 0:
            continue
        used = -(-kv // page)
        ids = [int(i) for i in block_table[s][:used]]
        for g in range(H_kv):
            keys = np.concatenate([k_pages[i, g] for i in ids])[:kv] if used else np.zeros((0, D))
            values = np.concatenate([v_pages[i, g] for i in ids])[:kv] if used else np.zeros((0, D))
            for i in range(n):
                if masks is None:
                    seen = np.arange(kv) <= kv - n + i
                else:
                    seen = np.array([j < kv - n or bool(int(masks[i]) >> (j - (kv - n)) & 1) for j in range(kv)], dtype=bool)
                for h in range(g * (H // H_kv), (g + 1) * (H // H_kv)):
                    if not seen.any():
                        out[r0 + i, h] = size[r0 + i, h] = 0.0
                        continue
                    e = keys[seen] @ q[r0 + i, h] * scale
                    p = np.exp(e - e.max())
                    p /= p.sum()
                    out[r0 + i, h] = p @ values[seen]
                    size[r0 + i, h] = p @ np.abs(values[seen])
    return out, size
