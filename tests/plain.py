"""Plain 64-bit forms of the operators around the path, in numpy."""
import numpy as np
import torch


def bf16(a):
    """a rounded to bf16, as float64."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16().double().numpy()


def page_grow(hist, new, page, es, free, head, table):
    """(table, slots, counts) of janus_page_grow."""
    table, slots, at, short = table.copy(), [], head, 0
    for b, (M, N) in enumerate(zip(hist, new)):
        had = -(-(M >> es) // page)
        given = {}
        for j in range(had, -(-((M + N) >> es) // page)):
            if at < len(free):
                given[j] = table[b, j] = free[at]
                at += 1
            else:
                short += 1
        for i in range(N):
            p = M + i + 1
            if p % (1 << es):
                slots.append(-1)
                continue
            c = (p >> es) - 1
            j = c // page
            have = table[b, j] if j < had else given.get(j, -1)
            slots.append(int(have) * page + c % page if have >= 0 else -1)
    return table, np.array(slots, np.int64), np.array([at - head, at, short], np.int32)


def positions(hist, new):
    return np.concatenate([np.arange(m, m + n) for m, n in zip(hist, new)]) if len(hist) else np.zeros(0, np.int64)


def rotate(x, pos, inv_freq, off, layout, mag=1.0, inverse=False):
    """x [tokens, heads, size] with its rotated elements turned, and the sum of the
    magnitudes of the two products behind each element."""
    x = x.astype(np.float64)
    y, m = x.copy(), np.abs(x)
    dim = 2 * len(inv_freq)
    for j, f in enumerate(inv_freq):
        a, b = (off + j, off + j + dim // 2) if layout == "half" else (off + 2 * j, off + 2 * j + 1)
        t = pos * f * (-1.0 if inverse else 1.0)
        c, s = mag * np.cos(t)[:, None], mag * np.sin(t)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        m[..., a] = m[..., b] = abs(mag) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, m


def attention(q, k, v, hist, new, rows_of, scale, es=0, tokens=None):
    """Dense causal attention, of all tokens or those listed.  rows_of(session, ids): pool rows.  Returns (out, lse, sum p |v|, and
    the largest sum |q k| * |scale| of a row's logits)."""
    T, H, _ = q.shape
    dv = v.shape[1]
    out, lse = np.zeros((T, H, dv)), np.full((T, H), -np.inf)
    mass, size = np.zeros((T, H, dv)), np.zeros((T, H))
    at = 0
    for b, (M, N) in enumerate(zip(hist, new)):
        for i in range(N):
            n = (M + i + 1) >> es
            if n > 0 and (tokens is None or at in tokens):
                r = rows_of(b, np.arange(n))
                kk, vv = k[r], v[r]
                x = q[at] @ kk.T * scale
                top = x.max(1)
                p = np.exp(x - top[:, None])
                l = p.sum(1)
                out[at] = p @ vv / l[:, None]
                mass[at] = p @ np.abs(vv) / l[:, None]
                lse[at] = top + np.log(l)
                size[at] = (np.abs(q[at]) @ np.abs(kk).T * abs(scale)).max(1)
            at += 1
    return out, lse, mass, size
