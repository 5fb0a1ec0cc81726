"""fp64 oracle of the paged key/value cache: rotary positions, the append, the attention
over pages. NumPy, one token and head at a time, written from the formulas in
include/dv.h."""
import math

import numpy as np


def freqs(rot, base=10000.0, rule="plain", factor=1.0, orig_len=0.0, low=1.0, high=32.0):
    """Radians per position of each of rot/2 pairs."""
    out = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2.0)) if rule == "ntk" else base
        f = b ** (-2.0 * i / rot)
        if rule == "linear":
            f /= factor
        elif rule == "parts":
            turns = orig_len * f / (2.0 * math.pi)
            g = min(max((turns - low) / (high - low), 0.0), 1.0)
            f = f * g + f / factor * (1.0 - g)
        out.append(f)
    return np.array(out)


def rope(x, pos, freq, layout="half", mscale=1.0, inverse=False):
    """x [T][H][dh] with its first 2 len(freq) elements rotated at pos [T]."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    n = len(freq)
    for t in range(x.shape[0]):
        for i in range(n):
            a = float(pos[t]) * float(freq[i]) * (-1.0 if inverse else 1.0)
            c, s = mscale * math.cos(a), mscale * math.sin(a)
            j0, j1 = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
            out[t, :, j0] = x[t, :, j0] * c - x[t, :, j1] * s
            out[t, :, j1] = x[t, :, j0] * s + x[t, :, j1] * c
    return out


def append(pool, x, table, seq, pos, heads=None):
    """A copy of pool [n_pages][H][page][dh] (fp64) with x [T][H][dh] in the tokens' rows."""
    pool = np.array(pool, dtype=np.float64)
    page = pool.shape[2]
    for t in range(len(pos)):
        if pos[t] < 0:
            continue
        g, r = int(table[seq[t], pos[t] // page]), int(pos[t]) % page
        for h in (range(pool.shape[1]) if heads is None else heads[t]):
            pool[g, int(h), r] = x[t, int(h)]
    return pool


def rows(pool, table_row, n, h):
    """Rows 0..n-1 of head h of a sequence, from its pages."""
    page = pool.shape[2]
    return np.array([pool[int(table_row[p // page]), h, p % page] for p in range(n)], dtype=np.float64).reshape(n, -1)


def attn(q, K, V, table, seq, pos, scale, group, heads=None):
    """Per (token, place): output, log-sum-exp, the largest sum of |products| of a logit (times |scale|) and
    sum_p p |V| (for error bounds)."""
    q = np.asarray(q, dtype=np.float64)
    T, n, dh = q.shape
    out, lse = np.zeros((T, n, dh)), np.full((T, n), -np.inf)
    mag, absv = np.zeros((T, n)), np.zeros((T, n, dh))
    for t in range(T):
        m = int(pos[t]) + 1
        if m <= 0:
            continue
        cache = {}
        for j in range(n):
            h = (j if heads is None else int(heads[t][j])) // group
            if h not in cache:
                cache[h] = rows(K, table[seq[t]], m, h), rows(V, table[seq[t]], m, h)
            k, v = cache[h]
            s = k @ q[t, j] * scale
            top = s.max()
            w = np.exp(s - top)
            out[t, j] = w @ v / w.sum()
            lse[t, j] = top + math.log(w.sum())
            mag[t, j] = abs(scale) * (np.abs(k) @ np.abs(q[t, j])).max()
            absv[t, j] = w @ np.abs(v) / w.sum()
    return out, lse, mag, absv


def layer(x, a, K, V, table, seq, pos, heads, scale, freq=None, layout="half", mscale=1.0):
    """The sparsified attention on pages: out[b] = bo + sum over the heads of b of H_i(x[b]) W^O_i, the heads' keys (rotated
    if freq is given) and values of every token in the pages before any attends. a: Wq, Wk, Wv, WoT [H*dh][d], bq, bk, bv,
    bo or none of them. Returns out, K, V."""
    x = np.asarray(x, dtype=np.float64)
    H, dh = K.shape[1], K.shape[3]
    qkv = []
    for w, b in (("Wq", "bq"), ("Wk", "bk"), ("Wv", "bv")):
        y = x @ np.asarray(a[w], dtype=np.float64).T
        qkv.append((y if a.get(b) is None else y + np.asarray(a[b], dtype=np.float64)).reshape(-1, H, dh))
    q, k, v = qkv
    if freq is not None:
        q, k = (rope(t, np.maximum(pos, 0), freq, layout, mscale) for t in (q, k))
    K, V = append(K, k, table, seq, pos, heads), append(V, v, table, seq, pos, heads)
    q = np.array([q[b, np.asarray(heads[b], dtype=int)] for b in range(len(x))]).reshape(len(x), -1, dh)
    h, _, _, _ = attn(q, K, V, table, seq, pos, scale, 1, heads)
    out = np.zeros(x.shape) if a.get("bo") is None else np.tile(np.asarray(a["bo"], dtype=np.float64), (len(x), 1))
    for b in range(len(x)):
        for j, i in enumerate(heads[b]):
            out[b] += h[b, j] @ np.asarray(a["WoT"][int(i) * dh:(int(i) + 1) * dh], dtype=np.float64)
    return out, K, V
