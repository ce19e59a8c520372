"""float64 reference of the operators around the attention: norm and rotation of queries and keys
with their gradients, appending to a paged cache, attention over it.  Plain NumPy; no code shared with
the GPU path."""
from __future__ import annotations

import numpy as np

from . import attention as A


def _pairs(rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _turn(x, pos, freq, interleaved, sign=1.0):
    """Rotates the pairs of x [T, heads, d] by sign * pos * freq."""
    rot = 0 if freq is None else 2 * len(freq)
    out = x.copy()
    if rot:
        ang = sign * np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)[None]
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        ia, ib = _pairs(rot, interleaved)
        a, b = x[..., ia], x[..., ib]
        out[..., ia] = a * c - b * s
        out[..., ib] = b * c + a * s
    return out


def norm_rope(x, w, eps, pos, freq, interleaved):
    """x [T, heads, d] -> y: x / sqrt(mean(x^2) + eps) * w (w None: x), rotated."""
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * np.asarray(w, np.float64)
    return _turn(x, pos, freq, interleaved)


def norm_rope_bwd(x, w, eps, pos, freq, interleaved, dy):
    """(dx, dw, magnitude of dx's terms per row, sum of |terms| of dw); dw None without w."""
    g = _turn(np.asarray(dy, np.float64), pos, freq, interleaved, -1.0)
    if w is None:
        return g, None, np.abs(g).max(-1, keepdims=True), None
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    xh = x * r
    dw, dw_abs = (g * xh).sum((0, 1)), np.abs(g * xh).sum((0, 1))
    g = g * w
    dx = r * (g - xh * np.mean(g * xh, -1, keepdims=True))
    size = r * (np.abs(g).max(-1, keepdims=True)
                + np.abs(xh).max(-1, keepdims=True) * np.mean(np.abs(g * xh), -1, keepdims=True))
    return dx, dw, size, dw_abs


def place(table, page_size, num_pages, b, t):
    """(page, slot) of token t of sequence b; None where the table holds no page for it."""
    if t < 0 or t // page_size >= table.shape[1]:
        return None
    page = int(table[b, t // page_size])
    return (page, t % page_size) if 0 <= page < num_pages else None


def append(k, v, kc, vc, table, kv_lens, cu):
    """Copies the rows of k, v [T, hkv, d] (already rotated) into copies of kc, vc [pages, page_size, hkv, d];
    returns them and the (page, slot, row) of every row stored."""
    kc, vc = np.array(kc, np.float64), np.array(vc, np.float64)
    stored = []
    for b in range(len(kv_lens)):
        n = int(cu[b + 1] - cu[b])
        for i in range(n):
            at = place(table, kc.shape[1], kc.shape[0], b, int(kv_lens[b]) - n + i)
            if at is not None:
                kc[at], vc[at] = k[cu[b] + i], v[cu[b] + i]
                stored.append((*at, int(cu[b]) + i))
    return kc, vc, stored


def paged_fwd(q, kc, vc, table, kv_lens, cu, causal, scale):
    """(out, lse, size) for the rows of q [T, hq, d] that belong to a sequence; size: the attention of |v|
    with the same weights, which errors of out are in proportion to.  Rows behind the last sequence: NaN."""
    q = np.asarray(q, np.float64)
    T, hq, d = q.shape
    out, size = np.full((T, hq, d), np.nan), np.full((T, hq, d), np.nan)
    lse = np.full((hq, T), np.nan)
    for b in range(len(kv_lens)):
        lo, hi = int(cu[b]), int(cu[b + 1])
        n, L = hi - lo, int(kv_lens[b])
        if n == 0:
            continue
        at = [place(table, kc.shape[1], kc.shape[0], b, t) for t in range(L)]
        js = [t for t in range(L) if at[t] is not None]
        k = np.array([kc[at[t]] for t in js], np.float64).reshape(len(js), kc.shape[2], d)
        v = np.array([vc[at[t]] for t in js], np.float64).reshape(len(js), kc.shape[2], d)
        o, l, a = np.zeros((n, hq, d)), np.full((hq, n), -np.inf), np.zeros((n, hq, d))
        group = hq // kc.shape[2]
        seen = np.array(js)[None] <= (np.arange(n)[:, None] + L - n) if causal else np.ones((n, len(js)), bool)
        for h in range(hq):
            if not len(js):
                break
            s = scale * q[lo:hi, h] @ k[:, h // group].T
            s = np.where(seen, s, -np.inf)
            m = s.max(1)
            live = np.isfinite(m)
            p = np.exp(s[live] - m[live, None])
            z = p.sum(1)
            l[h, live] = m[live] + np.log(z)
            o[live, h] = p @ v[:, h // group] / z[:, None]
            a[live, h] = p @ np.abs(v[:, h // group]) / z[:, None]
        out[lo:hi], lse[:, lo:hi], size[lo:hi] = o, l, a
    return out, lse, size


def gathered(kc, vc, table, kv_lens):
    """The sequences' keys and values end to end, as the varlen attention takes them (all pages there)."""
    ks, vs = [], []
    for b, L in enumerate(kv_lens):
        for t in range(int(L)):
            p, s = place(table, kc.shape[1], kc.shape[0], b, t)
            ks.append(kc[p, s])
            vs.append(vc[p, s])
    return np.array(ks), np.array(vs)


def paged_by_varlen(q, kc, vc, table, kv_lens, cu, causal, scale):
    """The same result from the oracle of the packed attention."""
    import torch
    k, v = gathered(kc, vc, table, kv_lens)
    cu_k = np.concatenate([[0], np.cumsum(kv_lens)]).astype(np.int32)
    return A.varlen_fwd(torch.from_numpy(np.asarray(q, np.float64)), torch.from_numpy(k), torch.from_numpy(v),
                        np.asarray(cu, np.int32), cu_k, causal, scale)
