"""Oracle for the fine tokens' own attention: norm and rotation of queries and
keys per head, a paged cache of keys and values, and new tokens' attention
over it.

Test infrastructure only (see the package docstring). Sec. 5.1 allows rotary
positions and Eq. 19's softmax attention over fine tokens; what they leave open
is read as follows:
* z = x / sqrt(mean(x^2) + eps) * gamma over a head's channels (no norm: z = x).
* Pair p of the first rot channels, (p, rot/2 + p) or (2p, 2p + 1), turns by
  its axis' coordinate times freqs[p]; the other channels stay.
* Query head h reads key/value head h // (n_heads / n_kv_heads).
* A token at row r of its sequence sees rows j <= r; with a window w > 0 those
  with j > r - w or j < sinks. A token that sees nothing gives zeros.

Everything is float64 and one row at a time; each function also returns the
magnitudes that bound an implementation's rounding errors.
"""
from __future__ import annotations

import numpy as np


def pair_members(rot: int, pairs_style: bool):
    """Channel indices (a, b) of the rot / 2 pairs."""
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if pairs_style else (p, rot // 2 + p)


def angles(positions, freqs, axis_pairs):
    """[T, rot / 2] angles of integer positions [n_axes, T]."""
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    return np.asarray(positions, dtype=np.float64)[axis].T * np.asarray(freqs, dtype=np.float64)


def rotate(z, ang, rot, pairs_style):
    """z [T, H, D] turned by ang [T, rot / 2]."""
    a, b = pair_members(rot, pairs_style)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = np.array(z, dtype=np.float64)
    y[..., a] = z[..., a] * c - z[..., b] * s
    y[..., b] = z[..., a] * s + z[..., b] * c
    return y


def _reach(z, rot, pairs_style):
    """Per channel: the length of its pair (what a rotation can carry into it)."""
    a, b = pair_members(rot, pairs_style)
    r = np.abs(z)
    r[..., a] = r[..., b] = np.abs(z[..., a]) + np.abs(z[..., b])
    return r


def norm_rope(x, gamma, eps, norm, ang, rot, pairs_style):
    """(y, magnitude) of rows x [T, H, D]."""
    x = np.asarray(x, dtype=np.float64)
    z = x
    if norm:
        z = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * (1.0 if gamma is None else gamma)
    return rotate(z, ang, rot, pairs_style), _reach(z, rot, pairs_style)


def norm_rope_backward(x, gamma, eps, norm, ang, rot, pairs_style, dy):
    """(dx, dgamma, magnitude of dx, magnitude of dgamma): the chain rule, with
    the rotation's transpose (the turn back)."""
    dy = np.asarray(dy, dtype=np.float64)
    dz, mag = rotate(dy, -ang, rot, pairs_style), _reach(dy, rot, pairs_style)
    if not norm:
        return dz, None, mag, None
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    xn = x * r
    gam = np.ones(x.shape[-1]) if gamma is None else np.asarray(gamma, dtype=np.float64)
    g = dz * gam
    dx = r * (g - xn * np.mean(g * xn, -1, keepdims=True))
    dx_mag = r * (mag * np.abs(gam) + np.abs(xn) * np.mean(mag * np.abs(gam * xn), -1, keepdims=True))
    return dx, np.sum(dz * xn, (0, 1)), dx_mag, np.sum(mag * np.abs(xn), (0, 1))


def token_rows(kv_len, cu_tokens):
    """(sequence, row) of every token that belongs to one; cu_tokens None: one each."""
    b = len(kv_len)
    cu = np.arange(b + 1) if cu_tokens is None else np.asarray(cu_tokens)
    return [(s, int(kv_len[s]) - int(cu[s + 1] - cu[s]) + i) for s in range(b) for i in range(int(cu[s + 1] - cu[s]))]


def place(table, row, page_size, n_pages):
    """(page, slot) of a row in one sequence's table, or None."""
    if row < 0 or row >= len(table) * page_size:
        return None
    page = int(table[row // page_size])
    return (page, row % page_size) if 0 <= page < n_pages else None


def visible(row, rows, window, sinks):
    """Which rows j < rows a token at `row` sees."""
    j = np.arange(rows)
    seen = j <= row
    return seen & ((j > row - window) | (j < sinks)) if window > 0 else seen


def paged_attention(q, k_pages, v_pages, table, kv_len, cu_tokens, scale, window=0, sinks=0):
    """(out, lse, score error scale, value magnitude) for q [T, Hq, D]; entries
    of tokens behind the last sequence are NaN. The score error scale is
    max_j scale * sum_d |q_d k_jd|, the value magnitude sum_j p_j |v_j|."""
    q = np.asarray(q, dtype=np.float64)
    n_pages, hk, ps, d = k_pages.shape
    hq = q.shape[1]
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, err = np.full(q.shape[:2], np.nan), np.full(q.shape[:2], np.nan)
    for t, (s, row) in enumerate(token_rows(kv_len, cu_tokens)):
        at = [(j, place(table[s], j, ps, n_pages)) for j in np.nonzero(visible(row, max(row + 1, 0), window, sinks))[0]]
        at = [pl for _, pl in at if pl is not None]
        pages, slots = np.array([a[0] for a in at], int), np.array([a[1] for a in at], int)
        for h in range(hq):
            if not at:
                out[t, h], mag[t, h], lse[t, h], err[t, h] = 0, 0, -np.inf, 0
                continue
            k = np.asarray(k_pages[pages, h * hk // hq, slots], dtype=np.float64)
            v = np.asarray(v_pages[pages, h * hk // hq, slots], dtype=np.float64)
            sc = scale * (k @ q[t, h])
            top = sc.max()
            p = np.exp(sc - top)
            lse[t, h] = top + np.log(p.sum())
            p /= p.sum()
            out[t, h], mag[t, h] = p @ v, p @ np.abs(v)
            err[t, h] = abs(scale) * (np.abs(k) @ np.abs(q[t, h])).max()
    return out, lse, err, mag
