"""fp64 reference of the calls on a cache in pages (numpy, from the definitions; shares no code with the HIP path).

Besides results the attention returns, per (token, head), what bounds of rounding errors need: the weighted sum of |v|, the
largest scale * sum |q_d k_d| over the visible rows and the number of those."""
from __future__ import annotations

import math

import numpy as np


def row_of(pages, table_row, page_size, r):
    """[Hkv][D] row r of a sequence."""
    return pages[table_row[r // page_size], :, r % page_size]


def gather(pages, table_row, page_size, n):
    """[n][Hkv][D] the first n rows."""
    if n == 0:
        return np.zeros((0, pages.shape[1], pages.shape[3]))
    return np.stack([row_of(pages, table_row, page_size, r) for r in range(n)]).astype(np.float64)


def rotate(x, cos, sin, rot, pairs):
    """x [heads][D] with its first `rot` elements turned by the angles whose cosines and sines are given."""
    y = np.array(x, dtype=np.float64)
    for j in range(rot // 2):
        a, b = (j, j + rot // 2) if pairs == "halves" else (2 * j, 2 * j + 1)
        y[:, a] = x[:, a] * cos[j] - x[:, b] * sin[j]
        y[:, b] = x[:, b] * cos[j] + x[:, a] * sin[j]
    return y


def append(k_pages, v_pages, page_table, lens, q, k, v, offsets, positions, rot_table, rot, pairs, page_size):
    """New (k_pages, v_pages, lens, q) in fp64; q, k, v [total][heads][D].  Page entries that name no page drop their rows."""
    kp, vp, lens = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64), np.array(lens)
    qo = None if q is None else np.array(q, dtype=np.float64)
    n_pages, cap = len(kp), page_table.shape[1] * page_size
    for b in range(len(lens)):
        n = offsets[b + 1] - offsets[b]
        fits = lens[b] >= 0 and lens[b] + n <= cap
        for t in range(n):
            at = offsets[b] + t
            pos = int(lens[b]) + t if positions is None else int(positions[at])
            cs = (None, None)
            if rot:
                entry = rot_table[min(max(pos, 0), len(rot_table) - 1)].astype(np.float64)
                cs = entry[:rot // 2], entry[rot // 2:]
            if q is not None:
                qo[at] = rotate(q[at].astype(np.float64), *cs, rot, pairs)
            if not fits:
                continue
            r = int(lens[b]) + t
            page = page_table[b][r // page_size]
            if 0 <= page < n_pages:
                kp[page, :, r % page_size] = rotate(k[at].astype(np.float64), *cs, rot, pairs)
                vp[page, :, r % page_size] = v[at]
        if fits:
            lens[b] += n
    return kp, vp, lens, qo


def attend(q, k, v, pos, scale, window=0, sinks=0, prefix=0):
    """q [n][Hq][D] at rows pos[n] of the own rows; k, v [prefix + rows][Hkv][D], the prefix ahead.  Returns dict of
    out [n][Hq][D], lse [n][Hq], absv [n][Hq][D], zabs [n][Hq], seen [n]."""
    n, Hq, D = q.shape
    Hkv, rows = k.shape[1], k.shape[0]
    G = Hq // Hkv
    j = np.arange(rows) - prefix
    i = np.asarray(pos)[:, None]
    see = j[None] <= i
    if window:
        see &= (j[None] > i - window) | (j[None] < sinks)
    see |= (j < 0)[None]
    out, absv = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse, zabs = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for h in range(Hq):
        kk, vv = k[:, h // G].astype(np.float64), v[:, h // G].astype(np.float64)
        used = see.any(0)                                    # rows that nobody sees may hold anything
        kk, vv = np.where(used[:, None], kk, 0.0), np.where(used[:, None], vv, 0.0)
        z = np.where(see, q[:, h].astype(np.float64) @ kk.T * scale, -np.inf)
        mag = np.where(see, np.abs(q[:, h]).astype(np.float64) @ np.abs(kk).T * scale, 0.0)
        for t in range(n):
            if not see[t].any():
                continue
            m = z[t].max()
            e = np.exp(z[t] - m)
            lse[t, h] = m + math.log(e.sum())
            w = e / e.sum()
            out[t, h], absv[t, h], zabs[t, h] = w @ vv, w @ np.abs(vv), mag[t].max()
    return dict(out=out, lse=lse, absv=absv, zabs=zabs, seen=see.sum(1))
