"""Plain 64-bit NumPy forms of the attention half of a decoder layer, written from the definitions: paged attention with a
shared prefix, the append with rotation, the gated block norm.  Test infrastructure only.

Operands are float64 arrays holding the exact values of the library's inputs.  ``attend`` also returns what error bounds are
made of: sum_j w_j |v_j| and sum_j |v_j| of every output and the largest sum_i |q_i k_i| of every row."""
from __future__ import annotations

import numpy as np


def gather(pages: np.ndarray, table: np.ndarray, n: int) -> np.ndarray:
    """[n, heads, dim] at positions 0..n-1 of pages [n_pages, page_size, heads, dim]."""
    ps = pages.shape[1]
    p = np.arange(n)
    return pages[table[p // ps], p % ps]


def attend(q, k_pages, v_pages, seq_len, table, prefix_pages, prefix_len, window, scale):
    """q [seqs, q_len, heads, dim] -> (out, lse, absout, absv, absqk)."""
    B, m, H, D = q.shape
    hk, ps = k_pages.shape[2], k_pages.shape[1]
    G = H // hk
    out, absout, absv = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    lse, absqk = np.full((B, m, H), -np.inf), np.zeros((B, m, H))
    for b in range(B):
        n = int(seq_len[b])
        row = np.array(table[b])
        for i in range(m):
            hi = n - m + i + 1
            if hi <= 0:
                continue
            lo = max(0, hi - window) if window else 0
            pos = np.arange(lo, hi)
            shared = pos < prefix_len
            ids = np.where(shared, np.asarray(prefix_pages)[np.minimum(pos // ps, max(len(prefix_pages) - 1, 0))] if len(prefix_pages) else 0,
                           row[pos // ps])
            k, v = k_pages[ids, pos % ps], v_pages[ids, pos % ps]  # [keys, hk, D]
            for j in range(hk):
                h = slice(j * G, (j + 1) * G)
                qh, kh, vh = q[b, i, h], k[:, j], v[:, j]
                s = qh @ kh.T * scale
                top = s.max(1, keepdims=True)
                e = np.exp(s - top)
                total = e.sum(1, keepdims=True)
                w = e / total
                out[b, i, h], absout[b, i, h], absv[b, i, h] = w @ vh, w @ np.abs(vh), np.abs(vh).sum(0)
                lse[b, i, h] = (top + np.log(total))[:, 0]
                absqk[b, i, h] = (np.abs(qh) @ np.abs(kh).T).max(1)
    return out, lse, absout, absv, absqk


def rotate(x, pos, table, interleaved):
    """x [tokens, heads, dim] turned by rows ``pos`` of table [positions, r] (cosines, then sines); table None, or a negative position: as it
    is."""
    y = x.copy()
    if table is None:
        return y
    r = table.shape[1]
    for t, p in enumerate(pos):
        if p < 0:
            continue
        for i in range(r // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
            c, s = table[p, i], table[p, r // 2 + i]
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def append(k, v, k_pages, v_pages, seq, pos, table, rope, interleaved):
    """New copies of the pages with the tokens' keys and values stored, and the number of slots written."""
    k_pages, v_pages = k_pages.copy(), v_pages.copy()
    ps, n = k_pages.shape[1], 0
    kr = rotate(k, pos, rope, interleaved)
    for t in range(len(pos)):
        if seq[t] < 0 or pos[t] < 0:
            continue
        page = table[seq[t], pos[t] // ps]
        k_pages[page, pos[t] % ps], v_pages[page, pos[t] % ps] = kr[t], v[t]
        n += 1
    return k_pages, v_pages, n


def block_norm(x, y, post, w_post, gate, scale, pre, w_pre, eps):
    """(x', h, |scale gate t|) for rows of float64."""
    t = np.zeros_like(x)
    if y is not None:
        t = y / np.sqrt((y * y).mean(1, keepdims=True) + eps) if post else y.copy()
        if w_post is not None:
            t = t * w_post
        if gate is not None:
            t = t * gate
        t = t * scale
    x2 = x + t
    h = x2 / np.sqrt((x2 * x2).mean(1, keepdims=True) + eps) if pre else x2.copy()
    if w_pre is not None:
        h = h * w_pre
    return x2, h, np.abs(t)
