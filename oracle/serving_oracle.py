"""Attention cache, attention and sampling around the linears, in numpy fp64.

No counterpart in the paper: these are the ordinary definitions, one token,
head and key at a time where that is the plainest way to say it.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rotate", "append", "visible_keys", "attend", "sample", "sample_row"]


def rotate(x, pos, cos, sin, interleaved):
    """x (heads, dim) turned at position `pos`; cos, sin (n_pos, rot / 2)."""
    y = np.array(x, np.float64)
    half = cos.shape[1]
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        c, s = np.float64(cos[pos, j]), np.float64(sin[pos, j])
        y[:, a] = x[:, a] * c - x[:, b] * s
        y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def append(q, k, v, k_pages, v_pages, token_start, own_len, pages, prefix_len, cos, sin, interleaved):
    """q (tokens, q_heads, dim), k and v (tokens, kv_heads, dim); returns the rotated q and copies of the two
    arrays (pages, kv_heads, page, dim) with the new tokens in them, all in fp64."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    k_pages, v_pages, q_out = np.array(k_pages, np.float64), np.array(v_pages, np.float64), np.empty_like(q)
    page = k_pages.shape[2]
    for s in range(len(own_len)):
        n = token_start[s + 1] - token_start[s]
        for i in range(n):
            t, at = token_start[s] + i, own_len[s] - n + i
            pos = max(0, prefix_len + at)
            q_out[t] = rotate(q[t], pos, cos, sin, interleaved)
            if at < 0:
                continue
            p = pages[s][at // page]
            if 0 <= p < len(k_pages):
                k_pages[p, :, at % page] = rotate(k[t], pos, cos, sin, interleaved)
                v_pages[p, :, at % page] = v[t]
    return q_out, k_pages, v_pages


def visible_keys(s, i, token_start, own_len, pages, prefix_pages, prefix_len, page):
    """(page, slot) of every key that new token i of sequence s sees."""
    n = token_start[s + 1] - token_start[s]
    seen = [(prefix_pages[j // page], j % page) for j in range(prefix_len)]
    return seen + [(pages[s][j // page], j % page) for j in range(max(0, own_len[s] - n + i + 1))]


def attend(q, k_pages, v_pages, token_start, own_len, pages, prefix_pages, prefix_len, scale):
    """q (tokens, q_heads, dim) -> (outputs, natural log-sum-exps, sum of |p v|) in fp64; a token that sees
    nothing: 0, -inf, 0."""
    q = np.asarray(q, np.float64)
    heads, dim = q.shape[1:]
    kv_heads, page = k_pages.shape[1:3]
    out, lse, mag = np.zeros_like(q), np.full(q.shape[:2], -np.inf), np.zeros_like(q)
    for s in range(len(own_len)):
        for i in range(token_start[s + 1] - token_start[s]):
            keys = visible_keys(s, i, token_start, own_len, pages, prefix_pages, prefix_len, page)
            if not keys:
                continue
            t = token_start[s] + i
            p, slot = np.array(keys).T
            for h in range(heads):
                g = h // (heads // kv_heads)
                x = np.asarray(k_pages[p, g, slot], np.float64) @ q[t, h] * scale
                top = x.max()
                w = np.exp(x - top)
                v = np.asarray(v_pages[p, g, slot], np.float64)
                out[t, h] = w @ v / w.sum()
                mag[t, h] = w @ np.abs(v) / w.sum()
                lse[t, h] = top + np.log(w.sum())
    return out, lse, mag


def sample_row(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, how far the decision was from another one: the least distance, as a share of the mass, between
    u or top_p and the edge of an interval that they fall in).  NaN logits count as -inf; a row without a
    logit above -inf gives -1."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    if z.size == 0 or z.max() == -np.inf:
        return -1, 1.0
    best = int(np.argmax(z))
    if not temperature > 0:
        return best, 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(z == z.max(), 1.0, np.exp((z - z.max()) / temperature))
    order = np.argsort(-z, kind="stable")
    margin = 1.0
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        before = np.cumsum(w[order]) - w[order]
        total = w[order].sum()
        margin = min(margin, np.abs(before / total - top_p).min())
        order = order[(before < top_p * total) | (np.arange(len(order)) == 0)]
    if min_p > 0:
        margin = min(margin, np.abs(w[order] - min_p).min())
        order = order[(w[order] >= min_p) | (np.arange(len(order)) == 0)]
    kept = np.sort(order)
    c = np.cumsum(w[kept])
    margin = min(margin, np.abs(c[:-1] / c[-1] - u).min() if len(kept) > 1 else 1.0)
    i = int(np.searchsorted(c, u * c[-1], side="right"))
    kept_w = np.flatnonzero(w[kept] > 0)
    return int(kept[min(i, kept_w[-1])]), float(margin)


def sample(z, u, temperature, top_k, top_p, min_p):
    rows = [sample_row(*a) for a in zip(z, u, temperature, top_k, top_p, min_p)]
    return np.array([r[0] for r in rows]), np.array([r[1] for r in rows])
