"""CPU oracle for the operators of a serving step (test infrastructure, NOT a product path).

Float64 numpy, one sequence, head and token after the other, from the definitions in the C header; imports nothing from
the package.  Caches are given as the values they stand for.
"""
from __future__ import annotations

import numpy as np


def spans(seq_start, T):
    """(first token, tokens) of every sequence."""
    return [(int(a), int(b) - int(a)) for a, b in zip(seq_start[:-1], seq_start[1:])]


def normed(x, g, eps):
    x = np.asarray(x, np.float64)
    return x if g is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(g, np.float64)


def rotated(x, cos, sin, interleaved):
    """x [heads, d], cos / sin [rot / 2]: plane j of the first rot values turned by its angle."""
    x = np.array(x, np.float64)
    if cos is None:
        return x
    half = len(cos)
    out = x.copy()
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        out[:, a] = x[:, a] * cos[j] - x[:, b] * sin[j]
        out[:, b] = x[:, b] * cos[j] + x[:, a] * sin[j]
    return out


def append(q, k, v, q_norm, k_norm, eps, cos, sin, interleaved, seq_start, kv_len, pages, page):
    """(q_out [T, Hq, d], {(page, slot): (k [Hkv, d], v [Hkv, d])}): a token of no sequence has NaN in q_out."""
    q_out = np.full(q.shape, np.nan)
    slots = {}
    for b, (t0, n) in enumerate(spans(seq_start, len(q))):
        for i in range(n):
            pos, t = int(kv_len[b]) - n + i, t0 + i
            if pos < 0:
                q_out[t] = 0
                continue
            c = s = None
            if cos is not None:
                known = pos < len(cos)
                c = cos[pos] if known else np.full(cos.shape[1], np.nan)
                s = sin[pos] if known else np.full(cos.shape[1], np.nan)
            q_out[t] = rotated(normed(q[t], q_norm, eps), c, s, interleaved)
            if pos // page < pages.shape[1]:
                slots[int(pages[b, pos // page]), pos % page] = (rotated(normed(k[t], k_norm, eps), c, s, interleaved),
                                                                np.asarray(v[t], np.float64))
    return q_out, slots


def attention(q, k_cache, v_cache, seq_start, kv_len, pages, scale, causal):
    """(o, spread, score): the output [T, Hq, d] (NaN for tokens of no sequence); sum_j p_j |v_j| of the same shape and
    the largest scale * sum |q k| of a row [T, Hq], which error bounds are made of.  Keys out of sight leave every sum."""
    T, Hq, d = q.shape
    page, Hkv = k_cache.shape[1], k_cache.shape[2]
    o, spread, score = np.full((T, Hq, d), np.nan), np.zeros((T, Hq, d)), np.zeros((T, Hq))
    for b, (t0, n) in enumerate(spans(seq_start, T)):
        ln = int(kv_len[b])
        at = [(int(pages[b, j // page]), j % page) for j in range(ln)]
        for h in range(Hq):
            if ln:
                pg, sl = np.array([x for x, _ in at]), np.array([x for _, x in at])
                K = k_cache[pg, sl, h // (Hq // Hkv)].astype(np.float64)
                V = v_cache[pg, sl, h // (Hq // Hkv)].astype(np.float64)
            for i in range(n):
                see = max(0, min(ln, ln - n + i + 1)) if causal else ln
                if see == 0:
                    o[t0 + i, h] = 0
                    continue
                qq = q[t0 + i, h].astype(np.float64)
                s = (K[:see] @ qq) * scale
                with np.errstate(invalid="ignore"):
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    o[t0 + i, h] = p @ V[:see]
                    spread[t0 + i, h] = p @ np.abs(V[:see])
                    score[t0 + i, h] = (np.abs(K[:see]) @ np.abs(qq)).max() * abs(scale)
    return o, spread, score


def verify(target, draft, tokens, u_accept, u_sample, seq_start):
    """(out, accepted, margin): margin[b] is the distance of the nearest comparison of sequence b from its border,
    relative to the values compared."""
    out, accepted, margin = np.full(len(target), -7), [], []
    for b, (t0, n) in enumerate(spans(seq_start, len(target))):
        a, near = 0, np.inf
        while a < n - 1:
            x = int(tokens[t0 + a])
            if not 0 <= x < target.shape[1]:
                break
            p, q = float(target[t0 + a, x]), 1.0 if draft is None else float(draft[t0 + a, x])
            left = float(u_accept[t0 + a]) * q
            if left != p:
                near = min(near, abs(left - p) / max(left, p))
            if not left < p:
                break
            a += 1
        accepted.append(a)
        if n == 0:
            margin.append(np.inf)
            continue
        p = target[t0 + a].astype(np.float64)
        w = p
        if a < n - 1:
            q = np.zeros_like(p)
            if draft is not None:
                q = draft[t0 + a].astype(np.float64)
            elif 0 <= int(tokens[t0 + a]) < len(p):
                q[int(tokens[t0 + a])] = 1.0
            with np.errstate(invalid="ignore"):
                w = np.maximum(p - q, 0)
            if w.sum() == 0:
                w = p
        w = np.maximum(w, 0)
        cum = np.cumsum(w)
        new = -1
        if np.isfinite(cum[-1]) and cum[-1] > 0:
            x = float(u_sample[b]) * cum[-1]
            over = np.nonzero((cum > x) & (w > 0))[0]
            new = int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])
            if x > 0:
                near = min(near, np.abs(cum - x).min() / cum[-1])
        out[t0:t0 + n] = -1
        out[t0:t0 + a] = tokens[t0:t0 + a]
        out[t0 + a] = new
        margin.append(near)
    return out, np.array(accepted), np.array(margin)
