"""Serving a batch of requests from one shared prefix (fp64 oracle; test infrastructure).

Each request's added tokens form its tail, kept in pages of a pool; a step of the batch plans
pages and slots, writes the new rows and attends.  Plain loops over requests and tokens.
"""
from __future__ import annotations

import numpy as np

NO_PAGES, TABLE_FULL, NO_TOKENS, BAD_LENGTH = 1, 2, 4, 8


def plan(have, add, page, free_pages, n_free, table, n_tok, n_pages):
    """Block tables and slot maps of a step; `table` is not changed in place.  Returns a dict."""
    n_req, max_pages = table.shape
    why, need = 0, 0
    for h, n in zip(have, add):
        if h < 0 or n < 0:
            why |= BAD_LENGTH
            continue
        need += -(-(h + n) // page) - (-(-h // page))
        if -(-(h + n) // page) > max_pages:
            why |= TABLE_FULL
    if need > min(n_free, len(free_pages)):
        why |= NO_PAGES
    if sum(n for h, n in zip(have, add) if h >= 0 and n >= 0) > n_tok:
        why |= NO_TOKENS
    out = dict(table=table.copy(), kv_len=np.array(have), q_start=np.zeros(n_req + 1, int), slots=np.full(n_tok, -1),
               positions=np.full(n_tok, -1), n_free=n_free, info=np.array([0, 0, why, min(need, 2 ** 31 - 1)]))
    if why:
        return out
    stack, t = list(free_pages[:n_free]), 0
    for r, (h, n) in enumerate(zip(have, add)):
        for pos in range(h, h + n):
            if pos % page == 0:
                out["table"][r, pos // page] = stack.pop()
            p = out["table"][r, pos // page]
            out["slots"][t] = p * page + pos % page if 0 <= p < n_pages else -1
            out["positions"][t] = pos
            t += 1
        out["kv_len"][r] = h + n
        out["q_start"][r + 1] = t
    out["n_free"] = len(stack)
    out["info"] = np.array([t, need, 0, need])
    return out


def rotate(x, pos, base):
    """Half-split rotary embedding of rows x [tokens][heads][d] at positions pos [tokens]."""
    d = x.shape[-1]
    a = np.asarray(pos, np.float64)[:, None, None] * base ** (-2.0 * np.arange(d // 2) / d)
    u, v = x[..., :d // 2], x[..., d // 2:]
    return np.concatenate([u * np.cos(a) - v * np.sin(a), v * np.cos(a) + u * np.sin(a)], -1)


def prefix_attend(Q, K, V, tails_k, tails_v, q_start, kv_len, scale):
    """Q [n_tok][n_q][d]; K, V [H][T][d] (T may be 0); tails: per request [H][len][d].  Rows of
    no request are NaN.  Returns (O, lse, A, S): A = sum_x p_x |v_x| and S = the largest
    scale * sum_f |q_f k_f| of the row's scores, for error bounds."""
    n_tok, n_q, d = Q.shape
    H = K.shape[0]
    O, A = np.full(Q.shape, np.nan), np.full(Q.shape, np.nan)
    lse, S = np.full((n_tok, n_q), np.nan), np.full((n_tok, n_q), np.nan)
    for r in range(len(kv_len)):
        n = q_start[r + 1] - q_start[r]
        for i in range(n):
            t, seen = q_start[r] + i, max(0, kv_len[r] - n + i + 1)
            for j in range(n_q):
                h = j // (n_q // H)
                k = np.concatenate([K[h], tails_k[r][h][:seen]])
                v = np.concatenate([V[h], tails_v[r][h][:seen]])
                if not len(k):
                    O[t, j], A[t, j], lse[t, j], S[t, j] = 0, 0, -np.inf, 0
                    continue
                s = scale * (k @ Q[t, j])
                m = s.max()
                p = np.exp(s - m)
                O[t, j], A[t, j] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
                lse[t, j] = m + np.log(p.sum())
                S[t, j] = scale * (np.abs(k) @ np.abs(Q[t, j])).max()
    return O, lse, A, S
