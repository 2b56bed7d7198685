"""Oracle for decoding from a paged key/value cache (fp64).

TEST INFRASTRUCTURE ONLY (see the package docstring).

Sec. 2.2 names a second query shape next to the scoring pass: a candidate continues a prompt and the answer is
rewarded.  The paper inherits what that takes from its serving engine; these are the definitions that
include/zo.h documents, written directly:

  cache_append     per-head RMS norm and rotary embedding of new rows at their positions in the cache, keys and values
                   into their slots
  attention_paged  softmax over the positions 0 .. pos of the row's sequence
  sample           temperature, top-k, top-p, min-p, then the inverse of the kept weights' running sum
  embed_rows       E[token] + E_pos[pos]

The cache is addressed one position at a time, sampling sorts: nothing is blocked, split or searched.
Pins: tests/test_oracle_decode.py.
"""
import numpy as np

from . import zo_oracle as _zo
from .zo_block import rms_norm


def row_places(cu_seqlens, kv_len):
    """(sequence, position) of every packed row."""
    cu = np.asarray(cu_seqlens, np.int64)
    return [(i, int(kv_len[i]) - int(cu[i + 1] - t)) for i in range(len(cu) - 1) for t in range(cu[i], cu[i + 1])]


def page_of(table, page_size, n_pages, seq, pos):
    """Page of a position, None when there is none in the pool."""
    if pos < 0 or pos // page_size >= table.shape[1]:
        return None
    pg = int(table[seq, pos // page_size])
    return pg if 0 <= pg < n_pages else None


def rotate(x, pos, theta):
    """Rotary embedding of heads x [.., dh] at position pos."""
    half = x.shape[-1] // 2
    ang = pos * float(theta) ** (-2.0 * np.arange(half) / (2 * half))
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def cache_append(q, k, v, cu_seqlens, n_heads, gamma_q, gamma_k, norm_eps, theta, K, V, table, kv_len, dtype="f64"):
    """Returns (Qout, K, V): new rows of queries, and the pools [page][kv head][slot][dh] with the new rows in."""
    q, k, v, K, V = (np.array(x, np.float64) for x in (q, k, v, K, V))
    n_pages, g, P, dh = K.shape
    for t, (i, pos) in enumerate(row_places(cu_seqlens, kv_len)):
        qh, kh = q[t].reshape(n_heads, dh), k[t].reshape(g, dh)
        if gamma_q is not None:
            qh, kh = rms_norm(qh, gamma_q, norm_eps), rms_norm(kh, gamma_k, norm_eps)
        if theta is not None and theta > 0:
            qh, kh = rotate(qh, pos, theta), rotate(kh, pos, theta)
        q[t] = _zo._round_out(qh, dtype).reshape(-1)
        page = page_of(table, P, n_pages, i, pos)
        if page is not None:
            K[page, :, pos % P] = _zo._round_out(kh, dtype)
            V[page, :, pos % P] = v[t].reshape(g, dh)
    return q, K, V


def attention_paged(q, cu_seqlens, n_heads, scale, K, V, table, kv_len, dtype="f64"):
    q = np.asarray(q, np.float64)
    n_pages, g, P, dh = K.shape
    out = np.zeros((q.shape[0], n_heads, dh))
    group = n_heads // g
    for t, (i, pos) in enumerate(row_places(cu_seqlens, kv_len)):
        at = [(page_of(table, P, n_pages, i, j), j % P) for j in range(pos + 1)]
        at = [(pg, sl) for pg, sl in at if pg is not None]
        if not at:
            continue
        pg, sl = np.array(at).T
        for h in range(n_heads):
            kh, vh = (np.asarray(X[pg, h // group, sl], np.float64) for X in (K, V))
            s = float(scale) * (kh @ q[t].reshape(n_heads, dh)[h])
            p = np.exp(s - s.max())
            out[t, h] = (p / p.sum()) @ vh
    return _zo._round_out(out.reshape(q.shape[0], -1), dtype)


def kept_tokens(z, temperature, top_k, top_p, min_p):
    """(kept tokens in order, their weights) of one row."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if len(order) == 0:
        return order, np.zeros(0)
    if not temperature > 0:
        return order[:1], np.ones(1)
    top = z[order[0]]
    w = (z[order] == top).astype(np.float64) if not np.isfinite(top) else np.exp(-(top - z[order]) / temperature)
    n_k = len(order) if top_k <= 0 else min(top_k, len(order))
    n = n_k
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[:n_k])[:-1]])
        n = int((before < top_p * w[:n_k].sum()).sum())
    if min_p > 0:
        n = min(n, int((w >= min_p).sum()))
    n = max(n, 1)
    return order[:n], w[:n]


def sample(z, temperature, top_k, top_p, min_p, u):
    """(tokens, prob, n_kept) of rows of logits; top_k, top_p, min_p may be None."""
    T = z.shape[0]
    token, prob, kept = np.full(T, -1, np.int32), np.zeros(T), np.zeros(T, np.int32)
    for t in range(T):
        idx, w = kept_tokens(z[t], temperature[t], 0 if top_k is None else int(top_k[t]),
                             1.0 if top_p is None else float(top_p[t]), 0.0 if min_p is None else float(min_p[t]))
        if len(idx) == 0:
            continue
        by_index = np.argsort(idx)
        cum = np.cumsum(w[by_index])
        target = min(max(float(u[t]), 0.0), 1.0) * cum[-1] if u[t] == u[t] else 0.0
        hit = np.nonzero(cum > target)[0]
        at = int(hit[0]) if len(hit) else int(np.nonzero(w[by_index])[0][-1])
        token[t], prob[t], kept[t] = idx[by_index[at]], w[by_index[at]] / cum[-1], len(idx)
    return token, prob, kept


def embed_rows(tokens, pos, E, E_pos, dtype="f64"):
    x = np.zeros((len(tokens), E.shape[1]))
    for t, tok in enumerate(tokens):
        if 0 <= tok < len(E):
            x[t] += E[tok]
        if E_pos is not None and 0 <= pos[t] < len(E_pos):
            x[t] += E_pos[pos[t]]
    return _zo._round_out(x, dtype)
