"""Token embeddings, the gated linear recurrence and token scores in float64.

TEST INFRASTRUCTURE ONLY (see ``oracle/ir.py``). Written straight from the
formulas, one step, token or row at a time; the gradients are hand-derived
adjoints of the formulas (pinned by finite differences and by an independent
library's autograd), without any of the product's reorderings.
"""
from __future__ import annotations

import numpy as np


def embedding(table, ids, scale):
    """out[i] = scale table[ids[i]]; id -1 gives zeros, another id out of range NaN."""
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    out = np.full((len(ids), table.shape[1]), np.nan)
    for i, v in enumerate(ids):
        if v == -1:
            out[i] = 0.0
        elif 0 <= v < len(table):
            out[i] = scale * table[v]
    return out


def embedding_grad(dout, ids, vocab, scale):
    """(dtable, sum of the absolute terms of each entry, tokens of each row)."""
    dout, ids = np.asarray(dout, np.float64), np.asarray(ids)
    d = np.zeros((vocab, dout.shape[1]))
    mag, cnt = np.zeros_like(d), np.zeros(vocab, np.int64)
    for i, v in enumerate(ids):
        if 0 <= v < vocab:
            d[v] += scale * dout[i]
            mag[v] += np.abs(scale * dout[i])
            cnt[v] += 1
    return d, mag, cnt


def sigmoid(z):
    z = np.asarray(z, np.float64)
    s = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, s) / (1.0 + s)


def _live(lens, T, B):
    n = np.full(B, T) if lens is None else np.clip(np.asarray(lens, np.int64), 0, T)
    return np.arange(T)[:, None] < n[None, :]


def gated_scan(z, x, h0, lens, coupled):
    """States h [T + 1, B, H] (h[0] = h0) and hs [T, B, H], zero where a sequence has ended."""
    z, x = np.asarray(z, np.float64), np.asarray(x, np.float64)
    T, B, H = z.shape
    live = _live(lens, T, B)
    h = np.zeros((T + 1, B, H))
    if h0 is not None:
        h[0] = h0
    hs = np.zeros((T, B, H))
    for t in range(T):
        h[t + 1] = h[t]
        for b in np.flatnonzero(live[t]):
            a = sigmoid(z[t, b])
            u = sigmoid(-z[t, b]) * x[t, b] if coupled else x[t, b]
            h[t + 1, b] = a * h[t, b] + u
            hs[t, b] = h[t + 1, b]
    return h, hs


def gated_scan_vjp(z, x, h0, lens, coupled, dhs, dhT):
    """(dz, dx, dh0) for the adjoints of hs and of the last state (None: zeros)."""
    z, x = np.asarray(z, np.float64), np.asarray(x, np.float64)
    T, B, H = z.shape
    live = _live(lens, T, B)
    h, _ = gated_scan(z, x, h0, lens, coupled)
    mu = np.zeros((B, H)) if dhT is None else np.array(dhT, np.float64)
    dz, dx = np.zeros((T, B, H)), np.zeros((T, B, H))
    for t in range(T - 1, -1, -1):
        for b in np.flatnonzero(live[t]):
            a, c = sigmoid(z[t, b]), sigmoid(-z[t, b])
            lam = mu[b] + (0.0 if dhs is None else np.asarray(dhs[t, b], np.float64))
            dx[t, b] = c * lam if coupled else lam
            dz[t, b] = lam * (h[t, b] - x[t, b] if coupled else h[t, b]) * a * c
            mu[b] = a * lam
    return dz, dx, mu


def token_scores(logits, tokens, scale, top):
    """dict of logp, lse, entropy, top_ids, top_logp of each row of logits.

    The largest logits come first, the lower class first among equals; a NaN
    counts as -infinity in that order. A row whose scaled logits are all below
    -1e30 (masked everywhere) has lse = logp = top_logp = -infinity and entropy 0;
    a row with NaN or +infinity has NaN.
    """
    z = np.asarray(logits, np.float64)
    R, V = z.shape
    out = {"logp": np.zeros(R), "lse": np.zeros(R), "entropy": np.zeros(R),
           "top_ids": np.zeros((R, top), np.int64), "top_logp": np.zeros((R, top))}
    for i in range(R):
        order = np.argsort(-np.where(np.isnan(z[i]), -np.inf, z[i]), kind="stable")[:top]
        y = scale * z[i]
        if np.isnan(y).any() or (y == np.inf).any():
            lp, lse, ent = np.full(V, np.nan), np.nan, np.nan
        elif (y < -1e30).all():
            lp, lse, ent = np.full(V, -np.inf), -np.inf, 0.0
        else:
            m = y.max()
            total = np.log(np.exp(y - m).sum())
            lse, lp = m + total, (y - m) - total
            some = lp > -np.inf
            ent = -(np.exp(lp[some]) * lp[some]).sum()
        out["lse"][i], out["entropy"][i] = lse, ent
        out["top_ids"][i], out["top_logp"][i] = order, lp[order]
        if tokens is not None:
            t = int(tokens[i])
            out["logp"][i] = 0.0 if t == -1 else lp[t] if 0 <= t < V else np.nan
    return out


def token_scores_vjp(logits, tokens, scale, dlogp, dentropy):
    """d(logits) for the adjoints of logp and of the entropy (None: zeros)."""
    z = np.asarray(logits, np.float64)
    R, V = z.shape
    s = token_scores(z, None, scale, 0)
    d = np.zeros((R, V))
    for i in range(R):
        lse, ent = s["lse"][i], s["entropy"][i]
        t = -1 if dlogp is None else int(tokens[i])
        if t != -1 and not 0 <= t < V:
            d[i] = np.nan
            continue
        if lse == -np.inf:
            continue
        lp = scale * z[i] - lse
        p = np.exp(lp)
        if t != -1:
            hot = np.zeros(V)
            hot[t] = 1.0
            d[i] += dlogp[i] * (hot - p)
        if dentropy is not None and dentropy[i] != 0:  # a row without adjoints is zero
            d[i] -= dentropy[i] * np.where(p > 0, p * (np.where(p > 0, lp, 0.0) + ent), 0.0)
    return d * scale
