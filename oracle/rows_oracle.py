"""CPU oracle of the row operators (top logits, distillation, beam selection, state reordering), plain numpy float64.

TEST INFRASTRUCTURE, NOT A PRODUCT PATH; it shares no code with the CUDA library.  Each function states the operator's
definition and nothing else: whole rows, no blocking, no reordering of sums.
"""
from __future__ import annotations

import numpy as np


def log_sum_exp(z, T):
    """log sum_v exp(z_v / T) along the last axis; -inf for a row of -inf, NaN where it holds NaN or +inf."""
    z = np.asarray(z, np.float64) / T
    m = z.max(-1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        lse = np.log(np.exp(z - np.where(np.isneginf(m), 0.0, m)).sum(-1)) + np.where(np.isneginf(m), 0.0, m)[..., 0]
    return np.where(np.isposinf(z).any(-1), np.nan, lse)


def log_softmax(z, T):
    """z_v / T - log sum_u exp(z_u / T) of one row; differences first, so that a row of huge equal values keeps its digits."""
    z = np.asarray(z, np.float64)
    d = (z - z.max()) / T
    return d - log_sum_exp(d, 1.0)


def top_logits(z, k, T):
    """(values, tokens, lse): the k largest of each row, descending, ties in token order, NaN below -inf."""
    z = np.asarray(z, np.float64)
    below = np.isnan(z)
    order = np.lexsort((np.broadcast_to(np.arange(z.shape[-1]), z.shape), np.where(below, 0.0, -z), below))[..., :k]
    return np.take_along_axis(z, order, -1), order.astype(np.int32), log_sum_exp(z, T)


def listed_mass(v, lse, T):
    """p of the listed logits v: against the target's log-sum-exp, or renormalised over the list where that is None."""
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        log_p = v / T - float(lse) if lse is not None else v if np.isneginf(v).all() else log_softmax(v, T)
        return np.where(np.isneginf(v), 0.0, np.exp(log_p))


def distill_row(z, values, tokens, lse, T, weight=1.0):
    """(loss, gradient * weight) of one row; lse None: renormalised over the list.  Gradient [V]."""
    z = np.asarray(z, np.float64)
    V = len(z)
    keep = np.asarray(tokens) >= 0
    y, v = np.asarray(tokens)[keep].astype(int), np.asarray(values, np.float64)[keep]
    if (np.asarray(tokens) >= V).any() or (np.asarray(tokens) < -1).any() or len(set(y.tolist())) < len(y):
        return np.nan, np.zeros(V)
    if len(y) == 0:
        return 0.0, np.zeros(V)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        p = listed_mass(v, lse, T)
        if np.isneginf(z).all():
            return (np.inf if (p > 0).any() else 0.0), np.zeros(V)
        log_q = log_softmax(z, T)
        q = np.exp(log_q)
        outside = np.ones(V, bool)
        outside[y] = False
        Q = q[outside].sum()
        R = max(0.0, 1.0 - p.sum()) if lse is not None and Q > 0 else 0.0
        loss = sum(a * (np.log(a) - b) for a, b in zip(p, log_q[y]) if a > 0)
        share = 0.0
        if R > 0:
            loss += R * (np.log(R) - np.log(Q))
            share = R / Q
        if np.isnan(q).any():
            return np.nan, np.full(V, np.nan)
        mass = p.sum() + R
        g = q * np.where(outside, mass - share, mass)
        g[y] -= p
    return loss, g * weight / T


def distill(z, values, tokens, lse, T, weight):
    """(loss [n], gradient [n, V], tolerance scale [n, V]); rows of weight 0 have no gradient."""
    loss, grad = [], []
    for n in range(len(z)):
        a, g = distill_row(z[n], values[n], tokens[n], None if lse is None else lse[n], T, weight[n])
        loss.append(a)
        grad.append(g if weight[n] != 0 else np.zeros(z.shape[1]))
    return np.array(loss), np.array(grad)


def beam_scores(logits, scores, T, finished=None, end_token=0):
    """[W, V] candidate scores of one entry."""
    W, V = logits.shape
    out = np.full((W, V), -np.inf)
    for w in range(W):
        s = float(scores[w])
        if not np.isfinite(s):
            continue
        if finished is not None and finished[w]:
            out[w, end_token] = s
            continue
        lse = log_sum_exp(logits[w], T)
        if np.isfinite(lse):
            out[w] = s + np.asarray(logits[w], np.float64) / T - lse
    return out


def beam_select(logits, scores, n_out, T, finished=None, end_token=0):
    """(scores, parents, tokens), each [B, n_out]; equal scores, -inf among them, in the order of (beam, token)."""
    V = logits.shape[2]
    s, at = [], []
    for b in range(len(logits)):
        c = beam_scores(logits[b], scores[b], T, None if finished is None else finished[b], end_token).ravel()
        at.append(np.argsort(-c, kind="stable")[:n_out])
        s.append(c[at[-1]])
    at = np.array(at, np.int32)
    return np.array(s), at // V, at % V


def beam_reorder(state, parents, lens=None):
    """state [B, W, S, ...]: beam m of entry b gets the first lens[b] steps of beam parents[b, m] (none of its own if < 0 or >= W)."""
    out = state.copy()
    B, W = parents.shape
    for b in range(B):
        n = state.shape[2] if lens is None else min(max(int(lens[b]), 0), state.shape[2])
        for m in range(W):
            if 0 <= parents[b, m] < W:
                out[b, m, :n] = state[b, parents[b, m], :n]
    return out
