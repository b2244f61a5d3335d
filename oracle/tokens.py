"""fp64 definitions of what stands around the layers of a token model (one token per column): embedding, norm with the
residual's addition, log probabilities with entropy and alternatives, clipping by the global norm; each with its
gradient as the formula says. No code shared with the library."""
from __future__ import annotations

import numpy as np


def _f64(a) -> np.ndarray:
    return np.asarray(a, dtype=np.float64)


def embed(table, ids, scale: float) -> np.ndarray:
    """X[:, j] = scale * table[ids[j]]; zero for an id that is no row of the table."""
    table, ids = _f64(table), np.asarray(ids, dtype=np.int64)
    X = np.zeros((table.shape[1], ids.size))
    known = (ids >= 0) & (ids < table.shape[0])
    X[:, known] = scale * table[ids[known]].T
    return X


def embed_gradient(vocab: int, ids, G, scale: float) -> np.ndarray:
    G, ids = _f64(G), np.asarray(ids, dtype=np.int64)
    dTable = np.zeros((vocab, G.shape[0]))
    known = (ids >= 0) & (ids < vocab)
    np.add.at(dTable, ids[known], scale * G[:, known].T)
    return dTable


def norm(S, weight, eps: float):
    """(Y, rstd) of the summed input S [d][m]."""
    S = _f64(S)
    rstd = 1.0 / np.sqrt(np.mean(S * S, axis=0) + eps)
    return _f64(weight)[:, None] * S * rstd, rstd


def norm_gradient(G, S, weight, eps: float, dS=None):
    """(dX, dweight) of L = <G, Y> + <dS, S>."""
    G, S, w = _f64(G), _f64(S), _f64(weight)[:, None]
    rstd = 1.0 / np.sqrt(np.mean(S * S, axis=0) + eps)
    dX = rstd * w * G - S * rstd ** 3 / S.shape[0] * np.sum(w * G * S, axis=0)
    if dS is not None:
        dX = dX + _f64(dS)
    return dX, np.sum(G * S * rstd, axis=1)


def log_softmax(logits) -> np.ndarray:
    """Per column; -infinity where the logit is, also where a column has nothing else."""
    x = _f64(logits)
    with np.errstate(invalid="ignore", divide="ignore"):
        most = np.max(x, axis=0)
        most = np.where(np.isneginf(most), 0.0, most)
        total = np.sum(np.exp(x - most), axis=0)
        lp = (x - most) - np.where(total == 0, 0.0, np.log(total))
    return lp


def _p_log_p(lp) -> np.ndarray:
    with np.errstate(invalid="ignore"):
        return np.where(np.isneginf(lp), 0.0, np.exp(lp) * lp)


def log_prob(logits, ids, top: int = 0):
    """(logp, entropy, top_logp, top_ids): ids None or outside the vocabulary give logp 0; alternatives are ordered by
    value, then by row; -infinity and NaN are none."""
    lp = log_softmax(logits)
    vocab, m = lp.shape
    logp = np.zeros(m)
    if ids is not None:
        ids = np.asarray(ids, dtype=np.int64)
        known = np.flatnonzero((ids >= 0) & (ids < vocab))
        logp[known] = lp[ids[known], known]
    entropy = -np.sum(_p_log_p(lp), axis=0)
    top_logp, top_ids = np.full((top, m), -np.inf), np.full((top, m), -1, dtype=np.int64)
    x = _f64(logits)
    for j in range(m if top else 0):
        rows = np.flatnonzero(~np.isnan(x[:, j]) & ~np.isneginf(x[:, j]))
        rows = rows[np.lexsort((rows, -x[rows, j]))][:top]
        top_ids[:rows.size, j] = rows
        top_logp[:rows.size, j] = lp[rows, j]
    return logp, entropy, top_logp, top_ids


def log_prob_gradient(logits, ids, g_logp=None, g_entropy=None) -> np.ndarray:
    """dL/dlogits of L = <g_logp, logp> + <g_entropy, entropy>; zero for masked logits."""
    lp = log_softmax(logits)
    vocab, m = lp.shape
    p = np.exp(lp)
    dx = np.zeros((vocab, m))
    if g_logp is not None:
        ids = np.asarray(ids, dtype=np.int64)
        known = np.flatnonzero((ids >= 0) & (ids < vocab))
        gl = np.zeros(m)
        gl[known] = _f64(g_logp)[known]
        dx -= p * gl
        dx[ids[known], known] += gl[known]
    if g_entropy is not None:
        H = -np.sum(_p_log_p(lp), axis=0)
        dx -= _f64(g_entropy) * (_p_log_p(lp) + p * H)
    dx[np.isneginf(_f64(logits))] = 0.0
    return dx


def grad_norm(tensors) -> float:
    return float(np.sqrt(sum(float(np.sum(_f64(t) ** 2)) for t in tensors)))


def grad_clip(tensors, max_norm: float):
    """(norm, factor): the factor is 1 where the norm is not larger than max_norm or not a finite number."""
    n = grad_norm(tensors)
    return n, max_norm / n if np.isfinite(n) and n > max_norm else 1.0
