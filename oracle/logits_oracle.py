"""Plain 64-bit oracle for the operators on rows of logits (TEST INFRASTRUCTURE ONLY; shares
no code with the HIP path and imports nothing from it).

Z is a numpy array of any float type, read as float64; a row at a time, by the definitions:
log p_j = scale z_j - log sum_i exp(scale z_i) over the columns above minus infinity.
"""

from __future__ import annotations

import numpy as np


def log_softmax(z, scale):
    """(log p, log of the sum); minus infinity throughout for a row of nothing else."""
    z = scale * np.asarray(z, np.float64)
    with np.errstate(invalid="ignore"):
        if np.isnan(z).any() or np.isposinf(z).any():
            return np.full(len(z), np.nan), np.nan
    live = z[z > -np.inf]
    if not len(live):
        return np.full(len(z), -np.inf), -np.inf
    top = live.max()
    lse = top + np.log(np.exp(live - top).sum())
    return (z - top) - np.log(np.exp(live - top).sum()), lse


def _plogp(log_p):
    p = np.exp(log_p)
    return p, np.where(p > 0, p * np.where(p > 0, log_p, 0.0), np.where(np.isnan(p), p, 0.0))


def alternatives(z, k):
    """The k largest logits' columns, ties to the lowest, -1 past the last one above -inf."""
    real = [j for j in range(len(z)) if z[j] > -np.inf]          # (a NaN is not)
    order = sorted(real, key=lambda j: (-float(z[j]), j))[:k]
    return np.array(order + [-1] * (k - len(order)), np.int64)


def logprob(Z, ids=None, scale=1.0, k=0):
    """dict of logp (with ids), lse, entropy, top_ids and top_logp."""
    Z = np.asarray(Z, np.float64)
    n, d = Z.shape
    out = dict(logp=np.zeros(n), lse=np.zeros(n), entropy=np.zeros(n),
               top_ids=np.full((n, k), -1, np.int64), top_logp=np.full((n, k), -np.inf))
    for i in range(n):
        log_p, out["lse"][i] = log_softmax(Z[i], scale)
        out["entropy"][i] = -_plogp(log_p)[1].sum()
        if ids is not None and 0 <= ids[i] < d:
            out["logp"][i] = log_p[ids[i]]
        if k:
            out["top_ids"][i] = top = alternatives(Z[i], k)
            out["top_logp"][i] = np.where(top >= 0, log_p[top], -np.inf)
    return out


def logprob_grad(Z, ids=None, scale=1.0, dlogp=None, dlse=None, dentropy=None):
    """scale (dlogp (e_t - p) + dlse p - dentropy p (log p + H)), e_t the given token's unit
    vector."""
    Z = np.asarray(Z, np.float64)
    n, d = Z.shape
    out = np.zeros((n, d))
    for i in range(n):
        given = ids is not None and 0 <= ids[i] < d
        gl = float(dlogp[i]) if dlogp is not None and given else 0.0
        gs = float(dlse[i]) if dlse is not None else 0.0
        ge = float(dentropy[i]) if dentropy is not None else 0.0
        log_p, lse = log_softmax(Z[i], scale)
        if (gl == 0 and gs == 0 and ge == 0) or lse == -np.inf:
            continue
        p, plogp = _plogp(log_p)
        row = gs * p - ge * (plogp - p * plogp.sum())
        row -= gl * p
        if given:
            row[ids[i]] += gl
        out[i] = scale * row
    return out


def teacher(ids, t, d, scale, lse=None):
    """(log q, q) of a row's entries, 0 for those that are no token."""
    ids, t = np.asarray(ids), scale * np.asarray(t, np.float64)
    ok = (ids >= 0) & (ids < d)
    log_q = np.where(ok, t, -np.inf)
    if lse is not None:
        log_q = log_q - lse
    elif ok.any() and log_q.max() > -np.inf:
        top = log_q.max()
        log_q = log_q - top - np.log(np.exp(log_q - top).sum())
    with np.errstate(invalid="ignore"):
        log_q = np.where(ok, log_q, -np.inf)
    return log_q, np.exp(log_q)


def distill(Z, ids, t, scale=1.0, t_scale=1.0, t_lse=None):
    Z = np.asarray(Z, np.float64)
    loss = np.zeros(len(Z))
    for i in range(len(Z)):
        log_p, _ = log_softmax(Z[i], scale)
        log_q, q = teacher(ids[i], t[i], Z.shape[1], t_scale, None if t_lse is None else float(t_lse[i]))
        for a in np.flatnonzero(q > 0):
            loss[i] += q[a] * (log_q[a] - log_p[ids[i][a]])
    return loss


def distill_grad(Z, ids, t, dloss, scale=1.0, t_scale=1.0, t_lse=None):
    Z = np.asarray(Z, np.float64)
    out = np.zeros(Z.shape)
    for i in range(len(Z)):
        log_p, lse = log_softmax(Z[i], scale)
        _, q = teacher(ids[i], t[i], Z.shape[1], t_scale, None if t_lse is None else float(t_lse[i]))
        if dloss[i] == 0 or q.sum() == 0 or lse == -np.inf:
            continue
        out[i] = np.exp(log_p) * q.sum()
        for a in np.flatnonzero(q > 0):
            out[i, ids[i][a]] -= q[a]
        out[i] *= scale * float(dloss[i])
    return out
