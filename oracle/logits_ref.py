"""Logits operators by their definitions, in float64 numpy: log probabilities
with entropy and alternatives, distillation from a teacher's alternatives, and
the gradients of both.  One row at a time, as the definitions read."""

from __future__ import annotations

import numpy as np


def distribution(row, scale: float):
    """(log probabilities, lse) of softmax(scale * row); a row of nothing but
    -inf has none: all -inf."""
    z = scale * np.asarray(row, dtype=np.float64)
    if np.isnan(z).any() or (z == np.inf).any():
        return np.full(z.shape, np.nan), np.nan
    top = z.max()
    if top == -np.inf:
        return np.full(z.shape, -np.inf), -np.inf
    log_sum = np.log(np.exp(z - top).sum())
    return (z - top) - log_sum, top + log_sum  # (z - lse would lose the sum beside a large maximum)


def entropy_of(logp):
    if np.isnan(logp).any():
        return np.nan
    p = np.exp(logp)
    return -(p[p > 0] * logp[p > 0]).sum()


def logprobs_ref(logits, ids, k: int, scale: float) -> dict:
    """logprob (None without ids), lse, entropy, top, top_ids."""
    logits = np.asarray(logits, dtype=np.float64)
    T, V = logits.shape
    out = dict(logprob=None if ids is None else np.zeros(T), lse=np.zeros(T), entropy=np.zeros(T),
               top=np.full((T, k), -np.inf), top_ids=np.full((T, k), -1, dtype=np.int32))
    for t in range(T):
        logp, out["lse"][t] = distribution(logits[t], scale)
        out["entropy"][t] = entropy_of(logp)
        if ids is not None and 0 <= ids[t] < V:
            out["logprob"][t] = logp[ids[t]]
        able = np.flatnonzero(logits[t] > -np.inf)  # (a NaN compares false)
        best = able[np.argsort(-logits[t, able], kind="stable")][:k]
        out["top_ids"][t, :len(best)] = best
        out["top"][t, :len(best)] = logp[best]
        if np.isnan(out["lse"][t]):
            out["top"][t] = np.nan
    return out


def logprobs_backward_ref(logits, ids, top_ids, scale: float, grad_logprob=None, grad_lse=None, grad_entropy=None,
                          grad_top=None):
    """Gradient of the logits: the Jacobians of log p_v, lse and the entropy in
    z = scale x applied to the outgoing gradients."""
    logits = np.asarray(logits, dtype=np.float64)
    T, V = logits.shape
    grad = np.zeros((T, V))
    for t in range(T):
        logp, lse = distribution(logits[t], scale)
        on_logp = np.zeros(V)  # gradient of every log p_v
        if grad_logprob is not None and 0 <= ids[t] < V:
            on_logp[ids[t]] += grad_logprob[t]
        if grad_top is not None:
            for v, g in zip(top_ids[t], grad_top[t]):
                if v >= 0:
                    on_logp[v] += g
        gz = 0.0 if grad_lse is None else grad_lse[t]
        gh = 0.0 if grad_entropy is None else grad_entropy[t]
        if lse == -np.inf or (not on_logp.any() and gz == 0 and gh == 0):
            continue
        p = np.exp(logp)
        d = on_logp + p * (gz - on_logp.sum())
        if gh != 0:
            own = np.where(p != 0, logp, 0)
            d -= gh * p * (own + entropy_of(logp))
        grad[t] = scale * d
    return grad


def taught(ids, teacher, V: int, renormalise: bool):
    """(kept slots, their q) of one row."""
    kept = [j for j in range(len(ids)) if 0 <= ids[j] < V and not teacher[j] == -np.inf]
    t = np.array([teacher[j] for j in kept], dtype=np.float64)
    if renormalise and kept:
        t = t - t.max()
        t = t - np.log(np.exp(t).sum())
    return kept, t


def distill_ref(logits, ids, teacher, scale: float, renormalise: bool):
    logits = np.asarray(logits, dtype=np.float64)
    T, V = logits.shape
    loss = np.zeros(T)
    for t in range(T):
        kept, logq = taught(ids[t], teacher[t], V, renormalise)
        if not kept:
            continue
        logp, _ = distribution(logits[t], scale)
        for j, lq in zip(kept, logq):
            loss[t] += np.exp(lq) * (lq - logp[ids[t][j]])
    return loss


def distill_backward_ref(grad_loss, logits, ids, teacher, scale: float, renormalise: bool):
    logits = np.asarray(logits, dtype=np.float64)
    T, V = logits.shape
    grad = np.zeros((T, V))
    for t in range(T):
        kept, logq = taught(ids[t], teacher[t], V, renormalise)
        logp, lse = distribution(logits[t], scale)
        if not kept or grad_loss[t] == 0 or lse == -np.inf:
            continue
        q = np.exp(logq)
        grad[t] = q.sum() * np.exp(logp)
        for j, own in zip(kept, q):
            grad[t, ids[t][j]] -= own
        grad[t] *= grad_loss[t] * scale
    return grad
