"""Row operators by their definitions, in float64 numpy: the key sort, the
router, dispatch and combine of expert layers, and embedding lookup, with their
gradients.  Loops over rows where that keeps the definition in sight."""

from __future__ import annotations

import numpy as np


def sort_keys_ref(keys, n_keys: int) -> dict:
    """order, position (int32, n) and offsets (int32, n_keys + 1)."""
    keys = np.asarray(keys).reshape(-1)
    inside = (keys >= 0) & (keys < n_keys)
    keys = np.where(inside, keys, n_keys).astype(np.int64)
    order = np.argsort(keys, kind="stable")
    position = np.empty_like(order)
    position[order] = np.arange(order.size)
    offsets = np.searchsorted(keys[order], np.arange(n_keys + 1), side="left")
    return dict(order=order.astype(np.int32), position=position.astype(np.int32), offsets=offsets.astype(np.int32))


def route_ref(logits, k: int, renormalise: bool):
    """(weights float64, ids int32) of every row."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    weights, ids = np.zeros((T, k)), np.full((T, k), -1, dtype=np.int32)
    for t in range(T):
        row = logits[t]
        able = [e for e in range(E) if row[e] > -np.inf]  # (a NaN compares false)
        chosen = sorted(able, key=lambda e: (-row[e], e))[:k]
        ids[t, :len(chosen)] = chosen
        if chosen:
            with np.errstate(invalid="ignore", over="ignore"):
                term = {e: np.exp(row[e] - row[chosen[0]]) for e in able}
            total = sum(term[e] for e in (chosen if renormalise else able))
            weights[t, :len(chosen)] = [term[e] / total for e in chosen]
        if np.isnan(row).any():
            weights[t] = np.nan
    return weights, ids


def route_backward_ref(grad_weights, logits, k: int, renormalise: bool):
    """Gradient (T, E) of the logits: the softmax's Jacobian applied to the
    chosen slots' gradients."""
    weights, ids = route_ref(logits, k, renormalise)
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    grad = np.zeros((T, E))
    for t in range(T):
        chosen = [e for e in ids[t] if e >= 0]
        if not chosen:
            continue
        over = chosen if renormalise else [e for e in range(E) if logits[t, e] > -np.inf]
        top = max(logits[t, e] for e in over)
        p = {e: np.exp(logits[t, e] - top) for e in over}
        total = sum(p.values())
        p = {e: v / total for e, v in p.items()}
        for e in over:  # d w_j / d l_e = w_j (delta - p_e)
            grad[t, e] = sum(weights[t, j] * grad_weights[t, j] * ((c == e) - p[e]) for j, c in enumerate(chosen))
    return grad


def dispatch_ref(x, ids, n_experts: int):
    """Rows (T k, C) in the order of their experts, zeros for dropped slots."""
    x = np.asarray(x, dtype=np.float64)
    k = np.asarray(ids).shape[1]
    plan = sort_keys_ref(ids, n_experts)
    rows = x[plan["order"] // k].copy() if plan["order"].size else np.zeros((0, x.shape[1]))
    rows[plan["offsets"][-1]:] = 0
    return rows, plan


def combine_ref(rows, weights, plan):
    """(out, sum of |terms|): sum of each token's kept rows times its weights."""
    rows, weights = np.asarray(rows, dtype=np.float64), np.asarray(weights, dtype=np.float64)
    T, k = weights.shape
    out, mag = np.zeros((T, rows.shape[1])), np.zeros((T, rows.shape[1]))
    for j in range(k):
        pos = plan["position"].reshape(T, k)[:, j]
        kept = pos < plan["offsets"][-1]
        term = weights[kept, j, None] * rows[pos[kept]]
        out[kept] += term
        mag[kept] += np.abs(term)
    return out, mag


def combine_backward_ref(grad_out, rows, weights, plan):
    """(grad_rows, grad_weights, sum of |terms| of grad_weights)."""
    g, rows, weights = (np.asarray(a, dtype=np.float64) for a in (grad_out, rows, weights))
    T, k = weights.shape
    grad_rows, grad_weights, mag = np.zeros_like(rows), np.zeros((T, k)), np.zeros((T, k))
    for j in range(k):
        pos = plan["position"].reshape(T, k)[:, j]
        kept = pos < plan["offsets"][-1]
        grad_rows[pos[kept]] = weights[kept, j, None] * g[kept]
        grad_weights[kept, j] = (g[kept] * rows[pos[kept]]).sum(1)
        mag[kept, j] = np.abs(g[kept] * rows[pos[kept]]).sum(1)
    return grad_rows, grad_weights, mag


def embed_ref(table, ids, scale: float):
    table, flat = np.asarray(table, dtype=np.float64), np.asarray(ids).reshape(-1)
    out = np.zeros((flat.size, table.shape[1]))
    for i, v in enumerate(flat):
        if 0 <= v < table.shape[0]:
            out[i] = scale * table[v]
    return out.reshape(np.asarray(ids).shape + (table.shape[1],))


def embed_backward_ref(grad_out, ids, table_rows: int, scale: float):
    """(grad_table, sum of |terms|, terms per row)."""
    flat = np.asarray(ids).reshape(-1)
    C = np.asarray(grad_out).shape[-1]
    g = np.asarray(grad_out, dtype=np.float64).reshape(flat.size, C)
    grad, mag = np.zeros((table_rows, C)), np.zeros((table_rows, C))
    count = np.zeros(table_rows, dtype=np.int64)
    inside = (flat >= 0) & (flat < table_rows)
    np.add.at(grad, flat[inside], scale * g[inside])
    np.add.at(mag, flat[inside], np.abs(scale * g[inside]))
    np.add.at(count, flat[inside], 1)
    return grad, mag, count
