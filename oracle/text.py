"""The operators of language models (embedding lookup in agents' tables and its gradient, distillation from a teacher's
top logits, a row's top logits) in fp64, entry by entry from their definitions."""
import numpy as np


def embed(E, tokens, scale):
    """E: (n, V, h); tokens: (n, T).  Rows of tokens outside [0, V) are zero."""
    n, V, h = E.shape
    out = np.zeros(tokens.shape + (h,))
    for i in range(n):
        for t, v in enumerate(tokens[i]):
            if 0 <= v < V:
                out[i, t] = scale * E[i, v].astype(np.float64)
    return out


def embed_grad(G, tokens, V, scale, old=None):
    """(gradient of the tables, the same sum over absolute values, terms per row); G: (n, T, h).  `old` is added to."""
    n, T, h = G.shape
    E = np.zeros((n, V, h)) if old is None else old.astype(np.float64).copy()
    size = np.abs(E)
    terms = np.zeros((n, V), dtype=np.int64)
    for i in range(n):
        for t, v in enumerate(tokens[i]):
            if 0 <= v < V:
                E[i, v] += scale * G[i, t].astype(np.float64)
                size[i, v] += abs(scale) * np.abs(G[i, t].astype(np.float64))
                terms[i, v] += 1
    return E, size, terms


def _log_softmax(x):
    m = x.max()
    return x - m - np.log(np.exp(x - m).sum())


def distill_row(s, u, ids, temperature, hard, label, weight):
    """(loss, gradient, size) of one row; size: the sum of |terms| of the loss, for bounds on its rounding."""
    V = len(s)
    s = s.astype(np.float64)
    grad = np.zeros(V)
    if weight == 0:
        return 0.0, grad, 0.0
    real = [k for k in range(len(ids)) if 0 <= ids[k] < V and not np.isneginf(u[k])]
    soft, labelled = hard < 1 and len(real) > 0, hard > 0 and label is not None and 0 <= label < V
    if np.isneginf(s).all() or not (soft or labelled):
        return 0.0, grad, 0.0
    if np.isnan(s).any() or np.isposinf(s).any():
        return np.nan, np.full(V, np.nan), np.nan
    with np.errstate(divide="ignore", invalid="ignore"):
        logq, logr = _log_softmax(s / temperature), _log_softmax(s)
    loss = size = 0.0
    if soft:
        logp = _log_softmax(np.array([u[k] for k in real], dtype=np.float64) / temperature)
        p = np.exp(logp)
        for j, k in enumerate(real):
            if p[j] > 0:
                term = (1 - hard) * temperature ** 2 * p[j] * (logp[j] - logq[ids[k]])
                loss += term
                size += abs(term) + (1 - hard) * temperature ** 2 * p[j]
            grad[ids[k]] -= (1 - hard) * temperature * p[j]
        grad += (1 - hard) * temperature * np.exp(logq)
    if labelled:
        loss -= hard * logr[label]
        size += hard * (abs(logr[label]) + 1)
        grad += hard * np.exp(logr)
        grad[label] -= hard
    return weight * loss, weight * grad, abs(weight) * size


def distill(logits, top, ids, temperature, hard, labels=None, weight=None, peer=None):
    """Every row of (n, T, V) logits against (n, T, K) entries; returns (loss, gradient, size)."""
    n, T, V = logits.shape
    loss, grad, size = np.zeros((n, T)), np.zeros((n, T, V)), np.zeros((n, T))
    for i in range(n):
        j = i if peer is None else min(max(int(peer[i]), 0), n - 1)
        for t in range(T):
            u, at = ([], []) if top is None else (top[j, t], ids[j, t])
            loss[i, t], grad[i, t], size[i, t] = distill_row(logits[i, t], u, at, temperature, hard, None if labels is None else int(labels[i, t]),
                                                             1.0 if weight is None else float(weight[i, t]))
    return loss, grad, size


def top_logits(rows, K):
    """(values, places) of the K largest of every row: by value from the largest down, then by place; NaN above +inf, -inf
    never: -inf and -1 fill up."""
    R, V = rows.shape
    values, ids = np.full((R, K), -np.inf), np.full((R, K), -1, dtype=np.int32)
    for r in range(R):
        x = rows[r].astype(np.float64)
        order = sorted((v for v in range(V) if not np.isneginf(x[v])), key=lambda v: (0, 0.0, v) if np.isnan(x[v]) else (1, -x[v], v))[:K]
        values[r, :len(order)] = x[order]
        ids[r, :len(order)] = order
    return values, ids
