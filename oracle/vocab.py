"""Float64 CPU oracle of the operators over discrete values: embedding rows and their gradient,
distillation from a teacher's top logits, adjusted logits, sampling with temperature, top-k, top-p and min-p.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Each function is the definition written
out for one row (or one id) after another; nothing is shared with the GPU package.
"""

import numpy as np


# ---- embedding ---------------------------------------------------------------------------------

def embed_forward(ids, table, scale, base=None):
    """scale table[id] for every id in [0, V), 0 for the others; added to base if given."""
    ids = np.asarray(ids)
    table = np.asarray(table, dtype=np.float64)
    out = np.zeros(ids.shape + (table.shape[1],))
    for at in np.ndindex(*ids.shape):
        if 0 <= ids[at] < len(table):
            out[at] = scale * table[ids[at]]
    return out if base is None else out + np.asarray(base, dtype=np.float64)


def embed_backward(ids, dout, V, scale):
    """scale times the sum of dout's rows at each id."""
    dout = np.asarray(dout, dtype=np.float64)
    g = np.zeros((V, dout.shape[-1]))
    for at in np.ndindex(*np.asarray(ids).shape):
        if 0 <= ids[at] < V:
            g[ids[at]] += scale * dout[at]
    return g


# ---- distillation ------------------------------------------------------------------------------

def _logsumexp(x):
    m = x.max() if len(x) else -np.inf
    return m if np.isinf(m) else m + np.log(np.exp(x - m).sum())


def distill_row(s, idx, top, lse, label, tau, alpha, tail):
    """Loss and gradient of one row over the classes of s (see include/tfm_vocab.h)."""
    s = np.asarray(s, dtype=np.float64)
    V = len(s)
    if V == 0 or s.max() == -np.inf:
        return 0.0, np.zeros(V)
    s = s - s.max()      # first: a row of the lowest values leaves no room for its log-sum-exp
    x = s / tau
    q = np.exp(x - _logsumexp(x))
    entries = {}
    for i, t in zip(idx, top):
        if 0 <= i < V and int(i) not in entries:
            entries[int(i)] = float(t)
    J = np.array(sorted(entries), dtype=int)
    t = np.array([entries[i] for i in J]) / tau
    out = np.ones(V, bool)
    out[J] = False
    p = np.zeros(V)
    if tail:
        p[J] = np.exp(t - lse)
    elif len(J) and t.max() > -np.inf:
        p[J] = np.exp(t - _logsumexp(t))
    rest = 0.0
    if tail and (s[out] > -np.inf).any():
        rest = max(0.0, 1.0 - p.sum())
    logq = x - _logsumexp(x)
    D = sum(p[i] * (np.log(p[i]) - logq[i]) for i in J if p[i] > 0)
    grad = (p.sum() + rest) * q - p
    if rest > 0:
        lqt = _logsumexp(logq[out])
        D += rest * (np.log(rest) - lqt)
        grad[out] -= rest * np.exp(logq[out] - lqt)
    loss, grad = alpha * tau * tau * D if alpha else 0.0, alpha * tau * grad
    if 0 <= label < V:
        l1 = s - _logsumexp(s)
        loss -= (1 - alpha) * l1[label]
        grad = grad + (1 - alpha) * np.exp(l1)
        grad[label] -= 1 - alpha
    return loss, grad


def distill_loss(s, idx, top, lse, labels, weights, n_class, tau, alpha, tail):
    """(loss, row losses, gradient [N][V]) of rows of logits; None where an array is left out."""
    N, V = s.shape
    w = np.ones(N) if weights is None else np.asarray(weights, dtype=np.float64)
    total = w.sum()
    rows, grad = np.zeros(N), np.zeros((N, V))
    for n in range(N):
        if w[n] == 0:
            continue
        nc = V if n_class is None else min(max(int(n_class[n]), 0), V)
        rows[n], g = distill_row(s[n, :nc], idx[n], top[n], None if lse is None else lse[n],
                                 -1 if labels is None else int(labels[n]), tau, alpha, tail)
        if total != 0:
            grad[n, :nc] = g * w[n] / total
    with np.errstate(invalid="ignore"):
        loss = (w * rows)[w != 0].sum() / total if total != 0 else 0.0
    return loss, rows, grad


# ---- adjusted logits ---------------------------------------------------------------------------

def adjust_row(s, n_class=None, history=(), repetition=1.0, presence=0.0, frequency=0.0,
               bias_idx=(), bias=(), allowed=None):
    """The logits of one row after penalties, biases and the mask (see include/tfm_vocab.h), and what
    the roundings of its steps are relative to: the sum of the magnitudes that a class went through."""
    x = np.array(s, dtype=np.float64)
    V = len(x)
    size = np.zeros(V)
    r = repetition if repetition > 0 else 1.0
    for v in range(V):
        c = sum(1 for t in history if t == v)
        if c:
            x[v] = x[v] / r if x[v] > 0 else x[v] * r
            size[v] += abs(x[v])
            less = presence + frequency * c
            size[v] += 2 * abs(frequency * c) + abs(presence)
            x[v] = x[v] - less
            size[v] += abs(x[v])
        for i, b in zip(bias_idx, bias):
            if i == v:
                x[v] = x[v] + b
                size[v] += abs(x[v])
                break
        if allowed is not None and not (int(allowed[v // 32]) >> (v % 32)) & 1:
            x[v] = -np.inf
        if n_class is not None and v >= n_class:
            x[v] = -np.inf
    return x, size


# ---- sampling ----------------------------------------------------------------------------------

def sample_row(s, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, log-probability) of one row's draw."""
    s = np.asarray(s, dtype=np.float64)
    s = np.where(np.isnan(s), -np.inf, s)
    if len(s) == 0 or s.max() == -np.inf:
        return -1, -np.inf
    rank = np.argsort(-s, kind="stable")
    rank = rank[s[rank] > -np.inf]
    if not temperature > 0:
        return int(rank[0]), 0.0
    with np.errstate(invalid="ignore"):
        x = np.where(s == s.max(), 0.0, (s - s.max()) / temperature)
    w = np.exp(x)
    kept = rank[:top_k] if top_k > 0 else rank
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[kept])])
        front = [i for i in range(len(kept)) if i == 0 or before[i] < top_p * before[-1]]
        kept = kept[:len(front)]
    if min_p > 0:
        kept = kept[:max(1, int((x[kept] >= np.log(min_p)).sum()))]
    kept = np.sort(kept)
    u = min(u, float(np.float32(1) - np.float32(2.0 ** -24))) if u > 0 else 0.0
    mass = np.cumsum(w[kept])
    at = int(np.flatnonzero(mass > u * mass[-1])[0])
    return int(kept[at]), float(x[kept[at]] - np.log(mass[-1]))
