"""fp64 definitions of what stands before and after the LM head: embedding rows and the
table's gradient, verified drafts, and the divergence from a teacher's top logits.

numpy float64 on the CPU, written from the formulas; shares no code with the kernels.
"""

import math

import numpy as np


def embed(table, tokens, seq, scale=1.0):
    """scale * table[tokens]; masked tokens (seq < 0) give 0, ids outside the table NaN."""
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for t, y in enumerate(tokens):
        if seq is None or seq[t] >= 0:
            out[t] = scale * table[y] if 0 <= y < len(table) else np.nan
    return out


def embed_backward(dx, tokens, seq, V, scale=1.0, start=None):
    """Gradient of the table: start (or 0) plus scale * dx[t] in row tokens[t]."""
    dx = np.asarray(dx, np.float64)
    dW = np.zeros((V, dx.shape[1])) if start is None else np.array(start, np.float64)
    for t, y in enumerate(tokens):
        if (seq is None or seq[t] >= 0) and 0 <= y < V:
            dW[y] += scale * dx[t]
    return dW


def distribution(z, temperature=1.0):
    """softmax(z / temperature), or None where z has no distribution."""
    y = np.asarray(z, np.float64) / temperature
    if np.isnan(y).any() or (y == np.inf).any() or (y == -np.inf).all():
        return None
    e = np.exp(y - y.max())
    return e / math.fsum(e)


def draw(weights, u):
    """The least v whose running sum exceeds u times the total."""
    run = np.cumsum(weights)
    over = np.nonzero((run > u * run[-1]) & (weights > 0))[0]
    return int(over[0]) if len(over) else int(np.nonzero(weights > 0)[0][-1])


def verify(logits, draft_logits, draft_tokens, n_draft, u, temperature=1.0):
    """One sequence: (tokens emitted, their log-probs).  logits [K + 1, V]; draft_logits
    [K, V] or None (drafts that were not sampled); n_draft drafts, u [K + 1]."""
    tokens, logp = [], []
    V = len(logits[0])
    K = len(u) - 1
    for a in range(n_draft + 1):
        p = distribution(logits[a], temperature)
        weights = p
        if a < n_draft:
            x = int(draft_tokens[a])
            if draft_logits is None:
                q = np.zeros(V)
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                q = distribution(draft_logits[a], temperature)
            if p is not None and q is not None and 0 <= x < V and u[a] * q[x] < p[x]:
                tokens.append(x)
                logp.append(math.log(p[x]))
                continue
            if p is not None and q is not None:
                rest = np.maximum(p - q, 0.0)
                weights = rest if rest.sum() > 0 else p
        break
    if p is None:
        return tokens + [-1], logp + [math.nan]
    v = draw(weights, u[K])
    return tokens + [v], logp + [math.log(p[v])]


def distill(logits, ids, teacher, mass, seq, seq_len, n_seq, temperature=1.0, scale=1.0):
    """(kl [T], loss, stats [2], dlogits [T, V]) of the divergence from the teacher's entries."""
    z = np.asarray(logits, np.float64)
    T, V = z.shape
    kl, dz, loss, count = np.zeros(T), np.zeros((T, V)), 0.0, 0
    for t in range(T):
        if seq[t] < 0:
            continue
        here = ids[t] >= 0
        k, l = ids[t][here], np.asarray(teacher[t], np.float64)[here] / temperature
        if len(k) == 0 or (l == -np.inf).all():
            continue
        count += 1
        if mass is None:
            top = l.max()
            lp = l - (top + math.log(math.fsum(np.exp(l - top))))
        else:
            lp = l - float(mass[t])
        p = np.exp(lp)
        y = z[t] / temperature
        m = y.max()
        lse = m + math.log(math.fsum(np.exp(y - m)))
        live = p > 0
        kl[t] = math.fsum(p[live] * (lp[live] - y[k[live]] + lse))
        w = scale / (n_seq * int(seq_len[seq[t]]))
        loss += w * kl[t]
        g = p.sum() * np.exp(y - lse)
        np.subtract.at(g, k, p)
        dz[t] = g * (w / temperature)
    return kl, loss, np.array([count, kl.sum()]), dz
