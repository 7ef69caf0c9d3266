"""The router's loss and its gradient in float64, from their definitions (a loop over sequences and tokens)."""
import numpy as np


def scores(l, score):
    """(p, softmax, log-sum-exp, 1 - sigmoid) of one row; a row of -inf alone has p = 0 and no lse."""
    if np.all(np.isneginf(l)):
        return np.zeros_like(l), np.zeros_like(l), 0.0, np.ones_like(l)
    m = l.max()
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        ex = np.exp(l - m)
        soft, lse = ex / ex.sum(), m + np.log(ex.sum())
        ls = np.minimum(l, 0.0) - np.log1p(np.exp(-np.abs(l)))  # log sigmoid
        sg = np.exp(ls - ls.max())
        om = np.exp(np.minimum(-l, 0.0) - np.log1p(np.exp(-np.abs(l))))
    return (soft if score == 0 else sg / sg.sum()), soft, lse, om


def members(T, mask, offsets):
    off = [0, T] if offsets is None else list(offsets)
    return [[t for t in range(off[s], off[s + 1]) if mask is None or mask[t]] for s in range(len(off) - 1)]


def loss(l, ids, k, mask, offsets, score, alpha, z_coef):
    T, E = l.shape
    seqs = members(T, mask, offsets)
    counts = np.zeros((len(seqs), E), np.int64)
    probs = np.zeros((len(seqs), E))
    bal = z = 0.0
    n = [len(v) for v in seqs]
    for s, toks in enumerate(seqs):
        for t in toks:
            for e in ids[t]:
                if 0 <= e < E:
                    counts[s, e] += 1
            p, _, lse, _ = scores(l[t], score)
            probs[s] += p / n[s]
            z += lse * lse
        if toks:
            bal += (E * counts[s] / (k * n[s]) * probs[s]).sum()
    n_seq, n_tok = sum(v > 0 for v in n), sum(n)
    bal, z = bal / max(1, n_seq), z / max(1, n_tok)
    total = (alpha * bal if alpha else 0.0) + (z_coef * z if z_coef else 0.0)
    return np.array([total, bal, z]), counts, probs, np.array(n + [n_seq, n_tok])


def grad(l, ids, k, mask, offsets, score, alpha, z_coef, counts, g, w=None, dw=None):
    """(dlogits, magnitude of the terms that each value is a sum of)"""
    T, E = l.shape
    seqs = members(T, mask, offsets)
    n_seq, n_tok = sum(bool(v) for v in seqs), sum(len(v) for v in seqs)
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    for s, toks in enumerate(seqs):
        for t in toks:
            f = E * counts[s] / (k * len(toks))
            p, soft, lse, om = scores(l[t], score)
            c = g * alpha / (n_seq * len(toks)) * p * (om if score else 1.0)
            out[t] += c * (f - (f * p).sum())
            mag[t] += np.abs(c) * (f + (f * p).sum())
            zt = g * z_coef * 2 / n_tok * lse * soft
            out[t] += zt
            mag[t] += np.abs(zt)
            if w is not None:
                ok = [j for j in range(k) if 0 <= ids[t][j] < E]
                dot = sum(w[t, j] * dw[t, j] for j in ok)
                adot = sum(abs(w[t, j] * dw[t, j]) for j in ok)
                for j in ok:
                    out[t, ids[t][j]] += w[t, j] * (dw[t, j] - dot)
                    mag[t, ids[t][j]] += abs(w[t, j]) * (abs(dw[t, j]) + adot)
    return out, mag
