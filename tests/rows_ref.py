"""Rows sorted by expert and back, low-rank adapters, and their gradients in float64, and how far fp32 sums may be off.

Every function returns values and, for each, a bound of the error that the operator's roundings can make: a sum of n
products in fp32 is off by at most n + 1 roundings of the sum of their magnitudes, each of `STEP` relative (2^-24 for an
operation rounded to nearest; 2^-23 is taken, as the matrix instructions' own roundings are not laid down to be to nearest).
"""
import numpy as np

STEP = 2.0 ** -23
# Half a step of a result's type, relative to the value.
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def rounded(v, err, dtype):
    """Bound after the value is rounded to its type."""
    return err + HALF[dtype] * (np.abs(v) + err)


def places(inv_perm, T, k, R):
    q = np.asarray(inv_perm[: T * k], np.int64).reshape(T, k)
    return np.where((q >= 0) & (q < R), q, -1)


def sort_rows(x, inv_perm, k, R, before, w=None):
    """`before`: what rows holds; rows that no slot has stay."""
    T = x.shape[0]
    out, err = before.copy(), np.zeros_like(before)
    q = places(inv_perm, T, k, R)
    for t, j in zip(*np.nonzero(q >= 0)):
        f = 1.0 if w is None else float(w[t, j])
        out[q[t, j]] = f * x[t]
        if w is not None:
            err[q[t, j]] = STEP * np.abs(out[q[t, j]])
    return out, err


def combine_rows(rows, inv_perm, T, k, w=None, add=None):
    q = places(inv_perm, T, k, rows.shape[0])
    y = np.zeros((T, rows.shape[1])) if add is None else add.copy()
    mag = np.abs(y)
    for t, j in zip(*np.nonzero(q >= 0)):
        v = (1.0 if w is None else float(w[t, j])) * rows[q[t, j]]
        y[t] += v
        mag[t] += np.abs(v)
    return y, (k + 1) * STEP * mag


def combine_rows_grad(dy, rows, inv_perm, k, before, w=None):
    T = dy.shape[0]
    drows, err = sort_rows(dy, inv_perm, k, before.shape[0], before, w)
    q = places(inv_perm, T, k, before.shape[0])
    dw, mag = np.zeros((T, k)), np.zeros((T, k))
    for t, j in zip(*np.nonzero(q >= 0)):
        dw[t, j] = dy[t] @ rows[q[t, j]]
        mag[t, j] = np.abs(dy[t]) @ np.abs(rows[q[t, j]])
    return drows, err, dw, (dy.shape[1] + 1) * STEP * mag


def segments(offsets, perm, T):
    """Adapter, places and rows of each segment (places whose row is outside [0, T) are left out)."""
    for l, (lo, hi) in enumerate(zip(offsets[:-1], offsets[1:])):
        p = np.arange(lo, hi)
        t = p if perm is None else np.asarray(perm, np.int64)[lo:hi]
        ok = (t >= 0) & (t < T)
        if ok.any():
            yield l, p[ok], t[ok]


def adapters(x, a, b, offsets, perm=None, scale=None, add=None, before=None, before_u=None):
    """y, its error, u, its error."""
    T, (L, N, r) = x.shape[0], b.shape
    y = np.zeros((T, N)) if before is None else before.copy()
    u = np.zeros((T, r)) if before_u is None else before_u.copy()
    ey, eu = np.zeros_like(y), np.zeros_like(u)
    for l, p, t in segments(offsets, perm, T):
        s = 1.0 if scale is None else float(scale[l])
        u[p] = x[t] @ a[l].T
        eu[p] = (x.shape[1] + 1) * STEP * (np.abs(x[t]) @ np.abs(a[l].T))
        d = s * (u[p] @ b[l].T)
        # Three products (of u's thirds) a rank, the factor, and the addition.
        e = abs(s) * ((3 * r + 3) * STEP * ((np.abs(u[p]) + eu[p]) @ np.abs(b[l].T)) + eu[p] @ np.abs(b[l].T))
        base = 0 if add is None else add[t]
        y[t] = base + d
        ey[t] = e + STEP * (np.abs(base) + np.abs(d) + e)
    return y, ey, u, eu


def adapters_grad(x, dy, u, a, b, offsets, perm=None, scale=None, add=None, before=None, da=0.0, db=0.0):
    """dx, da, db, each with its error; `da`, `db`: what is added to."""
    T, K = x.shape
    L, N, r = b.shape
    dx = np.zeros((T, K)) if before is None else before.copy()
    edx = np.zeros_like(dx)
    ga, gb = np.zeros((L, r, K)) + da, np.zeros((L, N, r)) + db
    ea, eb = np.zeros_like(ga), np.zeros_like(gb)
    for l, p, t in segments(offsets, perm, T):
        s = 1.0 if scale is None else float(scale[l])
        g = s * (dy[t] @ b[l])
        eg = (N + 2) * STEP * abs(s) * (np.abs(dy[t]) @ np.abs(b[l]))
        base = 0 if add is None else add[t]
        d = g @ a[l]
        e = (3 * r + 3) * STEP * ((np.abs(g) + eg) @ np.abs(a[l])) + eg @ np.abs(a[l])
        dx[t] = base + d
        edx[t] = e + STEP * (np.abs(base) + np.abs(d) + e)
        n = 3 * len(p) + 8  # the three thirds, then waves, chunks and what is added to
        ga[l] += g.T @ x[t]
        ea[l] = eg.T @ np.abs(x[t]) + n * STEP * ((np.abs(g) + eg).T @ np.abs(x[t])) + STEP * np.abs(ga[l])
        gb[l] += s * (dy[t].T @ u[p])
        eb[l] = n * STEP * abs(s) * (np.abs(dy[t]).T @ np.abs(u[p])) + STEP * np.abs(gb[l])
    return dx, edx, ga, ea, gb, eb
