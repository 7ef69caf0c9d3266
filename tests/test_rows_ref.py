"""The float64 forms of the row and adapter operators: their gradients against differences."""
import numpy as np

from tests import rows_ref as ref


def _difference(f, v, h=1e-6):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        old = v[i]
        v[i] = old + h
        hi = f()
        v[i] = old - h
        g[i] = (hi - f()) / (2 * h)
        v[i] = old
    return g


def test_combine_gradient():
    rng = np.random.default_rng(1)
    T, k, H, R = 4, 3, 5, 9
    inv = np.array([0, 4, -1, 7, 2, 8, -1, -1, -1, 5, 1, 12], np.int32)  # 12: past the rows; a token without any
    rows, w, dy = rng.standard_normal((R, H)), rng.standard_normal((T, k)), rng.standard_normal((T, H))
    f = lambda: (dy * ref.combine_rows(rows, inv, T, k, w)[0]).sum()
    drows, _, dw, _ = ref.combine_rows_grad(dy, rows, inv, k, np.zeros((R, H)), w)
    assert np.allclose(drows, _difference(f, rows), atol=1e-8) and np.allclose(dw, _difference(f, w), atol=1e-8)


def test_sorted_rows_gradient():
    rng = np.random.default_rng(2)
    T, k, H, R = 3, 2, 4, 6
    inv = np.array([5, 0, -1, 2, 3, -1], np.int32)
    x, w, d = rng.standard_normal((T, H)), rng.standard_normal((T, k)), rng.standard_normal((R, H))
    f = lambda: (d * ref.sort_rows(x, inv, k, R, np.zeros((R, H)), w)[0]).sum()
    dx = ref.combine_rows(d, inv, T, k, w)[0]
    dw = ref.combine_rows_grad(x, d, inv, k, np.zeros((R, H)), w)[2]
    assert np.allclose(dx, _difference(f, x), atol=1e-8) and np.allclose(dw, _difference(f, w), atol=1e-8)


def test_adapters_gradient():
    rng = np.random.default_rng(3)
    T, L, r, K, N = 7, 4, 2, 3, 5
    offsets, perm, scale = [0, 2, 2, 5, 6], rng.permutation(T), rng.standard_normal(L)  # an empty segment, a row in none
    x, a, b = rng.standard_normal((T, K)), rng.standard_normal((L, r, K)), rng.standard_normal((L, N, r))
    dy, add = rng.standard_normal((T, N)), rng.standard_normal((T, K))
    f = lambda: (dy * ref.adapters(x, a, b, offsets, perm, scale)[0]).sum()
    u = ref.adapters(x, a, b, offsets, perm, scale)[2]
    dx, _, da, _, db, _ = ref.adapters_grad(x, dy, u, a, b, offsets, perm, scale, before=np.zeros((T, K)))
    assert np.allclose(da, _difference(f, a), atol=1e-8) and np.allclose(db, _difference(f, b), atol=1e-8)
    assert np.allclose(dx, _difference(f, x), atol=1e-8)
    covered = perm[:6]
    more = ref.adapters_grad(x, dy, u, a, b, offsets, perm, scale, add=add, da=1.0, db=2.0)
    assert np.allclose(more[0][covered], (dx + add)[covered]) and np.allclose(more[2], da + 1) and np.allclose(more[4], db + 2)
