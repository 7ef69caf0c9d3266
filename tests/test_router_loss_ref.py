"""The float64 gradient of the router's loss against differences of its loss (CPU)."""
import numpy as np
import pytest

from tests import router_loss_ref as ref


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("offsets", [None, [0, 3, 3, 8]])
def test_gradient_equals_differences(score, offsets):
    rng = np.random.default_rng([score, offsets is None])
    T, E, k = 9, 7, 3
    l = rng.standard_normal((T, E)) * 2
    l[:, 5] = -np.inf
    ids = np.argsort(-l, axis=1)[:, :k]
    ids[4, 2] = -1
    mask = np.ones(T)
    mask[6] = 0
    alpha, zc, g = 0.3, 0.05, 1.7
    dw = rng.standard_normal((T, k))

    def gates(x):
        top = np.take_along_axis(x, np.where(ids >= 0, ids, 0), axis=1)
        top = np.where(ids >= 0, top, -np.inf)
        ex = np.exp(top - top.max(axis=1, keepdims=True))
        return ex / ex.sum(axis=1, keepdims=True)

    seqs = ref.members(T, mask, offsets)
    inside = {t for v in seqs for t in v}

    def total(x):
        v = g * ref.loss(x, ids, k, mask, offsets, score, alpha, zc)[0][0]
        return v + sum((gates(x) * dw)[t].sum() for t in inside)

    counts = ref.loss(l, ids, k, mask, offsets, score, alpha, zc)[1]
    d, _ = ref.grad(l, ids, k, mask, offsets, score, alpha, zc, counts, g, gates(l), dw)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            if np.isneginf(l[t, e]):
                assert d[t, e] == 0
                continue
            a, b = l.copy(), l.copy()
            a[t, e] += h
            b[t, e] -= h
            assert abs((total(a) - total(b)) / (2 * h) - d[t, e]) < 1e-8, (t, e)
