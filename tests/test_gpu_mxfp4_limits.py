"""The MXFP4 product where blocks are NaN and where scales reach the ends of their range, on each of its kernels."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import fp4_ref
from tests.gpu_common import log, torch_cuda

pytestmark = pytest.mark.gpu

# Up to 4, 16 and 32 tokens and few row blocks; tiles of 128 x 64, 128 x 96, 256 x 128 and 256 x 256, with whole and odd rows of
# y.  K = 288 is two tiles of columns, the second one with a single block; the kernels of many tokens go over four.
TNK = [(4, 200, 288), (16, 201, 288), (31, 200, 288), (70, 100, 288), (70, 4104, 288), (70, 4097, 288), (600, 7168, 288),
       (300, 7001, 288), (1500, 4104, 288), (1500, 5001, 1056), (2300, 7168, 288), (2300, 7001, 288)]


def _tiles(torch, code, scale):
    """Codes and scale bytes of a matrix in the product's layout, through the checkpoint's."""
    rows, cols = code.shape
    by, _ = fp4_ref.rowmajor(code, scale)
    out = torch.empty(damoe.mxfp4_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    damoe.mxfp4_pack(torch.from_numpy(by).cuda(), torch.from_numpy(np.ascontiguousarray(scale)).cuda(), rows, cols, out)
    return out


def _product(torch, x, tiles, N, yd=None, add=None):
    T, K = x.shape
    ws = torch.full((damoe.mxfp4_linear_workspace_size(T, N, K),), 0xFF, dtype=torch.uint8, device="cuda")
    y = torch.full((T, N), 7.0, dtype=yd or torch.float32, device="cuda")
    damoe.mxfp4_linear(x, T, K, tiles, N, y, ws, add=add)
    return y.double().cpu().numpy()


@pytest.mark.parametrize("T,N,K", TNK)
def test_nan_blocks(T, N, K):
    """A NaN block makes its row of x, or its column of w, NaN and nothing else: in the first block and the last, in the first
    row and the last, and where tiles of rows, tokens or columns end inside."""
    torch = torch_cuda()
    rng = np.random.default_rng([T, N, K])
    xv, wv = rng.standard_normal((T, K)), rng.standard_normal((N, K))
    xr, wr = sorted({0, T // 2, T - 1}), sorted({1, N // 3, N - 1})
    for i, r in enumerate(xr):
        xv[r, (0, K // 2, K - 1)[i % 3]] = (np.inf, np.nan, -np.inf)[i % 3]
    for i, r in enumerate(wr):
        wv[r, (K - 1, 0, K // 2)[i % 3]] = np.nan
    x = torch.from_numpy(xv.astype(np.float32)).cuda()
    code, scale = fp4_ref.quantise(wv.astype(np.float32))
    tiles = _tiles(torch, code, scale)
    xq, wq = fp4_ref.values(*fp4_ref.quantise(xv.astype(np.float32))), fp4_ref.values(code, scale)
    assert np.isnan(xq[xr]).any(axis=1).all() and np.isnan(wq[wr]).any(axis=1).all()
    want_nan = np.zeros((T, N), bool)
    want_nan[xr] = True
    want_nan[:, wr] = True
    ref, mag = np.nan_to_num(xq) @ np.nan_to_num(wq).T, np.abs(np.nan_to_num(xq)) @ np.abs(np.nan_to_num(wq)).T
    add = rng.standard_normal((T, N)).astype(np.float32)
    for yd in (torch.float32, torch.bfloat16):
        for a in (None, add):
            log(f"linear with NaN blocks T={T} N={N} K={K} {yd} add={a is not None}")
            d_add = None if a is None else torch.from_numpy(a).to(yd).cuda()
            got = _product(torch, x, tiles, N, yd, d_add)
            assert np.array_equal(np.isnan(got), want_nan)
            want = ref if a is None else ref + d_add.double().cpu().numpy()
            # Exact products, fewer than K sums in fp32 and one with `add`, one rounding to the result's type.
            tol = (K + 2) * 2.0 ** -24 * mag + 2.0 ** -23 * np.abs(want)
            tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if yd == torch.bfloat16 else 0.0)
            assert (np.abs(got - want) <= tol)[~want_nan].all()


@pytest.mark.parametrize("T,N", [(t, n) for t, n, k in TNK if k == 288])
def test_every_scale_of_weights_and_activations(T, N):
    """One product a result, under scales from 2^-127 to 2^127 on both sides: it is rounded once, to a subnormal number or
    infinity where it leaves fp32's range, though the two scales together leave it earlier."""
    torch = torch_cuda()
    log(f"linear of extreme scales T={T} N={N}")
    K = 288
    rng = np.random.default_rng([T, N])
    code, scale = np.zeros((N, K), np.uint8), rng.integers(0, 255, (N, K // 32)).astype(np.uint8)
    at = rng.integers(0, K, T)  # the columns of the rows of x that are not 0, and all columns of W
    code[:] = rng.integers(1, 8, (N, K))
    code |= (rng.integers(0, 2, (N, K)) << 3).astype(np.uint8)
    scale[: min(N, 255), :] = np.arange(min(N, 255), dtype=np.uint8)[:, None]
    e = rng.integers(-149, 128, T)
    e[: min(T, 4)] = [127, -149, -127, 100][: min(T, 4)]
    xv = np.zeros((T, K), np.float32)
    xv[np.arange(T), at] = np.exp2(e.astype(np.float64)).astype(np.float32)
    xq, wq = fp4_ref.values(*fp4_ref.quantise(xv)), fp4_ref.values(code, scale)
    got = _product(torch, torch.from_numpy(xv).cuda(), _tiles(torch, code, scale), N)
    want = xq[np.arange(T), at][:, None] * wq[:, at].T
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    assert (np.abs(want[want != 0]) < 2.0 ** -126).any() and (N <= 254 or np.isinf(want).any())  # both ends are met
    assert np.array_equal(got, want)


@pytest.mark.parametrize("T,N,K", TNK)
def test_sums_over_every_scale(T, N, K):
    """Sums of terms of one sign whose blocks lie anywhere in the scales' range."""
    torch = torch_cuda()
    log(f"linear, sums over every scale, T={T} N={N} K={K}")
    rng = np.random.default_rng([T, N, K, 1])
    code, scale = rng.integers(0, 8, (N, K)).astype(np.uint8), rng.integers(0, 255, (N, K // 32)).astype(np.uint8)
    ex = rng.integers(-140, 127, (T, K // 32)).astype(np.float64)
    xv = (np.abs(rng.standard_normal((T, K // 32, 32))) * np.exp2(ex)[:, :, None]).reshape(T, K)
    xv = np.minimum(xv, float(np.finfo(np.float32).max)).astype(np.float32)
    xq, wq = fp4_ref.values(*fp4_ref.quantise(xv)), fp4_ref.values(code, scale)
    got = _product(torch, torch.from_numpy(xv).cuda(), _tiles(torch, code, scale), N)
    want = xq @ wq.T
    # As for any sums: (K + 2) roundings of the terms' magnitude, here the result itself; below the normal range a rounding
    # is off by up to 2^-149 whatever the magnitude.
    tol = (K + 2) * (2.0 ** -24 * want + 2.0 ** -149)
    top = 2.0 ** 128
    inside, past = want + tol < top, want - tol >= top
    assert past.any() and inside.any() and not np.isnan(got).any()
    assert np.isinf(got[past]).all()
    bad = ~(np.abs(np.where(inside, got, 0.0) - np.where(inside, want, 0.0)) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])
