"""The bits that fp32 factors of the adapters keep: all from 2^-110 on, and of smaller ones against bf16 what is not below 2^-133.

One column and one rank are not 0 and the other factors are powers of two, so that every product and sum is exact, and a lost
bit shows.  A cut loses less than its step: the bound is 2^-133 for the factor, times the powers of two."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests.gpu_common import log, torch_cuda

pytestmark = pytest.mark.gpu

BIG = 2.0 ** 100


def small(torch, n, exponent):
    """n fp32 values of 2^exponent to 2^(exponent + 1), all 24 bits of the significand used (fewer in subnormal ones)."""
    g = torch.Generator().manual_seed(n - exponent)
    v = (1 + torch.randint(0, 1 << 23, (n,), generator=g).double() / (1 << 23))
    v[0] = 2 - 2.0 ** -23
    return (v * 2.0 ** exponent).float().cuda()


def zeros(torch, *s, dtype):
    return torch.zeros(*s, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")


@pytest.mark.parametrize("T,K,N", [(70, 8, 8), (2100, 2184, 648), (4200, 1160, 648)], ids=["one", "joined", "streamed"])
@pytest.mark.parametrize("r", [1, 16, 32, 64])
@pytest.mark.parametrize("exponent", [-20, -90, -110, -118, -130])
def test_bits_of_small_factors(T, K, N, r, exponent):
    torch = torch_cuda()
    log(f"T={T} K={K} N={N} r={r} 2^{exponent}")
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    ws = torch.empty(damoe.adapters_workspace_size(T, 1, r, K, N), dtype=torch.uint8, device="cuda")
    gws = torch.empty(damoe.adapters_grad_workspace_size(T, 1, r, K, N), dtype=torch.uint8, device="cuda")
    rank, v = r - 1, small(torch, T, exponent)

    def near(got, want, bf):
        err = (got.double() - want).abs()
        lost = BIG * 2.0 ** -133 if bf and exponent < -110 else 0.0
        assert float(err.max()) <= lost, (float(err.max()), lost)

    for w in ("bf16", "f32"):
        # u = v, then against B
        x, a, b = zeros(torch, T, K, dtype="f32"), zeros(torch, 1, r, K, dtype=w), zeros(torch, 1, N, r, dtype=w)
        x[:, 3], a[0, rank, 3], b[0, 5, rank] = v, 1, BIG
        y, u = zeros(torch, T, N, dtype="f32"), zeros(torch, T, r, dtype="f32")
        damoe.adapters(x, T, a, b, off, y, ws, u=u)
        assert torch.equal(u[:, rank], v)
        near(y[:, 5], v.double() * BIG, w == "bf16")
        # g = v, then against A and x
        for xt in ("bf16", "f32"):
            x = zeros(torch, T, K, dtype=xt)
            a.zero_(), b.zero_()
            dy, dx = zeros(torch, T, N, dtype="f32"), zeros(torch, T, K, dtype=xt)
            dy[:, 5], b[0, 5, rank], a[0, rank, 3] = v, 1, BIG
            x[0, 2] = BIG
            da, db = zeros(torch, 1, r, K, dtype="f32"), zeros(torch, 1, N, r, dtype="f32")
            damoe.adapters_grad(x, dy, u, T, a, b, off, da, db, gws, dx=dx)
            if xt == "f32":
                near(dx[:, 3], v.double() * BIG, w == "bf16")
            near(da[0, rank, 2].view(1), v[:1].double() * BIG, xt == "bf16")
    # u = v against dy
    for yt in ("bf16", "f32"):
        x, a, b = zeros(torch, T, K, dtype="f32"), zeros(torch, 1, r, K, dtype="f32"), zeros(torch, 1, N, r, dtype="f32")
        u, dy = zeros(torch, T, r, dtype="f32"), zeros(torch, T, N, dtype=yt)
        u[:, rank], dy[0, 4] = v, BIG
        da, db = zeros(torch, 1, r, K, dtype="f32"), zeros(torch, 1, N, r, dtype="f32")
        damoe.adapters_grad(x, dy, u, T, a, b, off, da, db, gws)
        near(db[0, 4, rank].view(1), v[:1].double() * BIG, yt == "bf16")
    # fp32 weights of bf16 rows
    x, a, b = zeros(torch, T, K, dtype="bf16"), zeros(torch, 1, r, K, dtype="f32"), zeros(torch, 1, N, r, dtype="f32")
    n = min(r, 8)
    x[:, 3], a[0, :n, 3] = BIG, v[:n]
    y, u = zeros(torch, T, N, dtype="bf16"), zeros(torch, T, r, dtype="f32")
    damoe.adapters(x, T, a, b, off, y, ws, u=u)
    near(u[:, :n], (v[:n].double() * BIG).expand(T, n), True)
