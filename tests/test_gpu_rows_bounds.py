"""What the row and adapter calls leave alone: the elements between rows, before and behind every output; results in the place of
what is added; strides that are given."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import rows_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_adapters import Case
from tests.test_gpu_rows import Batch, close, matrix

pytestmark = pytest.mark.gpu

GUARD = 64  # elements


def fenced(torch, shape, dtype):
    """A contiguous tensor of 7s with NaN before and behind it, and the whole."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * GUARD,), float("nan"), dtype=dtype, device="cuda")
    inner = whole[GUARD: GUARD + n].view(shape)
    inner.fill_(7)
    return inner, whole


def beside(m, whole):
    """The elements of `whole` that m, a view of it, does not have."""
    mask = whole.new_ones(whole.numel(), dtype=bool)
    mask.as_strided(m.shape, m.stride(), m.storage_offset()).fill_(False)
    return whole[mask]


def strided(torch, rows, cols, ld, dtype, shift, value=None):
    """A matrix with NaN before, between and behind its rows."""
    whole = torch.full((rows * ld + 2 * GUARD + shift,), float("nan"), dtype=dtype, device="cuda")
    m = whole[GUARD + shift:][: rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.randn(rows, cols, device="cuda") if value is None else torch.full((rows, cols), value, device="cuda"))
    return m, whole


@pytest.mark.parametrize("T,k,H", [(3, 2, 7), (40, 8, 1031), (2700, 16, 520), (5300, 1, 4099)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows(T, k, H, dtype):
    torch = torch_cuda()
    log(f"T={T} k={k} H={H} {dtype}")
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    b = Batch(torch, T, k, H, dtype, drop=0.1)
    for ld, shift in ((H + 1, 1), (H + 9, 0)):
        x, _ = strided(torch, T, H, ld, t, shift)
        rows, all_rows = strided(torch, b.R, H, ld, t, shift)
        y, all_y = strided(torch, T, H, ld, t, shift)
        drows, all_drows = strided(torch, b.R, H, ld, t, shift)
        dw, all_dw = fenced(torch, (T, k), torch.float32)
        damoe.sort_rows(x, T, k, H, b.d_inv, rows, w=b.d_w)
        damoe.combine_rows(rows, T, k, H, b.d_inv, y, w=b.d_w, add=x)
        damoe.combine_rows_grad(x, rows, T, k, H, b.d_inv, w=b.d_w, drows=drows, dw=dw)
        for m, whole in ((rows, all_rows), (y, all_y), (drows, all_drows), (dw, all_dw)):
            assert beside(m, whole).isnan().all() and m.isfinite().all()


SIZES = [(1, 1, 16, 136, 72), (70, 5, 9, 300, 648), (1000, 3, 20, 2184, 648), (700, 30, 40, 140, 33), (1500, 2, 8, 257, 130),
         (3000, 3, 48, 264, 520), (4200, 3, 4, 1160, 648), (4200, 3, 32, 1160, 650), (4200, 2, 128, 140, 72)]


@pytest.mark.parametrize("T,L,r,K,N", SIZES)
@pytest.mark.parametrize("x,w,y", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("bf16", "bf16", "f32")])
def test_adapters(T, L, r, K, N, x, w, y):
    torch = torch_cuda()
    log(f"T={T} L={L} r={r} K={K} N={N} x={x} w={w} y={y}")
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    c = Case(torch, T, L, r, K, N, x, w, y, free=min(3, T - 1))
    c.forward(), c.backward()
    covered = torch.from_numpy(np.sort(c.perm[: c.off[-1]])).long().cuda()
    free = torch.from_numpy(np.sort(c.perm[c.off[-1]:])).long().cuda()
    for ld, shift in ((1, 1), (8, 0)):
        out_y, all_y = strided(torch, T, N, N + ld, types[y], shift, 7)
        out_x, all_x = strided(torch, T, K, K + ld, types[x], shift, 7)
        u, all_u = fenced(torch, (T, r), torch.float32)
        da, all_da = fenced(torch, (L, r, K), torch.float32)
        db, all_db = fenced(torch, (L, N, r), torch.float32)
        c.forward(y=out_y, u=u)
        damoe.adapters_grad(c.dx_, c.d_dy, c.d_u, T, c.da_, c.db_, c.d_off, da, db, c.ws[1], perm=c.d_perm, scale=c.d_scale, add=c.d_addx,
                            dx=out_x)
        for m, whole in ((out_y, all_y), (out_x, all_x), (u, all_u), (da, all_da), (db, all_db)):
            assert beside(m, whole).isnan().all()
        n = int(c.off[-1])
        assert torch.equal(out_y[covered], c.d_y[covered]) and (out_y[free] == 7).all()
        assert torch.equal(out_x[covered], c.d_dx[covered]) and (out_x[free] == 7).all()
        assert torch.equal(u[:n], c.d_u[:n]) and (u[n:] == 7).all()
        assert torch.equal(da, c.d_ga) and torch.equal(db, c.d_gb)
        # In the place of what is added.
        out_y.copy_(c.d_add), out_x.copy_(c.d_addx)
        c.forward(y=out_y, add=out_y, u=None)
        damoe.adapters_grad(c.dx_, c.d_dy, c.d_u, T, c.da_, c.db_, c.d_off, da, db, c.ws[1], perm=c.d_perm, scale=c.d_scale, add=out_x,
                            dx=out_x)
        assert torch.equal(out_y[covered], c.d_y[covered]) and torch.equal(out_y[free], c.d_add[free])
        assert torch.equal(out_x[covered], c.d_dx[covered]) and torch.equal(out_x[free], c.d_addx[free])
        assert beside(out_y, all_y).isnan().all() and beside(out_x, all_x).isnan().all()
        assert torch.equal(da, c.d_ga) and torch.equal(db, c.d_gb)


def test_strides_that_are_given():
    """Rows in flat buffers, each with a stride of its own."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    T, K, N, L, r, k = 50, 70, 45, 3, 6, 2

    def flat(rows, cols, ld, v=None):
        v = rng.standard_normal((rows, cols)).astype(np.float32) if v is None else v
        buf = torch.full((rows * ld,), float("nan"), device="cuda")
        buf.view(rows, ld)[:, :cols] = torch.from_numpy(v).cuda()
        return buf, v.astype(np.float64)

    off = np.array([0, 11, 30, 47], np.int32)
    d_off = torch.from_numpy(off).cuda()
    (a, va), (b, vb) = (matrix(torch, rng.standard_normal(s), "f32") for s in ((L * r, K), (L * N, r)))
    a, b, va, vb = a.view(L, r, K), b.view(L, N, r), va.reshape(L, r, K), vb.reshape(L, N, r)
    x, vx = flat(T, K, K + 3)
    add, vadd = flat(T, N, N + 1)
    y, vy = flat(T, N, N + 6)
    u = torch.zeros(T, r, device="cuda")
    ws = torch.empty(damoe.adapters_workspace_size(T, L, r, K, N), dtype=torch.uint8, device="cuda")
    damoe.adapters(x, T, a, b, d_off, y, ws, add=add, u=u, ldx=K + 3, ld_add=N + 1, ldy=N + 6)
    want, err, wu, eu = ref.adapters(vx, va, vb, off, None, None, vadd, vy)
    close(y.view(T, -1)[:, :N], want, err, "f32", "y")
    dy, vdy = flat(T, N, N + 2)
    addx, vaddx = flat(T, K, K + 5)
    dx, vdx = flat(T, K, K + 4)
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    gws = torch.empty(damoe.adapters_grad_workspace_size(T, L, r, K, N), dtype=torch.uint8, device="cuda")
    damoe.adapters_grad(x, dy, u, T, a, b, d_off, da, db, gws, add=addx, dx=dx, ldx=K + 3, ldy=N + 2, ld_dx=K + 4, ld_add=K + 5)
    wx, ex, wa, ea, wb, eb = ref.adapters_grad(vx, vdy, u.double().cpu().numpy(), va, vb, off, None, None, vaddx, vdx)
    close(dx.view(T, -1)[:, :K], wx, ex, "f32", "dx")
    close(da, wa, ea, "f32", "da")
    close(db, wb, eb, "f32", "db")
    inv = rng.permutation(T * k).astype(np.int32)
    d_inv = torch.from_numpy(inv).cuda()
    rows, vr = matrix(torch, rng.standard_normal((T * k, K)), "f32", K + 2)
    before = vr.copy()
    damoe.sort_rows(x, T, k, K, d_inv, rows, ldx=K + 3)
    close(rows, *ref.sort_rows(vx, inv, k, T * k, before), None, "sort")
    out, _ = flat(T, K, K + 7)
    damoe.combine_rows(rows, T, k, K, d_inv, out, add=addx, ldy=K + 7, ld_add=K + 5)
    close(out.view(T, -1)[:, :K], *ref.combine_rows(rows.double().cpu().numpy(), inv, T, k, None, vaddx), "f32", "combine")
    dw = torch.zeros(T, k, device="cuda")
    damoe.combine_rows_grad(x, rows, T, k, K, d_inv, dw=dw, ldy=K + 3)
    close(dw, *ref.combine_rows_grad(vx, rows.double().cpu().numpy(), inv, k, before)[2:], "f32", "dw")
