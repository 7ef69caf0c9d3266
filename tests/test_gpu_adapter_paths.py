"""The adapters' ways through their kernels: one launch, two, many rows; the gradient of few rows, of many and of high ranks;
and what they leave of their workspaces."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import rows_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_adapters import Case
from tests.test_gpu_rows import close

pytestmark = pytest.mark.gpu

TYPES = [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "bf16"), ("bf16", "bf16", "f32"),
         ("f32", "f32", "bf16")]


@pytest.mark.parametrize("r", [1, 8, 12, 16, 24, 32, 40, 64, 128])
@pytest.mark.parametrize("x,w,y", TYPES)
def test_many_rows_and_whole_tiles_of_columns(r, x, w, y):
    torch = torch_cuda()
    log(f"r={r} x={x} w={w} y={y}")
    Case(torch, 4200, 3, r, 256, 512, x, w, y, free=5).check()


@pytest.mark.parametrize("T,L,r,K,N", [
    (3, 2, 64, 4160, 264),     # A of a segment too large for every block to read
    (70, 60, 16, 4096, 640),   # blocks enough for two launches
    (1000, 4, 16, 7300, 384),  # columns over blocks, a partial unit
    (1025, 2, 32, 136, 1100),  # the gradient's first rows past the few
    (1024, 1, 7, 130, 260), (3000, 2, 20, 256, 1300), (600, 1, 48, 384, 256), (4095, 5, 8, 128, 128), (4096, 1024, 3, 24, 40)])
@pytest.mark.parametrize("x,w,y", TYPES[:4])
def test_sizes_on_either_side_of_a_rule(T, L, r, K, N, x, w, y):
    torch = torch_cuda()
    log(f"T={T} L={L} r={r} K={K} N={N} x={x} w={w} y={y}")
    Case(torch, T, L, r, K, N, x, w, y).check()


@pytest.mark.parametrize("n", [1, 2, 3, 7])
def test_rows_shorter_than_a_load(n):
    torch = torch_cuda()
    for K, N in ((n, 40), (40, n), (n, n)):
        for dtype in ("bf16", "f32"):
            for T in (5, 1100):
                log(f"K={K} N={N} {dtype} T={T}")
                Case(torch, T, 2, 4, K, N, dtype, dtype, dtype).check()


def test_strides_and_alignment_of_many_rows():
    torch = torch_cuda()
    for dtype in ("bf16", "f32"):
        for kw in (dict(ld=3, shift=1), dict(ld=5, shift=3, mixed=False, free=40), dict(scale=False, add=False)):
            log(f"{dtype} {kw}")
            Case(torch, 4150, 4, 10, 264, 264, dtype, dtype, dtype, **kw).check()


@pytest.mark.parametrize("T,L,r,K,N", [(1, 1, 1, 1, 1), (1, 3, 16, 7168, 40), (100, 7, 9, 300, 500), (1024, 2, 64, 200, 300),
                                       (1025, 1, 16, 2048, 64), (2000, 1000, 5, 64, 64), (4095, 3, 16, 640, 72), (4096, 3, 128, 72, 640),
                                       (9000, 2, 33, 128, 128)])
def test_workspaces_end_where_they_are_said_to(T, L, r, K, N):
    """The bytes past the sizes that the library names, of T rows or of more, are as they were; fewer bytes are refused."""
    torch = torch_cuda()
    log(f"T={T} L={L} r={r} K={K} N={N}")
    for dtype in ("bf16", "f32"):
        c = Case(torch, T, L, r, K, N, dtype, dtype, dtype)
        sizes = [w.numel() for w in c.ws]
        c.ws = [torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda") for n in sizes]
        c.forward(), c.backward()
        for w, n in zip(c.ws, sizes):
            assert (w[n:] == 0xA5).all(), (dtype, n)
        want = [t.clone() for t in (c.d_y, c.d_dx, c.d_ga, c.d_gb)]
        c.ws = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes]
        c.forward(), c.backward()
        assert all(torch.equal(p, q) for p, q in zip(want, (c.d_y, c.d_dx, c.d_ga, c.d_gb)))


def test_values_that_are_not_finite_in_many_rows():
    """As in few rows: of their own segment, or of their own row, alone; infinite fp32 weights of bf16 rows stay infinite."""
    torch = torch_cuda()
    for x, w in (("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")):
        c = Case(torch, 4400, 4, 8, 256, 256, x, w, x, bounds=[0, 1000, 1001, 3000, 4300], add=False)
        c.forward(), c.backward()
        good = [t.clone() for t in (c.d_y, c.d_u, c.d_dx, c.d_ga, c.d_gb)]
        rows = lambda l: torch.from_numpy(c.perm[c.off[l]: c.off[l + 1]]).long().cuda()
        c.da_[0, 3, 5], c.dx_[int(rows(2)[70]), 11] = float("nan"), float("inf")
        c.da_[1, 2, 7] = float("inf")
        free = torch.from_numpy(c.perm[4300:]).long().cuda()
        c.dx_[free], c.d_dy[free] = float("nan"), float("inf")
        c.forward()
        assert c.d_y[rows(0)].isnan().all() and c.d_u[:1000, 3].isnan().all()
        assert c.d_u[1000, 2].isinf() and torch.equal(c.d_u[1000, 3:], good[1][1000, 3:])
        keep = torch.ones(4400, dtype=torch.bool, device="cuda")
        keep[rows(0)] = keep[rows(1)] = keep[rows(2)[70]] = False
        assert torch.equal(c.d_y[keep], good[0][keep])
        c.d_u.copy_(good[1])
        c.backward()
        assert torch.equal(c.d_ga[3], good[3][3]) and torch.equal(c.d_gb, good[4])
        # g's thirds may be 0, and 0 times infinity is NaN.
        assert not c.d_ga[2][:, 11].isfinite().any() and torch.equal(c.d_ga[2][:, 12:], good[3][2][:, 12:])
        assert torch.equal(c.d_dx[rows(2)], good[2][rows(2)]) and c.d_dx[rows(0)][:, 5].isnan().all()


def test_gradients_against_differences():
    """<dy, y> changes with a weight or a row as the gradient says: the change over a step of 2^-4, in which the sum is linear
    for one of x, A and B at a time, so that only fp32's roundings are left."""
    torch = torch_cuda()
    for T, L, K, N, r in ((40, 3, 72, 56, 5), (4100, 2, 128, 128, 16)):
        c = Case(torch, T, L, r, K, N, "f32", "f32", "f32", add=False)
        c.forward()
        c.backward(add=None)
        y0, u0 = c.d_y.double(), c.d_u.clone()
        named = torch.zeros(T, dtype=torch.bool, device="cuda")
        named[torch.from_numpy(c.perm[: c.off[-1]]).long().cuda()] = True
        rng = np.random.default_rng(T)
        l = int(np.argmax(np.diff(c.off)))
        t = int(c.perm[c.off[l]])
        for what, grad, at in ((c.dx_, c.d_dx, (t, int(rng.integers(K)))), (c.da_, c.d_ga, (l, int(rng.integers(r)), int(rng.integers(K)))),
                               (c.db_, c.d_gb, (l, int(rng.integers(N)), int(rng.integers(r))))):
            before = what[at].clone()
            what[at] += 2.0 ** -4
            step = float(what[at].double() - before.double())
            c.forward()
            what[at] = before
            moved = (c.d_y.double() - y0)[named] * c.d_dy.double()[named]
            # Each y is off by (K + 3 r + 4) steps of at most `size`, before and after; the gradient by as many of its terms.
            size = float((c.d_dy.double().abs()[named] * (y0.abs()[named] + c.d_y.double().abs()[named])).sum())
            slack = 2 * (3 * K + 3 * N + 6 * r + 8) * ref.STEP * (size / step + float(grad[at].abs()) + size)
            assert abs(float(moved.sum()) / step - float(grad[at])) <= slack, (what.shape, at)
        c.d_u.copy_(u0)


def test_graphs_of_every_way_replayed_between_eager_calls():
    torch = torch_cuda()
    for T, r, K in ((4, 16, 256), (90, 16, 8192), (1500, 8, 256), (4300, 16, 256), (4300, 40, 256)):
        log(f"T={T} r={r} K={K}")
        c, other = (Case(torch, T, 3, r, K, 264, seed=s) for s in (1, 2))
        outs = lambda c: [t.clone() for t in (c.d_y, c.d_u, c.d_dx, c.d_ga, c.d_gb)]
        c.forward(), c.backward()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.forward(), c.backward()
        for k in range(4):
            c.dx_.mul_(-0.5), c.d_ga.fill_(k), c.d_gb.fill_(k), c.d_y.fill_(k)
            g.replay()
            other.forward(), other.backward()
            got = outs(c)
            torch.cuda.synchronize()
            c.forward(), c.backward()
            assert all(torch.equal(p, q) for p, q in zip(got, outs(c))), k
            assert not torch.equal(got[3], other.d_ga)


def test_empty_segments_are_cleared_or_kept():
    """Segments without rows: zeros, or with accumulate what was there; of few rows and of many."""
    torch = torch_cuda()
    for T in (3, 700, 2000, 4500):
        for r in (4, 40):
            c = Case(torch, T, 200, r, 64, 72, bounds=[0] * 60 + [T // 2] * 100 + [T] * 41)
            c.forward()
            c.d_ga.fill_(float("nan")), c.d_gb.fill_(float("nan"))
            c.backward()
            full = np.flatnonzero(np.diff(c.off))
            empty = torch.from_numpy(np.setdiff1d(np.arange(200), full)).cuda()
            assert not c.d_ga[empty].any() and not c.d_gb[empty].any()
            assert c.d_ga[full].any() and c.d_ga.isfinite().all() and c.d_gb.isfinite().all()
            c.d_ga.fill_(3), c.d_gb.fill_(5)
            c.backward(accumulate=True)
            assert (c.d_ga[empty] == 3).all() and (c.d_gb[empty] == 5).all()


def test_offsets_that_end_before_the_rows_or_past_them():
    """Offsets past T are cut at T, so that nothing past the rows is touched."""
    torch = torch_cuda()
    for T in (20, 4300):
        c = Case(torch, T, 2, 8, 128, 128, mixed=False)
        c.forward()
        y = c.d_y.clone()
        c.d_off.copy_(torch.tensor([0, int(c.off[1]), T + 100000], dtype=torch.int32))
        c.forward(), c.backward()
        close(c.d_y, y.double().cpu().numpy(), np.zeros(y.shape), None, "y")


def test_offsets_that_decrease_stay_within_the_workspace():
    """Their results are unspecified; every place is below T, every slot one of those there are."""
    torch = torch_cuda()
    for T, r in ((700, 8), (2500, 8), (5000, 40)):
        log(f"T={T} r={r}")
        c = Case(torch, T, 64, r, 128, 256)
        sizes = [w.numel() for w in c.ws]
        c.ws = [torch.full((n + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda") for n in sizes]
        c.d_off.copy_(torch.tensor([0] + [T, 0] * 32, dtype=torch.int32))
        c.forward(), c.backward()
        for w, n in zip(c.ws, sizes):
            assert (w[n:] == 0xA5).all(), n


@pytest.mark.parametrize("T,L,r,K,N", [(2, 1, 1, 1 << 20, 9), (2, 1, 1, 9, 1 << 20), (1030, 1, 2, 1 << 17, 12), (1 << 20, 3, 2, 8, 9)])
def test_the_longest_rows_and_the_most_of_them(T, L, r, K, N):
    torch = torch_cuda()
    log(f"T={T} K={K} N={N}")
    for dtype in ("bf16", "f32"):
        Case(torch, T, L, r, K, N, dtype, dtype, dtype).check()
