"""Low-rank adapters of many segments and their gradient against float64 (tests/rows_ref.py)."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import rows_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_rows import close, matrix

pytestmark = pytest.mark.gpu


def tensor3(torch, v, dtype, shift=0):
    t = torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    buf = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")[shift:].view(t.shape)
    buf.copy_(t)
    return buf, t.double().numpy()


class Case:
    """Rows of T tokens over L adapters.  bounds: offsets, by default random ones with empty segments among them; free: rows in
    no segment; mixed: perm is a random order, else None."""

    def __init__(self, torch, T, L, r, K, N, x="bf16", w="bf16", y="bf16", bounds=None, free=0, mixed=True, scale=True, add=True,
                 ld=0, shift=0, seed=0):
        rng = np.random.default_rng([T, L, r, K, N, seed])
        self.torch, self.T, self.L, self.r, self.K, self.N, self.x, self.w, self.y = torch, T, L, r, K, N, x, w, y
        n = T - free
        if bounds is None:
            ids = rng.integers(0, L, n) if T < 4 * L else rng.choice(rng.integers(0, L, max(1, L // 2)), n)
            bounds = np.concatenate([[0], np.cumsum(np.bincount(ids, minlength=L))])
        self.off = np.asarray(bounds, np.int32)
        self.perm = rng.permutation(T).astype(np.int32) if mixed else None
        self.scale = rng.uniform(0.5, 2, L).astype(np.float32) if scale else None
        cu = lambda v: None if v is None else torch.from_numpy(v).cuda()
        self.d_off, self.d_perm, self.d_scale = cu(self.off), cu(self.perm), cu(self.scale)
        m = lambda rows, cols, t: matrix(torch, rng.standard_normal((rows, cols)), t, ld and cols + ld, shift)
        self.dx_, self.vx = m(T, K, x)
        self.da_, self.va = tensor3(torch, rng.standard_normal((L, r, K)) * K ** -0.5, w, shift)
        self.db_, self.vb = tensor3(torch, rng.standard_normal((L, N, r)) * r ** -0.5, w, shift)
        self.d_add, self.vadd = m(T, N, y) if add else (None, None)
        self.d_y, self.vy0 = m(T, N, y)
        self.d_dy, self.vdy = m(T, N, y)
        self.d_addx, self.vaddx = m(T, K, x) if add else (None, None)
        self.d_dx, self.vdx0 = m(T, K, x)
        self.d_u = torch.full((T, r), 7.0, device="cuda")
        size = damoe.adapters_workspace_size(T, L, r, K, N), damoe.adapters_grad_workspace_size(T, L, r, K, N)
        # 0xFF: whatever the calls read before they wrote it is NaN.
        self.ws = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in size]
        self.d_ga, self.d_gb = (torch.full(s, 3.0, device="cuda") for s in ((L, r, K), (L, N, r)))

    def forward(self, y=None, u="u", stream=None, **kw):
        kw = {"add": self.d_add, **kw}
        damoe.adapters(self.dx_, self.T, self.da_, self.db_, self.d_off, self.d_y if y is None else y, self.ws[0], perm=self.d_perm,
                       scale=self.d_scale, u=self.d_u if isinstance(u, str) else u, stream=stream, **kw)

    def backward(self, stream=None, **kw):
        kw = {"add": self.d_addx, "dx": self.d_dx, **kw}
        damoe.adapters_grad(self.dx_, self.d_dy, self.d_u, self.T, self.da_, self.db_, self.d_off, self.d_ga, self.d_gb, self.ws[1],
                            perm=self.d_perm, scale=self.d_scale, stream=stream, **kw)

    def check(self):
        torch = self.torch
        self.forward()
        y, ey, u, eu = ref.adapters(self.vx, self.va, self.vb, self.off, self.perm, self.scale, self.vadd, self.vy0,
                                    np.full((self.T, self.r), 7.0))
        close(self.d_y, y, ey, self.y, "y")
        close(self.d_u, u, eu, "f32", "u")
        again = torch.zeros_like(self.d_y)
        keep = np.ones(self.T, bool)
        for _, _, t in ref.segments(self.off, self.perm, self.T):
            keep[t] = False
        again[torch.from_numpy(keep).cuda()] = self.d_y[torch.from_numpy(keep).cuda()]
        self.forward(y=again, u=None)
        assert torch.equal(again, self.d_y)
        if self.d_add is not None:  # in the place of what is added
            again = self.d_add.clone()
            self.forward(y=again, add=again, u=None)
            assert torch.equal(again[torch.from_numpy(~keep).cuda()], self.d_y[torch.from_numpy(~keep).cuda()])
            assert torch.equal(again[torch.from_numpy(keep).cuda()], self.d_add[torch.from_numpy(keep).cuda()])
        # The gradient goes by the u that it is given.
        self.backward()
        given = self.d_u.double().cpu().numpy()
        dx, edx, da, ea, db, eb = ref.adapters_grad(self.vx, self.vdy, given, self.va, self.vb, self.off, self.perm, self.scale,
                                                    self.vaddx, self.vdx0)
        close(self.d_dx, dx, edx, self.x, "dx")
        close(self.d_ga, da, ea, "f32", "da")
        close(self.d_gb, db, eb, "f32", "db")
        one = self.d_ga.clone(), self.d_gb.clone()
        self.backward(dx=None, add=None)
        assert torch.equal(one[0], self.d_ga) and torch.equal(one[1], self.d_gb)
        self.backward(dx=None, add=None, accumulate=True)
        two = ref.adapters_grad(self.vx, self.vdy, given, self.va, self.vb, self.off, self.perm, self.scale,
                                da=one[0].double().cpu().numpy(), db=one[1].double().cpu().numpy())
        close(self.d_ga, two[2], two[3], "f32", "da, added")
        close(self.d_gb, two[4], two[5], "f32", "db, added")


SIZES = [(1, 1, 1, 1, 1), (1, 8, 16, 96, 64), (2, 1, 3, 700, 5), (7, 3, 5, 33, 17), (64, 64, 8, 256, 128), (65, 5, 16, 640, 72),
         (257, 70, 4, 130, 70), (300, 2, 32, 64, 257), (2048, 3, 33, 96, 100), (2101, 100, 16, 72, 264), (100, 2, 128, 200, 72),
         (40, 2, 100, 31, 66), (2050, 130, 64, 40, 33), (530, 1024, 2, 16, 24)]


@pytest.mark.parametrize("T,L,r,K,N", SIZES)
@pytest.mark.parametrize("x,w,y", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("bf16", "f32", "bf16"), ("f32", "bf16", "bf16"),
                                   ("bf16", "bf16", "f32")])
def test_sizes_and_types(T, L, r, K, N, x, w, y):
    torch = torch_cuda()
    log(f"T={T} L={L} r={r} K={K} N={N} x={x} w={w} y={y}")
    Case(torch, T, L, r, K, N, x, w, y).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [
    dict(bounds=[0, 0, 0, 0]), dict(bounds=[0, 0, 70, 70]), dict(bounds=[0, 1, 2, 90]), dict(bounds=[0, 16, 48, 64]),
    dict(bounds=[0, 63, 64, 65]), dict(bounds=[0, 15, 31, 99]), dict(free=40), dict(free=100), dict(mixed=False, free=3),
    dict(scale=False, add=False), dict(ld=3, free=1), dict(shift=1), dict(ld=5, shift=3, mixed=False)], ids=str)
def test_segments_strides_and_alignment(kw, dtype):
    torch = torch_cuda()
    log(f"{kw} {dtype}")
    Case(torch, 100, 3, 9, 136, 80, dtype, dtype, dtype, **kw).check()


@pytest.mark.parametrize("T", [700, 2500, 9000])
def test_long_segments_over_several_chunks(T):
    """Segments that begin and end inside of chunks, span whole ones, or fill one exactly."""
    torch = torch_cuda()
    for bounds in ([0, T // 3, T // 3 + 1, T], [0, 128, 256, T - 1], [0, 5, 6, T - T // 2], [0, 0, T, T]):
        log(f"T={T} {bounds}")
        Case(torch, T, 3, 6, 264, 40, bounds=bounds).check()


def test_rows_that_perm_does_not_name():
    """Entries of perm outside the rows leave their places out, and nothing beside them changes."""
    torch = torch_cuda()
    for bad in (-1, 90, 1 << 30, -(1 << 31)):
        c = Case(torch, 90, 4, 8, 64, 72, free=10)
        for p in (0, 17, 40, 79):
            c.perm[p] = bad
        c.d_perm.copy_(torch.from_numpy(c.perm))
        c.d_u.zero_()
        c.forward()
        y, ey, _, _ = ref.adapters(c.vx, c.va, c.vb, c.off, c.perm, c.scale, c.vadd, c.vy0)
        close(c.d_y, y, ey, "bf16", "y")


def test_values_that_are_not_finite():
    """They reach the rows of their own segment, or their own row, alone."""
    torch = torch_cuda()
    for dtype in ("bf16", "f32"):
        c = Case(torch, 200, 5, 8, 96, 80, dtype, dtype, dtype, bounds=[0, 40, 77, 78, 130, 190])
        c.check()
        rows = lambda l: torch.from_numpy(c.perm[c.off[l]: c.off[l + 1]]).long().cuda()
        good = [t.clone() for t in (c.d_y, c.d_u)]
        c.d_ga.zero_(), c.d_gb.zero_()
        c.backward()
        grads = [t.clone() for t in (c.d_dx, c.d_ga, c.d_gb)]
        c.da_[1, 3, 5], c.db_[3, 7, 2] = float("nan"), float("inf")
        x_row, free = int(rows(4)[9]), torch.from_numpy(c.perm[190:]).long().cuda()
        c.dx_[x_row, 11] = float("nan")
        c.dx_[free], c.d_dy[free], c.d_add[free] = float("nan"), float("nan"), float("inf")
        y = good[0].clone()
        c.forward(y=y)
        assert y[rows(1)].isnan().all() and not y[rows(3)][:, 7].isfinite().any() and y[x_row].isnan().all()
        same = torch.ones_like(y, dtype=torch.bool)
        same[rows(1)] = same[x_row] = False
        same[rows(3), 7] = False
        assert torch.equal(y[same], good[0][same])
        c.d_u.copy_(good[1])
        c.backward()
        dx, ga, gb = grads
        for l in (0, 2):
            assert torch.equal(c.d_dx[rows(l)], dx[rows(l)])
            assert torch.equal(c.d_ga[l], ga[l]) and torch.equal(c.d_gb[l], gb[l])
        assert c.d_dx[rows(1)][:, 5].isnan().all() and torch.equal(c.d_dx[rows(1)][:, 6:], dx[rows(1)][:, 6:])
        assert torch.equal(c.d_ga[1], ga[1]) and torch.equal(c.d_gb, gb)
        assert c.d_ga[4][:, 11].isnan().all() and torch.equal(c.d_ga[4][:, 12:], ga[4][:, 12:])


def test_large_values_keep_their_range():
    """The parts that u is split into neither overflow nor lose its sign: values next to fp32's and bf16's largest."""
    torch = torch_cuda()
    big = float(torch.finfo(torch.float32).max)
    x = torch.zeros(2, 8, device="cuda")
    x[0, 0], x[1, 0] = big, -big
    a = torch.zeros(1, 1, 8, dtype=torch.bfloat16, device="cuda")
    a[0, 0, 0] = 1
    b = torch.full((1, 5, 1), 0.5, dtype=torch.bfloat16, device="cuda")
    y, off = torch.zeros(2, 5, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    ws = torch.empty(damoe.adapters_workspace_size(2, 1, 1, 8, 5), dtype=torch.uint8, device="cuda")
    damoe.adapters(x, 2, a, b, off, y, ws)
    assert (y[0] == big / 2).all() and (y[1] == -big / 2).all()


def test_many_segments_of_experts_and_rows_past_32_bit_offsets():
    torch = torch_cuda()
    T, K, N, r = 700000, 8192, 16, 2
    x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")  # 11 GB
    at = torch.tensor([0, 5, 524288, T - 1], device="cuda")
    x[at] = torch.randn(4, K, device="cuda").to(x.dtype)
    a, b = torch.randn(3, r, K, device="cuda").to(x.dtype), torch.randn(3, N, r, device="cuda").to(x.dtype)
    off = torch.tensor([0, 6, 600000, T], dtype=torch.int32, device="cuda")
    y, u = torch.zeros(T, N, dtype=x.dtype, device="cuda"), torch.zeros(T, r, device="cuda")
    ws = torch.empty(damoe.adapters_workspace_size(T, 3, r, K, N), dtype=torch.uint8, device="cuda")
    damoe.adapters(x, T, a, b, off, y, ws, u=u)
    rows = at.cpu().numpy()
    vx, va, vb = x[at].double().cpu().numpy(), a.double().cpu().numpy(), b.double().cpu().numpy()
    want, err, wu, eu = ref.adapters(vx, va[[0, 1, 2]], vb, [0, 2, 3, 4])
    close(y[at], want, err, "bf16", "y")
    close(u[at], wu, eu, "f32", "u")
    assert int((y != 0).any(dim=1).sum()) == 4
    dy = torch.zeros_like(y)
    dy[at] = torch.randn(4, N, device="cuda").to(x.dtype)
    da, db = torch.empty(3, r, K, device="cuda"), torch.empty(3, N, r, device="cuda")
    gws = torch.empty(damoe.adapters_grad_workspace_size(T, 3, r, K, N), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)
    damoe.adapters_grad(x, dy, u, T, a, b, off, da, db, gws, dx=dx)
    wx, ex, wa, ea, wb, eb = ref.adapters_grad(vx, dy[at].double().cpu().numpy(), u[at].double().cpu().numpy(), va, vb, [0, 2, 3, 4])
    close(dx[at], wx, ex, "bf16", "dx")
    close(da, wa, ea, "f32", "da")
    close(db, wb, eb, "f32", "db")
    dx[at] = 0
    assert not dx.any(), rows


def test_equal_bits_streams_and_graphs():
    """Two calls at once on two streams with workspaces of their own, and graphs replayed between eager calls."""
    torch = torch_cuda()
    cases = [Case(torch, 800, 5, 16, 520, 264, seed=s, free=9) for s in range(2)]
    outs = lambda c: [t.clone() for t in (c.d_y, c.d_u, c.d_dx, c.d_ga, c.d_gb)]
    for c in cases:
        c.forward(), c.backward()
    want = [outs(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c in cases:
            c.d_ga.zero_(), c.d_gb.zero_(), c.d_u.zero_()
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for c, s in zip(cases, streams):
            c.forward(stream=s), c.backward(stream=s)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(p, q) for p, q in zip(outs(c)[2:], w[2:]))
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.forward(), c.backward()
        graphs.append(g)
    for k in range(3):
        for c in cases:
            c.dx_.mul_(-0.5), c.da_.mul_(1.5)
            c.d_ga.fill_(k)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        replayed = [outs(c) for c in cases]
        for c, got in zip(cases, replayed):
            c.forward(), c.backward()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, outs(c)))
