"""The adapters' two launches at sizes that take them: rows that stream (from 4096 on) and rows whose sums are joined.  One launch
leaves the workspace as it is, so each case shows which way it goes."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import rows_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_adapter_paths import TYPES
from tests.test_gpu_adapters import Case
from tests.test_gpu_rows import close

pytestmark = pytest.mark.gpu

# Whole tiles of columns and 8 more (tiles of 128 bf16 or 64 fp32 columns a wave); whole units of 128 columns and 8 more.
STREAM = dict(T=4200, L=3, K=1160, N=648)
JOIN = dict(T=2100, L=3, K=2184, N=648)


def two_launches(c):
    c.ws[0].fill_(0xFF)
    c.forward(y=c.d_y.clone(), u=None)
    wrote = bool((c.ws[0] != 0xFF).any())
    c.ws[0].fill_(0xFF)
    return wrote


def outputs(c):
    return [t.clone() for t in (c.d_y, c.d_u, c.d_dx, c.d_ga, c.d_gb)]


@pytest.mark.parametrize("r", [4, 8, 12, 16, 24, 32])
@pytest.mark.parametrize("x,w,y", TYPES)
def test_rows_that_stream(r, x, w, y):
    torch = torch_cuda()
    log(f"r={r} x={x} w={w} y={y}")
    c = Case(torch, r=r, x=x, w=w, y=y, free=5, **STREAM)
    assert two_launches(c)
    c.check()


@pytest.mark.parametrize("r", [6, 8, 16, 24, 64, 128])
@pytest.mark.parametrize("x,w,y", TYPES[:5])
def test_rows_whose_sums_are_joined(r, x, w, y):
    torch = torch_cuda()
    log(f"r={r} x={x} w={w} y={y}")
    c = Case(torch, r=r, x=x, w=w, y=y, free=5, **JOIN)
    assert two_launches(c)
    c.check()


@pytest.mark.parametrize("kw", [dict(ld=3, shift=1), dict(ld=5, shift=3, mixed=False, free=40), dict(scale=False, add=False),
                                dict(bounds=[0, 1, 2050, 2050, 4200]), dict(bounds=[0, 128, 256, 4199, 4199]), dict(free=4200),
                                dict(bounds=[0, 5, 20, 37, 4100])], ids=str)
@pytest.mark.parametrize("x,w,r", [("bf16", "bf16", 10), ("f32", "f32", 5), ("bf16", "f32", 8), ("bf16", "bf16", 32)])
def test_strides_alignment_and_segments_of_rows_that_stream(kw, x, w, r):
    torch = torch_cuda()
    log(f"{kw} {x} {w} r={r}")
    c = Case(torch, **{**STREAM, "L": 4}, r=r, x=x, w=w, y=x, **kw)
    assert two_launches(c) or kw.get("free") == 4200
    c.check()


@pytest.mark.parametrize("sizes", [STREAM, JOIN], ids=["streamed", "joined"])
@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_values_that_are_not_finite(sizes, x, w):
    """Of their own segment, or of their own row, alone."""
    torch = torch_cuda()
    T, n = sizes["T"], sizes["T"] // 4
    c = Case(torch, **{**sizes, "L": 4}, r=8, x=x, w=w, y=x, bounds=[0, n, n + 1, 3 * n, T - 100], add=False)
    assert two_launches(c)
    c.forward(), c.backward()
    good = outputs(c)
    rows = lambda l: torch.from_numpy(c.perm[c.off[l]: c.off[l + 1]]).long().cuda()
    c.da_[0, 3, 5], c.dx_[int(rows(2)[70]), 11] = float("nan"), float("inf")
    c.da_[1, 2, 7], c.db_[2, 640, 3] = float("inf"), float("nan")
    free = torch.from_numpy(c.perm[T - 100:]).long().cuda()
    c.dx_[free], c.d_dy[free] = float("nan"), float("inf")
    c.forward()
    assert c.d_y[rows(0)].isnan().all() and c.d_u[:n, 3].isnan().all()
    assert c.d_u[n, 2].isinf() and torch.equal(c.d_u[n, 3:], good[1][n, 3:])
    assert c.d_y[rows(2), 640].isnan().all()
    keep = torch.ones(c.d_y.shape, dtype=torch.bool, device="cuda")
    keep[rows(0)] = keep[rows(1)] = keep[rows(2)[70]] = False
    keep[rows(2), 640] = False
    assert torch.equal(c.d_y[keep], good[0][keep])
    assert not c.d_y[rows(2)[70]].isfinite().any()


def test_entries_out_of_range():
    """perm's outside the rows leave their places out; offsets are cut at T; what decreasing ones give stays within the buffers."""
    torch = torch_cuda()
    for sizes in (STREAM, JOIN):
        T = sizes["T"]
        for bad in (-1, T, 1 << 30, -(1 << 31)):
            c = Case(torch, **sizes, r=16, free=10)
            assert two_launches(c)
            for p in (0, 17, 140, T - 11):
                c.perm[p] = bad
            c.d_perm.copy_(torch.from_numpy(c.perm))
            c.forward(u=None)
            y, ey, _, _ = ref.adapters(c.vx, c.va, c.vb, c.off, c.perm, c.scale, c.vadd, c.vy0)
            close(c.d_y, y, ey, "bf16", "y")
        c = Case(torch, **sizes, r=16, mixed=False)
        c.forward()
        y = c.d_y.clone()
        c.d_off[-1] += 100000
        c.d_y.zero_()
        c.forward()
        assert torch.equal(c.d_y, y)
        size = c.ws[0].numel()
        c.ws[0] = torch.full((size + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
        c.d_off.copy_(torch.tensor([0, T, 0, T], dtype=torch.int32))
        c.forward()
        assert (c.ws[0][size:] == 0xA5).all()


@pytest.mark.parametrize("sizes,r", [(STREAM, 4), (STREAM, 16), (STREAM, 32), (JOIN, 8), (JOIN, 16), (JOIN, 24)])
def test_graphs_replayed_between_eager_calls(sizes, r):
    torch = torch_cuda()
    log(f"{sizes} r={r}")
    c, other = (Case(torch, **sizes, r=r, seed=s) for s in (1, 2))
    assert two_launches(c)
    c.forward(), c.backward()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward(), c.backward()
    for k in range(4):
        c.dx_.mul_(-0.5), c.d_ga.fill_(k), c.d_gb.fill_(k), c.d_y.fill_(k), c.d_u.fill_(k)
        g.replay()
        other.forward(), other.backward()
        got = outputs(c)
        torch.cuda.synchronize()
        c.d_y.fill_(k + 9), c.d_u.fill_(k + 9)
        c.forward(), c.backward()
        assert all(torch.equal(p, q) for p, q in zip(got, outputs(c))), k


@pytest.mark.parametrize("sizes,r", [(dict(T=800, L=5, K=520, N=264), 16), (STREAM, 8), (STREAM, 32), (JOIN, 16)])
def test_calls_at_once_on_two_streams(sizes, r):
    """With workspaces of their own; every output is another value before each round."""
    torch = torch_cuda()
    log(f"{sizes} r={r}")
    cases = [Case(torch, **sizes, r=r, seed=s) for s in range(2)]  # a random order of all rows: no row is left out
    for c in cases:
        c.forward(), c.backward()
    want = [outputs(c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for k in range(3):
        for c in cases:
            for t in (c.d_y, c.d_u, c.d_dx, c.d_ga, c.d_gb):
                t.fill_(k + 11)
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(2):
            for c, s in zip(cases, streams):
                c.forward(stream=s)
            for c, s in zip(cases, streams):
                c.backward(stream=s)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(p, q) for p, q in zip(outputs(c), w)), k


@pytest.mark.parametrize("ends", [[0, 0, 0, 0], [0, 3, 3, 9]], ids=["none", "stale"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_without_rows(ends, dtype):
    """da and db are 0, or with accumulate what they were, whatever the offsets hold."""
    torch = torch_cuda()
    L, r, K, N = 3, 5, 700, 33
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    new = lambda *s: torch.ones(*s, dtype=t, device="cuda")
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for ws in (0, damoe.adapters_grad_workspace_size(0, L, r, K, N)):
        da, db = torch.full((L, r, K), 3.0, device="cuda"), torch.full((L, N, r), float("nan"), device="cuda")
        call = lambda **kw: damoe.adapters_grad(new(0, K), new(0, N), torch.empty(0, r, device="cuda"), 0, new(L, r, K), new(L, N, r), off, da, db,
                                                torch.empty(ws, dtype=torch.uint8, device="cuda"), dx=new(0, K), **kw)
        call()
        assert not da.any() and not db.any()
        da.fill_(3), db.fill_(5)
        call(accumulate=True)
        assert (da == 3).all() and (db == 5).all()
        call(perm=torch.empty(0, dtype=torch.int32, device="cuda"), add=new(0, K))
        assert not da.any() and not db.any()
