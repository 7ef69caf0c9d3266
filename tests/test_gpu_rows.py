"""Rows sorted by expert and back, and the gradient, against float64 (tests/rows_ref.py)."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import rows_ref as ref
from tests.gpu_common import log, torch_cuda

pytestmark = pytest.mark.gpu


def matrix(torch, v, dtype, ld=0, shift=0):
    """Device matrix of the values rounded to the type, with rows `ld` apart (0: side by side), `shift` elements from a 16-byte
    boundary, NaN between its rows; and its values in float64."""
    t = torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    r, c = t.shape
    buf = torch.full((max(r, 1) * max(ld, c) + shift,), float("nan"), dtype=t.dtype, device="cuda")
    m = buf[shift:].view(max(r, 1), -1)[:r, :c]
    m.copy_(t)
    return m, t.double().numpy()


def close(got, want, err, dtype, what):
    got = got.double().cpu().numpy()
    bound = ref.rounded(want, err, dtype) if dtype else err
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], bound[bad][:4])


class Batch:
    """T tokens of k slots over a matrix of R rows: `drop` of the slots have none, the token `bare` not one."""

    def __init__(self, torch, T, k, H, dtype, R=None, drop=0.0, ld=0, shift=0, seed=0, cut=None):
        rng = np.random.default_rng([T, k, H, seed])
        self.torch, self.T, self.k, self.H, self.dtype = torch, T, k, H, dtype
        self.R = T * k if R is None else R
        self.rng, self.ld, self.shift = rng, ld, shift
        q = rng.permutation(max(self.R, T * k))[: T * k]
        if cut is None:
            q = np.where(q < self.R, q, -1)
        q[rng.random(T * k) < drop] = -1
        if T > 2 and drop:
            q.reshape(T, k)[1] = -1
        self.inv = q.astype(np.int32)
        self.d_inv = torch.from_numpy(self.inv).cuda()
        self.w = rng.standard_normal((T, k)).astype(np.float32)
        self.d_w = torch.from_numpy(self.w).cuda()

    def new(self, rows):
        return matrix(self.torch, self.rng.standard_normal((rows, self.H)), self.dtype, self.ld, self.shift)

    def check(self, weighted=True):
        torch, T, k, H, R = self.torch, self.T, self.k, self.H, self.R
        w, d_w = (self.w, self.d_w) if weighted else (None, None)
        x, vx = self.new(T)
        out, before = self.new(R)
        damoe.sort_rows(x, T, k, H, self.d_inv, out, w=d_w)
        close(out, *ref.sort_rows(vx, self.inv, k, R, before, w), self.dtype if weighted else None, "sort")
        rows, vr = self.new(R)
        untouched = np.setdiff1d(np.arange(R), self.inv)
        rows[torch.from_numpy(untouched).cuda()] = float("nan")  # rows that no slot has are not read
        for add in (False, True):
            base, vb = self.new(T)
            y, _ = self.new(T)
            damoe.combine_rows(rows, T, k, H, self.d_inv, y, w=d_w, add=base if add else None)
            want, err = ref.combine_rows(vr, self.inv, T, k, w, vb if add else None)
            close(y, want, err, self.dtype, "combine")
            if add:
                damoe.combine_rows(rows, T, k, H, self.d_inv, base, w=d_w, add=base)
                assert torch.equal(base, y)
        dy, vd = self.new(T)
        drows, before = self.new(R)
        dw = torch.full((T, k), 7.0, device="cuda")
        damoe.combine_rows_grad(dy, rows, T, k, H, self.d_inv, w=d_w, drows=drows, dw=dw)
        want, err, want_w, err_w = ref.combine_rows_grad(vd, vr, self.inv, k, before, w)
        close(drows, want, err, self.dtype if weighted else None, "drows")
        close(dw, want_w, err_w, "f32", "dw")
        # One output alone, and in the rows' own place.
        dw2 = torch.full((T, k), 7.0, device="cuda")
        damoe.combine_rows_grad(dy, rows, T, k, H, self.d_inv, w=d_w, dw=dw2)
        assert torch.equal(dw, dw2)
        alone, _ = matrix(torch, before, self.dtype, self.ld, self.shift)
        damoe.combine_rows_grad(dy, None, T, k, H, self.d_inv, w=d_w, drows=alone)
        assert torch.equal(alone, drows)
        damoe.combine_rows_grad(dy, rows, T, k, H, self.d_inv, w=d_w, drows=rows, dw=dw2)
        touched = torch.from_numpy(self.inv[self.inv >= 0]).long().cuda()
        touched = touched[touched < R]
        assert torch.equal(rows[touched], drows[touched]) and torch.equal(dw, dw2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,H", [(1, 1, 1), (1, 8, 7168), (3, 2, 63), (5, 16, 2047), (9, 3, 2049), (37, 8, 520), (2, 4, 8192),
                                   (1030, 8, 264), (1025, 5, 7)])
def test_sizes(T, k, H, dtype):
    torch = torch_cuda()
    log(f"T={T} k={k} H={H} {dtype}")
    b = Batch(torch, T, k, H, dtype)
    b.check()
    b.check(weighted=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(drop=0.4), dict(drop=1.0), dict(R=20, drop=0.1), dict(R=20, cut=True), dict(R=500),
                                dict(ld=301, drop=0.2), dict(shift=1), dict(ld=293, shift=3, drop=0.5)], ids=str)
def test_masked_slots_capacity_strides_and_alignment(kw, dtype):
    torch = torch_cuda()
    log(f"{kw} {dtype}")
    b = Batch(torch, 13, 4, 292, dtype, **kw)
    b.check()
    b.check(weighted=False)


def test_no_tokens_and_no_rows():
    torch = torch_cuda()
    x, rows = torch.ones(0, 8, device="cuda"), torch.ones(0, 8, device="cuda")
    inv, dw = torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(3, 2, device="cuda")
    damoe.sort_rows(x, 0, 2, 8, inv, torch.ones(4, 8, device="cuda"))
    damoe.combine_rows(rows, 0, 2, 8, inv, x)
    damoe.combine_rows_grad(x, rows, 0, 2, 8, inv, drows=rows, dw=dw)
    # Tokens all of whose slots lie elsewhere, and a matrix without rows.
    inv = torch.tensor([-1, 0, 1, -1, 5, 2], dtype=torch.int32, device="cuda")
    x = torch.ones(3, 8, device="cuda")
    y, add = torch.full((3, 8), 7.0, device="cuda"), torch.rand(3, 8, device="cuda")
    damoe.sort_rows(x, 3, 2, 8, inv, rows)
    damoe.combine_rows(rows, 3, 2, 8, inv, y, add=add)
    assert torch.equal(y, add)
    damoe.combine_rows(rows, 3, 2, 8, inv, y)
    assert not y.any()
    damoe.combine_rows_grad(x, rows, 3, 2, 8, inv, drows=rows, dw=dw)
    assert not dw.any()


def test_values_that_are_not_finite():
    """They stay in their own tokens and columns; a NaN of any bits stays one in bf16."""
    torch = torch_cuda()
    T, k, H = 4, 2, 40
    inv = torch.arange(T * k, dtype=torch.int32, device="cuda")
    for t in (torch.bfloat16, torch.float32):
        rows = torch.ones(T * k, H, device="cuda", dtype=t)
        rows[2, 3], rows[5, 7] = float("inf"), float("nan")
        if t == torch.float32:
            rows.view(torch.int32)[0, 1] = 0x7FFFFFFF
        y = torch.empty(T, H, device="cuda", dtype=t)
        damoe.combine_rows(rows, T, k, H, inv, y)
        assert y[1, 3] == float("inf") and y[2, 7].isnan()
        y[1, 3] = y[2, 7] = 2
        if t == torch.float32:
            assert y[0, 1].isnan()
            y[0, 1] = 2
        assert (y == 2).all()
    x = torch.ones(2, H, device="cuda", dtype=torch.bfloat16)
    x.view(torch.int16)[0, 5], x[1, 6] = 0x7F81, float("-inf")
    out = torch.empty(2, H, device="cuda", dtype=torch.bfloat16)
    damoe.sort_rows(x, 2, 1, H, inv, out, w=torch.tensor([[2.0], [0.5]], device="cuda"))
    assert out[0, 5].isnan() and out[1, 6] == float("-inf") and int((~out.isfinite()).sum()) == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_past_32_bit_offsets(dtype):
    torch = torch_cuda()
    H = 8192
    R = (1 << 32) // H + 70000
    big = torch.empty(R, H, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    inv = torch.tensor([R - 1, 1, (1 << 32) // H + 5, 0], dtype=torch.int32, device="cuda")
    x = torch.randn(2, H, device="cuda").to(big.dtype)
    w = torch.tensor([[1.0, 2.0], [4.0, 0.5]], device="cuda")  # exact factors
    for low in (0, 1, 5, 69999):
        big[low] = 7
    damoe.sort_rows(x, 2, 2, H, inv, big, w=w)
    for t, j in np.ndindex(2, 2):
        assert torch.equal(big[int(inv[2 * t + j])], x[t] * float(w[t, j]))
    assert (big[5] == 7).all() and (big[69999] == 7).all()
    y = torch.empty_like(x)
    damoe.combine_rows(big, 2, 2, H, inv, y)
    want = (x.float() * w.sum(dim=1, keepdim=True)).to(x.dtype)
    assert torch.equal(y, want) or float((y.double() - want.double()).abs().max()) <= 2.0 ** -8 * float(want.abs().max())
    dw = torch.empty(2, 2, device="cuda")
    damoe.combine_rows_grad(x, big, 2, 2, H, inv, drows=big, dw=dw)
    for t, j in np.ndindex(2, 2):
        assert torch.equal(big[int(inv[2 * t + j])], x[t])
    n = (x.double() ** 2).sum(dim=1, keepdim=True).cpu()
    assert ((dw.double().cpu() - n * w.double().cpu()).abs() <= (H + 1) * ref.STEP * n * w.double().cpu()).all()
    assert (big[5] == 7).all() and (big[69999] == 7).all()


def test_equal_bits_on_another_stream_and_in_a_replayed_graph():
    torch = torch_cuda()
    T, k, H = 700, 6, 777
    b = Batch(torch, T, k, H, "bf16", drop=0.2)
    x, rows, dy = (b.new(n)[0] for n in (T, b.R, T))
    out = [torch.zeros(b.R, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, H, dtype=torch.bfloat16, device="cuda"),
           torch.zeros(b.R, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, device="cuda")]

    def calls(out, stream=None):
        damoe.sort_rows(x, T, k, H, b.d_inv, out[0], w=b.d_w, stream=stream)
        damoe.combine_rows(rows, T, k, H, b.d_inv, out[1], w=b.d_w, add=dy, stream=stream)
        damoe.combine_rows_grad(dy, rows, T, k, H, b.d_inv, w=b.d_w, drows=out[2], dw=out[3], stream=stream)

    calls(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = [torch.zeros_like(t) for t in out]
    side.wait_stream(torch.cuda.current_stream())
    calls(other, side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, other))
    replayed = [torch.zeros_like(t) for t in out]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(replayed)
    for _ in range(3):
        x.mul_(0.5), rows.add_(1), dy.neg_()
        for t in replayed:
            t.zero_()
        g.replay()
        for t in out:
            t.zero_()
        calls(out)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, replayed))


@pytest.mark.parametrize("T,k,H", [(1 << 20, 16, 1), (1 << 20, 1, 24), (1, 16, 1 << 20), (65536, 8, 40)])
def test_the_most_tokens_and_the_longest_rows(T, k, H):
    """Against torch: with gates of powers of two, and values of a few bits, every sum is exact."""
    torch = torch_cuda()
    log(f"T={T} k={k} H={H}")
    g = torch.Generator(device="cuda").manual_seed(1)
    R = T * k
    inv = torch.randperm(R, generator=g, device="cuda").to(torch.int32)
    inv[torch.rand(R, generator=g, device="cuda") < 0.1] = -1
    small = lambda *s: torch.randint(-4, 5, s, generator=g, device="cuda").bfloat16()
    x, rows, add = small(T, H), small(R, H), small(T, H)
    w = 2.0 ** torch.randint(-2, 3, (T, k), generator=g, device="cuda").float()
    ok = inv >= 0
    token, place = torch.arange(R, device="cuda") // k, inv.long()
    want = torch.zeros(R, H, device="cuda")
    want[place[ok]] = w.view(-1)[ok][:, None] * x[token[ok]].float()
    out = torch.zeros(R, H, dtype=torch.bfloat16, device="cuda")
    damoe.sort_rows(x, T, k, H, inv, out, w=w)
    assert torch.equal(out.float(), want)
    taken = torch.where(ok[:, None], rows[place.clamp_min(0)].float(), 0).view(T, k, H)
    y = torch.empty_like(x)
    damoe.combine_rows(rows, T, k, H, inv, y, w=w, add=add)
    total = add.float()
    for j in range(k):
        total = total + w[:, j, None] * taken[:, j]
    assert torch.equal(y, total.bfloat16())
    dw, out2 = torch.empty(T, k, device="cuda"), torch.zeros_like(out)
    damoe.combine_rows_grad(x, rows, T, k, H, inv, w=w, drows=out2, dw=dw)
    assert torch.equal(out2, out)
    for j in range(k):
        assert torch.equal(dw[:, j], (x.float() * taken[:, j]).sum(dim=1))
