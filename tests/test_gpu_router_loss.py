"""The router's loss and its gradient against float64 (tests/router_loss_ref.py)."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe, synth
from tests import router_loss_ref as ref
from tests.gpu_common import log, torch_cuda

pytestmark = pytest.mark.gpu

# A probability in fp32: the argument of exp2 is off by 2^-24 of up to 60 (the logits' spread here), the two
# exponentials, the reciprocal and the quotient by 2^-22 together, the row's sum by one rounding for each of at most
# 16 values a lane and 6 exchanges; a mean adds at most 64 roundings (tokens of a wave, blocks of a sequence).  160
# roundings of 2^-24 are 1e-5.
REL = 160 * 2.0 ** -24


class Case:
    def __init__(self, torch, T, E, k, offsets=None, mask=None, dtype="f32", seed=0, bias=1.0, edit=None, ld=None, shift=0):
        rng = np.random.default_rng([T, E, k, seed])
        l = rng.standard_normal((T, E)) * 1.5 + bias * rng.standard_normal(E)
        ids = np.argsort(-l, axis=1, kind="stable")[:, :k].astype(np.int32)
        self.dw = (rng.standard_normal((T, k)) * 1e-2).astype(np.float32)
        w = np.exp(rng.standard_normal((T, k)))
        self.w = (w / w.sum(axis=1, keepdims=True)).astype(np.float32)
        if edit:
            edit(l, ids)
        self.T, self.E, self.k, self.ids = T, E, k, ids
        self.off, self.mask = offsets, mask
        self.S = 1 if offsets is None else len(offsets) - 1
        self.ld = ld or E
        t = torch.from_numpy(np.ascontiguousarray(l, np.float32))
        t = t.to(torch.bfloat16) if dtype == "bf16" else t
        self.l = t.double().numpy()
        self.shift = shift
        buf = torch.full((T * self.ld + shift + 8,), float("nan"), dtype=t.dtype, device="cuda")
        self.logits = buf[shift:]
        self.logits[: T * self.ld].view(T, self.ld)[:, :E] = t.cuda()
        cu = lambda a, d: None if a is None else torch.from_numpy(np.ascontiguousarray(a, d)).cuda()
        self.d_ids, self.d_w, self.d_dw = cu(ids, np.int32), cu(self.w, np.float32), cu(self.dw, np.float32)
        self.d_mask, self.d_off = cu(mask, np.uint8), cu(offsets, np.int32)
        self.counts = torch.full((self.S, E), -7, dtype=torch.int32, device="cuda")
        self.probs = torch.full((self.S, E), 7.0, device="cuda")
        self.tokens = torch.full((self.S + 2,), -7, dtype=torch.int32, device="cuda")
        self.loss = torch.full((3,), 7.0, device="cuda")
        self.ws = torch.full((damoe.router_loss_workspace_size(T, E, self.S),), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws[:4] = 0  # the error word

    def forward(self, score, alpha, zc, stream=None):
        damoe.router_loss(self.logits, self.d_ids, self.T, self.E, self.k, self.loss, self.counts, self.tokens, self.ws,
                          mask=self.d_mask, seq_offsets=self.d_off, S=self.S, score=score, alpha=alpha, z_coef=zc,
                          probs=self.probs, ld=self.ld, stream=stream)

    def backward(self, out, score, alpha, zc, dloss=None, gates=True, ldd=None, stream=None):
        damoe.router_loss_grad(self.logits, self.d_ids, self.T, self.E, self.k, self.counts, self.tokens, out,
                               mask=self.d_mask, seq_offsets=self.d_off, S=self.S, score=score, alpha=alpha, z_coef=zc,
                               dloss=dloss, w=self.d_w if gates else None, dw=self.d_dw if gates else None, ld=self.ld,
                               ldd=ldd or self.E, stream=stream)

    def check(self, torch, score, alpha=0.7, zc=0.02, g=1.5):
        want, counts, probs, tokens = ref.loss(self.l, self.ids, self.k, self.mask, self.off, score, alpha, zc)
        self.forward(score, alpha, zc)
        assert np.array_equal(self.counts.cpu().numpy(), counts)
        assert np.array_equal(self.tokens.cpu().numpy(), tokens)
        np.testing.assert_allclose(self.probs.double().cpu().numpy(), probs, rtol=REL, atol=1e-30)
        # A small lse is the difference of larger terms: off by 2^-22 of them.
        z_abs = 2.0 ** -20 * (1 + min(want[2], 1e30))
        with np.errstate(over="ignore"):
            want = want.astype(np.float32).astype(np.float64)  # a z past fp32 is infinite
        np.testing.assert_allclose(self.loss.double().cpu().numpy(), want, rtol=REL, atol=z_abs)
        dloss = torch.full((1,), g, device="cuda")
        out = torch.full((self.T, self.E), 7.0, dtype=self.logits.dtype, device="cuda")
        self.backward(out, score, alpha, zc, dloss)
        d, mag = ref.grad(self.l, self.ids, self.k, self.mask, self.off, score, alpha, zc, counts, g,
                          self.w.astype(np.float64), self.dw.astype(np.float64))
        tol = 2 * REL * mag + 1e-30
        if self.logits.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(d) + tol)  # one rounding
        got = out.double().cpu().numpy()
        bad = ~(np.abs(got - d) <= tol)
        assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], d[bad][:4])


SHAPES = [(1, 8, 8), (1, 1, 1), (3, 37, 5), (16, 64, 2), (17, 100, 16), (64, 256, 8), (130, 384, 8), (509, 256, 8),
          (70, 512, 4), (33, 1000, 6), (20, 1024, 16), (40, 1023, 3), (9000, 8, 2)]


@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,k", SHAPES)
def test_one_sequence(T, E, k, score):
    torch = torch_cuda()
    for dtype in ("f32", "bf16"):
        log(f"router loss T={T} E={E} k={k} score={score} {dtype}")
        Case(torch, T, E, k, dtype=dtype).check(torch, score)


@pytest.mark.parametrize("offsets,T", [([0, 5, 5, 37, 38, 100], 100), ([0, 0, 0, 64], 64), ([0, 1, 2, 3, 4, 5, 6, 7], 20),
                                       ([0] + list(range(1, 130)), 129), ([0, 17, 300], 517), ([0, 0], 30),
                                       ([0] + [40] * 300 + [50], 60)])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
def test_sequences(offsets, T, score):
    """Ragged sequences, empty ones, tokens behind the last one; padding inside them."""
    torch = torch_cuda()
    log(f"router loss sequences {offsets[:8]} T={T}")
    mask = (np.random.default_rng(T).random(T) < 0.8).astype(np.uint8)
    for m in (None, mask):
        Case(torch, T, 48, 4, offsets=offsets, mask=m).check(torch, score)


def test_many_sequences():
    """Thousands of sequences of 0 to 5 tokens, and a long run of empty ones."""
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    n = rng.integers(0, 6, 5000)
    n[1000:4500] = 0
    off = np.concatenate([[0], np.cumsum(n)]).tolist()
    for score in (0, 1):
        Case(torch, off[-1] + 9, 40, 3, offsets=off, mask=(rng.random(off[-1] + 9) < 0.9).astype(np.uint8)).check(torch, score)
    Case(torch, 50, 16, 2, offsets=[0] + [30] * 5000 + [45]).check(torch, 0)


@pytest.mark.parametrize("T,E,k,lengths,dtype", [
    (40, 64, 8, [1] * 20 + [0, 3, 0, 9], "f32"), (99, 37, 4, [1] * 99, "bf16"), (513, 256, 8, [400] + [1] * 100, "f32"),
    (120, 1000, 6, [4] * 29, "bf16"), (130, 1023, 3, [3, 5] * 16, "f32"), (1030, 384, 8, [0, 0, 7] * 140 + [21], "f32"),
    (4096, 48, 2, [64] * 64, "f32"), (4097, 48, 2, [64] * 64 + [1], "f32"), (5003, 48, 2, [0, 1, 2, 3, 4] * 500, "bf16"),
    (16500, 40, 2, [16] * 1031, "f32")])
def test_short_sequences(T, E, k, lengths, dtype):
    torch = torch_cuda()
    off = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    assert off[-1] <= T
    for score in (0, 1):
        log(f"router loss of {len(lengths)} short sequences T={T} E={E} {dtype} score={score}")
        mask = (np.random.default_rng(T).random(T) < 0.85).astype(np.uint8)
        Case(torch, T, E, k, offsets=off, mask=mask, dtype=dtype).check(torch, score)


def test_many_tokens_ragged():
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    T = 20011
    off = np.concatenate([[0], np.sort(rng.choice(T, 12, replace=False)), [T - 7]])
    off = np.maximum.accumulate(off)
    off[-2] = min(off[-2], off[-1])
    Case(torch, T, 40, 6, offsets=off.tolist(), mask=(rng.random(T) < 0.9).astype(np.uint8)).check(torch, 0)


@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
def test_special_rows(score):
    """Experts switched off, rows of -inf alone, the type's lowest value, huge logits, masked slots, an id held
    twice, and NaN in rows that do not count."""
    torch = torch_cuda()
    T, E, k = 41, 64, 4
    mask = np.ones(T, np.uint8)
    mask[[3, 20]] = 0

    def edit(l, ids):
        l[:, 10:20] = -np.inf
        l[5] = -np.inf
        l[6] = -np.finfo(np.float32).max / 4  # one value throughout: a uniform row
        l[7, 1:] = -np.finfo(np.float32).max  # a single expert is left
        l[8] = 50.0 + np.arange(E) / 8
        l[9] = -95.0 - np.arange(E) / 8       # sigmoids below the normal range
        l[3] = np.nan
        l[20] = np.inf
        ids[11] = -1
        ids[12, 1] = -1
        ids[13, :] = ids[13, 0]               # one expert in every slot
        ids[14, 2] = ids[14, 0]

    c = Case(torch, T, E, k, mask=mask, edit=edit)
    c.check(torch, score, zc=0.0)  # row 6 has a z past fp32: a loss without it
    assert damoe.read_device_error(c.ws) == 0
    # With the z-loss, without the rows whose z is past fp32.
    mask[[6, 7]] = 0
    Case(torch, T, E, k, mask=mask, edit=edit, offsets=[0, 19, 41]).check(torch, score)


def test_nan_in_a_valid_row():
    torch = torch_cuda()

    def edit(l, ids):
        l[2, 5] = np.nan

    c = Case(torch, 40, 32, 2, offsets=[0, 10, 40], edit=edit)
    c.forward(0, 1.0, 0.1)
    assert torch.isnan(c.loss).all()
    assert torch.isnan(c.probs[0]).all() and torch.isfinite(c.probs[1]).all()
    out = torch.zeros((40, 32), device="cuda")
    c.backward(out, 0, 1.0, 0.1)
    rows = torch.isnan(out).any(dim=1).cpu().numpy()
    assert rows[2] and rows.sum() == 1


def test_nan_among_switched_off_experts():
    torch = torch_cuda()

    def edit(l, ids):
        l[7] = -np.inf
        l[7, 3] = np.nan

    c = Case(torch, 200, 32, 2, edit=edit)
    c.forward(0, 1.0, 0.1)
    assert torch.isnan(c.loss).all() and torch.isnan(c.probs).all()
    out = torch.zeros((200, 32), device="cuda")
    c.backward(out, 0, 1.0, 0.1, gates=False)
    assert torch.isnan(out[7]).all() and torch.isfinite(out[:7]).all() and torch.isfinite(out[8:]).all()


def test_nothing_valid():
    torch = torch_cuda()
    for T, mask, off in [(30, np.zeros(30, np.uint8), None), (30, None, [0, 0, 0]), (0, None, None)]:
        c = Case(torch, T, 16, 2, mask=mask, offsets=off)
        c.forward(0, 1.0, 1.0)
        assert c.loss.tolist() == [0, 0, 0] and (c.counts == 0).all() and (c.probs == 0).all() and (c.tokens == 0).all()
        out = torch.full((T, 16), 7.0, device="cuda")
        c.backward(out, 0, 1.0, 1.0)
        assert (out == 0).all()


def test_invalid_ids_are_flagged():
    torch = torch_cuda()

    def edit(l, ids):
        ids[4, 1] = 32
        ids[9, 0] = 2 ** 31 - 1
        ids[10, 0] = -2 ** 31

    c = Case(torch, 20, 32, 3, edit=edit)
    c.check(torch, 0)
    assert damoe.read_device_error(c.ws) == damoe.DEVERR_EXPERT_ID
    assert damoe.read_device_error(c.ws) == 0


@pytest.mark.parametrize("E,ld,shift", [(64, 64, 1), (64, 67, 0), (64, 68, 0), (63, 80, 2), (384, 386, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(E, ld, shift, dtype):
    torch = torch_cuda()
    T, k = 50, 4
    c = Case(torch, T, E, k, ld=ld, shift=shift, dtype=dtype)
    c.check(torch, 0)
    # The gradient into rows of its own stride leaves what lies between them alone.
    want = torch.zeros((T, E), dtype=c.logits.dtype, device="cuda")
    c.backward(want, 0, 0.7, 0.02)
    buf = torch.full((T * (E + 5) + 4,), 7.0, dtype=c.logits.dtype, device="cuda")
    c.backward(buf[shift:], 0, 0.7, 0.02, ldd=E + 5)
    view = buf[shift: shift + T * (E + 5)].view(T, E + 5)
    d, mag = ref.grad(c.l, c.ids, k, None, None, 0, 0.7, 0.02, c.counts.cpu().numpy(), 1.0, c.w.astype(np.float64),
                      c.dw.astype(np.float64))
    tol = 2 * REL * mag + 1e-30
    tol = tol + (2.0 ** -8 * (np.abs(d) + tol) if dtype == "bf16" else 0.0)
    assert (np.abs(view[:, :E].double().cpu().numpy() - d) <= tol).all()
    assert (view[:-1, E:] == 7.0).all() and (buf[:shift] == 7.0).all()
    # In place.
    c.backward(c.logits, 0, 0.7, 0.02, ldd=ld)
    assert (np.abs(c.logits[: T * ld].view(T, ld)[:, :E].double().cpu().numpy() - d) <= tol).all()
    assert (np.abs(want.double().cpu().numpy() - d) <= tol).all()


def test_largest_batch():
    """2^20 tokens of 1024 experts: rows past every 32-bit offset, and every output of the forward call but probs."""
    torch = torch_cuda()
    T, E, k = 1 << 20, 1024, 16
    base = Case(torch, 64, E, k, seed=3)
    rep = T // 64
    logits = base.logits[: 64 * E].view(64, E).repeat(rep, 1)
    ids, w, dw = base.d_ids.repeat(rep, 1), base.d_w.repeat(rep, 1), base.d_dw.repeat(rep, 1)
    ws = torch.zeros(damoe.router_loss_workspace_size(T, E), dtype=torch.uint8, device="cuda")
    counts, tokens = torch.zeros((1, E), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    loss = torch.zeros(3, device="cuda")
    damoe.router_loss(logits, ids, T, E, k, loss, counts, tokens, ws, alpha=1.0, z_coef=1.0)
    want, c, _, _ = ref.loss(base.l, base.ids, k, None, None, 0, 1.0, 1.0)
    assert np.array_equal(counts.cpu().numpy(), c * rep) and tokens.tolist() == [T, 1, T]
    # 2048 tokens a block, 256 a wave, and 512 blocks: up to 300 roundings more than REL counts.
    np.testing.assert_allclose(loss.double().cpu().numpy(), want, rtol=REL + 300 * 2.0 ** -24)
    damoe.router_loss_grad(logits, ids, T, E, k, counts, tokens, logits, alpha=1.0, z_coef=1.0, w=w, dw=dw)  # in place
    d, mag = ref.grad(base.l, base.ids, k, None, None, 0, 0.0, 0.0, c, 1.0, base.w.astype(np.float64), base.dw.astype(np.float64))
    # The loss's share of a row's gradient is 1 / T of what it is for 64 tokens.
    d2, mag2 = ref.grad(base.l, base.ids, k, None, None, 0, 1.0, 1.0, c, 1.0 / rep)
    for t0 in (0, T // 2, T - 64):
        got = logits[t0: t0 + 64].double().cpu().numpy()
        assert (np.abs(got - d - d2) <= 2 * REL * (mag + mag2) + 1e-30).all(), t0


def test_two_batches_at_once():
    torch = torch_cuda()
    cs = [Case(torch, T, 64, 4, offsets=off, seed=9) for T, off in ((50, None), (3000, [0, 700, 701, 2990]))]
    want, outs = [], []
    for c in cs:
        c.forward(1, 0.5, 0.1)
        o = torch.zeros((c.T, 64), device="cuda")
        c.backward(o, 1, 0.5, 0.1)
        want.append((c.loss.clone(), c.counts.clone(), c.probs.clone(), o))
        outs.append(torch.zeros_like(o))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for c, s, o in zip(cs, streams, outs):
            c.forward(1, 0.5, 0.1, s)
            c.backward(o, 1, 0.5, 0.1, stream=s)
    torch.cuda.synchronize()
    for c, w, o in zip(cs, want, outs):
        assert all(torch.equal(a, b) for a, b in zip(w, (c.loss, c.counts, c.probs, o)))


def test_gates_alone_and_loss_alone():
    torch = torch_cuda()
    c = Case(torch, 60, 48, 5)
    c.forward(0, 0.0, 0.0)
    assert c.loss[0].item() == 0.0 and c.loss[1].item() > 0 and c.loss[2].item() > 0
    out = torch.zeros((60, 48), device="cuda")
    c.backward(out, 0, 0.0, 0.0)
    d, mag = ref.grad(c.l, c.ids, c.k, None, None, 0, 0.0, 0.0, c.counts.cpu().numpy(), 1.0, c.w.astype(np.float64),
                      c.dw.astype(np.float64))
    assert (np.abs(out.double().cpu().numpy() - d) <= 2 * REL * mag).all()
    c.backward(out, 1, 0.7, 0.02, gates=False)
    d, mag = ref.grad(c.l, c.ids, c.k, None, None, 1, 0.7, 0.02, c.counts.cpu().numpy(), 1.0)
    assert (np.abs(out.double().cpu().numpy() - d) <= 2 * REL * mag).all()


@pytest.mark.parametrize("T", [48, 9000])
def test_repeats_streams_and_graphs(T):
    """Equal bits from call to call, on another stream, and in two captured graphs replayed among eager work."""
    torch = torch_cuda()
    off = [0, T // 3, T - 5]
    cs = [Case(torch, T, 64, 4, offsets=off, seed=s) for s in (1, 2)]
    outs = [torch.zeros((T, 64), device="cuda") for _ in cs]

    def step(c, o, stream=None):
        c.forward(0, 0.5, 0.1, stream)
        c.backward(o, 0, 0.5, 0.1, stream=stream)

    def results(c, o):
        return [t.clone() for t in (c.loss, c.counts, c.probs, c.tokens, o)]

    eager = []
    for c, o in zip(cs, outs):
        step(c, o)
        eager.append(results(c, o))
        step(c, o)
        assert all(torch.equal(a, b) for a, b in zip(eager[-1], results(c, o)))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(cs[0], outs[0], side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager[0], results(cs[0], outs[0])))
    torch.cuda.synchronize()
    graphs = []
    for c, o in zip(cs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(c, o, side)
        graphs.append(g)
    torch.cuda.synchronize()
    kept = [c.logits.clone() for c in cs]
    for rep in range(3):
        for c, o, keep in zip(cs, outs, kept):
            c.logits.copy_(keep.flip(0) if rep == 1 else keep)  # eager work between replays
            for t in (c.loss, c.probs, o):
                t.fill_(float("nan"))
            c.counts.fill_(-1)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        if rep != 1:
            for c, o, e in zip(cs, outs, eager):
                assert all(torch.equal(a, b) for a, b in zip(e, results(c, o))), rep


def test_router_then_loss_then_gradient():
    """As they are used: the router's logits, ids and gates, its loss and gradient, through Path."""
    torch = torch_cuda()
    from paper_2607_23099_amd.moe import DeviceLayer, Gate, Path
    sh = synth.TINY
    T = 77
    path = Path(DeviceLayer(sh), T + 10)
    path.prepare_loss(S=2)
    gate = Gate(sh)
    path.fill_x(T, 5)
    path.router(gate, T)
    off, dw = torch.tensor([0, 30, T], dtype=torch.int32, device="cuda"), torch.randn(T, sh.k, device="cuda")
    path.router_loss(T, 0.01, 0.001, seq_offsets=off)
    path.router_loss_grad(T, 0.01, 0.001, seq_offsets=off, dw=dw)
    l = path.logits[:T].double().cpu().numpy()
    ids, w = path.ids[: T * sh.k].view(T, sh.k).cpu().numpy(), path.w[: T * sh.k].view(T, sh.k).double().cpu().numpy()
    want, counts, probs, tokens = ref.loss(l, ids, sh.k, None, [0, 30, T], 0, 0.01, 0.001)
    np.testing.assert_allclose(path.loss.double().cpu().numpy(), want, rtol=REL, atol=2.0 ** -20 * (1 + want[2]))
    assert np.array_equal(path.loss_counts.cpu().numpy(), counts)
    d, mag = ref.grad(l, ids, sh.k, None, [0, 30, T], 0, 0.01, 0.001, counts, 1.0, w, dw.double().cpu().numpy())
    assert (np.abs(path.dlogits[:T].double().cpu().numpy() - d) <= 2 * REL * mag + 1e-30).all()
    assert (path.dlogits[T:] == 0).all()
    # The routing's own histogram counts the same assignments.
    path.route(T)
    assert np.array_equal(path.counts.cpu().numpy(), counts.sum(axis=0))
