"""What the binding of the MXFP4 calls and the router's loss refuses (no GPU: every call ends before the library's)."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2607_23099_amd import build, damoe
from paper_2607_23099_amd.moe import MxLinear, Path


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(damoe.LIB_PATH):
        build.build_damoe()


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _bytes(n):
    return torch.zeros(n, dtype=torch.uint8)


class Batch:
    """A routed batch's tensors, good ones, any of which a call may replace."""
    T, E, k, S = 8, 64, 4, 2

    def __init__(self):
        T, E, k, S = self.T, self.E, self.k, self.S
        self.t = dict(logits=torch.zeros(T, E), ids=_i32(T, k), loss=torch.zeros(3), counts=_i32(S, E), tokens=_i32(S + 2),
                      ws=_bytes(damoe.router_loss_workspace_size(T, E, S)), mask=torch.ones(T, dtype=torch.uint8),
                      seq_offsets=_i32(S + 1), probs=torch.zeros(S, E), dlogits=torch.zeros(T, E), w=torch.zeros(T, k),
                      dw=torch.zeros(T, k), dloss=torch.zeros(1))

    def forward(self, **kw):
        t = {**self.t, **kw}
        damoe.router_loss(t["logits"], t["ids"], self.T, self.E, self.k, t["loss"], t["counts"], t["tokens"], t["ws"],
                          mask=t["mask"], seq_offsets=t["seq_offsets"], S=self.S, probs=t["probs"], alpha=1.0, stream=0)

    def backward(self, **kw):
        t = {**self.t, **kw}
        damoe.router_loss_grad(t["logits"], t["ids"], self.T, self.E, self.k, t["counts"], t["tokens"], t["dlogits"],
                               mask=t["mask"], seq_offsets=t["seq_offsets"], S=self.S, dloss=t["dloss"], w=t["w"],
                               dw=t["dw"], alpha=1.0, stream=0)


def test_offsets_of_another_number_of_sequences():
    b = Batch()
    for call in (b.forward, b.backward):
        for n in (2, 4, 40):
            with pytest.raises(ValueError, match="seq_offsets"):
                call(seq_offsets=_i32(n))
    # Through the buffers' object: three sequences in buffers made for two.
    path = Path.__new__(Path)
    path.dl = type("Layer", (), {"shape": type("Shape", (), {"E": b.E, "k": b.k})})
    path.loss_S, path.T_max, path.logits, path.ids, path.w = 2, b.T, b.t["logits"], b.t["ids"], b.t["w"]
    path.loss, path.loss_counts, path.loss_tokens, path.loss_ws = (b.t[n] for n in ("loss", "counts", "tokens", "ws"))
    path.loss_probs, path.dlogits = b.t["probs"], b.t["dlogits"]
    for call in (path.router_loss, path.router_loss_grad):
        with pytest.raises(ValueError, match="seq_offsets"):
            call(b.T, 0.1, seq_offsets=torch.tensor([0, 2, 5, 8], dtype=torch.int32), stream=0)


@pytest.mark.parametrize("name", ["counts", "tokens", "loss", "probs"])
def test_outputs_and_counts_of_another_type_or_size(name):
    b = Batch()
    t = b.t[name]
    bad = [t.to(torch.int64), t.double(), t.to(torch.float32 if t.dtype == torch.int32 else torch.int32), t.reshape(-1)[:-1],
           torch.zeros(2 * t.numel(), dtype=t.dtype)[::2], torch.zeros(1, dtype=t.dtype).expand(t.numel())]
    for v in bad:
        with pytest.raises(ValueError, match=name):
            b.forward(**{name: v})
        if name in ("counts", "tokens"):  # what torch's own counting gives is int64
            with pytest.raises(ValueError, match=name):
                b.backward(**{name: v})


def _wider(t):
    """The tensor's rows a column too short, a row too few, side by side in no matrix, and expanded."""
    r, c = t.shape
    flat = torch.zeros(r * c - 1, dtype=t.dtype)
    return [t[:, :-1], t[:-1], t.new_zeros(r, 2 * c)[:, ::2], flat, t.new_zeros(c, r).t(), t.new_zeros(r, c - 1)]


def test_matrices_that_do_not_hold_the_rows():
    b = Batch()
    for name, calls in [("logits", (b.forward, b.backward)), ("dlogits", (b.backward,))]:
        for v in _wider(b.t[name]):
            for call in calls:
                with pytest.raises(ValueError, match=name):
                    call(**{name: v})
    T, N, K = 5, 64, 96
    good = dict(x=torch.zeros(T, K), y=torch.zeros(T, N), add=torch.zeros(T, N))
    tiles, ws = _bytes(damoe.mxfp4_bytes(N, K)), _bytes(damoe.mxfp4_linear_workspace_size(T, N, K))
    for name in good:
        for v in _wider(good[name]):
            t = {**good, name: v}
            with pytest.raises(ValueError, match=f"^{name}:"):
                damoe.mxfp4_linear(t["x"], T, K, tiles, N, t["y"], ws, add=t["add"], stream=0)
        # A stride given with the call: the last row has to end inside.
        ld, cols = 128, good[name].shape[1]
        for flat in (torch.zeros((T - 1) * ld + cols - 1), torch.zeros(T - 1, ld), torch.zeros(T, ld)[:, : cols - 1]):
            t = {**good, name: flat}
            with pytest.raises(ValueError, match=f"^{name}:"):
                damoe.mxfp4_linear(t["x"], T, K, tiles, N, t["y"], ws, add=t["add"], stream=0,
                                   **{{"x": "ldx", "y": "ldy", "add": "ld_add"}[name]: ld})
    codes, scales = _bytes(T * K // 2), _bytes(T * K // 32)
    for v in _wider(good["x"]):
        with pytest.raises(ValueError, match="^x:"):
            damoe.mxfp4_quantise(v, T, K, codes, scales, damoe.LAYOUT_ROWMAJOR, stream=0)
        with pytest.raises(ValueError, match="^x:"):
            damoe.mxfp4_dequantise(codes, scales, T, K, v, damoe.LAYOUT_ROWMAJOR, stream=0)


def test_row_strides_that_the_binding_takes():
    """What holds the rows is taken, whatever its form: the stride that the library is given."""
    x = torch.zeros(6, 40)
    assert damoe._ld("x", x, 6, 40, None) == 40 and damoe._ld("x", x, 5, 32, None) == 40
    assert damoe._ld("x", x[:, 3:35], 6, 32, None) == 40 and damoe._ld("x", x[::2], 3, 40, None) == 80
    assert damoe._ld("x", x[2:3, :32], 1, 32, None) >= 32  # of one row, any
    assert damoe._ld("x", x[:, :1], 6, 1, None) == 40
    assert damoe._ld("x", x.view(-1), 6, 40, None) == 40 and damoe._ld("x", x.view(2, 3, 40), 6, 40, None) == 40
    assert damoe._ld("x", x.view(-1)[3:], 5, 32, 40) == 40 and damoe._ld("x", x[:, 3:35], 6, 32, 40) == 40
    assert damoe._ld("x", x[1:], 5, 40, 40) == 40 and damoe._ld("x", x[:0], 0, 40, None) == 40
    assert damoe._ld("x", x[:0].view(-1), 0, 40, 40) == 40
    assert damoe._ld("x", x[:1].expand(6, 40), 6, 40, None) == 0  # refused by the library: a stride below the columns


def test_buffers_that_do_not_hold_the_codes():
    rows, cols = 48, 384
    x = torch.zeros(rows, cols)
    for layout in (damoe.LAYOUT_ROWMAJOR, damoe.LAYOUT_FRAG16, damoe.LAYOUT_TILE32):
        n, row = damoe.mxfp4_bytes(rows, cols, layout), layout == damoe.LAYOUT_ROWMAJOR
        assert damoe._codes_bytes(rows, cols, layout) == n
        codes, scales = _bytes(n), _bytes(rows * cols // 32) if row else None
        bad = [("codes", codes[:-1], scales), ("codes", _bytes(2 * n)[::2], scales)]
        bad += [("scales", codes, scales[:-1]), ("scales", codes, _bytes(2 * scales.numel())[::2])] if row else []
        for name, c, s in bad:
            with pytest.raises(ValueError, match=f"^{name}:"):
                damoe.mxfp4_quantise(x, rows, cols, c, s, layout, stream=0)
            with pytest.raises(ValueError, match=f"^{name}:"):
                damoe.mxfp4_dequantise(c, s, rows, cols, x, layout, stream=0)
    for r, c in [(1, 32), (33, 288), (31, 256), (32, 257 * 32)]:
        assert damoe._codes_bytes(r, c, damoe.LAYOUT_TILE32) == damoe.mxfp4_bytes(r, c)
    codes, scales, tiles = _bytes(rows * cols // 2), _bytes(rows * cols // 32), _bytes(damoe.mxfp4_bytes(rows, cols))
    for name, a in [("codes", (codes[:-1], scales, tiles)), ("scales", (codes, scales[:-1], tiles)),
                    ("tiles", (codes, scales, tiles[:-1]))]:
        with pytest.raises(ValueError, match=f"^{name}:"):
            damoe.mxfp4_pack(a[0], a[1], rows, cols, a[2], stream=0)
    T = 3
    y, ws = torch.zeros(T, rows), _bytes(damoe.mxfp4_linear_workspace_size(T, rows, cols))
    with pytest.raises(ValueError, match="^w_tiles:"):
        damoe.mxfp4_linear(x, T, cols, tiles[:-1], rows, y, ws, stream=0)
    # A workspace with gaps counts bytes that it has not side by side.
    with pytest.raises(ValueError, match="^ws:"):
        damoe.mxfp4_linear(x, T, cols, tiles, rows, y, _bytes(2 * ws.numel())[::2], stream=0)
    b = Batch()
    with pytest.raises(ValueError, match="^ws:"):
        b.forward(ws=_bytes(2 * b.t["ws"].numel())[::2])


def test_tensors_of_the_host_or_another_device():
    """A kernel would fault on memory that is not the current device's."""
    b = Batch()
    for call in (b.forward, b.backward):
        with pytest.raises(ValueError, match="current device"):
            call()
    T, N, K = 5, 64, 96
    x, y = torch.zeros(T, K), torch.zeros(T, N)
    tiles, ws = _bytes(damoe.mxfp4_bytes(N, K)), _bytes(damoe.mxfp4_linear_workspace_size(T, N, K))
    codes, scales = _bytes(T * K // 2), _bytes(T * K // 32)
    calls = [lambda x=x, rows=T, **kw: damoe.mxfp4_quantise(x, rows, K, codes, scales, damoe.LAYOUT_ROWMAJOR, **kw),
             lambda x=x, rows=T, **kw: damoe.mxfp4_dequantise(codes, scales, rows, K, x, damoe.LAYOUT_ROWMAJOR, **kw),
             lambda x=x, rows=T, **kw: damoe.mxfp4_linear(x, rows, K, tiles, N, y, ws, **kw)]
    for call in calls + [lambda rows=T, **kw: damoe.mxfp4_pack(codes, scales, rows, K, _bytes(4352), **kw)]:
        for kw in (dict(stream=0), {}):
            with pytest.raises(ValueError, match="current device"):
                call(**kw)
        call(rows=0, stream=0)  # without rows, nothing is launched
    for call in calls:
        with pytest.raises(damoe.DamoeError, match="unsupported"):
            call(x=x.half(), stream=0)


@pytest.mark.gpu
def test_one_tensor_of_the_host_among_the_device_s():
    """Refused, whichever it is; the same call without it runs."""
    b = Batch()
    b.t = {n: t.cuda() for n, t in b.t.items()}
    for call, names in [(b.forward, "logits ids loss counts tokens ws mask seq_offsets probs"),
                        (b.backward, "logits ids counts tokens mask seq_offsets dlogits w dw dloss")]:
        call()
        for n in names.split():
            with pytest.raises(ValueError, match="device"):
                call(**{n: b.t[n].cpu()})
    T, N, K = 5, 64, 96
    t = dict(x=torch.zeros(T, K), w=_bytes(damoe.mxfp4_bytes(N, K)), y=torch.zeros(T, N), add=torch.zeros(T, N),
             ws=_bytes(damoe.mxfp4_linear_workspace_size(T, N, K)))
    t = {n: v.cuda() for n, v in t.items()}

    def linear(**kw):
        a = {**t, **kw}
        damoe.mxfp4_linear(a["x"], T, K, a["w"], N, a["y"], a["ws"], add=a["add"])

    linear()
    for n in t:
        with pytest.raises(ValueError, match="device"):
            linear(**{n: t[n].cpu()})
    codes, scales = _bytes(T * K // 2).cuda(), _bytes(T * K // 32).cuda()
    for c, s in [(codes.cpu(), scales), (codes, scales.cpu())]:
        for call in (lambda: damoe.mxfp4_quantise(t["x"], T, K, c, s, damoe.LAYOUT_ROWMAJOR),
                     lambda: damoe.mxfp4_dequantise(c, s, T, K, t["x"], damoe.LAYOUT_ROWMAJOR),
                     lambda: damoe.mxfp4_pack(c, s, T, K, _bytes(4352).cuda())):
            with pytest.raises(ValueError, match="device"):
                call()
    torch.cuda.synchronize()


def test_calls_by_words():
    """damoe_call_words: the call's own status for its arguments in order, and a refusal of any other number of words."""
    P, Q, big = 0x10000, 0x20000, 1 << 40  # never dereferenced: every call ends before a launch
    call = damoe.lib().damoe_call_words
    loss = [P, 1, 64, P, 0, 0, 8, 64, 4, 1, 0, 1.0, 0.0, P, P, 0, P, P, big, 0]
    grad = [P, 1, 64, P, 0, 0, 0, 0, P, P, 8, 64, 4, 1, 0, 1.0, 0.0, 0, Q, 64, 0]
    linear = [P, 0, 512, 4, 512, P, 64, 0, 0, Q, 0, 64, P, big, 0]
    bad, unsupported, workspace = -1, -2, -3
    # The position of an argument and a value that the call refuses there.
    refusals = [
        (0, damoe._LOSS_WORDS, loss, {bad: [(0, 0), (0, P + 2), (2, 63), (3, 0), (6, -1), (7, 0), (8, 17), (9, 2), (10, 2), (13, 0),
                                            (14, 0), (16, 0), (17, 0), (17, P + 8)], unsupported: [(1, 2)], workspace: [(18, 255)]}),
        (1, damoe._GRAD_WORDS, grad, {bad: [(0, 0), (2, 63), (4, P), (5, P), (8, 0), (9, 0), (10, -1), (11, 0), (12, 17), (13, 2),
                                            (14, 2), (18, 0), (18, Q + 2), (19, 63)], unsupported: [(1, 2)]}),
        (2, damoe._LINEAR_WORDS, linear, {bad: [(0, 0), (2, 511), (3, -1), (4, 0), (5, 0), (5, P + 8), (6, 0), (9, 0), (11, 63),
                                                (12, 0), (12, P + 8)], unsupported: [(1, 2), (4, 48), (10, 2)], workspace: [(13, 0)]})]
    for fn, pack, good, wrong in refusals:
        for status, changes in wrong.items():
            for i, v in changes:
                words = pack(*good[:i], v, *good[i + 1:])
                assert call(fn, words, len(good)) == status, (fn, i, v)
        for n in (0, len(good) - 1, len(good) + 1):
            assert call(fn, pack(*good), n) == bad
        assert call(fn, None, len(good)) == bad
    assert call(3, damoe._LINEAR_WORDS(*linear), 15) == call(-1, b"", 0) == bad


def test_products_that_the_library_does_not_have():
    """Refused where the object is made, not at its first call."""
    w = torch.zeros(64, 32, dtype=torch.bfloat16)
    for weight, T_max in [(w, -1), (w, (1 << 20) + 1), (w[:, :24], 8), (w[:, :0], 8), (w[:0], 8),
                          (w[:1].expand(1 << 20, 32).as_strided((1 << 20, 8192), (0, 0)), 8),  # 4.6 GB of tiles
                          (w.as_strided((64, 8192), (0, 0)), 1 << 20), (w.as_strided(((1 << 20) + 1, 32), (0, 0)), 8)]:
        with pytest.raises(ValueError, match="no product"):
            MxLinear(weight, T_max)
