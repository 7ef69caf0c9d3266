"""Refusals, sizes and no-ops of the MXFP4 calls and the router's loss (no GPU: every call ends before a launch)."""
import os

import pytest

from paper_2607_23099_amd import build, damoe

P, Q = 0x10000, 0x20000  # never dereferenced
BAD, UNSUPPORTED, WORKSPACE = -1, -2, -3
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(damoe.LIB_PATH):
        build.build_damoe()


def _q(x=P, dtype=0, rows=32, cols=256, ldx=256, layout=0, codes=P, scales=P):
    return damoe.lib().damoe_mxfp4_quantise(x, dtype, rows, cols, ldx, layout, codes, scales, None)


def _dq(x=P, dtype=0, rows=32, cols=256, ldx=256, layout=0, codes=P, scales=P):
    return damoe.lib().damoe_mxfp4_dequantise(codes, scales, rows, cols, layout, x, dtype, ldx, None)


@pytest.mark.parametrize("call", [_q, _dq])
def test_quantise_refusals(call):
    for kw in [dict(x=None), dict(codes=None), dict(scales=None), dict(rows=-1), dict(cols=0), dict(cols=-32),
               dict(ldx=255), dict(codes=P + 8), dict(x=P + 1), dict(dtype=1, x=P + 2)]:
        assert call(**kw) == BAD, kw
    for kw in [dict(dtype=2), dict(dtype=-1), dict(layout=3), dict(layout=-1), dict(cols=48), dict(layout=1, rows=17),
               dict(layout=1, cols=96, ldx=96), dict(cols=(1 << 20) + 32, ldx=1 << 21), dict(rows=1 << 36),
               dict(rows=0, cols=33, ldx=64), dict(rows=0, layout=1, cols=96)]:
        assert call(**kw) == UNSUPPORTED, kw
    for layout in (0, 1, 2):
        assert call(rows=0, layout=layout) == 0


def test_mxfp4_bytes():
    assert damoe.mxfp4_bytes(3, 96, damoe.LAYOUT_ROWMAJOR) == 3 * 48
    assert damoe.mxfp4_bytes(32, 256, damoe.LAYOUT_FRAG16) == 32 * 256 * 17 // 32
    assert damoe.mxfp4_bytes(1, 32) == 4352 and damoe.mxfp4_bytes(33, 288) == 4 * 4352
    for bad in [(0, 32, 0), (-1, 32, 0), (1, 0, 0), (1, 33, 0), (16, 96, 1), (8, 128, 1), (1, 32, 3), (1 << 36, 32, 0)]:
        assert damoe.mxfp4_bytes(*bad) == 0, bad


def test_pack_refusals():
    f = damoe.lib().damoe_mxfp4_pack
    assert f(P, P, 0, 32, P, None) == 0
    for a in [(None, P, 1, 32, P), (P, None, 1, 32, P), (P, P, 1, 32, None), (P + 8, P, 1, 32, P), (P, P, 1, 32, P + 4),
              (P, P, -1, 32, P), (P, P, 1, 0, P)]:
        assert f(*a, None) == BAD, a
    for a in [(P, P, 1, 40, P), (P, P, 0, 40, P), (P, P, 1 << 36, 32, P)]:
        assert f(*a, None) == UNSUPPORTED, a


def _lin(x=P, xd=0, ldx=512, T=4, K=512, w=P, N=64, add=None, lda=0, y=Q, yd=0, ldy=64, ws=P, wsb=BIG):
    return damoe.lib().damoe_mxfp4_linear(x, xd, ldx, T, K, w, N, add, lda, y, yd, ldy, ws, wsb, None)


def test_linear_refusals():
    for kw in [dict(x=None), dict(w=None), dict(y=None), dict(ws=None), dict(T=-1), dict(N=0), dict(K=0), dict(ldx=511),
               dict(ldy=63), dict(add=P, lda=63), dict(x=P + 1), dict(xd=1, x=P + 2), dict(y=Q + 1), dict(yd=1, y=Q + 2),
               dict(w=P + 8), dict(ws=P + 8), dict(add=P + 1, lda=64)]:
        assert _lin(**kw) == BAD, kw
    for kw in [dict(xd=2), dict(yd=-1), dict(K=48), dict(T=(1 << 20) + 1), dict(N=(1 << 20) + 1, ldy=1 << 21),
               dict(K=(1 << 20) + 32, ldx=1 << 21), dict(T=1 << 20, K=8192, ldx=8192), dict(N=1 << 20, ldy=1 << 20, K=8192, ldx=8192)]:
        assert _lin(**kw) == UNSUPPORTED, kw
    need = damoe.mxfp4_linear_workspace_size(4, 64, 512)
    assert need >= 256 and _lin(wsb=0) == WORKSPACE
    assert _lin(T=0) == 0 and _lin(T=0, x=None, y=None, ws=None) == 0
    for bad in [(-1, 64, 512), (4, 0, 512), (4, 64, 0), (4, 64, 40), (1 << 20, 64, 8192)]:
        assert damoe.mxfp4_linear_workspace_size(*bad) == 0, bad


def test_linear_workspace_holds_every_smaller_call():
    for N, K in [(64, 512), (7168, 2048), (4096, 7168), (33, 8192), (20000, 256)]:
        sizes = [damoe.mxfp4_linear_workspace_size(T, N, K) for T in range(0, 1200)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), (N, K)


def _loss(logits=P, dtype=1, ld=64, ids=P, mask=None, off=None, T=8, E=64, k=4, S=1, score=0, loss=P, counts=P, probs=None,
          tokens=P, ws=P, wsb=BIG):
    return damoe.lib().damoe_router_loss(logits, dtype, ld, ids, mask, off, T, E, k, S, score, 1.0, 0.0, loss, counts, probs,
                                         tokens, ws, wsb, None)


def _grad(logits=P, dtype=1, ld=64, ids=P, w=None, dw=None, mask=None, off=None, counts=P, tokens=P, T=8, E=64, k=4, S=1,
          score=0, dl=Q, ldd=64):
    return damoe.lib().damoe_router_loss_grad(logits, dtype, ld, ids, w, dw, mask, off, counts, tokens, T, E, k, S, score, 1.0,
                                              0.0, None, dl, ldd, None)


COMMON = [dict(logits=None), dict(T=-1), dict(T=(1 << 20) + 1), dict(E=0), dict(E=1025, ld=2000), dict(k=0), dict(k=17), dict(E=3, k=4),
          dict(ld=63), dict(S=0), dict(S=2), dict(S=(1 << 20) + 1, off=P), dict(score=2), dict(score=-1), dict(logits=P + 2),
          dict(dtype=0, logits=P + 1), dict(counts=None), dict(tokens=None)]


def test_router_loss_refusals():
    for kw in COMMON + [dict(ids=None), dict(loss=None), dict(ws=None), dict(ws=P + 8)]:
        assert _loss(**kw) == BAD, kw
    for kw in [dict(dtype=2), dict(dtype=-1)]:
        assert _loss(**kw) == UNSUPPORTED, kw
    need = damoe.router_loss_workspace_size(8, 64, 1)
    assert need > 0 and _loss(wsb=need - 1 if need <= 256 else 255) == WORKSPACE
    for bad in [(-1, 64, 1), (8, 0, 1), (8, 1025, 1), (8, 64, 0), ((1 << 20) + 1, 64, 1)]:
        assert damoe.router_loss_workspace_size(*bad) == 0, bad
    # Enough for every smaller batch.
    for E, S in [(64, 1), (256, 37)]:
        for t_max in (1, 100, 8191, 8193, 16500, 40000):
            assert all(damoe.router_loss_workspace_size(T, E, S) <= damoe.router_loss_workspace_size(t_max, E, S)
                       for T in range(0, t_max, 97))


def test_router_loss_grad_refusals():
    more = [dict(dl=None), dict(ldd=63), dict(dl=P, ldd=80), dict(w=P), dict(dw=P), dict(w=P, dw=P, ids=None), dict(dl=Q + 2)]
    for kw in COMMON + more:
        assert _grad(**kw) == BAD, kw
    for kw in [dict(dtype=2), dict(dtype=-1)]:
        assert _grad(**kw) == UNSUPPORTED, kw
    assert _grad(T=0) == 0 and _grad(T=0, logits=None, dl=None) == 0


def test_tensor_forms_that_the_binding_refuses():
    torch = pytest.importorskip("torch")
    a = torch.zeros(8, 64)
    with pytest.raises(ValueError):  # a transposed matrix has no rows of neighbours
        damoe.mxfp4_quantise(torch.zeros(256, 32).t(), 32, 256, a, a, damoe.LAYOUT_ROWMAJOR, stream=0)
    with pytest.raises(ValueError):
        damoe.router_loss_grad(a, a, 8, 64, 4, a, a, a.to(torch.bfloat16), stream=0)
    with pytest.raises(ValueError):
        damoe.mxfp4_linear(a, 8, 64, a, 64, a, a, add=a.to(torch.bfloat16), stream=0)
    with pytest.raises(damoe.DamoeError):  # fp16 is no type of these calls
        damoe.mxfp4_quantise(a.half(), 8, 64, a, a, damoe.LAYOUT_ROWMAJOR, stream=0)


def test_lists_that_the_binding_refuses():
    torch = pytest.importorskip("torch")
    T, E, k, S = 8, 64, 4, 2
    a = torch.zeros(T, E)
    ids = torch.zeros(T, k, dtype=torch.int32)
    off = torch.zeros(S + 1, dtype=torch.int32)
    w = torch.zeros(T, k)
    mask = torch.ones(T, dtype=torch.uint8)
    good = dict(mask=mask, seq_offsets=off)

    def loss(ids=ids, **kw):
        damoe.router_loss(a, ids, T, E, k, a, a, a, a[0], S=S, stream=0, **{**good, **kw})

    def grad(ids=ids, **kw):
        damoe.router_loss_grad(a, ids, T, E, k, a, a, a, S=S, stream=0, **{**good, "w": w, "dw": w, **kw})

    bad = [dict(ids=ids.long()), dict(ids=ids[:-1]), dict(ids=torch.zeros(k, T, dtype=torch.int32).t()), dict(mask=mask.long()),
           dict(mask=mask[:-1]), dict(mask=torch.ones(2 * T, dtype=torch.uint8)[::2]), dict(seq_offsets=off.long()),
           dict(seq_offsets=off[:-1])]
    for kw in bad:
        with pytest.raises(ValueError):
            loss(**kw)
        with pytest.raises(ValueError):
            grad(**kw)
    for kw in [dict(dw=torch.zeros(1, 1).expand(T, k)), dict(w=w.double()), dict(dw=w[:-1]), dict(dloss=torch.zeros((), dtype=torch.float64))]:
        with pytest.raises(ValueError):
            grad(**kw)
    with pytest.raises(damoe.DamoeError, match="workspace"):  # the lists are good: the library's own check is next
        loss()
    with pytest.raises(damoe.DamoeError, match="invalid argument"):
        loss(ids=None)
    damoe.router_loss_grad(a, None, 0, E, k, a, a, a, stream=0)  # no gates, no tokens
    with pytest.raises(ValueError):
        damoe.mxfp4_quantise(torch.zeros(4, 8, 64).transpose(0, 1), 32, 64, a, a, damoe.LAYOUT_ROWMAJOR, stream=0)


def test_objects_refuse_what_their_buffers_do_not_hold():
    torch = pytest.importorskip("torch")
    from paper_2607_23099_amd.moe import MxLinear, Path

    lin = MxLinear.__new__(MxLinear)
    lin.N, lin.K, lin.T_max = 64, 32, 4
    lin.tiles = lin.ws = torch.zeros(1, dtype=torch.uint8)
    x = torch.zeros(4, 32)
    for args, kw in [((torch.zeros(5, 32),), {}), ((torch.zeros(4, 64),), {}), ((x.to("meta"),), {}), ((x, torch.zeros(4, 63)), {}),
                     ((x,), dict(add=torch.zeros(1, 64))), ((x,), dict(add=torch.zeros(1, 64).expand(4, 64).to("meta")))]:
        with pytest.raises(ValueError):
            lin(*args, stream=0, **kw)
    path = Path.__new__(Path)
    path.loss_S, path.T_max = 0, 4
    for call in (path.router_loss, path.router_loss_grad):
        with pytest.raises(RuntimeError):
            call(4, 0.1)
    path.loss_S = 1
    for call in (path.router_loss, path.router_loss_grad):
        with pytest.raises(ValueError):
            call(5, 0.1)


def test_router_loss_workspace_holds_every_smaller_batch():
    for E, S in [(64, 2), (64, 15), (256, 64), (384, 65), (40, 5000)]:
        sizes = [damoe.router_loss_workspace_size(T, E, S) for T in list(range(0, 5000, 7)) + [8192, 16384, 16385, 70000, 1 << 20]]
        assert all(0 < a <= b for a, b in zip(sizes, sizes[1:])), (E, S)
