"""The router's loss and gradient where a valid row holds a NaN or +inf, and past 32-bit offsets, against float64."""
import numpy as np
import pytest

from paper_2607_23099_amd import damoe
from tests import router_loss_ref as ref
from tests.gpu_common import log, torch_cuda
from tests.test_gpu_router_loss import REL, Case

pytestmark = pytest.mark.gpu


# One block, blocks of one wave, blocks of eight; rows of fours, twos and single columns.
@pytest.mark.parametrize("T,E,offsets", [(40, 32, [0, 10, 40]), (60, 37, [0, 10, 11, 40, 50, 60]), (300, 384, [0, 200, 300]),
                                         (200, 1000, [0, 120, 200])])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("value", [np.nan, np.inf], ids=["nan", "inf"])
def test_a_valid_row_with_nan_or_inf(T, E, offsets, score, value):
    """It makes the mean probabilities of its sequence, the losses and its row of the gradient NaN, whichever of the two
    terms is asked for, and nothing else."""
    torch = torch_cuda()
    at = 7

    def edit(l, ids):
        l[at, 5] = value

    for dtype in ("f32", "bf16"):
        for alpha, zc in [(0.7, 0.0), (0.0, 0.02), (0.7, 0.02)]:
            log(f"router loss with {value} T={T} E={E} score={score} alpha={alpha} z={zc} {dtype}")
            c = Case(torch, T, E, 4, offsets=offsets, dtype=dtype, edit=edit)
            clean = c.l.copy()
            clean[at] = 0.0  # the other rows' results do not depend on this one's logits
            _, counts, probs, tokens = ref.loss(clean, c.ids, 4, None, offsets, score, alpha, zc)
            c.forward(score, alpha, zc)
            assert torch.isnan(c.loss).all(), c.loss.tolist()
            assert np.array_equal(c.counts.cpu().numpy(), counts) and np.array_equal(c.tokens.cpu().numpy(), tokens)
            assert torch.isnan(c.probs[0]).all()
            np.testing.assert_allclose(c.probs[1:].double().cpu().numpy(), probs[1:], rtol=REL, atol=1e-30)
            for gates in (False, True):
                out = torch.zeros((T, E), dtype=c.logits.dtype, device="cuda")
                c.backward(out, score, alpha, zc, gates=gates)
                assert torch.isnan(out[at]).all(), int(torch.isnan(out[at]).sum())
                g = (c.w.astype(np.float64), c.dw.astype(np.float64)) if gates else ()
                d, mag = ref.grad(clean, c.ids, 4, None, offsets, score, alpha, zc, counts, 1.0, *g)
                tol = 2 * REL * mag + 1e-30
                tol = tol + (2.0 ** -8 * (np.abs(d) + tol) if dtype == "bf16" else 0.0)
                bad = ~(np.abs(out.double().cpu().numpy() - d) <= tol)
                bad[at] = False
                assert not bad.any(), np.argwhere(bad)[:4].tolist()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("score", [0, 1], ids=["softmax", "sigmoid"])
def test_the_last_rows_of_the_largest_batch(dtype, score):
    """2^20 rows 2100 elements apart: element offsets past 2^31 and byte offsets past 2^32.  All rows but the last 64 are NaN
    and do not count, so a row taken from any other place shows, forward and backward."""
    torch = torch_cuda()
    T, E, k, ld, n = 1 << 20, 1024, 16, 2100, 64
    log(f"router loss, the last rows of {T} x {E}, {dtype}, score={score}")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    c = Case(torch, n, E, k, dtype=dtype, seed=5)
    buf = torch.full((T, ld), float("nan"), dtype=dt, device="cuda")
    buf[T - n:, :E] = c.logits[: n * E].view(n, E)
    ids = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    w, dw = torch.zeros((T, k), device="cuda"), torch.zeros((T, k), device="cuda")
    for t, s in ((ids, c.d_ids), (w, c.d_w), (dw, c.d_dw)):
        t[T - n:] = s
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[T - n:] = 1
    ws = torch.zeros(damoe.router_loss_workspace_size(T, E), dtype=torch.uint8, device="cuda")
    loss, counts = torch.zeros(3, device="cuda"), torch.zeros((1, E), dtype=torch.int32, device="cuda")
    probs, tokens = torch.zeros((1, E), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    damoe.router_loss(buf, ids, T, E, k, loss, counts, tokens, ws, mask=mask, score=score, alpha=0.7, z_coef=0.02, probs=probs)
    want, want_c, want_p, _ = ref.loss(c.l, c.ids, k, None, None, score, 0.7, 0.02)
    assert tokens.tolist() == [n, 1, n] and np.array_equal(counts.cpu().numpy(), want_c)
    np.testing.assert_allclose(probs.double().cpu().numpy(), want_p, rtol=REL, atol=1e-30)
    np.testing.assert_allclose(loss.double().cpu().numpy(), want, rtol=REL, atol=2.0 ** -20 * (1 + want[2]))
    damoe.router_loss_grad(buf, ids, T, E, k, counts, tokens, buf, mask=mask, score=score, alpha=0.7, z_coef=0.02, w=w, dw=dw)
    d, mag = ref.grad(c.l, c.ids, k, None, None, score, 0.7, 0.02, want_c, 1.0, c.w.astype(np.float64), c.dw.astype(np.float64))
    tol = 2 * REL * mag + 1e-30
    tol = tol + (2.0 ** -8 * (np.abs(d) + tol) if dtype == "bf16" else 0.0)
    assert (np.abs(buf[T - n:, :E].double().cpu().numpy() - d) <= tol).all()
    for a in range(0, T - n, 1 << 17):
        rows = buf[a: min(a + (1 << 17), T - n)]
        assert (rows[:, :E] == 0).all() and torch.isnan(rows[:, E:]).all()
