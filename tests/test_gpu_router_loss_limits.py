"""The router's loss and gradient where a valid row holds a NaN or +inf, against float64."""
import numpy as np
import pytest

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
