"""damoe_call_words: integers that the callee's type does not hold are refused (no GPU: every call ends before a launch)."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2607_23099_amd import build, damoe
from tests.test_rows_adapters_cpu import BAD, BIG, CALLS, UNSUPPORTED, P, Q


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(damoe.LIB_PATH):
        build.build_damoe()


LINEAR = dict(x=P, xdtype=1, ldx=64, T=4, K=64, w=P, N=64, add=0, ld_add=0, y=Q, ydtype=1, ldy=64, ws=P, ws_bytes=BIG, stream=0)
INTEGERS = {"dtype", "xdtype", "ydtype", "wdtype", "T", "k", "H", "R", "L", "r", "K", "N", "accumulate"}


@pytest.mark.parametrize("fn,pack,good", [c[:3] for c in CALLS] + [(2, damoe._LINEAR_WORDS, LINEAR)],
                         ids=["sort", "combine", "combine_grad", "adapters", "adapters_grad", "mxfp4_linear"])
def test_integers_past_32_bits(fn, pack, good):
    """2^32 tokens are not none, and 2^32 + 8 rows are not 8."""
    call = damoe.lib().damoe_call_words
    # A call that ends early by itself, with another status.
    quiet, status = ({**good, "r": 129}, UNSUPPORTED) if "r" in good else ({**good, "T": 0}, 0)
    assert call(fn, pack(*quiet.values()), len(quiet)) == status
    for name in INTEGERS & set(good):
        for far in (1 << 32, -(1 << 32), 1 << 62):
            words = {**quiet, name: quiet[name] + far}
            assert call(fn, pack(*words.values()), len(words)) == BAD, (name, far)


@pytest.mark.parametrize("size", [damoe.adapters_workspace_size, damoe.adapters_grad_workspace_size], ids=["forward", "gradient"])
def test_workspaces_of_sizes_past_32_bits(size):
    """0, as for any size that the calls do not take, and not the size of what is left of them."""
    good = [100, 3, 8, 64, 48]
    assert size(*good) > 0
    for i in range(len(good)):
        for far in (1 << 32, -(1 << 32), 1 << 62):
            assert size(*good[:i], good[i] + far, *good[i + 1:]) == 0
