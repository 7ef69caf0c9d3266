"""Rows whose last piece is not all lanes', on the kernels for many rows as on those for few (the gradient goes by blocks of
tokens from 40 MB of rows on)."""
import pytest

from tests.gpu_common import log, torch_cuda
from tests.test_gpu_rows import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,k,H,dtype,kw", [
    (2600, 8, 516, "f32", dict(drop=0.1)),                        # 129 lanes' pieces: one in the third
    (1400, 16, 1031, "bf16", dict(drop=0.3, ld=1035, shift=1)),   # the last piece has 7 elements
    (1000, 4, 2731, "f32", dict(R=3000, cut=True, shift=1)),      # slots past the rows
    (2700, 1, 8184, "bf16", dict(R=3000)),
])
def test_many_rows_against_float64(T, k, H, dtype, kw):
    torch = torch_cuda()
    assert T * k * H * (2 if dtype == "bf16" else 4) >= 40 << 20
    log(f"T={T} k={k} H={H} {dtype} {kw}")
    b = Batch(torch, T, k, H, dtype, **kw)
    b.check()
    b.check(weighted=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [2, 8, 9, 255, 257, 511, 513, 1023, 1025])
def test_lanes_past_the_end_of_a_row(H, dtype):
    """16 slots, whose places come from 16 lanes, in rows of which a piece's last lanes have nothing."""
    torch = torch_cuda()
    log(f"H={H} {dtype}")
    Batch(torch, 9, 16, H, dtype, drop=0.2, ld=H + 1).check()
