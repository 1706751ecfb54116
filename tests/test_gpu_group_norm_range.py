"""GPU tests of hilo_group_norm where magnitudes, offsets and row counts are out of the ordinary, against 64 bits."""
import pytest
import torch

from .gpu_helpers import lib_ready
from .test_gpu_e4m3_128 import check
from .test_gpu_group_norm import Images, rng

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    return lib_ready()


@pytest.mark.parametrize("rows", [60, 300, 30000])
@pytest.mark.parametrize("per", [1, 8, 64])
def test_offsets_whose_squares_leave_fp32(H, rows, per):
    """Offsets of 1e20 and deviations of 1e15: only the squares about the mean have to be in range, whose sum here is
    at most 30000 * 64 * (5e15)^2 = 5e37. One kernel (60 and 300 rows) and two (30000). The tolerance is that of
    ordinary sizes."""
    p = Images(1, rows, 128, 128 // per, "f32", cond=False, weights=False)
    g = rng(rows + per)
    sign = torch.where(torch.rand(128 // per, generator=g, device="cuda") < 0.5, -1.0, 1.0).repeat_interleave(per)
    p.buf[:] = 1e20 * sign + 1e15 * torch.randn(rows, 128, generator=g, device="cuda").clamp(-5, 5)
    y, _ = p.run(H, "none", "f32")
    want, off = p.exact("none", 1e-5)
    assert torch.isfinite(y).all()
    check(y, want, off, "f32")
