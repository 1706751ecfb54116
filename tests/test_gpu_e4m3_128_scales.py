"""GPU tests of the products with a scale per 128 at the ends of what their scales may be, in every kernel: a row's scale and
a weight's, each from the smallest to the largest, whose product is in fp32's normal range."""
import pytest
import torch

from .gemm128_shapes import GATED, PLAIN
from .gpu_helpers import lib_ready
from .test_gpu_e4m3_128 import F8, Problem, check, gated_exact, run_gated, run_gemm
from .test_gpu_e4m3_128_kernels import name

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    return lib_ready()


# scales of rows and of weights, as powers of two (each times a gain of 2^-2 to 2^2; the problem's own are 2^-6.6 and so / sqrt(k))
ENDS = [(118, -118), (-118, 118), (60, 40), (-50, -40)]


@pytest.mark.parametrize("shape", [(*k, *shapes[-1]) for k, shapes in PLAIN.items()], ids=name)
@pytest.mark.parametrize("rows2,weights2", ENDS)
def test_gemm_scales_far_apart(H, shape, rows2, weights2):
    """Results of 2^-90 to 2^100: the bound for ordinary scales times a power of two. No step on the way is subnormal: the
    products of scales are 2^-114 at least."""
    p = Problem(*shape[3:], bias=False)
    p.a_scale *= 2.0 ** rows2
    p.w_scale[0] *= 2.0 ** weights2
    assert torch.isfinite(p.a_scale).all() and (p.a_scale.abs().min() > 0) and (p.w_scale[0].abs().min() > 0)
    y = run_gemm(H, p, "f32")
    assert torch.isfinite(y).all()
    want, off = p.exact()
    check(y, want, off, "f32")


@pytest.mark.parametrize("shape", [(*k, *shapes[-1]) for k, shapes in GATED.items()], ids=name)
def test_gated_scales_far_apart(H, shape):
    p = Problem(*shape[3:], two=True, bias=False)
    p.a_scale *= 2.0 ** 110
    for s in p.w_scale:
        s *= 2.0 ** -110
    y, _ = run_gated(H, p, "silu", "f32")
    h, off = gated_exact(p, "silu")
    check(y, h, off, "f32")


@pytest.mark.parametrize("shape", [(*k, *shapes[0]) for k, shapes in PLAIN.items()], ids=name)
def test_the_largest_products_of_scales(H, shape):
    """Products of scales of 2^127 and codes of 2^-9, the smallest: nothing is out of range, nor are blocks of zeros NaN."""
    rows, k, n = shape[3:]
    p = Problem(rows, k, n, bias=False)
    p.a[:] = 1  # 2^-9
    p.w[0][:] = 1
    p.w[0][n // 2:] = 0
    p.a_scale[:] = 2.0 ** 63
    p.w_scale[0][:] = 2.0 ** 64 / 4096
    p.w_scale[0][:, 0] = 2.0 ** 64
    assert (p.a[0, 0].view(F8).float() == 2.0 ** -9).item()
    y = run_gemm(H, p, "f32")
    want, off = p.exact()
    assert torch.isfinite(y).all() and (y[:, n // 2:] == 0).all() and want.max() < 3e38
    check(y, want, off, "f32")
