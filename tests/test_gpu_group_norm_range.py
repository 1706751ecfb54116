"""GPU tests of hilo_group_norm where magnitudes, offsets and row counts are out of the ordinary, against 64 bits."""
import pytest
import torch

from .gpu_helpers import lib_ready
from .test_gpu_e4m3_128 import check, check_codes
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


def constant_images(H, dtype, B, rows, d, groups, seed):
    """Every image's groups of one value each, in 32 bits out, with b_norm and w_norm: the result, and b_norm."""
    g = rng(seed)
    x = (100 * torch.randn(B, 1, groups, 1, generator=g, device="cuda")).to(dtype)
    x = x.expand(B, rows, groups, d // groups).reshape(B * rows, d).contiguous()
    w, b = torch.randn(2, d, generator=g, device="cuda")
    shape = H.GroupNormShape(B=B, rows=rows, d=d, groups=groups, vec_dtype=H.HILO_F32, y_dtype=H.HILO_F32,
                             x_dtype={torch.bfloat16: H.HILO_BF16, torch.float16: H.HILO_F16, torch.float32: H.HILO_F32}[dtype])
    y = torch.empty(B * rows, d, device="cuda")
    n = H.hilo_group_norm_workspace_bytes(shape)
    H.hilo_group_norm(shape, H.NormVectors(w_norm=w, b_norm=b), x, y, None, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    return y, b


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("d,groups", [(64, 8), (64, 64), (160, 16), (256, 1), (512, 32)])
def test_a_constant_group_is_its_bias(H, dtype, d, groups):
    """Of equal values the mean is that value, whatever their number: 0 times the weight is left, and the bias."""
    bad = []
    for rows in list(range(1, 130)) + [255, 256, 257, 399, 500, 777, 1000, 1380, 3001, 5000, 20001, 70007]:
        y, b = constant_images(H, dtype, 3, rows, d, groups, rows)
        if not torch.equal(y, b.expand_as(y)):
            bad.append((rows, (y - b).abs().max().item()))
    assert not bad, bad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d,groups", [(9000, 2048, 2048), (33, 4112, 257), (20000, 512, 512), (100, 8192, 16), (3001, 144, 36)])
def test_a_constant_group_is_its_bias_of_many_groups(H, dtype, rows, d, groups):
    y, b = constant_images(H, dtype, 2, rows, d, groups, rows)
    assert torch.equal(y, b.expand_as(y))


@pytest.mark.parametrize("offset", [1e3, 1e6])
@pytest.mark.parametrize("rows,d,groups", [(1, 64, 4), (7, 64, 8), (60, 160, 16), (333, 512, 32), (1380, 1152, 36), (777, 64, 1),
                                           (30000, 128, 32), (20000, 512, 512), (70007, 64, 8)])
def test_an_offset_costs_its_roundings(H, rows, d, groups, offset):
    """With A the largest |x| of a group, S the largest distance from its mean and u = 2^-24: a mean is rounded once by a
    thread (u A), three times among its eight channels, once each among threads, CTAs and clusters; a batch of four
    rows is two roundings, and each of J joins one, which weighs half in the mean over the joins (J: rows / 2560 + 4 at
    these sizes, as for ordinary ones). What corrects a mean is a sum of distances from it, at most 64 terms one after another:
    64 u S. That is the mean's error; squares about it add its own square, and 100 + J roundings of theirs."""
    p = Images(1, rows, d, groups, "f32", cond=False, weights=False, offset=0.0)
    g = rng(rows)
    p.buf += offset * torch.randn(groups, generator=g, device="cuda").sign().repeat_interleave(d // groups)
    y, _ = p.run(H, "none", "f32")
    x = p.buf.double().view(rows, groups, -1)
    mean = x.mean((0, 2), keepdim=True)
    A, S = x.abs().amax((0, 2), keepdim=True), (x - mean).abs().amax((0, 2), keepdim=True)
    var = (x - mean).square().mean((0, 2), keepdim=True)
    u, J = 2.0 ** -24, rows / 2560 + 4
    off_mean = (9 + J / 2) * u * A + 64 * u * S
    root = torch.sqrt(var + 1e-5)
    rel = 0.5 * ((100 + J) * u + off_mean ** 2 / (var + 1e-5)) + 8 * u  # (of the root, with its own and the product's roundings)
    want = (x - mean) / root
    off = off_mean / root + want.abs() * rel + off_mean / root * rel
    check(y.view_as(x), want, off, "f32")


@pytest.mark.parametrize("B,rows,d,groups,out", [(100003, 16, 64, 4, "f32"), (70001, 1, 16, 1, "e4m3"), (300000, 3, 32, 8, "bf16"),
                                                 (2000, 40, 1024, 256, "f32")])
def test_very_many_images(H, B, rows, d, groups, out):
    p = Images(B, rows, d, groups, "bf16")
    y, sc = p.run(H, "silu", out)
    want, off = p.exact("silu", 1e-5)
    if out == "e4m3":
        check_codes(y, sc, want, off)
    else:
        check(y, want, off, out)


@pytest.mark.parametrize("B,rows,d,groups", [(1, 3500, 16, 1), (2, 3000, 16, 4), (1, 1700, 32, 8), (3, 900, 48, 6), (40, 1000, 16, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_narrow_images_to_codes(H, B, rows, d, groups, dtype):
    """Codes take half a warp a row: of 16 channels a thread has up to 224 rows (what shared memory holds of 16-bit values, 3584
    rows, by sixteen). Their sum is off by 112 half steps of the mean at most (of fp32, at most 112 rows, what corrects it
    leaves one); with about ten for what follows that is within ordinary sizes' 66 whole steps."""
    p = Images(B, rows, d, groups, dtype)
    y, sc = p.run(H, "silu", "e4m3")
    want, off = p.exact("silu", 1e-5)
    check_codes(y, sc, want, off)


@pytest.mark.parametrize("rows", [50, 20000])
def test_images_share_scale_and_shift(H, rows):
    """vec_row 0: one row of scale and shift for all images."""
    p = Images(3, rows, 64, 8)
    one = p.cond[:1].clone()
    p.cond = one.expand(3, -1).contiguous()
    want, off = p.exact("silu", 1e-5)
    shape = H.GroupNormShape(B=3, rows=rows, d=64, groups=8, act=H.HILO_ACT_SILU, y_dtype=H.HILO_F32, vec_row=0)
    n = H.hilo_group_norm_workspace_bytes(shape)
    y = torch.empty(3 * rows, 64, device="cuda")
    vectors = H.NormVectors(scale=one[:, :64], shift=one[:, 64:128], w_norm=p.w, b_norm=p.b)
    H.hilo_group_norm(shape, vectors, p.buf, y, None, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    check(y, want, off, "f32")
