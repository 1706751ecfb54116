"""GPU tests of the 8-bit linear operators with a scale for each block of 128
(hilo_quantize_e4m3_128, hilo_gemm_e4m3_128, hilo_gated_e4m3_128) against
plain 64-bit forms.

Quantisation is compared bit for bit with the same fp32 steps in torch. Products
are compared element by element with the exact sum over the codes: the tensor
core adds a block's 128 products in fp32 (each addition off by at most 2^-23 of
what it adds up, truncating or not), the kernel multiplies two scales, adds each
of the blocks (one rounding each) and the bias, and the result is rounded once,
by at most half a step of its type. So with S = sum |a w| the fp32 value is off by at
most (128 + blocks + 4) 2^-23 (S + |bias|).
"""
import math

import numpy as np
import pytest
import torch

from .gpu_helpers import lib_ready

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": F8}


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def code(H, name):
    return {"bf16": H.HILO_BF16, "f16": H.HILO_F16, "f32": H.HILO_F32, "e4m3": H.HILO_E4M3}[name]


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def count(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


# ------------------------------------------------------------ quantisation ---


def block_max(x, tall):
    """Largest magnitudes of blocks of `tall` rows x 128 columns, and the same for every element; NaNs left out."""
    rows, cols = x.shape
    down, across = -(-rows // tall), -(-cols // 128)
    y = torch.zeros(down * tall, across * 128, dtype=torch.float64 if x.dtype == torch.float64 else torch.float32, device="cuda")
    y[:rows, :cols] = torch.nan_to_num(x.to(y.dtype).abs(), nan=0.0, posinf=math.inf)
    m = y.view(down, tall, across, 128).amax(3).amax(1)
    return m, m.repeat_interleave(tall, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def quantised(x, tall):
    """Codes and scales by the definition, in fp32 steps."""
    m, each = block_max(x, tall)
    fix = lambda v: torch.where(v > 0, v.clamp(min=2.0 ** -100), torch.full_like(v, 448.0))  # noqa: E731
    most = torch.tensor(448.0, device="cuda")  # (on the device: torch divides by, or into, a number of the host's in two roundings)
    y = x.float() * (most / fix(each))
    return y.clamp(-448, 448).to(F8), fix(m) / most


def same_codes(a, b):
    a, b = a.view(torch.uint8), b.view(torch.uint8)
    nan = (a & 0x7F) == 0x7F
    assert torch.equal(nan, (b & 0x7F) == 0x7F)
    assert torch.equal(a[~nan], b[~nan])


def run_quant(H, x, tile, pad=0, dpad=0, spare=0, n_rows=None, ld_more=0):
    rows, cols = x.shape
    names = {v: k for k, v in DT.items()}
    buf = torch.full((rows + spare, cols + pad), float("nan"), dtype=x.dtype, device="cuda")
    buf[:rows, :cols] = x
    dst = torch.full((rows + spare, cols + dpad), 0x55, dtype=torch.uint8, device="cuda")
    down, across = -(-(rows + spare) // 128), -(-cols // 128)
    ld = (across if tile else rows + spare) + ld_more
    scale = torch.full((down if tile else across, ld), -7.0, device="cuda")
    H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=rows + spare, cols=cols, dtype=code(H, names[x.dtype]), tile=tile,
                                             src_row=cols + pad, dst_row=cols + dpad, scale_ld=ld), buf, n_rows, dst, scale)
    torch.cuda.synchronize()
    return dst, scale


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,dpad,spare,ld", [
    (1, 16, 0, 0, 0, 0), (1, 4096, 0, 0, 0, 0), (3, 128, 16, 0, 0, 1), (7, 144, 0, 32, 5, 0), (130, 272, 48, 16, 130, 3),
    (33, 1168, 0, 0, 0, 0), (4096, 2064, 16, 0, 3, 5)])
@pytest.mark.parametrize("tile", [0, 1])
def test_quantise_bit_for_bit(H, dtype, rows, cols, pad, dpad, spare, ld, tile):
    g = rng(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(8 * torch.rand(rows, 1, generator=g, device="cuda") - 6))
    x = x.to(DT[dtype])
    if rows > 2:
        x[1] = 0
    dst, scale = run_quant(H, x, tile, pad, dpad, spare, count(rows) if spare else None, ld)
    want, sc = quantised(x, 128 if tile else 1)
    same_codes(dst[:rows, :cols], want)
    if tile:
        assert torch.equal(scale[:sc.shape[0], :sc.shape[1]], sc)
        assert (scale[sc.shape[0]:] == -7).all() and (scale[:, sc.shape[1]:] == -7).all()
    else:
        assert torch.equal(scale[:, :rows], sc.t())
        assert (scale[:, rows:] == -7).all()
    assert (dst[rows:] == 0x55).all() and (dst[:, cols:] == 0x55).all()


def test_scales_of_every_mantissa(H):
    """amax / 448 is correctly rounded: all 2^23 mantissas of an fp32, each at one of 200 exponents."""
    rows = 1 << 23
    at = torch.arange(rows, device="cuda", dtype=torch.int32)
    amax = ((at % 200 + 27) << 23 | at).view(torch.float32)  # from 2^-100
    x = torch.zeros(rows, 16, device="cuda")
    x[:, 3] = -amax
    codes, scale = torch.empty(rows, 16, dtype=torch.uint8, device="cuda"), torch.empty(1, rows, device="cuda")
    H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=rows, cols=16, dtype=H.HILO_F32), x, None, codes, scale)
    assert torch.equal(scale[0], amax / torch.full((), 448.0, device="cuda"))
    assert (codes[:, 3] == 0xFE).all() and (codes[:, :3] == 0).all()


@pytest.mark.parametrize("n", [-3, 0, 2, 7, 9, 100])
@pytest.mark.parametrize("tile", [0, 1])
def test_quantise_counts_rows_on_the_device(H, n, tile):
    x = torch.randn(9, 144, generator=rng(1), device="cuda")
    dst, scale = run_quant(H, x, tile, n_rows=count(n))
    there = min(max(n, 0), 9)
    if there:
        want, sc = quantised(x[:there], 128 if tile else 1)
        same_codes(dst[:there], want)
        assert torch.equal(scale[:, :] if tile else scale[:, :there], sc if tile else sc.t())
    assert (dst[there:] == 0x55).all()
    if not tile:
        assert (scale[:, there:] == -7).all()
    elif not there:
        assert (scale == -7).all()


@pytest.mark.parametrize("tile", [0, 1])
def test_quantise_extremes(H, tile):
    """Blocks of zeros, of the smallest and the largest numbers, infinities, NaNs, ties between codes."""
    x = torch.zeros(256, 896, device="cuda")
    x[:, 128:256] = 2.0 ** -140 * torch.randn(256, 128, generator=rng(2), device="cuda")
    x[:, 256:384] = torch.finfo(torch.float32).max
    x[:, 384:512] = torch.randn(256, 128, generator=rng(3), device="cuda")
    x[5, 390] = float("nan")
    x[:, 512:640] = torch.randn(256, 128, generator=rng(4), device="cuda")
    x[7, 600] = -float("inf")
    x[:, 640:768] = 448.0 * torch.exp2(-torch.arange(128, device="cuda") / 7.0).round()
    steps = torch.arange(127, device="cuda") / 16.0 + 1.0  # between codes, with 448 to make the factor 1
    x[:, 768:895], x[:, 895] = steps, 448.0
    dst, scale = run_quant(H, x, tile)
    want, sc = quantised(x, 128 if tile else 1)
    same_codes(dst, want)
    assert torch.equal(scale, sc if tile else sc.t())
    value = dst.view(F8).float() * (scale.repeat_interleave(128, 0) if tile else scale.t()).repeat_interleave(128, 1)[:, :896]
    assert torch.isnan(value[5, 390]) and (value[:, :128] == 0).all()
    assert torch.isfinite(value[:, 128:384]).all()


def test_quantise_far_rows(H):
    """Offsets past 2^32 bytes in source and destination."""
    rows, cols, row = 5, 144, 1 << 30
    src = torch.empty(rows * row, dtype=torch.bfloat16, device="cuda")
    dst = torch.empty(rows * row, dtype=torch.uint8, device="cuda")
    x = torch.randn(rows, cols, generator=rng(5), device="cuda").bfloat16()
    src.view(rows, row)[:, :cols] = x
    scale = torch.empty(2, rows, device="cuda")
    H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=rows, cols=cols, src_row=row, dst_row=row), src, None, dst, scale)
    want, sc = quantised(x, 1)
    same_codes(dst.view(rows, row)[:, :cols].contiguous(), want)
    assert torch.equal(scale, sc.t())


# ---------------------------------------------------------------- products ---


class Problem:
    """Rows and weights in codes, with gains that differ from block to block; buffers with room around them."""

    def __init__(self, rows, k, n, two=False, bias=True, spare=0, pad=0, seed=0):
        g = rng(1000 * rows + 10 * k + n + seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        gain = lambda *s: torch.exp2(4 * torch.rand(*s, generator=g, device="cuda") - 2)  # noqa: E731
        self.rows, self.k, self.n, self.cap = rows, k, n, rows + spare
        kb, nb = -(-k // 128), -(-n // 128)
        self.a = torch.full((self.cap, k + pad), 0x7F, dtype=torch.uint8, device="cuda")  # (NaN where nobody looks)
        self.a[:rows, :k] = (100 * r(rows, k)).clamp(-448, 448).to(F8).view(torch.uint8)
        self.a_scale = torch.full((kb, self.cap + pad), float("nan"), device="cuda")
        self.a_scale[:, :rows] = 0.01 * gain(kb, rows)
        self.w, self.w_scale, self.bias = [], [], []
        for _ in range(2 if two else 1):
            w = torch.full((n, k + pad), 0x7F, dtype=torch.uint8, device="cuda")
            w[:, :k] = (100 * r(n, k)).clamp(-448, 448).to(F8).view(torch.uint8)
            self.w.append(w)
            s = torch.full((nb, kb + (1 if pad else 0)), float("nan"), device="cuda")
            s[:, :kb] = 0.01 / math.sqrt(k) * gain(nb, kb)
            self.w_scale.append(s)
            self.bias.append(r(n).bfloat16() if bias else None)

    def strides(self):
        return dict(a_row=self.a.shape[1], w_row=self.w[0].shape[1], a_scale_ld=self.a_scale.shape[1],
                    w_scale_ld=self.w_scale[0].shape[1])

    def exact(self, i=0):
        """(the products with bias in 64 bits, how far an fp32 value of them may be off)."""
        rows, k, n = self.rows, self.k, self.n
        a = self.a[:rows, :k].view(F8).double() * self.a_scale[:, :rows].double().t().repeat_interleave(128, 1)[:, :k]
        s = self.w_scale[i][:, :-(-k // 128)].double()
        w = self.w[i][:, :k].view(F8).double() * s.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
        y, size = a @ w.t(), a.abs() @ w.abs().t()
        if self.bias[i] is not None:
            y, size = y + self.bias[i].double(), size + self.bias[i].double().abs()
        return y, (128 + -(-k // 128) + 4) * 2.0 ** -23 * size


def check(got, want, off, dtype, what=""):
    half = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]  # half a step, of the value
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0  # half of the smallest step
    err = (got.double() - want).abs()
    bound = off + half * (want.abs() + off) + tiny
    worst = (err / bound.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound, at most {err.max().item():.3e}"
    return worst


def run_gemm(H, p, out="bf16", n_rows=None, opad=0, stream=None, into=None):
    y = torch.full((p.cap, p.n + opad), 3.0, dtype=DT[out], device="cuda") if into is None else into
    H.hilo_gemm_e4m3_128(H.Gemm128Shape(rows=p.cap, k=p.k, n=p.n, out_dtype=code(H, out), out_row=p.n + opad, **p.strides()),
                         p.a, p.a_scale, p.w[0], p.w_scale[0], p.bias[0], n_rows, y, stream)
    return y


SIZES = [(1, 16, 16), (1, 128, 128), (1, 4096, 144), (2, 144, 400), (15, 272, 128), (16, 1168, 256), (17, 128, 272), (31, 640, 144),
         (33, 2048, 128), (64, 272, 144), (65, 400, 272), (127, 128, 16), (129, 1168, 144), (200, 272, 400), (256, 1024, 512),
         (257, 144, 128), (512, 256, 272), (513, 272, 144), (700, 1168, 272), (1000, 16, 16), (2389, 512, 528), (1499, 304, 2224),
         (1300, 1168, 2064), (513, 272, 4752), (2389, 160, 4112), (300, 512, 7200)]


@pytest.mark.parametrize("out", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_gemm(H, rows, k, n, out):
    p = Problem(rows, k, n, bias=out != "f16")
    y = run_gemm(H, p, out)
    want, off = p.exact()
    check(y, want, off, out, f"{rows}x{k}x{n} {out}")


@pytest.mark.parametrize("rows,k,n", [(1, 144, 144), (40, 272, 272), (130, 400, 144), (600, 272, 400)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_gemm_strides_and_counted_rows(H, rows, k, n, out):
    """Padded rows and scales, NaN codes in the padding and behind the counted rows, outputs that stay as they were."""
    p = Problem(rows, k, n, spare=300, pad=48)
    y = run_gemm(H, p, out, n_rows=count(rows), opad=32)
    want, off = p.exact()
    check(y[:rows, :n], want, off, out)
    assert (y[rows:] == 3).all() and (y[:, n:] == 3).all()


@pytest.mark.parametrize("cap", [5, 600])
@pytest.mark.parametrize("n_rows", [-1, 0, 1, 1 << 30])
def test_gemm_counts_at_the_ends(H, cap, n_rows):
    p = Problem(cap, 272, 144)
    y = run_gemm(H, p, "f32", n_rows=count(n_rows))
    there = min(max(n_rows, 0), cap)
    want, off = p.exact()
    if there:
        check(y[:there], want[:there], off[:there], "f32")
    assert (y[there:] == 3).all()


@pytest.mark.parametrize("rows", [3, 40, 600])
def test_gemm_nan_stays_in_its_row_and_feature(H, rows):
    p = Problem(rows, 272, 272, bias=False)
    want, off = p.exact()
    p.a[1, 130] = 0x7F
    p.w[0][200, 5] = 0xFF
    y = run_gemm(H, p, "f32")
    bad = torch.zeros(rows, 272, dtype=torch.bool, device="cuda")
    bad[1], bad[:, 200] = True, True
    assert torch.equal(torch.isnan(y), bad)
    check(torch.where(bad, 0.0, y.double()), torch.where(bad, 0.0, want), off, "f32")


def test_gemm_saturates_fp16(H):
    p = Problem(20, 128, 128, bias=False)
    p.a_scale *= 1e6
    y = run_gemm(H, p, "f16")
    want, _ = p.exact()
    big = want.abs() > 65600
    assert big.any() and torch.equal(y.double()[big], want[big].sign() * 65504)


def test_gemm_far_rows(H):
    """Offsets past 2^32 elements in rows, weights and outputs."""
    for rows in (6, 530):
        row = 1 << 23 if rows > 512 else 1 << 30
        p = Problem(rows, 144, 144)
        a = torch.zeros(rows * row, dtype=torch.uint8, device="cuda")
        a.view(rows, row)[:, :144] = p.a
        y = torch.zeros(rows * row, dtype=torch.bfloat16, device="cuda")
        H.hilo_gemm_e4m3_128(H.Gemm128Shape(rows=rows, k=144, n=144, a_row=row, out_row=row), a, p.a_scale, p.w[0], p.w_scale[0],
                             p.bias[0], None, y)
        want, off = p.exact()
        check(y.view(rows, row)[:, :144], want, off, "bf16")
        del a, y
        torch.cuda.empty_cache()


# ------------------------------------------------------------------- gated ---


def act_exact(g, act):
    z = g if act == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    return g * torch.sigmoid(z)


def gated_exact(p, act):
    """h in 64 bits, and how far the fp32 value may be off: gate and up by what the products are, the activation's
    slope is at most 1.2 (SiLU 1.1, GELU 1.13); its exponential and division are within 2^-19 of the value."""
    (g, og), (u, ou) = p.exact(0), p.exact(1)
    h = act_exact(g, act) * u
    off = 1.2 * og * (u.abs() + ou) + act_exact(g, act).abs() * ou + 2.0 ** -19 * h.abs()
    # (the argument of the exponential is off by 2^-22 of itself: of the value, so much again)
    z = (g if act == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)).abs()
    return h, off + 2.0 ** -22 * z * h.abs()


def run_gated(H, p, act="silu", out="bf16", n_rows=None, opad=0, into=None):
    y = torch.zeros(p.cap, p.n + opad, dtype=torch.uint8 if out == "e4m3" else DT[out], device="cuda") if into is None else into[0]
    sc = torch.full((-(-p.n // 128), p.cap + 1), -7.0, device="cuda") if into is None else into[1]
    if into is None:
        y.fill_(3)
    H.hilo_gated_e4m3_128(H.Gemm128Shape(rows=p.cap, k=p.k, n=p.n, act=H.HILO_ACT_SILU if act == "silu" else H.HILO_ACT_GELU,
                                         out_dtype=code(H, out), out_row=p.n + opad, out_scale_ld=p.cap + 1, **p.strides()),
                          p.a, p.a_scale, p.w[0], p.w_scale[0], p.w[1], p.w_scale[1], p.bias[0], p.bias[1], n_rows, y,
                          sc if out == "e4m3" else None)
    return y, sc


def check_codes(y, sc, h, off):
    """Each scale is that of the block's largest value, and each code is no further from the value than half a step:
    2^-4 of it, or half the smallest code, 2^-10, of the scale."""
    rows, n = h.shape
    m, _ = block_max(h, 1)
    least = block_max((h.abs() - off).clamp(min=0), 1)[0]  # of the values as they may be in fp32
    most = block_max(h.abs() + off, 1)[0]
    scale = sc[:, :rows].t().double()
    fp32 = m * 2.0 ** -22  # the division's rounding, and that of the value
    zero = most == 0  # (of scale 1, by definition)
    assert (scale[zero] == 1).all()
    assert (zero | ((scale * 448 >= least - fp32) & (scale * 448 <= most + fp32))).all()
    each = scale.repeat_interleave(128, 1)[:, :n]
    err = (y[:rows, :n].view(F8).double() * each - h).abs()
    # (a code of the value as it is in fp32: half a step beyond what that is off)
    bound = off + (h.abs() + off) * 2.0 ** -4 + each * 2.0 ** -10 + h.abs() * 2.0 ** -20
    assert (err <= bound).all(), (err / bound).max().item()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("out", ["bf16", "f16", "f32", "e4m3"])
@pytest.mark.parametrize("rows,k,n", SIZES)
def test_gated(H, rows, k, n, out, act):
    p = Problem(rows, k, n, two=True, bias=act == "gelu")
    y, sc = run_gated(H, p, act, out)
    h, off = gated_exact(p, act)
    if out == "e4m3":
        check_codes(y, sc, h, off)
        assert (sc[:, rows:] == -7).all()
    else:
        check(y, h, off, out)


@pytest.mark.parametrize("rows,k,n", [(1, 144, 144), (40, 272, 272), (130, 400, 144), (600, 272, 400)])
@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_gated_strides_and_counted_rows(H, rows, k, n, out):
    p = Problem(rows, k, n, two=True, spare=300, pad=48)
    y, sc = run_gated(H, p, "gelu", out, n_rows=count(rows), opad=32)
    h, off = gated_exact(p, "gelu")
    if out == "e4m3":
        check_codes(y, sc, h, off)
        assert (sc[:, rows:] == -7).all()
    else:
        check(y[:rows, :n], h, off, out)
    assert (y[rows:] == 3).all() and (y[:, n:] == 3).all()


@pytest.mark.parametrize("rows", [3, 40, 600])
def test_gated_large_and_empty_blocks(H, rows):
    """Gates far out on both sides: e^-g overflows and vanishes; blocks whose values are all zero have scale 1."""
    p = Problem(rows, 128, 272, two=True, bias=False)
    p.w_scale[0] *= 1000
    p.w[1][:128] = 0
    y, sc = run_gated(H, p, "silu", "e4m3")
    assert (sc[0, :rows] == 1).all() and (y[:, :128].view(F8).float() == 0).all()
    h, off = gated_exact(p, "silu")
    check_codes(y, sc, h, off)
    y, _ = run_gated(H, p, "gelu", "f32")
    h, off = gated_exact(p, "gelu")
    check(y, h, off, "f32")


def test_gated_halves_of_one_matrix(H):
    p = Problem(70, 272, 256, two=True)
    w, s = torch.cat(p.w), torch.cat(p.w_scale)
    want, _ = run_gated(H, p, "silu", "f32")
    p.w, p.w_scale = [w[:256], w[256:]], [s[:2], s[2:]]
    got, _ = run_gated(H, p, "silu", "f32")
    assert torch.equal(got, want)


# --------------------------------------------------- together, and as they run ---


@pytest.mark.parametrize("rows", [1, 50, 300, 1000])
def test_feed_forward(H, rows):
    """Rows to codes, up, gated, to codes, and down again: each step against 64 bits from what it was given."""
    d, f = 400, 656
    g = rng(rows)
    x = torch.randn(rows, d, generator=g, device="cuda").bfloat16()
    weights = [torch.randn(f, d, generator=g, device="cuda") / 20, torch.randn(f, d, generator=g, device="cuda") / 20,
               torch.randn(d, f, generator=g, device="cuda") / 25]
    p, q = Problem(rows, d, f, two=True, bias=False), Problem(rows, f, d, bias=True)
    into = [(p, 0), (p, 1), (q, 0)]
    for w, (pr, i) in zip(weights, into):
        n, k = w.shape
        pr.w[i], pr.w_scale[i] = torch.empty(n, k, dtype=torch.uint8, device="cuda"), torch.empty(-(-n // 128), -(-k // 128), device="cuda")
        H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=n, cols=k, dtype=H.HILO_F32, tile=1), w, None, pr.w[i], pr.w_scale[i])
    p.a, p.a_scale = torch.empty(rows, d, dtype=torch.uint8, device="cuda"), torch.empty(4, rows, device="cuda")
    q.a, q.a_scale = torch.empty(rows, f, dtype=torch.uint8, device="cuda"), torch.empty(6, rows, device="cuda")
    y = torch.empty(rows, d, device="cuda")

    def step():
        H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=rows, cols=d), x, None, p.a, p.a_scale)
        H.hilo_gated_e4m3_128(H.Gemm128Shape(rows=rows, k=d, n=f, act=H.HILO_ACT_SILU, out_dtype=H.HILO_E4M3), p.a, p.a_scale,
                              p.w[0], p.w_scale[0], p.w[1], p.w_scale[1], None, None, None, q.a, q.a_scale)
        H.hilo_gemm_e4m3_128(H.Gemm128Shape(rows=rows, k=f, n=d, out_dtype=H.HILO_F32), q.a, q.a_scale, q.w[0], q.w_scale[0],
                             q.bias[0], None, y)

    step()
    torch.cuda.synchronize()
    h, off = gated_exact(p, "silu")
    check_codes(q.a, q.a_scale, h, off)
    want, off = q.exact()
    check(y, want, off, "f32")
    # the whole of it, against unquantised arithmetic: three roundings to e4m3 of both operands and the middle
    full = (act_exact(x.double() @ weights[0].double().t(), "silu") * (x.double() @ weights[1].double().t())) @ weights[2].double().t()
    full += q.bias[0].double()
    rel = ((y.double() - full).norm() / full.norm()).item()
    assert rel < 0.12, rel
    # captured, replayed on other rows
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    y.zero_()
    graph.replay()
    assert torch.equal(y, first)
    x.copy_(torch.randn(rows, d, generator=g, device="cuda").bfloat16())
    graph.replay()
    replayed = y.clone()
    step()
    assert torch.equal(y, replayed) and not torch.equal(y, first)


@pytest.mark.parametrize("rows", [1, 100, 900])
def test_repeats_itself_on_two_streams(H, rows):
    p = Problem(rows, 2064, 528)
    q = Problem(rows, 1040, 400, two=True)
    torch.cuda.synchronize()
    want, codes = run_gemm(H, p, "f32"), run_gated(H, q, "silu", "e4m3")
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    ys, hs = [torch.zeros_like(want) for _ in range(8)], [(torch.zeros_like(codes[0]), torch.zeros_like(codes[1])) for _ in range(8)]
    torch.cuda.synchronize()
    for y, h in zip(ys, hs):
        with torch.cuda.stream(one):
            run_gemm(H, p, "f32", into=y)
        with torch.cuda.stream(two):
            run_gated(H, q, "silu", "e4m3", into=h)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)
    assert all(torch.equal(h[0], codes[0]) and torch.equal(h[1][:, :rows], codes[1][:, :rows]) for h in hs)


def test_rows_do_not_depend_on_their_neighbours(H):
    """A row of a batch gives what it gives alone, to the order of the fp32 sums."""
    p = Problem(300, 1168, 272)
    y = run_gemm(H, p, "f32")
    want, off = p.exact()
    for r in (0, 17, 299):
        one = torch.zeros(1, 272, device="cuda")
        H.hilo_gemm_e4m3_128(H.Gemm128Shape(rows=1, k=1168, n=272, out_dtype=H.HILO_F32), p.a[r:r + 1], p.a_scale[:, r:r + 1].contiguous(),
                             p.w[0], p.w_scale[0], p.bias[0], None, one)
        assert ((one - y[r:r + 1]).abs() <= 2 * off[r:r + 1]).all()
