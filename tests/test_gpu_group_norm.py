"""GPU tests of hilo_group_norm against group norm in 64 bits on the same inputs.

Tolerance, per element, with A the largest |x| of the group and u = 2^-23. A thread adds
up at most 28 rows (one kernel: what its shared memory holds) or joins J batches of four (two
kernels; at these sizes J is at most rows / 2560 + 4), each join off by at most u A. Its eight
channels follow, a lane's entries of the group (at most 32), the lanes (five steps), the CTAs'
pairs (at most four a lane and five steps): half a u each and as much for each weight, less
than 64 u A together. So the mean is off by at most (J + 64) u A, the squares by (J + 64) u of
themselves and the mean's error squared, their root by half of that. (A thread's error of its
mean times that mean's distance from the group's, of either sign, is left out: the bar is below
the bound.) The
difference to the mean, its product, the vectors and the sum are six roundings more.
The activations' slope is at most 1.2, their exponential and division are within
2^-19 of the value. Then one rounding to the output's type.
"""
import math

import pytest
import torch

from .gpu_helpers import lib_ready
from .test_gpu_e4m3_128 import DT, act_exact, check, check_codes, code

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Images:
    def __init__(self, B, rows, d, groups, dtype="bf16", vec="bf16", cond=True, weights=True, pad=0, offset=1.0, seed=0):
        g = rng(B + 10 * rows + 100 * d + seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.B, self.rows, self.d, self.groups, self.dtype, self.vec = B, rows, d, groups, dtype, vec
        x = r(B * rows, d) * torch.exp2(2 * torch.rand(d, generator=g, device="cuda") - 1) + offset * r(d)
        self.buf = torch.full((B * rows, d + pad), float("nan"), dtype=DT[dtype], device="cuda")
        self.buf[:, :d] = x.to(DT[dtype])
        self.cond = (0.3 * r(B, 2 * d + 16)).to(DT[vec]) if cond else None
        self.w = (1 + 0.2 * r(d)).to(DT[vec]) if weights else None
        self.b = (0.2 * r(d)).to(DT[vec]) if weights else None

    def vectors(self, H):
        c, d = self.cond, self.d
        return H.NormVectors(scale=None if c is None else c[:, :d], shift=None if c is None else c[:, d:2 * d], w_norm=self.w, b_norm=self.b)

    def exact(self, act, eps):
        B, n, d, G = self.B, self.rows, self.d, self.groups
        x = self.buf[:, :d].double().view(B, n, G, d // G)
        mean, top = x.mean((1, 3), keepdim=True), x.abs().amax((1, 3), keepdim=True)
        var = (x - mean).square().mean((1, 3), keepdim=True)
        J = B * n / 2560 + 2 + 64
        u = 2.0 ** -23
        off_mean = J * u * top
        root = torch.sqrt(var + eps)
        rel = 0.5 * (J * u * var + off_mean ** 2) / (var + eps) + 4 * u
        one = lambda v, none: torch.full((B, 1, d), none, dtype=torch.float64, device="cuda") if v is None else v.double().view(-1, 1, d).expand(B, 1, d)  # noqa: E731
        s = None if self.cond is None else self.cond[:, :d].contiguous()
        t = None if self.cond is None else self.cond[:, d:2 * d].contiguous()
        a = one(self.w, 1.0) * (1 + one(s, 0.0))
        b = one(self.b, 0.0) * (1 + one(s, 0.0)) + one(t, 0.0)
        z = ((x - mean) / root).view(B, n, d)
        y = z * a + b
        off = (a.abs() * ((off_mean / root).expand_as(x).reshape(B, n, d) + z.abs() * (rel.expand_as(x).reshape(B, n, d) + 6 * u))
               + 3 * u * (y.abs() + b.abs()))
        if act != "none":
            zarg = (y if act == "silu" else 2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)).abs()
            h = act_exact(y, act)
            off = 1.2 * off + (2.0 ** -19 + 2.0 ** -22 * zarg) * h.abs()
            y = h
        return y.view(B * n, d), off.view(B * n, d)

    def run(self, H, act="none", out="bf16", eps=1e-5, ypad=0, in_place=False, into=None, ws=None, more_ws=0):
        B, n, d = self.B, self.rows, self.d
        acts = {"none": H.HILO_ACT_NONE, "silu": H.HILO_ACT_SILU, "gelu": H.HILO_ACT_GELU}
        shape = H.GroupNormShape(B=B, rows=n, d=d, groups=self.groups, act=acts[act], eps=eps, x_dtype=code(H, self.dtype),
                                 y_dtype=code(H, out), vec_dtype=code(H, self.vec), x_row=self.buf.shape[1],
                                 y_row=self.buf.shape[1] if in_place else d + ypad, vec_row=2 * d + 16, y_scale_ld=B * n + 3)
        if in_place:
            y = self.buf
        elif into is not None:
            y = into
        else:
            y = torch.zeros(B * n, d + ypad, dtype=torch.uint8 if out == "e4m3" else DT[out], device="cuda")
            y.fill_(3)
        sc = torch.full((-(-d // 128), B * n + 3), -7.0, device="cuda") if out == "e4m3" else None
        nb = H.hilo_group_norm_workspace_bytes(shape)
        ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws  # (NaNs: nothing in it counts)
        H.hilo_group_norm(shape, self.vectors(H) if self.cond is not None or self.w is not None else None, self.buf, y, sc, ws, nb)
        return y, sc


SIZES = [(1, 1, 16, 1), (1, 1, 128, 32), (2, 3, 128, 32), (1, 7, 144, 36), (3, 17, 320, 32), (1, 64, 512, 32), (2, 333, 256, 8),
         (1, 1024, 512, 32), (3, 1380, 1152, 36), (1, 900, 2048, 32), (2, 100, 4096, 32), (1, 77, 8192, 16), (1, 50, 4112, 257),
         (5, 4, 48, 48), (1, 20000, 128, 32), (1, 5000, 640, 1), (70, 40, 64, 4), (1, 65536, 64, 8), (1, 9000, 8192, 8192), (2, 3000, 4112, 257),
         (1, 70000, 320, 32), (3, 30001, 144, 36), (500, 9, 2048, 32), (2, 20000, 512, 512),
         (1, 7000, 2048, 128), (1, 16384, 512, 64)]


@pytest.mark.parametrize("B,rows,d,groups", SIZES)
@pytest.mark.parametrize("dtype,out,act", [("bf16", "bf16", "silu"), ("f16", "f16", "gelu"), ("f32", "f32", "none"), ("bf16", "e4m3", "silu"),
                                           ("f32", "e4m3", "gelu"), ("f16", "f32", "silu")])
def test_group_norm(H, B, rows, d, groups, dtype, out, act):
    p = Images(B, rows, d, groups, dtype, vec="f32" if dtype == "f32" else "bf16")
    y, sc = p.run(H, act, out)
    want, off = p.exact(act, 1e-5)
    if out == "e4m3":
        check_codes(y, sc, want, off)
        assert (sc[:, B * rows:] == -7).all()
    else:
        check(y, want, off, out)


@pytest.mark.parametrize("cond,weights", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("out", ["bf16", "e4m3"])
def test_group_norm_without_some_vectors(H, cond, weights, out):
    p = Images(2, 150, 160, 10, "f16", cond=cond, weights=weights, pad=32)
    y, sc = p.run(H, "silu", out, ypad=48)
    want, off = p.exact("silu", 1e-5)
    if out == "e4m3":
        check_codes(y, sc, want, off)
    else:
        check(y[:, :160], want, off, out)
    assert (y[:, 160:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B,rows,d", [(2, 300, 320), (1, 30000, 128)])
def test_group_norm_in_place(H, dtype, B, rows, d):
    p = Images(B, rows, d, 32, dtype, pad=16)
    want, off = p.exact("silu", 1e-5)
    y, _ = p.run(H, "silu", dtype, in_place=True)
    check(y[:, :d], want, off, dtype)
    assert torch.isnan(y[:, d:]).all()


@pytest.mark.parametrize("offset", [100.0, 10000.0])
def test_group_norm_far_from_zero(H, offset):
    """An offset far above the deviation costs its own rounding, no more."""
    p = Images(1, 3000, 128, 128, "f32", cond=False, weights=False, offset=offset)
    y, _ = p.run(H, "none", "f32")
    want, off = p.exact("none", 1e-5)
    check(y, want, off, "f32")


def test_group_norm_constant_and_eps(H):
    p = Images(1, 200, 64, 8, "f32", cond=False, weights=False)
    p.buf[:, :64] = 3.0
    y, _ = p.run(H, "none", "f32")
    assert (y == 0).all()
    y, sc = p.run(H, "silu", "e4m3")
    assert (y == 0).all() and (sc[:, :200] == 1).all()
    p.buf[:, :8] += 1e-3 * torch.randn(200, 8, generator=rng(3), device="cuda")
    y, _ = p.run(H, "none", "f32", eps=1e-2)
    want, off = p.exact("none", 1e-2)
    check(y, want, off, "f32")


@pytest.mark.parametrize("rows", [500, 40000])
def test_group_norm_specials_stay_in_their_group(H, rows):
    p = Images(3, rows, 256, 16, "bf16", cond=False, weights=False)
    p.buf[rows + 77, 40] = float("inf")
    p.buf[2 * rows + 3, 255] = float("nan")
    y, _ = p.run(H, "none", "f32")
    bad = torch.isnan(y).view(3, rows, 16, 16)
    want = torch.zeros_like(bad)
    want[1, :, 2], want[2, :, 15] = True, True
    assert torch.equal(bad, want)


def test_group_norm_far_rows(H):
    """Offsets past 2^32 elements in rows of x and y."""
    rows, d, row = 6, 128, 1 << 30
    p = Images(2, 3, d, 32, "bf16")
    big = torch.empty(rows * row, dtype=torch.bfloat16, device="cuda")
    big.view(rows, row)[:, :d] = p.buf
    want, off = p.exact("silu", 1e-5)
    shape = H.GroupNormShape(B=2, rows=3, d=d, groups=32, act=H.HILO_ACT_SILU, x_row=row, y_row=row, vec_row=2 * d + 16)
    nb = H.hilo_group_norm_workspace_bytes(shape)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    H.hilo_group_norm(shape, p.vectors(H), big, big, None, ws, nb)
    check(big.view(rows, row)[:, :d], want, off, "bf16")


def test_group_norm_one_row_of_the_widest_stride(H):
    p = Images(1, 1, 256, 32, "f32", cond=False)
    want, off = p.exact("silu", 1e-5)
    far = (1 << 39) - 16
    shape = H.GroupNormShape(B=1, rows=1, d=256, groups=32, act=H.HILO_ACT_SILU, x_dtype=H.HILO_F32, y_dtype=H.HILO_F32, x_row=far,
                             y_row=far, vec_row=far + 8)
    nb = H.hilo_group_norm_workspace_bytes(shape)
    y = torch.empty(1, 256, device="cuda")
    H.hilo_group_norm(shape, p.vectors(H), p.buf, y, None, torch.empty(nb, dtype=torch.uint8, device="cuda"), nb)
    check(y, want, off, "f32")


@pytest.mark.parametrize("B,rows,d", [(1, 600, 512), (2, 40000, 128)])
def test_group_norm_captured_and_on_two_streams(H, B, rows, d):
    p, q = Images(B, rows, d, 32), Images(B, rows, d, 32, seed=1)
    want, other = p.run(H, "silu")[0], q.run(H, "silu")[0]
    torch.cuda.synchronize()
    y = torch.zeros_like(want)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(H, "silu", into=y, ws=ws)
    one = torch.cuda.Stream()
    z = torch.zeros_like(other)
    torch.cuda.synchronize()
    for _ in range(10):
        graph.replay()
        with torch.cuda.stream(one):
            q.run(H, "silu", into=z)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, other)
    p.buf.copy_(q.buf)
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(y, want)


FIRST = r"""
import torch
from tests.gpu_helpers import lib_ready
H = lib_ready()
x = torch.randn(600, 256, device="cuda").bfloat16()
big = torch.randn(60000, 256, device="cuda").bfloat16()
w = torch.randn(512, 256, device="cuda").bfloat16()
E = lambda *s, t=torch.uint8: torch.zeros(*s, dtype=t, device="cuda")
codes, scale, wc, ws = E(600, 256), E(2, 600, t=torch.float32), E(512, 256), E(4, 2, t=torch.float32)
h, hs, y = E(600, 256), E(2, 600, t=torch.float32), E(600, 512, t=torch.float32)
z, work = torch.zeros_like(big), E(1 << 20)

def norm(rows, src, dst, sc, out):
    s = H.GroupNormShape(B=1, rows=rows, d=256, groups=16, act=H.HILO_ACT_SILU, y_dtype=out)
    H.hilo_group_norm(s, None, src, dst, sc, work, H.hilo_group_norm_workspace_bytes(s))

def step():
    norm(60000, big, z, None, H.HILO_BF16)
    norm(600, x, codes, scale, H.HILO_E4M3)
    H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=512, cols=256, tile=1), w, None, wc, ws)
    up = H.Gemm128Shape(rows=600, k=256, n=256, act=H.HILO_ACT_GELU, out_dtype=H.HILO_E4M3)
    H.hilo_gated_e4m3_128(up, codes, scale, wc, ws, wc[256:], ws[2:], None, None, None, h, hs)
    for rows in (1, 600):
        s = H.Gemm128Shape(rows=rows, k=256, n=512, out_dtype=H.HILO_F32, a_scale_ld=600)
        H.hilo_gemm_e4m3_128(s, h, hs, wc, ws, None, None, y)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (z, codes, scale, h, hs, y)]
for t in (z, codes, scale, h, hs, y):
    t.zero_()
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (z, codes, scale, h, hs, y))) and y.abs().max() > 0
print("the same")
"""


def test_first_calls_inside_a_capture(H):
    """A process whose very first calls are captured: nothing that they set up needs a stream."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-3000:]


def test_group_norm_into_a_product(H):
    """A 1x1 convolution in 8 bits behind a group norm: codes and scales go from one to the other."""
    B, rows, d, n = 2, 200, 320, 272
    p = Images(B, rows, d, 32)
    codes, sc = p.run(H, "silu", "e4m3")
    h, off = p.exact("silu", 1e-5)
    check_codes(codes, sc, h, off)
    w = torch.randn(n, d, generator=rng(9), device="cuda") / 18
    wc, ws = torch.empty(n, d, dtype=torch.uint8, device="cuda"), torch.empty(3, 3, device="cuda")
    H.hilo_quantize_e4m3_128(H.Quant128Shape(rows=n, cols=d, dtype=H.HILO_F32, tile=1), w, None, wc, ws)
    y = torch.empty(B * rows, n, device="cuda")
    H.hilo_gemm_e4m3_128(H.Gemm128Shape(rows=B * rows, k=d, n=n, out_dtype=H.HILO_F32, a_scale_ld=B * rows + 3), codes, sc, wc, ws,
                         None, None, y)
    rel = ((y.double() - h @ w.double().t()).norm() / (h @ w.double().t()).norm()).item()
    assert rel < 0.06, rel  # (two operands, each off by 2^-4 at most, a third of it in the mean square)
