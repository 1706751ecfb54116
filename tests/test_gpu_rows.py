"""hilo_row_positions, hilo_rope and hilo_gate_norm against their formulas in 64 bits.

Tolerances (u = half a step of the output's dtype, 2^-24 of fp32):
  positions  equal: sums of whole numbers, one division, one addition, each correctly rounded
  rope       (|a| + |b|) 2^-20 + u |out|: the angle in turns is off by at most 2^-25 + 2^-26 (2 pi times
             that is below 2^-21), the sine and cosine by two units, each product and sum by half of one
  norms      a thread adds at most 32 terms in a row and 7 levels follow, so a sum is off by at most 40 2^-24
             of the sum of its terms' magnitudes and a norm of n values x by 2^-18 (|xhat| + r mean|x|)
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from .gpu_helpers import lib_ready

pytestmark = pytest.mark.gpu
TYPES = {0: torch.bfloat16, 1: torch.float32, 2: torch.float16}
BF16, F32, F16, E4M3 = 0, 1, 2, 3
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def half_step(t):
    return torch.finfo(t).eps / 2


# -------------------------------------------------------------- positions --

@pytest.mark.parametrize("B,Hh,W,T,levels,lf,regions", [
    (1, 8, 12, 3, 1, 0, 0), (3, 16, 8, 0, 2, 0, 0), (2, 12, 20, 5, 2, 0, 1), (2, 8, 16, 1, 1, 4, 0), (1, 32, 32, 7, 1, 2, 0),
    (9, 4, 4, 2, 1, 0, 0)])
def test_row_positions(H, B, Hh, W, T, levels, lf, regions):
    sh = H.Shape(B=B, H=Hh, W=W, d=128, T=T, levels=levels, lf=lf)
    rng = np.random.default_rng(Hh + W + B)
    N = Hh * W
    score = torch.from_numpy(rng.random((B, N)).astype(np.float32)).cuda()
    mask = torch.from_numpy((rng.random((B, N)) < 0.1).astype(np.uint8)).cuda()
    keep = torch.from_numpy(rng.integers(0, N // 2, B).astype(np.int32)).cuda()
    mid = torch.from_numpy(rng.integers(0, N // 3, B).astype(np.int32)).cuda()
    sp = H.SplitBuffers.alloc(sh)
    (H.hilo_split_regions if regions else H.hilo_split)(sh, score, mask, keep, mid, sp)
    cap = H.hilo_row_capacity(sh)
    org = H.RowPositions(t_img=2.5, h0=-0.37 * Hh, w0=0.11 * W, txt0=-3.25, txt_step=0.3)
    pos = torch.full((B * T + cap + 4, 3), math.nan, device="cuda")
    H.hilo_row_positions(sh, sp, org, pos, cap)
    H.hilo_sync_status()
    got, f = pos.cpu().numpy(), np.float32
    lab = sp.labels.cpu().numpy().reshape(B, Hh, W)
    src, cnt, cu = sp.row_src.cpu().numpy(), sp.counts.cpu().numpy().reshape(B, 3), sp.cu_img.cpu().numpy()
    for r in range(B * T):
        want = f(float(f(r % T)) * float(f(0.3)) + float(f(-3.25)))
        assert np.all(got[r] == want)
    for b in range(B):
        for r in range(cu[b], cu[b + 1]):
            i = r - cu[b]
            if i < cnt[b, 0]:
                h, w = f(src[r] // W), f(src[r] % W)
            else:
                s = lf if lf else 2 if i < cnt[b, 0] + cnt[b, 1] else 4
                top, left = s * (src[r] // (W // s)), s * (src[r] % (W // s))
                at = [(p, q) for p in range(top, top + s) for q in range(left, left + s)
                      if lf or lab[b, p, q] == (1 if s == 2 else 2)]
                h, w = (f(sum(x[a] for x in at)) / f(len(at)) for a in (0, 1))
            want = [f(2.5), f(h + f(-0.37 * Hh)), f(w + f(0.11 * W))]
            assert np.array_equal(got[B * T + r], np.array(want, dtype=f)), (b, r)
    assert np.all(np.isnan(got[B * T + cu[B]:]))
    # a smaller capacity: the first rows, no more
    pos.fill_(math.nan)
    H.hilo_row_positions(sh, sp, org, pos, 3)
    assert np.array_equal(pos.cpu().numpy()[:B * T + 3], got[:B * T + 3]) and bool(pos[B * T + 3:].isnan().all())


CHECKED = r"""
import torch
from paper_2606_13898_gb300 import hilo as H
assert H.library_path().endswith("_build_checks/libhilo.so"), H.library_path()
sh = H.Shape(B=1, H=8, W=8, d=128, T=2)
sp = H.SplitBuffers.alloc(sh)
sp.labels.zero_()
sp.row_src.copy_(torch.arange(64))
sp.counts.copy_(torch.tensor([64, 0, 0]))
sp.cu_img.copy_(torch.tensor([0, 64]))
sp.row_src[9] = 64  # one past the grid: its labels would be another image's
pos = torch.full((66, 3), -7.0, device="cuda")
H.hilo_row_positions(sh, sp, H.RowPositions(t_img=1.0), pos, 64)
try:
    H.hilo_sync_status()
    raise SystemExit("no check fired")
except H.HiloError as e:
    assert e.status == H.HILO_ERR_CHECK and "check 7" in str(e), str(e)
assert bool((pos[11] == -7).all()) and bool((pos[10] == torch.tensor([1.0, 1.0, 0.0], device="cuda")).all())
"""


def test_positions_on_the_checks_build():
    """A row source outside the grid is caught before anything is addressed with it, and its row skipped."""
    from paper_2606_13898_gb300 import build
    env = dict(os.environ, HILO_LIBRARY=build.build(variant="checks"))
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider", "-k", "row_positions",
                        "tests/test_gpu_rows.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-3000:] + r.stderr[-2000:]
    r = subprocess.run([sys.executable, "-c", CHECKED], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr


# ------------------------------------------------------------------- rope --

def rope_reference(x, pos, dims, theta, interleaved, per_axis):
    x = x.double()
    D, i, out = sum(dims), 0, x.clone()
    mag = torch.zeros_like(x)
    for a, n in enumerate(dims):
        for j in range(n // 2):
            f = theta ** (-2.0 * j / n) if per_axis else theta ** (-2.0 * i / D)
            t = (pos[:, a].double() * f)[:, None]
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + D // 2)
            out[..., lo] = x[..., lo] * t.cos() - x[..., hi] * t.sin()
            out[..., hi] = x[..., lo] * t.sin() + x[..., hi] * t.cos()
            mag[..., lo] = mag[..., hi] = x[..., lo].abs() + x[..., hi].abs()
            i += 1
    return out, mag


ROPE = [
    # rows, heads, head_dim, dims, dtype, interleaved, per_axis, theta
    (1, 1, 64, (64,), BF16, 0, 1, 1e4),
    (5, 3, 128, (16, 56, 56), BF16, 1, 1, 1e4),
    (130, 48, 128, (16, 56, 56), BF16, 0, 0, 256.0),
    (77, 2, 80, (16, 32, 32), F16, 1, 0, 1e6),
    (33, 5, 256, (64, 96, 96), F32, 0, 1, 1e4),
    (260, 1, 96, (24, 24, 24, 24), F32, 1, 1, 1e4),
    (40, 4, 128, (8, 4, 4), F16, 0, 1, 1e4),    # 16 of 128 channels, the rest copied
    (40, 4, 64, (30, 2), BF16, 1, 0, 500.0),    # odd shares
    (3, 300, 8 * 3, (16,), F32, 0, 1, 1e4),
    (6000, 4, 64, (64,), BF16, 1, 1, 1e4),
]


@pytest.mark.parametrize("rows,heads,hd,dims,dtype,inter,per_axis,theta", ROPE)
def test_rope(H, rows, heads, hd, dims, dtype, inter, per_axis, theta):
    g, t = gen(rows + heads), TYPES[dtype]
    x = torch.randn(rows + 3, heads, hd, generator=g, device="cuda").to(t)
    pos = torch.randint(-800, 800, (rows + 3, len(dims)), generator=g, device="cuda").float() / 12
    pos[rows // 2, 0] = 123456.75
    pos[0, -1] = -99999.3
    n = torch.tensor([rows], dtype=torch.int32, device="cuda")
    y = torch.full_like(x, math.nan)
    sh = H.RopeShape(rows=rows + 3, heads=heads, head_dim=hd, dtype=dtype, axis_dims=dims, theta=theta, interleaved=inter,
                     per_axis=per_axis)
    H.hilo_rope(sh, x, pos, n, y)
    want, mag = rope_reference(x[:rows], pos[:rows], dims, theta, inter, per_axis)
    tol = mag * 2.0 ** -20 + half_step(t) * want.abs() + (2.0 ** -25 if dtype == F16 else 0)
    assert bool(((y[:rows].double() - want).abs() <= tol).all())
    assert bool(y[rows:].isnan().all())
    # in place, all rows, on rows of a wider buffer whose other columns stay
    wide = torch.full((rows + 3, heads * hd + 16), 7.0, dtype=t, device="cuda")
    wide[:, 8:-8] = x.reshape(rows + 3, -1)
    sh2 = H.RopeShape(rows=rows + 3, heads=heads, head_dim=hd, dtype=dtype, axis_dims=dims, theta=theta, interleaved=inter,
                      per_axis=per_axis, x_row=wide.stride(0), x_head=hd, y_row=wide.stride(0), y_head=hd)
    part = wide[:, 8:]
    H.hilo_rope(sh2, part, pos, None, part)
    assert torch.equal(wide[:rows, 8:-8].reshape(rows, heads, hd), y[:rows])
    assert bool((wide[:, :8] == 7).all()) and bool((wide[:, -8:] == 7).all())
    # a count beyond the rows, heads outermost in y
    z = torch.full((heads, rows + 3, hd), math.nan, dtype=t, device="cuda")
    n.fill_(1 << 30)
    sh3 = H.RopeShape(rows=rows, heads=heads, head_dim=hd, dtype=dtype, axis_dims=dims, theta=theta, interleaved=inter,
                      per_axis=per_axis, y_row=hd, y_head=(rows + 3) * hd)
    H.hilo_rope(sh3, x, pos, n, z)
    assert torch.equal(z[:, :rows].transpose(0, 1), y[:rows]) and bool(z[:, rows:].isnan().all())


@pytest.mark.parametrize("per_axis,theta", [(0, 1e4), (1, 1e4), (1, 1e6), (0, 1.5), (1, 1e30)])
@pytest.mark.parametrize("inter", [0, 1])
def test_rope_at_far_positions(H, inter, per_axis, theta):
    """Positions up to 2^24: the angle is off by less than 2^-21 radians there, beside sine, cosine, products and sum
    of a few 2^-24; at 2^30 by 2^30 * 2^-47 = 2^-17."""
    rows, heads, hd, dims = 64, 2, 128, (64, 32, 32)
    g = gen(inter + per_axis)
    x = torch.randn(rows, heads, hd, generator=g, device="cuda")
    sh = H.RopeShape(rows=rows, heads=heads, head_dim=hd, dtype=F32, axis_dims=dims, theta=theta, interleaved=inter,
                     per_axis=per_axis)
    for top, off in ((2.0 ** 24, 2.0 ** -20), (2.0 ** 30, 2.0 ** -16)):
        pos = top * (2 * torch.rand(rows, 3, generator=g, device="cuda") - 1)
        pos[0], pos[1], pos[2] = top, -top, 0.75 * top + 0.5
        y = torch.empty_like(x)
        H.hilo_rope(sh, x, pos, None, y)
        want, mag = rope_reference(x, pos, dims, theta, inter, per_axis)
        assert bool(((y.double() - want).abs() <= mag * off + 2.0 ** -24 * want.abs()).all()), float(((y.double() - want).abs() / mag).max())


def test_rope_gradient(H):
    """Rotating by the negated positions undoes the rotation and is its gradient: against differences of
    f(x) = sum(w * rope(x)) in fp32, whose rounding is 2^-24 of f per evaluation."""
    rows, heads, hd, dims = 7, 2, 64, (16, 24, 24)
    g = gen(1)
    x, w = (torch.randn(rows, heads, hd, generator=g, device="cuda") for _ in range(2))
    pos = 50 * torch.randn(rows, 3, generator=g, device="cuda")
    sh = H.RopeShape(rows=rows, heads=heads, head_dim=hd, dtype=F32, axis_dims=dims, interleaved=0, per_axis=0)
    y, grad, back = (torch.empty_like(x) for _ in range(3))
    H.hilo_rope(sh, x, pos, None, y)
    H.hilo_rope(sh, y, -pos, None, back)
    assert float((back - x).abs().max()) <= 2.0 ** -18 * float(x.abs().max())
    H.hilo_rope(sh, w, -pos, None, grad)
    step = 0.5
    for r, h, c in ((0, 0, 0), (3, 1, 31), (6, 1, 63), (2, 0, 40)):
        vals = []
        for s in (step, -step):
            xs = x.clone()
            xs[r, h, c] += s
            H.hilo_rope(sh, xs, pos, None, y)
            vals.append(float((w.double() * y.double()).sum()))
        diff = (vals[0] - vals[1]) / (2 * step)  # f is linear: exact but for rounding
        assert abs(diff - float(grad[r, h, c])) <= 2.0 ** -18 * 4


# -------------------------------------------------------------- gate norm --

def norm_reference(kind, x):
    """(norm(x), its error bound at fp32 sums)."""
    if kind == 0:
        return x, torch.zeros_like(x)
    mean = x.mean(-1, keepdim=True) if kind == 1 else torch.zeros_like(x[:, :1])
    r = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + 1e-6)
    n = (x - mean) * r
    return n, 2.0 ** -18 * (n.abs() + (r * x.abs().mean(-1, keepdim=True) if kind == 1 else 0))


class Case:
    def __init__(self, H, B, T, rows, d, norm, branch, types, weights, resid, parts="mid", spare=5, seed=0, vec_row=None):
        self.H, self.types, self.parts = H, types, parts
        self.B, self.T, self.d, self.norm, self.branch, self.resid = B, T, d, norm, branch, resid
        ut, yt, uo, ht, vt = types
        g = gen(seed + d)
        self.cap = sum(rows) + spare
        R = B * T + self.cap
        self.cu = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
        self.total = B * T + sum(rows)
        self.u = (torch.randn(R, d, generator=g, device="cuda") * 2 + 1.5).to(TYPES[ut])
        self.y = torch.randn(R, d, generator=g, device="cuda").to(TYPES[yt])
        self.u[self.total:], self.y[self.total:] = math.nan, math.nan
        self.vec_row = 3 * d if vec_row is None else vec_row
        self.mod = [torch.randn(B, max(3 * d, 8), generator=g, device="cuda").to(TYPES[vt]) for _ in range(2)]
        self.w = [torch.randn(3, d, generator=g, device="cuda").to(TYPES[vt]) for _ in range(2)]
        self.weights = weights
        first, last = parts == "in", parts == "out"
        self.vec = [H.NormVectors(gate=None if first else m[:, 2 * d:], scale=m[:, d:2 * d], shift=m[:, :d],
                                  w_branch=w[0] if weights else None, w_norm=w[1] if weights else None,
                                  b_norm=w[2] if weights else None) for m, w in zip(self.mod, self.w)]
        self.shape = H.NormShape(B=B, T=T, cap=self.cap, d=d, norm=norm, norm_branch=branch, resid_scale=resid, u_dtype=ut,
                                 y_dtype=yt, u_out_dtype=uo, h_dtype=ht, vec_dtype=vt, vec_row=self.vec_row)
        self.first, self.last, self.R = first, last, R

    def run(self, u_out=None, h=None, h_scale=None, u=None):
        u = self.u if u is None else u
        bt = self.B * self.T
        self.H.hilo_gate_norm(self.shape, self.vec[0] if self.T else None, self.vec[1], self.cu, u if self.T else None, u[bt:],
                              None if self.first else self.y, u_out, h, h_scale)

    def reference(self):
        """u', h and their error bounds (without the last rounding) over the rows that there are."""
        B, T, d, cu = self.B, self.T, self.d, self.cu.tolist()
        img = torch.empty(self.total, dtype=torch.long, device="cuda")
        stream = torch.ones(self.total, dtype=torch.long, device="cuda")
        for b in range(B):
            img[b * T:(b + 1) * T] = b
            img[B * T + cu[b]:B * T + cu[b + 1]] = b
        stream[:B * T] = 0
        at = img if self.vec_row else torch.zeros_like(img)
        mod = torch.stack([m.double()[:, :3 * d] for m in self.mod])[stream, at]
        shift, scale, gate = mod.split(d, -1)
        w = torch.stack([x.double() for x in self.w])[stream]
        u, e_u = self.u[:self.total].double(), 0.0
        if not self.first:
            z, e_z = norm_reference(self.branch, self.y[:self.total].double())
            if self.weights:
                z, e_z = z * w[:, 0], e_z * w[:, 0].abs()
            e_u = gate.abs() * e_z + 2.0 ** -22 * ((self.resid * u).abs() + (gate * z).abs())
            u = self.resid * u + gate * z
        n, e_n = norm_reference(self.norm, u)
        if not self.first:
            r = 1.0 if self.norm == 0 else 1 / torch.sqrt(u.var(-1, correction=0, keepdim=True) + 1e-6) if self.norm == 1 else \
                1 / torch.sqrt((u * u).mean(-1, keepdim=True) + 1e-6)
            e_n = e_n + 2 * r * (e_u + (e_u.mean(-1, keepdim=True) if self.norm else 0))
        b = 0.0
        if self.weights:
            n, e_n, b = n * w[:, 1], e_n * w[:, 1].abs(), w[:, 2]
        h = (n + b) * (1 + scale) + shift
        e_h = e_n * (1 + scale).abs() + 2.0 ** -21 * ((n.abs() + abs(b)) * (1 + scale).abs() + shift.abs())
        return u, e_u, h, e_h


NORM = [
    # B, T, rows, d, norm, branch, (u, y, u_out, h, vectors), weights, residual scale
    (1, 0, [1], 8, 1, 0, (F32, BF16, F32, BF16, BF16), 0, 1.0),
    (2, 3, [7, 0], 64, 2, 2, (BF16, F32, F32, F32, F32), 1, 0.5),
    (3, 5, [2, 9, 1], 248, 1, 1, (F32, F32, BF16, F16, BF16), 1, 1.0),
    (2, 1, [40, 11], 264, 2, 0, (BF16, BF16, BF16, BF16, F32), 0, -0.7),
    (1, 64, [300], 512, 1, 0, (F32, BF16, F32, F16, BF16), 0, 1.0),
    (4, 7, [1, 30, 0, 77], 1000, 1, 2, (BF16, BF16, F32, BF16, BF16), 1, 1.0),
    (2, 9, [500, 600], 1152, 2, 1, (F32, BF16, F32, F32, F32), 1, 0.3),
    (1, 2, [900], 2056, 1, 0, (F32, BF16, F32, BF16, BF16), 0, 1.0),
    (2, 77, [333, 129], 3072, 1, 2, (F32, BF16, F32, F16, BF16), 1, 1.0),
    (1, 0, [1000], 4096, 2, 1, (F32, F32, F32, F32, F32), 1, 1.0),
]


@pytest.mark.parametrize("parts", ["mid", "in", "out"])
@pytest.mark.parametrize("B,T,rows,d,norm,branch,types,weights,resid", NORM)
def test_gate_norm(H, B, T, rows, d, norm, branch, types, weights, resid, parts):
    c = Case(H, B, T, rows, d, norm, branch, types, weights, resid, parts)
    u_out = None if c.first else torch.full((c.R, d), math.nan, dtype=TYPES[types[2]], device="cuda")
    h = None if c.last else torch.full((c.R, d), math.nan, dtype=TYPES[types[3]], device="cuda")
    c.run(u_out, h)
    H.hilo_sync_status()
    u, e_u, hr, e_h = c.reference()
    for got, want, e in ((u_out, u, e_u), (h, hr, e_h)):
        if got is None:
            continue
        tol = e + half_step(got.dtype) * want.abs() + 1e-7
        assert bool(((got[:c.total].double() - want).abs() <= tol).all())
        assert bool(got[c.total:].isnan().all())


def test_gate_norm_in_place_shared_vectors_and_repeats(H):
    """u_out on u's own rows; one row of vectors for all images (vec_row 0); the same bits twice."""
    c = Case(H, 3, 4, [50, 3, 20], 640, 1, 1, (F32, BF16, F32, BF16, BF16), 1, 1.0, vec_row=0)
    u, e_u, hr, e_h = c.reference()
    first = torch.empty_like(c.u)
    h1, h2 = (torch.empty(c.R, c.d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.run(first, h1)
    buf = c.u.clone()
    c.run(buf, h2, u=buf)
    assert torch.equal(buf[:c.total], first[:c.total]) and torch.equal(h1[:c.total], h2[:c.total])
    assert bool(((buf[:c.total].double() - u).abs() <= e_u + 2.0 ** -24 * u.abs() + 1e-7).all())
    assert bool(((h2[:c.total].double() - hr).abs() <= e_h + 2.0 ** -8 * hr.abs() + 1e-7).all())


@pytest.mark.parametrize("d", [72, 512, 1024, 3072])
def test_gate_norm_e4m3(H, d):
    """Codes and scales are hilo_quantize_rows_e4m3's of the fp32 rows; a row of zeros has scale 1."""
    kw = dict(B=2, T=3, rows=[30, 11], d=d, norm=1, branch=0, weights=0, resid=1.0)
    a = Case(H, types=(F32, BF16, F32, F32, BF16), **kw)
    b = Case(H, types=(F32, BF16, F32, E4M3, BF16), **kw)
    for c in (a, b):
        for m in c.mod:
            m[0, :2 * d] = 0
            m[0, d:2 * d] = -1  # image 0: h = 0
    h = torch.full((a.R, d), math.nan, device="cuda")
    a.run(None, h)
    q = torch.full((a.R, d), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((a.R,), -1.0, device="cuda")
    b.run(None, q, s)
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    H.hilo_quantize_rows_e4m3(h, H.HILO_F32, a.total, d, q2, s2)
    assert torch.equal(q[:a.total], q2[:a.total]) and torch.equal(s[:a.total], s2[:a.total])
    assert bool((q[a.total:] == 0x55).all()) and bool((s[a.total:] == -1).all())
    assert float(s[0]) == 1.0 and bool((s[3:6] != 1.0).all())


def test_gate_norm_fp16_saturates(H):
    c = Case(H, 1, 0, [9], 128, 2, 0, (F32, BF16, F32, F16, F32), 0, 1.0, parts="in")
    c.mod[1][:, :128] = 1e6
    h = torch.empty(c.R, 128, dtype=torch.float16, device="cuda")
    c.run(None, h)
    assert bool((h[:9] == 65504).all())


def test_a_bad_row_stays_alone(H):
    """An infinity or NaN in one row leaves the others as they are."""
    c = Case(H, 1, 3, [200], 1152, 1, 2, (F32, BF16, F32, BF16, BF16), 0, 1.0)
    outs = []
    for bad in (False, True):
        if bad:
            c.u[17, 5], c.y[90, 1000], c.y[91, 3] = math.inf, math.nan, -math.inf
        u, h = torch.zeros_like(c.u), torch.zeros(c.R, c.d, dtype=torch.bfloat16, device="cuda")
        c.run(u, h)
        outs.append((u, h))
    keep = torch.ones(c.R, dtype=torch.bool, device="cuda")
    keep[[17, 90, 91]] = False
    assert all(torch.equal(x[keep], y[keep]) for x, y in zip(*outs))
    assert bool(outs[1][1][[17, 90, 91]].isnan().any(1).all())
