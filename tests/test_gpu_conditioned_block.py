"""The conditioned block and the layers that the new operators make together, against 64 bits.

hilo_block_forward_mod rounds what hilo_block_forward rounds (16-bit GEMM
operands, attention inputs and probabilities) and the sub-layers' outputs once
more to bf16, half a step (2^-8) of a branch whose own operands were rounded
by as much; its tolerance is that of the other block tests (max-abs 2e-2,
rel-L2 1e-2).
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2606_13898_gb300 import inputs as I

from .gpu_helpers import assert_block_close, lib_ready

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def rot(x, pos, dims, theta, interleaved, per_axis):
    """x [rows, heads, hd] in 64 bits."""
    D, i, out = sum(dims), 0, x.clone()
    for a, n in enumerate(dims):
        for j in range(n // 2):
            f = theta ** (-2.0 * j / n) if per_axis else theta ** (-2.0 * i / D)
            t = (pos[:, a].double() * f)[:, None]
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + D // 2)
            out[..., lo], out[..., hi] = x[..., lo] * t.cos() - x[..., hi] * t.sin(), x[..., lo] * t.sin() + x[..., hi] * t.cos()
            i += 1
    return out


def norm(x, kind):
    if kind == 0:
        return x
    if kind == 1:
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)


def weights(w, d):
    def t(a):
        return torch.from_numpy(I.bf16_bits_to_f32(a)).double().cuda()
    return [{f: t(getattr(getattr(w, s), f)) for f in ("w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2")
             if getattr(getattr(w, s), f) is not None} for s in ("txt", "img")]


def vectors(H, d, B, seed, wide=False):
    """BlockMod's four NormVectors over one product per stream: six rows of d per image."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    mods = [(0.4 * torch.randn(B, 6 * d, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2)]
    ws = [(1 + 0.2 * torch.randn(6, d, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2)]
    vec = {}
    for s, m, w in zip(("txt", "img"), mods, ws):
        for k, part in enumerate(("attn", "mlp")):
            c = [m[:, (3 * k + i) * d:(3 * k + i + 1) * d] for i in range(3)]
            vec[f"{s}_{part}"] = H.NormVectors(shift=c[0], scale=c[1], gate=c[2], w_branch=w[3 * k] if wide else None,
                                               w_norm=w[3 * k + 1] if wide else None, b_norm=w[3 * k + 2] if wide else None)
    return vec, mods, ws


def block_reference(w, u, n_txt, cu, T, heads, mods, ws, wide, kind, branch, resid, pos, axes, mlp, n_img=None):
    """The conditioned block in 64 bits; u [rows, d], text rows first."""
    d, B = u.shape[1], len(cu) - 1
    rows = u.shape[0]
    stream = (torch.arange(rows, device="cuda") >= n_txt).long()
    img = torch.empty(rows, dtype=torch.long, device="cuda")
    joint = []
    for b in range(B):
        img[b * T:(b + 1) * T] = b
        img[n_txt + cu[b]:n_txt + cu[b + 1]] = b
        joint.append(torch.cat([torch.arange(b * T, (b + 1) * T), torch.arange(n_txt + cu[b], n_txt + cu[b + 1])]).cuda())
    mod = torch.stack([m.double() for m in mods])[stream, img].view(rows, 6, d)
    wv = torch.stack([x.double() for x in ws])[stream]

    def linear(x, name):
        return torch.cat([x[:n_txt] @ w[0]["w_" + name].T + w[0]["b_" + name], x[n_txt:] @ w[1]["w_" + name].T + w[1]["b_" + name]])

    def before(x, k):
        h = norm(x, kind)
        if wide:
            h = h * wv[:, 3 * k + 1] + wv[:, 3 * k + 2]
        return h * (1 + mod[:, 3 * k + 1]) + mod[:, 3 * k]

    def after(x, y, k):
        z = norm(y, branch)
        if wide:
            z = z * wv[:, 3 * k]
        return resid * x + mod[:, 3 * k + 2] * z

    q, k, v = linear(before(u, 0), "qkv").view(rows, 3, heads, d // heads).unbind(1)
    if pos is not None:
        q, k = (rot(x, pos[:rows], **axes) for x in (q, k))
    o = torch.zeros_like(q)
    size = torch.ones(rows, dtype=torch.float64, device="cuda")
    if n_img is not None:
        size[n_txt:] = n_img[:rows - n_txt].double()
    for at in joint:
        s = torch.einsum("ihc,jhc->hij", q[at], k[at]) / math.sqrt(d // heads) + size[at].log()
        o[at] = torch.einsum("hij,jhc->ihc", s.softmax(-1), v[at])
    u = after(u, linear(o.reshape(rows, d), "o"), 0)
    if mlp:
        u = after(u, linear(torch.nn.functional.gelu(linear(before(u, 1), "1"), approximate="tanh"), "2"), 1)
    return u


BLOCKS = [
    # B, T, image rows, d, heads, mlp, norm, norm_branch, weights, residual scale, axes, interleaved, per_axis
    (1, 64, [300], 512, 8, 1, 1, 0, False, 1.0, (16, 24, 24), 1, 1),
    (3, 5, [40, 0, 257], 256, 2, 1, 2, 2, True, 0.8, (16, 56, 56), 0, 0),
    (2, 0, [130, 77], 384, 3, 0, 1, 1, True, 1.0, None, 0, 0),
    (1, 33, [129], 1024, 8, 1, 1, 0, True, 1.0, (44, 42, 42), 1, 1),
]


@pytest.mark.parametrize("B,T,lens,d,heads,mlp,kind,branch,wide,resid,axes,inter,per_axis", BLOCKS)
@pytest.mark.parametrize("prop", [False, True])
def test_conditioned_block(H, B, T, lens, d, heads, mlp, kind, branch, wide, resid, axes, inter, per_axis, prop):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cap, n_txt = int(cu[-1]) + 30, B * T
    w = I.make_weights(d, bool(mlp), seed=d + B)
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    u = torch.randn(n_txt + cap, d, generator=g, device="cuda").to(torch.bfloat16)
    vec, mods, ws = vectors(H, d, B, seed=3, wide=wide)
    mod = H.BlockMod(vec_row=6 * d, norm=kind, norm_branch=branch, resid_scale=resid, axis_dims=axes, interleaved=inter,
                     per_axis=per_axis, **vec)
    pos = None if axes is None else 20 * torch.randn(n_txt + cap, 3, generator=g, device="cuda")
    n_img = (1 + torch.randint(0, 4, (cap,), generator=g, device="cuda")).float() if prop else None
    sh = H.Shape(B=B, H=32, W=32, d=d, T=T, heads=heads, mlp=mlp)
    dw, cud = H.DeviceWeights.from_host(w), torch.from_numpy(cu).cuda()
    ws_bytes = H.hilo_block_workspace_bytes(sh, cap)
    scratch = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    out = torch.full((n_txt + cap, d), math.nan, device="cuda")
    H.hilo_block_forward_mod(sh, dw, mod, pos, cud, cap, u if T else None, u[n_txt:], H.HILO_BF16, n_img, out, scratch, ws_bytes)
    H.hilo_sync_status()
    rows = n_txt + int(cu[-1])
    ref = block_reference(weights(w, d), u[:rows].double(), n_txt, cu.tolist(), T, heads, mods, ws, wide, kind, branch, resid,
                          pos, None if axes is None else dict(dims=axes, theta=1e4, interleaved=inter, per_axis=per_axis), mlp,
                          n_img)
    assert_block_close(out[:rows].cpu().numpy(), ref.cpu().numpy(), "conditioned block")
    assert bool(out[rows:].isnan().all())
    # fp32 rows, in place
    buf = u.float()
    H.hilo_block_forward_mod(sh, dw, mod, pos, cud, cap, buf, buf[n_txt:], H.HILO_F32, n_img, buf, scratch, ws_bytes)
    assert torch.equal(buf[:rows], out[:rows])


def test_without_conditioning_it_is_the_plain_block(H):
    B, T, d, heads, lens = 2, 17, 512, 4, [200, 61]
    cu = torch.tensor([0, 200, 261], dtype=torch.int32, device="cuda")
    cap, n_txt = 261, B * T
    dw = H.DeviceWeights.from_host(I.make_weights(d, True, seed=1))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    u = torch.randn(n_txt + cap, d, generator=g, device="cuda").to(torch.bfloat16)
    sh = H.Shape(B=B, H=32, W=32, d=d, T=T, heads=heads, mlp=1)
    nb = H.hilo_block_workspace_bytes(sh, cap)
    scratch = torch.empty(nb, dtype=torch.uint8, device="cuda")
    none = H.NormVectors()
    mod = H.BlockMod(none, none, none, none, vec_row=0)
    a, b = (torch.empty(n_txt + cap, d, device="cuda") for _ in range(2))
    H.hilo_block_forward(sh, dw, cu, cap, u, u[n_txt:], H.HILO_BF16, a, scratch, nb)
    H.hilo_block_forward_mod(sh, dw, mod, None, cu, cap, u, u[n_txt:], H.HILO_BF16, None, b, scratch, nb)
    H.hilo_sync_status()
    assert_block_close(b.cpu().numpy(), a.double().cpu().numpy())


def test_hot_path_with_conditioning(H):
    """score, split, pack, positions, two conditioned blocks, unpack: eagerly and from a captured graph."""
    wl = I.tiny_layer(mlp=True)
    batch = I.make_batch(wl)
    ws = [I.make_weights(wl.d, True, seed=s) for s in (1, 2)]
    sh = H.Shape(B=wl.B, H=wl.H, W=wl.W, d=wl.d, T=wl.T, heads=wl.heads, mlp=1, levels=wl.levels)
    hp = H.HotPath(sh, [H.DeviceWeights.from_host(w) for w in ws])
    axes = dict(axis_dims=(16, 24, 24), interleaved=1, per_axis=1)
    vecs = [vectors(H, wl.d, wl.B, seed=s) for s in (5, 6)]
    origin = H.RowPositions(t_img=1.0, h0=-16.0, w0=-16.0, txt0=16.0, txt_step=1.0)
    hp.enable_mod([H.BlockMod(vec_row=6 * wl.d, **v[0], **axes) for v in vecs], origin)
    x, text = H.bf16_from_bits(batch.x), H.bf16_from_bits(batch.text)
    mask, kk, km = (torch.from_numpy(a).cuda() for a in (batch.mask, batch.k_keep, batch.k_mid))
    hp.run(x, text, mask, kk, km, mod=True)
    H.hilo_sync_status()
    cu = hp.split.cu_img.tolist()
    n_txt = wl.B * wl.T
    rows = n_txt + cu[-1]
    u = torch.cat([text.reshape(n_txt, wl.d), hp.packed[:cu[-1]]]).double()
    for w, (_, mods, wv) in zip(ws, vecs):
        u = block_reference(weights(w, wl.d), u, n_txt, cu, wl.T, wl.heads, mods, wv, False, 1, 0, 1.0, hp.pos[:rows],
                            dict(dims=(16, 24, 24), theta=1e4, interleaved=1, per_axis=1), 1)
    # the second block's inputs carry the first one's error: twice the tolerance of one block
    assert_block_close(hp.out[:rows].cpu().numpy() / 2, u.cpu().numpy() / 2)
    tok = hp.split.tok_row.long()
    assert torch.equal(hp.y.view(-1, wl.d), hp.out_img[tok])
    want = hp.y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hp.run(x, text, mask, kk, km, mod=True)
    hp.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(hp.y, want)
    with pytest.raises(ValueError):
        hp.run(x, text, mask, kk, km, mod=True, fp8=True)
    # enabled again, the path keeps the positions that the graph writes
    pos = hp.pos
    hp.enable_mod(hp.mods, H.RowPositions(t_img=2.0))
    assert hp.pos is pos
    with pytest.raises(ValueError):
        hp.enable_mod(hp.mods[:1], origin)
    with pytest.raises(ValueError):
        H.HotPath(sh, hp.weights).run(x, text, mask, kk, km, mod=True)


def test_prompt_layer(H):
    """A causal layer with grouped heads over packed prompts, as makes the text rows: norm, product, rotation of
    the q and k heads in place, attention on the product's columns, product, residual and norm."""
    lens, d, heads, kv, hd = [130, 1, 61, 300], 512, 8, 2, 64
    n, cols = sum(lens), (heads + 2 * kv) * hd
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    u = torch.randn(n, d, generator=g, device="cuda").to(torch.bfloat16)
    w_qkv = (0.05 * torch.randn(cols, d, generator=g, device="cuda")).to(torch.bfloat16)
    w_o = (0.05 * torch.randn(d, heads * hd, generator=g, device="cuda")).to(torch.bfloat16)
    gain = (1 + 0.1 * torch.randn(2, d, generator=g, device="cuda")).to(torch.bfloat16)
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(m, device="cuda") for m in lens]).float()[:, None].contiguous()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    B = len(lens)
    ns = H.NormShape(B=B, T=0, cap=n, d=d, norm=H.HILO_NORM_RMS, u_dtype=H.HILO_BF16)
    h = torch.empty(n, d, **bf)
    H.hilo_gate_norm(ns, None, H.NormVectors(w_norm=gain[0]), cu, None, u, None, None, h, None)
    qkv = h @ w_qkv.T
    rs = H.RopeShape(rows=n, heads=heads + kv, head_dim=hd, dtype=H.HILO_BF16, axis_dims=(64,), interleaved=0, x_row=cols,
                     x_head=hd, y_row=cols, y_head=hd)
    H.hilo_rope(rs, qkv, pos, None, qkv)
    q, k, v = qkv.unflatten(1, (-1, hd)).split([heads, kv, kv], 1)
    sh = H.AttnShape(B=B, heads=heads, kv_heads=kv, head_dim=hd, rows_q=n, rows_k=n, q_row=cols, q_head=hd, k_row=cols, k_head=hd,
                     v_row=cols, v_head=hd)
    nb = H.hilo_attention_workspace_bytes(sh)
    a = torch.empty(n, heads * hd, **bf)
    H.hilo_attention(sh, cu, cu, q, k, v, a, torch.empty(nb, dtype=torch.uint8, device="cuda"), nb)
    y = a @ w_o.T
    u2, h2 = torch.empty(n, d, device="cuda"), torch.empty(n, d, **bf)
    H.hilo_gate_norm(ns, None, H.NormVectors(w_norm=gain[1]), cu, None, u, y, u2, h2, None)
    H.hilo_sync_status()
    ud = u.double()
    qkv_r = (norm(ud, 2) * gain[0].double()) @ w_qkv.double().T
    x = qkv_r.view(n, -1, hd)
    qk = rot(x[:, :heads + kv], pos, (64,), 1e4, 0, 1)
    o = torch.zeros(n, heads, hd, dtype=torch.float64, device="cuda")
    for b in range(B):
        at = slice(int(cu[b]), int(cu[b + 1]))
        kk, vv = (t.repeat_interleave(heads // kv, 1) for t in (qk[at, heads:], x[at, heads + kv:]))
        s = torch.einsum("ihc,jhc->hij", qk[at, :heads], kk) / 8
        s = s.masked_fill(torch.ones_like(s[0]).triu(1).bool(), -math.inf)
        o[at] = torch.einsum("hij,jhc->ihc", s.softmax(-1), vv)
    u_r = ud + o.reshape(n, -1) @ w_o.double().T
    # five roundings to bf16 on the way (h, qkv, rotated, a, y), each half a step of 2^-8 of a branch whose size
    # is about u's own: below 1e-2 together in the norm of the whole
    rel = float((u2.double() - u_r).norm() / u_r.norm())
    assert rel <= 1e-2, rel
    h_r = norm(u_r, 2) * gain[1].double()
    assert float((h2.double() - h_r).norm() / h_r.norm()) <= 1e-2 + 2.0 ** -8


CAPTURED = r"""
import torch
from paper_2606_13898_gb300 import hilo as H
n, d = 300, 512
u = torch.randn(n, d, device="cuda")
h = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
out = torch.empty_like(h)
pos = torch.arange(n, device="cuda").float()[:, None].contiguous()
cu = torch.tensor([0, 100, n], dtype=torch.int32, device="cuda")
ns = H.NormShape(B=2, T=0, cap=n, d=d, norm=H.HILO_NORM_RMS)
rs = H.RopeShape(rows=n, heads=8, head_dim=64, dtype=H.HILO_BF16, axis_dims=(64,))
sh = H.AttnShape(B=2, heads=8, kv_heads=8, head_dim=64, rows_q=n, rows_k=n)
nb = H.hilo_attention_workspace_bytes(sh)
ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()


def layer():
    H.hilo_gate_norm(ns, None, H.NormVectors(), cu, None, u, None, None, h, None)
    H.hilo_rope(rs, h, pos, None, h)
    H.hilo_attention(sh, cu, cu, h, h, h, out, ws, nb)


graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):  # the process's first calls of these kernels
    layer()
out.zero_()
graph.replay()
torch.cuda.synchronize()
got = out.clone()
layer()
H.hilo_sync_status()
assert torch.equal(got, out) and bool(out.isfinite().all()) and float(out.float().abs().max()) > 0.1
"""


def test_first_calls_in_a_capture(H):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CAPTURED], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
