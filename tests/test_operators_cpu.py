"""What the conditioning, position and attention entry points refuse, before any device work: NULL, unaligned
and overlapping buffers, shapes outside the supported sets, workspaces that are too small. Nothing here needs a
GPU; the addresses are never dereferenced."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest

ARG, SHAPE, WORKSPACE = -1, -2, -4
A, U, O = 4096, 4100, 4104  # aligned; to 4 bytes only; to 8 bytes only


@pytest.fixture(scope="module")
def H():
    from paper_2606_13898_gb300 import build
    from paper_2606_13898_gb300 import hilo

    build.build()
    hilo.lib()
    return hilo


def refused(H, rc, code):
    assert rc == code, (rc, H.lib().hilo_last_error())
    assert H.lib().hilo_last_error() != b""


def ref(x):
    return ctypes.byref(x)


# -------------------------------------------------------------- attention --

def attn(H, **kw):
    base = dict(B=2, heads=8, kv_heads=2, head_dim=128, rows_q=300, rows_k=5000)
    return H.AttnShape(**{**base, **kw}).c()


def call_attn(H, s, cu_q=A, cu_k=A, q=A, k=A, v=A, out=A, ws=A, n=1 << 40):
    return H.lib().hilo_attention(ref(s), cu_q, cu_k, q, k, v, out, ws, n, None)


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE),
    (dict(kv_heads=-2), SHAPE), (dict(heads=129, kv_heads=1), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(dtype=1), ARG), (dict(dtype=7), ARG), (dict(causal=2), ARG), (dict(causal=-1), ARG), (dict(scale=-1.0), ARG),
    (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG), (dict(rows_q=-1), SHAPE), (dict(rows_k=-1), SHAPE),
    (dict(rows_q=(1 << 30) + 1), SHAPE), (dict(rows_k=(1 << 30) + 1), SHAPE),
    (dict(rows_q=1 << 30, heads=128, kv_heads=1), SHAPE),  # 2^30 tiles of one token each
    (dict(q_row=0), ARG), (dict(q_row=-1024), ARG), (dict(k_row=1028), ARG), (dict(v_head=4), ARG), (dict(k_head=0), ARG),
    (dict(q_head=1 << 39), ARG), (dict(out_row=1028), ARG),
    (dict(out_row=512), ARG),                 # rows of out inside one another's heads
    (dict(out_head=64), ARG),                 # heads of out inside one another
    (dict(out_row=128, out_head=128), ARG),
])
def test_attention_shapes(H, bad, code):
    s = attn(H, **bad)
    refused(H, call_attn(H, s), code)
    assert H.lib().hilo_attention_workspace_bytes(ref(s)) == 0
    with pytest.raises(H.HiloError):
        H.hilo_attention_workspace_bytes(H.AttnShape(**{**dict(B=2, heads=8, kv_heads=2, head_dim=128, rows_q=300, rows_k=5000),
                                                        **bad}))


@pytest.mark.parametrize("bad,code", [
    (dict(cu_q=None), ARG), (dict(cu_k=None), ARG), (dict(q=None), ARG), (dict(k=None), ARG), (dict(v=None), ARG),
    (dict(out=None), ARG), (dict(q=O), ARG), (dict(k=O), ARG), (dict(v=O), ARG), (dict(out=O), ARG), (dict(ws=O), ARG),
    (dict(cu_q=A + 2), ARG), (dict(cu_k=A + 1), ARG), (dict(ws=None), WORKSPACE), (dict(n=0), WORKSPACE)])
def test_attention_buffers(H, bad, code):
    refused(H, call_attn(H, attn(H), **bad), code)


def test_attention_workspace(H):
    L = H.lib()
    assert L.hilo_attention_workspace_bytes(None) == 0
    refused(H, L.hilo_attention(None, A, A, A, A, A, A, A, 1 << 40, None), ARG)
    s = attn(H)
    n = L.hilo_attention_workspace_bytes(ref(s))
    assert n > 1 << 20
    refused(H, call_attn(H, s, n=n - 1), WORKSPACE)
    # sequences too short to be cut need next to nothing; heads outermost in out is a layout like another
    assert 0 < L.hilo_attention_workspace_bytes(ref(attn(H, rows_k=128))) <= 64
    assert L.hilo_attention_workspace_bytes(ref(attn(H, out_row=128, out_head=300 * 128))) == n
    refused(H, call_attn(H, attn(H, out_row=128, out_head=299 * 128)), ARG)


def test_attention_scales_that_overflow_in_base_two(H):
    """The kernel works with scale * log2(e), which has to be finite as well."""
    for scale in (3.0e38, 2.0 ** 127):
        refused(H, call_attn(H, attn(H, scale=scale), n=0), ARG)
    for scale in (1.7e38, 1e-45, 0.0):
        refused(H, call_attn(H, attn(H, scale=scale), n=0), WORKSPACE)


def test_attention_dense_strides(H):
    s = attn(H)
    assert (s.q_row, s.q_head, s.k_row, s.k_head, s.v_row, s.v_head, s.out_row, s.out_head) == (1024, 128, 256, 128, 256, 128,
                                                                                             1024, 128)


# ------------------------------------------------------------------- rope --

def rope(H, **kw):
    base = dict(rows=10, heads=4, head_dim=128, dtype=0, axis_dims=(16, 56, 56))
    return H.RopeShape(**{**base, **kw}).c()


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(rows=-1), SHAPE), (dict(heads=0), SHAPE), (dict(heads=65537), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(head_dim=12), SHAPE), (dict(head_dim=264), SHAPE), (dict(axis_dims=(130,)), SHAPE),
    (dict(axis_dims=(64, 80)), SHAPE), (dict(axis_dims=(15, 17)), SHAPE), (dict(axis_dims=(0, 16)), SHAPE),
    (dict(axis_dims=(-16, 32)), SHAPE), (dict(axis_dims=(24,)), SHAPE), (dict(interleaved=2), ARG), (dict(per_axis=-1), ARG),
    (dict(theta=1.0), ARG), (dict(theta=math.inf), ARG), (dict(theta=math.nan), ARG), (dict(theta=-5.0), ARG),
    (dict(x_row=0), ARG), (dict(x_head=4), ARG), (dict(y_row=516), ARG), (dict(y_row=-512), ARG), (dict(y_head=1 << 39), ARG),
    (dict(y_row=128, y_head=128), ARG), (dict(y_row=256), ARG), (dict(dtype=1, x_row=514), ARG)])
def test_rope_shapes(H, bad, code):
    s = rope(H, **bad)
    refused(H, H.lib().hilo_rope(ref(s), A, A, None, 2 * A, None), code)


def test_rope_buffers(H):
    L, s = H.lib(), rope(H)
    for args in ((None, A, None, A), (A, None, None, A), (A, A, None, None), (O, A, None, A), (A, A, None, O), (A, A + 2, None, A),
                 (A, A, A + 1, A)):
        refused(H, L.hilo_rope(ref(s), *args, None), ARG)
    refused(H, L.hilo_rope(None, A, A, None, A, None), ARG)
    for bad in (dict(x_row=1024), dict(y_head=256, y_row=1024)):  # in place, with other strides
        refused(H, L.hilo_rope(ref(rope(H, **bad)), A, A, None, A, None), ARG)
    with pytest.raises(ValueError):
        rope(H, axis_dims=(16,) * 5)
    with pytest.raises(ValueError):
        rope(H, axis_dims=())


# -------------------------------------------------------------- gate norm --

def norm(H, **kw):
    base = dict(B=2, T=3, cap=10, d=64)
    return H.NormShape(**{**base, **kw}).c()


def call_norm(H, s, txt=None, img=None, cu=A, u_txt=A, u_img=A, y=A, u_out=2 * A, h=3 * A, h_scale=None):
    L = H.lib()
    vec = H.hilo_norm_vectors()
    return L.hilo_gate_norm(ref(s), ref(txt or vec), ref(img or vec), cu, u_txt, u_img, y, u_out, h, h_scale, None)


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), SHAPE), (dict(T=-1), SHAPE), (dict(cap=-1), SHAPE), (dict(B=1 << 20, T=1 << 12), SHAPE), (dict(d=0), SHAPE),
    (dict(d=60), SHAPE), (dict(d=4104), SHAPE), (dict(norm=3), ARG), (dict(norm=-1), ARG), (dict(norm_branch=3), ARG),
    (dict(vec_dtype=2), ARG), (dict(vec_row=-8), ARG), (dict(vec_row=68), ARG), (dict(eps=-1e-6), ARG), (dict(eps=math.nan), ARG),
    (dict(eps=math.inf), ARG), (dict(resid_scale=math.inf), ARG), (dict(u_dtype=2), ARG), (dict(y_dtype=3), ARG),
    (dict(u_out_dtype=2), ARG), (dict(h_dtype=4), ARG)])
def test_norm_shapes(H, bad, code):
    refused(H, call_norm(H, norm(H, **bad)), code)


def test_norm_buffers(H):
    s = norm(H)
    for bad in (dict(cu=None), dict(u_txt=None), dict(u_img=None), dict(u_txt=O), dict(u_img=O), dict(y=O), dict(u_out=O),
                dict(h=O), dict(u_out=None, h=None), dict(y=None)):
        refused(H, call_norm(H, s, **bad), ARG)
    L, vec = H.lib(), H.hilo_norm_vectors()
    refused(H, L.hilo_gate_norm(ref(s), None, ref(vec), A, A, A, A, 2 * A, 3 * A, None, None), ARG)
    refused(H, L.hilo_gate_norm(ref(s), ref(vec), None, A, A, A, A, 2 * A, 3 * A, None, None), ARG)
    refused(H, L.hilo_gate_norm(None, ref(vec), ref(vec), A, A, A, A, 2 * A, 3 * A, None, None), ARG)
    for n in ("gate", "scale", "shift", "w_branch", "w_norm", "b_norm"):
        v = H.hilo_norm_vectors(**{n: O})
        refused(H, call_norm(H, s, img=v), ARG)
        refused(H, call_norm(H, s, txt=v), ARG)
    refused(H, call_norm(H, norm(H, h_dtype=H.HILO_E4M3)), ARG)          # no scale
    refused(H, call_norm(H, norm(H, h_dtype=H.HILO_E4M3), h_scale=A + 2), ARG)
    # in place with another dtype
    refused(H, call_norm(H, norm(H, u_dtype=0, u_out_dtype=1), u_txt=2 * A), ARG)
    refused(H, call_norm(H, norm(H, u_dtype=0, u_out_dtype=1), u_img=2 * A + 6 * 64 * 4), ARG)


# -------------------------------------------------------------- positions --

def test_row_positions(H):
    L = H.lib()
    s = H.Shape(B=1, H=8, W=8, d=128, T=4).c()
    o = H.RowPositions().c()
    sp = H.hilo_split_out(*([A] * 5))
    refused(H, L.hilo_row_positions(None, ref(sp), ref(o), A, 64, None), ARG)
    refused(H, L.hilo_row_positions(ref(H.Shape(B=1, H=7, W=8, d=128).c()), ref(sp), ref(o), A, 64, None), SHAPE)
    refused(H, L.hilo_row_positions(ref(H.Shape(B=1, H=8, W=8, d=128, T=-1).c()), ref(sp), ref(o), A, 64, None), SHAPE)
    refused(H, L.hilo_row_positions(ref(s), None, ref(o), A, 64, None), ARG)
    refused(H, L.hilo_row_positions(ref(s), ref(H.hilo_split_out()), ref(o), A, 64, None), ARG)
    for args in ((None, A, 64), (ref(o), None, 64), (ref(o), A, -1), (ref(o), A + 2, 64)):
        refused(H, L.hilo_row_positions(ref(s), ref(sp), *args, None), ARG)


# ------------------------------------------------------ conditioned block --

def test_conditioned_block(H):
    L = H.lib()
    sh = H.Shape(B=1, H=8, W=8, d=256, T=4, heads=2, mlp=1)
    w = H.hilo_block_weights(*(H.hilo_stream_weights(*([A] * 8)) for _ in range(2)))
    none = H.NormVectors()
    good = dict(vec_row=0, axis_dims=(16, 56, 56))
    n = L.hilo_block_workspace_bytes(ref(sh.c()), 64)

    def call(mod, pos=A, n_img=None, shape=sh, ws=n):
        m = None if mod is None else ref(H.BlockMod(none, none, none, none, **{**good, **mod}).c(pos))
        return L.hilo_block_forward_mod(ref(shape.c()), ref(w), m, A, 64, A, A, 0, n_img, A, A, ws, None)

    refused(H, call(None), ARG)
    for bad in (dict(norm=0), dict(norm=5), dict(norm_branch=4), dict(vec_dtype=2), dict(vec_row=4), dict(eps=math.nan),
                dict(resid_scale=math.nan), dict(theta=0.5), dict(interleaved=3)):
        refused(H, call(bad), ARG)
    for bad in (dict(axis_dims=(16, 64, 64)), dict(axis_dims=(8, 4)), dict(axis_dims=(3, 13))):
        refused(H, call(bad), SHAPE)
    refused(H, call({}, pos=A + 2), ARG)
    refused(H, call({}, n_img=A + 2), ARG)
    refused(H, call({}, shape=H.Shape(B=1, H=8, W=8, d=256, T=4, heads=3, mlp=1)), SHAPE)
    refused(H, call({}, ws=n - 1), WORKSPACE)
    bad = H.BlockMod(none, none, H.NormVectors(gate=O), none, **good).c(A)
    refused(H, L.hilo_block_forward_mod(ref(sh.c()), ref(w), ref(bad), A, 64, A, A, 0, None, A, A, n, None), ARG)
    with pytest.raises(ValueError):
        H.BlockMod(none, none, none, none, **good).c(None)
    with pytest.raises(ValueError):
        H.BlockMod(none, none, none, none, vec_row=0).c(A)


def test_structs_follow_their_vectors(H):
    """The structs carry the present addresses: a replaced vector or its replaced memory gives a rebuilt struct, and two
    calls with the same conditioning have structs of their own."""
    import torch

    v = H.NormVectors(gate=torch.empty(8), scale=torch.empty(8))
    c = v.c()
    assert v.c() is c and c.gate == v.gate.data_ptr() and c.shift is None
    v.gate = torch.empty(8)
    assert v.c() is not c and v.c().gate == v.gate.data_ptr()
    m = H.BlockMod(v, v, v, v, vec_row=64, axis_dims=(16, 16))
    a, b = m.c(A), m.c(2 * A)
    assert a.pos == A and b.pos == 2 * A and a.rot.axes == 2 and b.img_mlp.gate == v.gate.data_ptr()
    v.gate.data = torch.empty(8)  # the same tensor object over other memory
    assert v.c().gate == v.gate.data_ptr() and m.c(A).txt_attn.gate == v.gate.data_ptr()
    m.txt_attn = H.NormVectors(shift=torch.empty(8))
    assert m.c(A).txt_attn.gate is None and m.c(A).txt_attn.shift == m.txt_attn.shift.data_ptr()


SANITIZED = r"""
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include "hilo.h"

static int calls = 0;
#define REFUSED(expr) do { int rc_ = (expr); ++calls; if (rc_ == HILO_OK || !strlen(hilo_last_error())) { \
    printf("not refused: %s\n", #expr); return 1; } } while (0)

int main(void) {
  void* A = (void*)(uintptr_t)4096;   /* never dereferenced */
  int32_t big[] = {INT32_MIN, -1, 0, 1, 7, 64, 128, 4096, 65536, 1 << 30, INT32_MAX};
  int64_t far[] = {INT64_MIN, -8, 0, 8, 12, 512, (int64_t)1 << 38, ((int64_t)1 << 39) - 8, INT64_MAX};
  const int nb = sizeof big / sizeof big[0], nf = sizeof far / sizeof far[0];
  size_t total = 0;
  int i, j, k;
  for (i = 0; i < nb; ++i) for (j = 0; j < nb; ++j) for (k = 0; k < nf; ++k) {
    hilo_attn_shape a = {big[i], big[j], big[(i + j) % nb], k & 1 ? 64 : 128, i & 1, HILO_BF16, big[(j + k) % nb], big[k % nb],
                         0.0f, far[k], far[(k + 1) % nf], far[(k + 2) % nf], 128, far[k], 128, far[(k + i) % nf], far[(k + j) % nf]};
    hilo_rope_shape r = {big[i], big[j], big[(i + k) % nb], HILO_BF16, far[k], far[(k + i) % nf], far[(k + j) % nf], 512,
                         {1 + k % 4, {big[i], big[j], 16, 16}, 0, 1, 1e4}};
    hilo_norm_shape n = {big[i], big[j], big[k % nb], big[(i + 3) % nb], 1, 0, 1, 0, 1, 0, 0, 1e-6f, 1.0f, far[k]};
    hilo_norm_vectors v;
    hilo_shape s = {big[i], 8, 8, 256, big[j], 2, 1, 1, 0};
    hilo_split_out sp = {A, A, A, A, A};
    hilo_positions_origin o = {0, 0, 0, 0, 0};
    memset(&v, 0, sizeof v);
    hilo_attn_shape b = {1 + k, 8, 2, 128, 1, HILO_F16, i < 4 ? 1 << 24 : 5, j < 4 ? 1 << 30 : 7, 0.5f, 1024, 128, 256, 128, 256,
                         128, far[(k + i) % nf], far[(k + j) % nf]};
    total += hilo_attention_workspace_bytes(&a) + hilo_attention_workspace_bytes(&b);
    REFUSED(hilo_attention(&b, A, A, A, A, A, A, NULL, 0, NULL));
    r.rows = INT32_MAX;
    r.heads = 65536;
    REFUSED(hilo_attention(&a, A, A, A, A, A, A, NULL, 0, NULL));
    REFUSED(hilo_rope(&r, A, A, NULL, NULL, NULL));
    r.rot.theta = -1.0;
    REFUSED(hilo_rope(&r, A, A, NULL, A, NULL));
    REFUSED(hilo_gate_norm(&n, &v, &v, A, A, A, NULL, A, A, NULL, NULL));
    REFUSED(hilo_row_positions(&s, &sp, &o, (float*)A, -1 - i, NULL));
  }
  REFUSED(hilo_block_forward_mod(NULL, NULL, NULL, NULL, 0, NULL, NULL, 0, NULL, NULL, NULL, 0, NULL));
  printf("%d %d\n", calls, total > 0);
  return 0;
}
"""


def test_extreme_arguments_under_sanitizers(tmp_path):
    """Every combination of extreme counts and strides ends in a status and a message, without undefined arithmetic."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    probe = subprocess.run([gcc, "-fsanitize=address", "-fsanitize=undefined", "-x", "c", "-", "-o", str(tmp_path / "probe")],
                           input="int main(void){return 0;}", capture_output=True, text=True)
    if probe.returncode != 0:
        pytest.skip("the C compiler has no sanitizer runtime")
    from paper_2606_13898_gb300 import build
    lib = os.path.dirname(build.build(variant="asan"))
    src, exe = tmp_path / "host.c", tmp_path / "host"
    src.write_text(SANITIZED)
    r = subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-fsanitize=address", "-fsanitize=undefined",
                        "-fno-omit-frame-pointer", "-I", build.INCLUDE, str(src), "-o", str(exe), "-L", lib, "-lhilo",
                        f"-Wl,-rpath,{lib}"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "runtime error" not in r.stderr, r.stdout[-2000:] + r.stderr[-4000:]
    calls, some = (int(x) for x in r.stdout.split())
    assert calls > 5000 and some == 1
