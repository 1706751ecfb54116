"""What the 8-bit products with a scale per 128, their quantisation and group norm refuse, before any device work. Nothing
here needs a GPU; the addresses are never dereferenced."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest

ARG, SHAPE, WORKSPACE = -1, -2, -4
A, U, O = 4096, 4100, 4104  # aligned; to 4 bytes only; to 8 bytes only
FAR = 1 << 39


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


# ------------------------------------------------------------ quantisation --

def call_quant(H, src=A, n_rows=A, dst=A, scale=A, **kw):
    s = H.Quant128Shape(**{**dict(rows=300, cols=4096, dtype=0), **kw}).c()
    return H.lib().hilo_quantize_e4m3_128(ref(s), src, n_rows, dst, scale, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), ARG), (dict(dtype=-1), ARG), (dict(tile=2), ARG), (dict(tile=-1), ARG), (dict(rows=-1), SHAPE),
    (dict(rows=(1 << 30) + 1, scale_ld=1 << 31), SHAPE), (dict(cols=0), SHAPE), (dict(cols=8), SHAPE), (dict(cols=-16), SHAPE),
    (dict(cols=4100), SHAPE), (dict(cols=(1 << 30) + 16), SHAPE), (dict(cols=0x7ffffff0), SHAPE),
    (dict(rows=1 << 30, cols=4096, scale_ld=1 << 31), SHAPE),
    (dict(src_row=4080), ARG), (dict(src_row=4104), ARG), (dict(src_row=FAR), ARG), (dict(src_row=-4096), ARG),
    (dict(dst_row=4080), ARG), (dict(dst_row=4100), ARG), (dict(dst_row=FAR), ARG), (dict(scale_ld=299), ARG),
    (dict(scale_ld=-1), ARG), (dict(scale_ld=FAR), ARG), (dict(tile=1, scale_ld=31), ARG)])
def test_quantisation_shapes(H, bad, code):
    refused(H, call_quant(H, **bad), code)


@pytest.mark.parametrize("bad", [dict(src=None), dict(dst=None), dict(scale=None), dict(src=O), dict(dst=O), dict(scale=A + 2),
                                 dict(n_rows=A + 1)])
def test_quantisation_buffers(H, bad):
    refused(H, call_quant(H, **bad), ARG)
    refused(H, H.lib().hilo_quantize_e4m3_128(None, A, None, A, A, None), ARG)


# ---------------------------------------------------------------- products --

def call_gemm(H, a=A, a_scale=A, w=A, w_scale=A, bias=None, n_rows=None, out=A, **kw):
    s = H.Gemm128Shape(**{**dict(rows=300, k=4096, n=1024), **kw}).c()
    return H.lib().hilo_gemm_e4m3_128(ref(s), a, a_scale, w, w_scale, bias, n_rows, out, None)


def call_gated(H, a=A, a_scale=A, w_gate=A, s_gate=A, w_up=A, s_up=A, b_gate=None, b_up=None, n_rows=None, out=A, out_scale=A, **kw):
    s = H.Gemm128Shape(**{**dict(rows=300, k=4096, n=1024, act=H.HILO_ACT_SILU, out_dtype=H.HILO_E4M3), **kw}).c()
    return H.lib().hilo_gated_e4m3_128(ref(s), a, a_scale, w_gate, s_gate, w_up, s_up, b_gate, b_up, n_rows, out, out_scale, None)


@pytest.mark.parametrize("bad,code", [
    (dict(act=3), ARG), (dict(act=-1), ARG), (dict(out_dtype=4), ARG), (dict(out_dtype=-1), ARG), (dict(rows=-1), SHAPE),
    (dict(rows=(1 << 30) + 1), SHAPE), (dict(k=0), SHAPE), (dict(k=-16), SHAPE), (dict(k=4104), SHAPE), (dict(k=0x7ffffff0), SHAPE),
    (dict(n=0), SHAPE), (dict(n=1000), SHAPE), (dict(n=-1024), SHAPE), (dict(n=0x7ffffff0), SHAPE),
    (dict(rows=1 << 30, n=1 << 14), SHAPE), (dict(a_row=4080), ARG), (dict(a_row=4104), ARG), (dict(a_row=FAR), ARG),
    (dict(w_row=4080), ARG), (dict(w_row=4104), ARG), (dict(w_row=-4096), ARG), (dict(out_row=1008), ARG), (dict(out_row=1032), ARG),
    (dict(out_row=FAR), ARG), (dict(a_scale_ld=299), ARG), (dict(a_scale_ld=FAR), ARG), (dict(w_scale_ld=31), ARG),
    (dict(w_scale_ld=FAR), ARG)])
def test_product_shapes(H, bad, code):
    refused(H, call_gemm(H, **bad), code)
    refused(H, call_gated(H, **bad), code)


def test_what_only_one_of_them_takes(H):
    for act in (H.HILO_ACT_SILU, H.HILO_ACT_GELU):
        refused(H, call_gemm(H, act=act), ARG)
    refused(H, call_gated(H, act=H.HILO_ACT_NONE), ARG)
    refused(H, call_gemm(H, out_dtype=H.HILO_E4M3), ARG)
    for bad in (dict(out_scale_ld=299), dict(out_scale_ld=FAR), dict(out_scale=None), dict(out_scale=A + 2)):
        refused(H, call_gated(H, **bad), ARG)


@pytest.mark.parametrize("bad", [dict(a=None), dict(a_scale=None), dict(out=None), dict(a=O), dict(out=O), dict(a_scale=A + 2),
                                 dict(n_rows=A + 2)])
def test_product_buffers(H, bad):
    refused(H, call_gemm(H, **bad), ARG)
    refused(H, call_gated(H, **bad), ARG)


def test_product_weights(H):
    for bad in (dict(w=None), dict(w_scale=None), dict(w=O), dict(w_scale=A + 2), dict(bias=A + 1)):
        refused(H, call_gemm(H, **bad), ARG)
        refused(H, call_gemm(H, rows=0, **bad), ARG)
    for bad in (dict(w_gate=None), dict(w_up=None), dict(s_gate=None), dict(s_up=None), dict(w_gate=O), dict(w_up=O),
                dict(s_gate=A + 2), dict(s_up=A + 1), dict(b_gate=A + 1), dict(b_up=A + 1)):
        refused(H, call_gated(H, **bad), ARG)
    L = H.lib()
    refused(H, L.hilo_gemm_e4m3_128(None, A, A, A, A, None, None, A, None), ARG)
    refused(H, L.hilo_gated_e4m3_128(None, A, A, A, A, A, A, None, None, None, A, A, None), ARG)


# -------------------------------------------------------------- group norm --

def norm(H, **kw):
    return H.GroupNormShape(**{**dict(B=2, rows=300, d=512), **kw})


def call_norm(H, vec=None, x=A, y=2 * A, y_scale=None, ws=A, n=1 << 40, **kw):
    s = norm(H, **kw).c()
    return H.lib().hilo_group_norm(ref(s), None if vec is None else ref(vec), x, y, y_scale, ws, n, None)


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), SHAPE), (dict(B=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(B=1 << 16, rows=1 << 15), SHAPE),
    (dict(B=0x7fffffff, rows=0x7fffffff), SHAPE), (dict(d=0), SHAPE), (dict(d=8, groups=8), SHAPE), (dict(d=520, groups=8), SHAPE),
    (dict(d=8208, groups=16), SHAPE), (dict(d=-512), SHAPE), (dict(groups=0), SHAPE), (dict(groups=-32), SHAPE), (dict(groups=33), SHAPE),
    (dict(groups=1024), SHAPE), (dict(act=3), ARG), (dict(act=-1), ARG), (dict(x_dtype=3), ARG), (dict(x_dtype=-1), ARG),
    (dict(y_dtype=4), ARG), (dict(vec_dtype=2), ARG), (dict(vec_dtype=3), ARG), (dict(eps=-1e-6), ARG), (dict(eps=math.nan), ARG),
    (dict(eps=math.inf), ARG), (dict(x_row=496), ARG), (dict(x_row=520), ARG), (dict(x_row=FAR), ARG), (dict(y_row=496), ARG),
    (dict(y_row=516), ARG), (dict(y_row=-512), ARG), (dict(vec_row=-8), ARG), (dict(vec_row=516), ARG), (dict(vec_row=FAR), ARG),
    (dict(y_dtype=3, y_scale_ld=599), ARG), (dict(y_dtype=3, y_scale_ld=FAR), ARG)])
def test_group_norm_shapes(H, bad, code):
    refused(H, call_norm(H, **bad), code)
    assert H.lib().hilo_group_norm_workspace_bytes(ref(norm(H, **bad).c())) == 0
    with pytest.raises(H.HiloError):
        H.hilo_group_norm_workspace_bytes(norm(H, **bad))


def test_group_norm_buffers(H):
    L = H.lib()
    for bad in (dict(x=None), dict(y=None), dict(x=O), dict(y=O), dict(ws=O), dict(y_dtype=3), dict(y_dtype=3, y_scale=A + 2),
                dict(y_dtype=1, y=A), dict(y=A, y_row=528), dict(x_dtype=2, y=A)):
        refused(H, call_norm(H, **bad), ARG)
    for n in ("scale", "shift", "w_norm", "b_norm"):
        refused(H, call_norm(H, vec=H.hilo_norm_vectors(**{n: O})), ARG)
    for n in ("gate", "w_branch"):
        refused(H, call_norm(H, vec=H.hilo_norm_vectors(**{n: A})), ARG)
    refused(H, L.hilo_group_norm(None, None, A, A, None, A, 1 << 40, None), ARG)
    assert L.hilo_group_norm_workspace_bytes(None) == 0
    need = L.hilo_group_norm_workspace_bytes(ref(norm(H).c()))
    assert need > 0
    refused(H, call_norm(H, ws=None), WORKSPACE)
    refused(H, call_norm(H, n=need - 1), WORKSPACE)
    refused(H, call_norm(H, n=0, y=A), WORKSPACE)  # in place is well


def test_group_norm_workspace_bound(H):
    """A pair per group and cluster of chunks: the workspace does not grow with the rows."""
    for d, groups in ((128, 32), (512, 32), (8192, 8192), (1152, 36)):
        for B, rows in ((1, 1 << 30), (7, 1 << 20), (5000, 3)):
            n = H.hilo_group_norm_workspace_bytes(norm(H, B=B, rows=rows, d=d, groups=groups))
            assert 8 * groups * B <= n <= 8 * groups * (114 + 2 * B), (d, groups, B, rows, n)


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
  void* O = (void*)(uintptr_t)4104;
  int32_t big[] = {INT32_MIN, -16, 0, 16, 48, 128, 4096, 65536, 1 << 30, INT32_MAX - 15, INT32_MAX};
  int64_t far[] = {INT64_MIN, -16, 0, 16, 24, 4096, (int64_t)1 << 38, ((int64_t)1 << 39) - 16, INT64_MAX};
  const int nb = sizeof big / sizeof big[0], nf = sizeof far / sizeof far[0];
  size_t total = 0;
  int i, j, k;
  for (i = 0; i < nb; ++i) for (j = 0; j < nb; ++j) for (k = 0; k < nf; ++k) {
    hilo_quant128_shape q = {big[i], big[j], k % 3, (i + k) & 1, far[k], far[(k + i) % nf], far[(k + j) % nf]};
    hilo_gemm128_shape g = {big[i], big[j], big[(i + k) % nb], HILO_ACT_NONE, HILO_F32, far[k], far[(k + i) % nf], far[(k + j) % nf],
                            far[(k + 1) % nf], far[(k + 2) % nf], far[(k + 3) % nf]};
    hilo_gemm128_shape w = {big[i], big[j], big[k % nb], HILO_ACT_SILU, HILO_E4M3, ((int64_t)1 << 39) - 16, ((int64_t)1 << 39) - 16,
                            ((int64_t)1 << 39) - 16, ((int64_t)1 << 39) - 1, ((int64_t)1 << 39) - 1, ((int64_t)1 << 39) - 1};
    hilo_group_norm_shape n = {big[i], big[j], 16 << (k % 10), 1 << (i % 5), k % 3, k % 3, (i + j) % 4, j & 1, 1e-6f,
                               ((int64_t)1 << 39) - 16, ((int64_t)1 << 39) - 16, far[k], ((int64_t)1 << 39) - 1};
    hilo_group_norm_shape m = {big[i], 3, big[j], big[(j + k) % nb], 0, 0, 0, 0, 1e-6f, far[k], far[(k + i) % nf], 0, far[(k + j) % nf]};
    total += hilo_group_norm_workspace_bytes(&n) + hilo_group_norm_workspace_bytes(&m);
    REFUSED(hilo_quantize_e4m3_128(&q, O, NULL, A, A, NULL));
    REFUSED(hilo_gemm_e4m3_128(&g, A, A, A, A, O, NULL, O, NULL));
    REFUSED(hilo_gated_e4m3_128(&w, A, A, A, A, A, NULL, NULL, NULL, NULL, A, A, NULL));
    REFUSED(hilo_group_norm(&n, NULL, A, A, NULL, NULL, 0, NULL));
    REFUSED(hilo_group_norm(&m, NULL, A, A, NULL, NULL, 0, NULL));
  }
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
    assert calls == 5 * 11 * 11 * 9 and some == 1
