"""What hilo_group_norm takes at the ends of its ranges, before any device work. Nothing here needs a GPU; the addresses
are never dereferenced."""
import ctypes

import pytest

SHAPE, WORKSPACE = -2, -4


@pytest.fixture(scope="module")
def H():
    from paper_2606_13898_gb300 import build
    from paper_2606_13898_gb300 import hilo

    build.build()
    hilo.lib()
    return hilo


def call(H, ws_bytes, **kw):
    """A call whose workspace is too small unless its shape is refused before."""
    s = H.GroupNormShape(**kw).c()
    rc = H.lib().hilo_group_norm(ctypes.byref(s), None, 4096, 8192, None, 4096, ws_bytes, None)
    return rc, H.lib().hilo_group_norm_workspace_bytes(ctypes.byref(s))


@pytest.mark.parametrize("kw", [dict(B=1 << 29, rows=1, d=16, groups=1), dict(B=1 << 29, rows=2, d=64, groups=8),
                                dict(B=1 << 30, rows=1, d=16, groups=16), dict(B=1 << 30, rows=0, d=128),
                                dict(B=0x7fffffff, rows=0, d=16, groups=1), dict(B=(1 << 20) + 1, rows=1, d=8192, groups=8192),
                                dict(B=1 << 28, rows=1, d=128, groups=64)])
def test_shapes_whose_grids_are_too_large_are_refused(H, kw):
    """Four CTAs an image, and an eighth of one a group: no grid passes 2^31 - 1, and the caller sees a shape's error."""
    assert call(H, 0, **kw) == (SHAPE, 0)


@pytest.mark.parametrize("kw", [dict(B=(1 << 29) - 1, rows=2, d=16, groups=16), dict(B=(1 << 29) - 1, rows=1, d=16, groups=1),
                                dict(B=1 << 20, rows=1, d=8192, groups=8192), dict(B=1 << 28, rows=4, d=64, groups=32),
                                dict(B=1, rows=1 << 30, d=8192, groups=8192)])
def test_the_largest_shapes_are_taken(H, kw):
    """(With no workspace, which is the only thing wrong with them.)"""
    rc, need = call(H, 0, **kw)
    assert rc == WORKSPACE and need >= 8 * kw["B"] * kw["groups"]
