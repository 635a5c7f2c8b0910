"""Descriptors of packed attention and layer norm as a C caller may leave them: layouts that a call does not read, strides whose products pass
64 bits, numbers that do not fit a field.  CPU only; no call here reaches a kernel."""
import ctypes
import os
import subprocess

import pytest

ONE = ctypes.c_void_p(256)      # non-null and aligned; never dereferenced on these paths


@pytest.fixture(scope="module")
def dsv():
    import paper_2502_07590_amd as m
    if not os.path.exists(m.library_path()):
        from paper_2502_07590_amd.build import build_library
        build_library()
    m.load_library()
    return m


def fwd(dsv, p, ws, ws_bytes):
    return dsv.load_library().dsv_packed_attn_fwd(p.c, *[ONE] * 6, None, ONE, ws, ws_bytes, None)


def bwd(dsv, p, ws, ws_bytes):
    return dsv.load_library().dsv_packed_attn_bwd(p.c, *[ONE] * 6, None, *[ONE] * 5, ws, ws_bytes, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [(1 << 26, 128), (0x5555555555555555, -1), (1 << 62, 1 << 62), (-8, 3), (-(1 << 63), -(1 << 63))])
def test_the_forward_reads_no_layout_of_the_backward(dsv, dtype, left):
    p = dsv.Packed(8, 8, 80000, 1, 10000, 8, 2, 128, dtype, 0.1)     # a call in pieces: the workspace check comes before any launch
    need = dsv.packed_attn_fwd_workspace(p)
    assert need > 0
    for name in ("dO", "dq", "dk", "dv"):
        setattr(p._c, name, left)
    assert dsv.packed_attn_fwd_workspace(p) == need
    assert fwd(dsv, p, ONE, need - 1) == -3
    assert bwd(dsv, p, ONE, 0) in (-1, -2)                             # which the backward does read
