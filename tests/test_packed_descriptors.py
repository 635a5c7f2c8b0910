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


# heads * stride just below a multiple of 2^64: in 64 bits the last head would lie before the first
FAR = (1 << 40) - 8


@pytest.mark.parametrize("name", ["dq", "dk", "dv"])
def test_output_rows_on_one_another_behind_64_bits(dsv, name):
    heads = 15728640
    p = dsv.Packed(1, 2, 2, 2, 2, heads, heads, 64, "bf16", 0.1)
    for other in ("q", "k", "v", "o", "dO", "dq", "dk", "dv"):
        setattr(p._c, other, (64, 128))
    assert bwd(dsv, p, None, 0) == -3
    setattr(p._c, name, (0, FAR))
    assert bwd(dsv, p, None, 0) == -1
    p = dsv.Norm(2, 64, "bf16", heads=(1 << 30) - 1)
    p._c.dx = (0, (1 << 34) + (1 << 6))
    assert dsv.load_library().dsv_layer_norm_bwd(p.c, *[ONE] * 8, None, 0, None) == -1


def test_layouts_under_address_and_undefined_sanitizers(tmp_path):
    """Strides over their range, in host code built with sanitizers; device code is built as always and never launched."""
    from concurrent.futures import ThreadPoolExecutor

    from paper_2502_07590_amd.build import CSRC, HIPCC_FLAGS, _hipcc
    here = os.path.dirname(os.path.abspath(__file__))
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-g"]
    flags = [f for f in HIPCC_FLAGS if f != "-O3"] + ["-O1"]

    def run(cmd, **kw):
        res = subprocess.run(cmd, capture_output=True, text=True, **kw)
        assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout[-2000:]}\n{res.stderr[-4000:]}"
        return res

    def compile_one(src):
        obj = str(tmp_path / (src + ".o"))
        run([_hipcc(), *flags, *san, "-c", os.path.join(CSRC, src), "-o", obj])
        return obj

    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, ["api_packed.hip", "packed_fwd.hip", "packed_bwd.hip", "norm.hip"]))
    main_o, exe = str(tmp_path / "main.o"), str(tmp_path / "layouts_san")
    run([_hipcc(), "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", *san, "-I", os.path.join(os.path.dirname(here), "include"), "-c", "-x", "c++",
         os.path.join(here, "sanitize", "packed_layouts_main.cpp"), "-o", main_o])
    run([_hipcc(), "--offload-arch=gfx950", *san, "-o", exe, main_o, *objs])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    assert "packed layouts sanitizer run ok" in run([exe], env=env).stdout


PACKED = dict(n_seq=3, total_q=300, total_k=400, max_q=200, max_k=300, Hq=8, Hkv=2, d=128, dtype="bf16", scale=0.1)
NORM = dict(tokens=100, n=128, dtype="bf16", eps=1e-5, heads=4)


@pytest.mark.parametrize("far", [1 << 31, (1 << 32) + 4, 1 << 64, -(1 << 31) - 1, -(1 << 32)])
def test_numbers_outside_a_field_are_refused(dsv, far):
    """Cut to 32 bits they would describe another call: 2^32 + 4 heads four, 2^32 tokens none."""
    for name in ("n_seq", "total_q", "total_k", "Hq", "Hkv", "d"):
        with pytest.raises(dsv.DsvError, match=name):
            dsv.Packed(**{**PACKED, name: far})
    for name in ("tokens", "n", "heads"):
        with pytest.raises(dsv.DsvError, match=name):
            dsv.Norm(**{**NORM, name: far})


def test_limits_that_are_none(dsv):
    """No sequence is longer than all tokens, and those fit a field: a limit that does not, limits nothing."""
    plain = dsv.Packed(**{**PACKED, "max_q": (1 << 31) - 1, "max_k": (1 << 31) - 1})
    for far in (1 << 31, 1 << 32, (1 << 32) + 4, 1 << 64):
        p = dsv.Packed(**{**PACKED, "max_q": far, "max_k": far})
        assert (p._c.max_q, p._c.max_k) == ((1 << 31) - 1,) * 2
        assert dsv.packed_attn_fwd_workspace(p) == dsv.packed_attn_fwd_workspace(plain)
        assert dsv.packed_attn_bwd_workspace(p) == dsv.packed_attn_bwd_workspace(plain) > 0
    for name in ("max_q", "max_k"):
        with pytest.raises(dsv.DsvError, match=name):
            dsv.Packed(**{**PACKED, name: -(1 << 32)})
