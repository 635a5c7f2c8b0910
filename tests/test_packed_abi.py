"""The entry points of packed attention and layer norm: what they refuse, on the host, before anything touches a GPU, and the
reference the GPU tests compare with, against brute force and differences.  CPU only."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import packed_ref as ref


@pytest.fixture(scope="module")
def dsv():
    import paper_2502_07590_amd as m
    if not os.path.exists(m.library_path()):
        from paper_2502_07590_amd.build import build_library
        build_library()
    m.load_library()
    return m


ONE = ctypes.c_void_p(256)      # non-null and aligned; never dereferenced on these paths
PACKED = dict(n_seq=3, total_q=300, total_k=400, max_q=200, max_k=300, Hq=8, Hkv=2, d=128, dtype="bf16", scale=0.1)


def fwd(dsv, p, ptrs=None, ws=ONE, ws_bytes=1 << 40):
    """Q, K, V, cu_q, cu_k, O, O_tail, lse"""
    return dsv.load_library().dsv_packed_attn_fwd(p.c, *(ptrs or [ONE] * 6 + [None, ONE]), ws, ws_bytes, None)


def bwd(dsv, p, ptrs=None, ws=ONE, ws_bytes=1 << 40):
    """Q, K, V, cu_q, cu_k, O, O_tail, lse, dO, dQ, dK, dV"""
    return dsv.load_library().dsv_packed_attn_bwd(p.c, *(ptrs or [ONE] * 6 + [None] + [ONE] * 5), ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(n_seq=0), -1), (dict(total_q=-1), -1), (dict(total_k=-1), -1), (dict(max_q=-1), -1), (dict(max_k=-2), -1),
    (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=7), -1), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=math.inf), -1),
    (dict(scale=math.nan), -1), (dict(d=80), -2), (dict(dtype=torch.float16), -2), (dict(total_q=1 << 29), -2), (dict(total_k=1 << 30), -2),
    (dict(total_q=1 << 27, Hq=64, Hkv=1), -2), (dict(n_seq=1 << 23), -2)])
def test_descriptors_that_are_refused(dsv, change, status):
    p = dsv.Packed(**{**PACKED, **change})
    assert fwd(dsv, p) == status and bwd(dsv, p) == status
    assert dsv.packed_attn_fwd_workspace(p) == 0 and dsv.packed_attn_bwd_workspace(p) == 0


def test_pointers_strides_and_workspaces_that_are_refused(dsv):
    p = dsv.Packed(**PACKED)
    for i in (0, 1, 2, 3, 4, 5, 7):
        for bad in (None, ctypes.c_void_p(258 if i in (3, 4, 7) else 264)):
            ptrs = [ONE] * 6 + [None, ONE]
            ptrs[i] = bad
            assert fwd(dsv, p, ptrs) == -1, i
            assert bwd(dsv, p, ptrs + [ONE] * 4) == -1, i
    for i in (8, 9, 10, 11):
        for bad in (None, ctypes.c_void_p(264)):
            ptrs = [ONE] * 6 + [None] + [ONE] * 5
            ptrs[i] = bad
            assert bwd(dsv, p, ptrs) == -1, i
    assert fwd(dsv, p, [ONE] * 6 + [ctypes.c_void_p(264), ONE]) == -1                       # tail off its 16 bytes
    assert fwd(dsv, dsv.Packed(**{**PACKED, "dtype": "f32"}), [ONE] * 8) == -1              # a tail of fp32
    need = dsv.packed_attn_bwd_workspace(p)
    assert need > 0
    for ws, n in ((None, need), (ONE, need - 1), (ctypes.c_void_p(264), need)):
        assert bwd(dsv, p, ws=ws, ws_bytes=n) == -3
    few = dsv.Packed(8, 8, 80000, 1, 10000, 8, 2, 128, "bf16", 0.1)
    need = dsv.packed_attn_fwd_workspace(few)
    assert need > 0
    for ws, n in ((None, need), (ONE, need - 1), (ctypes.c_void_p(264), need)):
        assert fwd(dsv, few, ws=ws, ws_bytes=n) == -3
    for name in ("q", "k", "v", "o"):
        for strides in ((1024, 4), (1028, 128), (-1024, 128), (1024, -128), (1 << 41, 128)):
            p = dsv.Packed(**PACKED)
            setattr(p._c, name, strides)
            assert fwd(dsv, p) == -1 and bwd(dsv, p) == -1, (name, strides)
    for name in ("dO", "dq", "dk", "dv"):
        p = dsv.Packed(**PACKED)
        setattr(p._c, name, (1028, 128))
        assert bwd(dsv, p) == -1
    for name, call in (("o", fwd), ("dq", bwd), ("dk", bwd), ("dv", bwd)):
        for strides in ((0, 128), (1024, 0), (128, 128), (64, 1024), (136, 256)):           # rows of an output on one another
            p = dsv.Packed(**PACKED)
            setattr(p._c, name, strides)
            assert call(dsv, p) == -1, (name, strides)
    p = dsv.Packed(**PACKED)
    p._c.causal = 2
    assert fwd(dsv, p) == -1
    p = dsv.Packed(**PACKED)
    p._c.flags = 1
    assert fwd(dsv, p) == -1
    lib = dsv.load_library()
    assert lib.dsv_packed_attn_fwd(None, *[ONE] * 8, ONE, 0, None) == -1 and lib.dsv_packed_attn_fwd_workspace(None) == 0


def test_nothing_to_do_needs_no_tensors(dsv):
    p = dsv.Packed(**{**PACKED, "total_q": 0})
    assert fwd(dsv, p, [None, ONE, ONE, ONE, ONE, None, None, None], ws=None, ws_bytes=0) == 0
    both = dsv.Packed(**{**PACKED, "total_q": 0, "total_k": 0})
    assert bwd(dsv, both, [None, None, None, ONE, ONE] + [None] * 7, ws=None, ws_bytes=0) == 0


def test_norm_refusals(dsv):
    lib = dsv.load_library()
    ok = dict(tokens=100, n=128, dtype="bf16", eps=1e-5, heads=4)

    def nf(p, ptrs=None):       # X, gamma, beta, Y, mean, rstd
        return lib.dsv_layer_norm_fwd(p.c, *(ptrs or [ONE] * 6), None)

    def nb(p, ptrs=None, ws=ONE, n=1 << 40):       # X, gamma, mean, rstd, dY, dX, dgamma, dbeta
        return lib.dsv_layer_norm_bwd(p.c, *(ptrs or [ONE] * 8), ws, n, None)

    for change, status in ((dict(tokens=-1), -1), (dict(n=0), -1), (dict(heads=0), -1), (dict(eps=-1e-5), -1), (dict(eps=math.inf), -1), (dict(eps=math.nan), -1),
                           (dict(n=8193), -2), (dict(dtype=torch.float16), -2), (dict(tokens=1 << 30), -2)):
        p = dsv.Norm(**{**ok, **change})
        assert nf(p) == status and nb(p) == status, change
        assert dsv.layer_norm_bwd_workspace(p) == 0
    p = dsv.Norm(**ok)
    for i in (0, 3, 4, 5):
        for bad in (None, ctypes.c_void_p(257)):
            ptrs = [ONE] * 6
            ptrs[i] = bad
            assert nf(p, ptrs) == -1, i
    for i in range(8):
        for bad in (None, ctypes.c_void_p(257)):
            ptrs = [ONE] * 8
            ptrs[i] = bad
            if i != 1 or bad is not None:           # gamma may be missing
                assert nb(p, ptrs) == -1, i
    need = dsv.layer_norm_bwd_workspace(p)
    for ws, n in ((None, need), (ONE, need - 1), (ctypes.c_void_p(264), need)):
        assert nb(p, ws=ws, n=n) == -3
    for name, call in (("y", nf), ("dx", nb)):
        for strides in ((0, 128), (512, 64), (512, 0), (100, 512), (-512, 128)):
            p = dsv.Norm(**ok)
            setattr(p._c, name, strides)
            assert call(p) == -1, (name, strides)
    p = dsv.Norm(**ok)
    p._c.x = (-512, 128)
    assert nf(p) == -1 and nb(p) == -1
    p = dsv.Norm(**{**ok, "tokens": 0})
    assert nf(p, [None] * 6) == 0 and nb(p, [None] * 8, None, 0) == 0


def test_tensors_that_the_binding_refuses(dsv):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    p = dsv.Packed(1, 4, 4, 4, 4, 2, 2, 64, "bf16", 0.1)
    with pytest.raises(dsv.DsvError):
        dsv.packed_attn_fwd(p, x, x, x, cu, cu)            # host tensors
    with pytest.raises(dsv.DsvError):
        dsv.packed_attn_bwd(p, x, x, x, cu, cu, x, torch.zeros(2, 4), x)
    n = dsv.Norm(4, 64, "bf16", heads=2)
    with pytest.raises(dsv.DsvError):
        dsv.layer_norm_fwd(n, x)
    with pytest.raises(dsv.DsvError):
        dsv.layer_norm_bwd(n, x, None, torch.zeros(4, 2), torch.zeros(4, 2), x)
    from paper_2502_07590_amd import binding as b
    c, cpu = b._CPacked.from_buffer_copy(p._c), torch.device("cpu")
    assert (c.q.row, c.q.head, c.dv.row, c.dv.head) == (128, 64, 128, 64)      # contiguous until a tensor says otherwise
    for bad in (x[:3], x.float(), x.transpose(1, 2), torch.zeros(4, 2, 128, dtype=torch.bfloat16)[:, :, ::2], x[0]):
        with pytest.raises(dsv.DsvError):
            b._rows(c, "q", bad, (4, 2, 64), torch.bfloat16, cpu)
    b._rows(c, "q", x.transpose(0, 1).contiguous().transpose(0, 1), (4, 2, 64), torch.bfloat16, cpu)
    assert (c.q.row, c.q.head) == (64, 256)
    b._rows(c, "q", x[:, :1], (4, 1, 64), torch.bfloat16, cpu)
    assert (c.q.row, c.q.head) == (128, 64)                 # an axis of one step
    for bad in (cu.long(), cu[:1], torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(dsv.DsvError):
            b._flat("cu_q", bad, (2,), torch.int32, cpu)


# ---------------------------------------------------------------------------------------------- the reference itself
def test_reference_attention_is_the_formula_and_its_gradients_the_differences():
    lq, lk, Hq, Hkv, d, scale = [3, 0, 5, 1], [4, 2, 2, 0], 4, 2, 8, 0.7
    g = torch.Generator().manual_seed(3)
    Q, dO = (torch.randn(sum(lq), Hq, d, generator=g, dtype=torch.float64) for _ in range(2))
    K, V = (torch.randn(sum(lk), Hkv, d, generator=g, dtype=torch.float64) for _ in range(2))
    cq, ck = ref.cu_of(lq), ref.cu_of(lk)
    for causal in (False, True):
        out = ref.attention(Q, K, V, cq, ck, scale, causal, dO)
        O, lse = out["O"][0], out["lse"][0]
        for s in range(4):                                 # one row, one key at a time
            for i in range(lq[s]):
                for h in range(Hq):
                    keys = [j for j in range(lk[s]) if not causal or j <= i + lk[s] - lq[s]]
                    t = int(cq[s]) + i
                    if not keys:
                        assert lse[h, t] == -math.inf and (O[t, h] == 0).all() and (out["dQ"][0][t, h] == 0).all()
                        continue
                    rows = [int(ck[s]) + j for j in keys]
                    x = torch.tensor([scale * float(Q[t, h] @ K[r, h // 2]) for r in rows], dtype=torch.float64)
                    z = float(sum(math.exp(v) for v in x))
                    assert abs(float(lse[h, t]) - math.log(z)) < 1e-12
                    o = sum(math.exp(float(v)) / z * V[r, h // 2] for v, r in zip(x, rows))
                    assert torch.allclose(O[t, h], o, atol=1e-12)

        def loss(**kw):
            a = {**dict(Q=Q, K=K, V=V), **kw}
            return float((ref.attention(a["Q"], a["K"], a["V"], cq, ck, scale, causal)["O"][0] * dO).sum())

        for name, x in (("Q", Q), ("K", K), ("V", V)):
            for at in [(0, 0, 0), (x.shape[0] - 1, x.shape[1] - 1, d - 1), (2, 1, 3)]:
                up, down = x.clone(), x.clone()
                up[at] += 1e-5
                down[at] -= 1e-5
                diff = (loss(**{name: up}) - loss(**{name: down})) / 2e-5
                assert abs(diff - float(out["d" + name][0][at])) < 1e-8 * max(1, abs(diff)), (name, at)


def test_reference_norm_is_torchs_and_its_gradients_the_differences():
    g = torch.Generator().manual_seed(4)
    X, dY = (torch.randn(3, 2, 7, generator=g, dtype=torch.float64) for _ in range(2))
    gamma, beta = (torch.randn(7, generator=g, dtype=torch.float64) for _ in range(2))
    out = ref.norm(X, gamma, beta, 1e-3, dY)
    assert torch.allclose(out["Y"][0], torch.nn.functional.layer_norm(X, (7,), gamma, beta, 1e-3), atol=1e-12)

    def loss(x, a, b):
        return float((ref.norm(x, a, b, 1e-3)["Y"][0] * dY).sum())

    for at in ((0, 0, 0), (2, 1, 6)):
        e = torch.zeros_like(X)
        e[at] = 1e-6
        assert abs((loss(X + e, gamma, beta) - loss(X - e, gamma, beta)) / 2e-6 - float(out["dX"][0][at])) < 1e-7
    e = torch.zeros(7, dtype=torch.float64)
    e[3] = 1e-6
    assert abs((loss(X, gamma + e, beta) - loss(X, gamma - e, beta)) / 2e-6 - float(out["dgamma"][0][3])) < 1e-7
    assert abs((loss(X, gamma, beta + e) - loss(X, gamma, beta - e)) / 2e-6 - float(out["dbeta"][0][3])) < 1e-7


def test_host_code_under_address_and_undefined_sanitizers(tmp_path):
    """Split plans and workspace sizes over the range of a descriptor's numbers; device code is built as always and never launched."""
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
    main_o, exe = str(tmp_path / "main.o"), str(tmp_path / "packed_san")
    run([_hipcc(), "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", *san, "-I", os.path.join(os.path.dirname(here), "include"), "-c", "-x", "c++",
         os.path.join(here, "sanitize", "packed_checks_main.cpp"), "-o", main_o])
    run([_hipcc(), "--offload-arch=gfx950", *san, "-o", exe, main_o, *objs])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    assert "packed checks sanitizer run ok" in run([exe], env=env).stdout
