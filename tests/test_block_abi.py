"""Rotary positions, gated norms and the 8-bit cache: what their entry points refuse, on the host, before anything touches a GPU; and the references the GPU
tests compare with, against differentiation, differences and brute force.  CPU only."""
import ctypes
import math
import os

import pytest
import torch

import block_ref as ref


@pytest.fixture(scope="module")
def dsv():
    import paper_2502_07590_amd as m
    if not os.path.exists(m.library_path()):
        from paper_2502_07590_amd.build import build_library
        build_library()
    m.load_library()
    return m


ONE = ctypes.c_void_p(256)      # non-null and aligned; never dereferenced on these paths
ODD = ctypes.c_void_p(257)
ROTARY = dict(tokens=100, heads=4, d=128, dtype="bf16", pairs=[16, 24, 24], layout="axis_halves", gain=1.0)
GATED = dict(tokens=100, n=128, n_seg=3, dtype="bf16", eps=1e-6)
CACHE = dict(n_seq=3, total=300, max_new=200, Hq=8, Hkv=2, d=128, dtype="bf16", n_pages=50, page=64, max_pages=20, scale=0.1)


def changed(p, name, value):
    setattr(p._c, name, value)
    return p


# ---------------------------------------------------------------------------------------------- rotary
def rotary(dsv, p, ptrs=None):     # X, pos, freq, Y
    lib = dsv.load_library()
    got = {f(p.c, *(ptrs or [ONE, ONE, ONE, ctypes.c_void_p(512)]), None) for f in (lib.dsv_rotary_fwd, lib.dsv_rotary_bwd)}
    assert len(got) == 1
    return got.pop()


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), -1), (dict(heads=0), -1), (dict(d=0), -1), (dict(pairs=[65]), -1), (dict(pairs=[-1, 3]), -1), (dict(pairs=[0, 0]), -1),
    (dict(pairs=[2 ** 31 - 1] * 3), -1), (dict(gain=math.inf), -1), (dict(gain=math.nan), -1), (dict(dtype=torch.float16), -2), (dict(d=8193), -2),
    (dict(tokens=1 << 25), -2), (dict(tokens=1 << 20, heads=1024), -2)])
def test_rotary_descriptors_that_are_refused(dsv, change, status):
    assert rotary(dsv, dsv.Rotary(**{**ROTARY, **change})) == status


def test_rotary_pointers_and_strides_that_are_refused(dsv):
    p = dsv.Rotary(**ROTARY)
    for i in range(4):
        for bad in (None, ODD):
            ptrs = [ONE, ONE, ONE, ctypes.c_void_p(512)]
            ptrs[i] = bad
            assert rotary(dsv, p, ptrs) == -1, (i, bad)
    for strides in ((512, 100), (127, 512), (512, 0), (-512, 128), (1 << 41, 128)):
        assert rotary(dsv, changed(dsv.Rotary(**ROTARY), "y", strides)) == -1, strides
    for strides in ((-512, 128), (512, -128), (512, 1 << 40)):
        assert rotary(dsv, changed(dsv.Rotary(**ROTARY), "x", strides)) == -1, strides
    assert rotary(dsv, changed(dsv.Rotary(**ROTARY), "y", (1024, 128)), [ONE] * 4) == -1      # in place, other strides
    for name, value in (("layout", 3), ("layout", -1), ("axes", 0), ("axes", 4), ("flags", 1)):
        assert rotary(dsv, changed(dsv.Rotary(**ROTARY), name, value)) == -1, name
    assert rotary(dsv, dsv.Rotary(**{**ROTARY, "tokens": 0}), [None, None, ONE, None]) == 0
    lib = dsv.load_library()
    assert lib.dsv_rotary_fwd(None, ONE, ONE, ONE, ONE, None) == -1
    with pytest.raises(dsv.DsvError):
        dsv.Rotary(**{**ROTARY, "layout": "thirds"})
    with pytest.raises(dsv.DsvError):
        dsv.Rotary(**{**ROTARY, "pairs": [1, 1, 1, 1]})
    with pytest.raises(dsv.DsvError):
        dsv.Rotary(**{**ROTARY, "tokens": 1 << 31})


def test_frequencies(dsv):
    """Against the formulas, and what they promise: linear divides all, base keeps the fastest and divides the slowest, parts keeps and divides by turns."""
    n, base, L = 64, 10000.0, 4096.0
    plain, gain = dsv.rotary_freqs(n, base)
    i = torch.arange(n, dtype=torch.float64)
    assert gain == 1.0 and torch.allclose(plain, base ** (-i / n), rtol=1e-14, atol=0)
    lin, gain = dsv.rotary_freqs(n, base, "linear", 8)
    assert gain == 1.0 and torch.allclose(lin * 8, plain, rtol=1e-14, atol=0)
    stretched, gain = dsv.rotary_freqs(n, base, "base", 8)
    assert gain == 1.0 and stretched[0] == 1 and abs(float(stretched[-1] * 8 / plain[-1]) - 1) < 1e-12 and (stretched[1:] < plain[1:]).all()
    parts, gain = dsv.rotary_freqs(n, base, "parts", 8, original=L, low=1, high=32)
    turns = L * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.allclose(parts[turns <= 1] * 8, plain[turns <= 1], rtol=1e-14, atol=0)
    between = (turns > 1) & (turns < 32)
    keep = (turns[between] - 1) / 31
    assert between.any() and torch.allclose(parts[between], plain[between] * (keep + (1 - keep) / 8), rtol=1e-12, atol=0)
    assert abs(gain - (0.1 * math.log(8) + 1)) < 1e-6
    three, _ = dsv.rotary_freqs([16, 0, 24], base)
    assert torch.equal(three, torch.cat([dsv.rotary_freqs(16, base)[0], dsv.rotary_freqs(24, base)[0]]))
    assert dsv.rotary_freqs(1, base, "base", 4)[0].tolist() == [1.0]
    for bad in (dict(pairs=-1), dict(base=1.0), dict(base=math.nan), dict(factor=0.5), dict(factor=math.inf), dict(scaling="parts"), dict(scaling="parts", original=4096, low=3, high=3),
                dict(scaling="cubic"), dict(scaling="parts", original=math.inf)):
        with pytest.raises(dsv.DsvError):
            dsv.rotary_freqs(**{**dict(pairs=8, factor=2.0), **bad})


@pytest.mark.parametrize("layout", ["interleaved", "halves", "axis_halves"])
def test_the_rotary_reference(layout):
    """Its pairs cover the turned channels once; it keeps lengths, and scores depend on the difference of positions alone; back is the transpose."""
    pairs, d = [3, 5, 2], 24
    lo, hi, axis = zip(*ref.pairs_of(pairs, layout))
    assert sorted(lo + hi) == list(range(20)) and [axis.count(a) for a in range(3)] == pairs
    g = torch.Generator().manual_seed(1)
    q, k = torch.randn(1, 1, d, generator=g, dtype=torch.float64), torch.randn(1, 1, d, generator=g, dtype=torch.float64)
    f = ref.freqs(pairs)

    def score(a, b):
        x, _ = ref.rotary(q, torch.tensor([a]), f, pairs, layout)
        y, _ = ref.rotary(k, torch.tensor([b]), f, pairs, layout)
        return float((x * y).sum())

    assert abs(score([5, 2, 9], [3, 7, 1]) - score([105, 12, 10], [103, 17, 2])) < 1e-12 and abs(score([5, 2, 9], [3, 7, 1]) - score([5, 2, 9], [3, 7, 2])) > 1e-3
    pos = torch.randint(-50, 50, (6, 3), generator=g)
    X, dY = (torch.randn(6, 2, d, generator=g, dtype=torch.float64) for _ in range(2))
    y, _ = ref.rotary(X, pos, f, pairs, layout, 1.3)
    dx, _ = ref.rotary(dY, pos, f, pairs, layout, 1.3, back=True)
    assert abs(float((y * dY).sum() - (X * dx).sum())) < 1e-10                     # <R x, dy> = <x, R^T dy>
    assert torch.equal(y[..., 20:], X[..., 20:])


# ---------------------------------------------------------------------------------------------- gated norm
def gated_fwd(dsv, p, ptrs=None):      # X, Y, cu, gate, scale, shift, Z, H, stats
    return dsv.load_library().dsv_gated_norm_fwd(p.c, *(ptrs or [ONE] * 7 + [ctypes.c_void_p(512), ONE]), None)


def gated_bwd(dsv, p, ptrs=None, ws=ONE, ws_bytes=1 << 40):      # X, Y, cu, gate, scale, stats, dZ, dH, dX, dY, dgate, dscale, dshift
    return dsv.load_library().dsv_gated_norm_bwd(p.c, *(ptrs or [ONE] * 13), ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), -1), (dict(n=0), -1), (dict(n_seg=0), -1), (dict(eps=-1e-6), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1), (dict(residual=math.nan), -1),
    (dict(residual=math.inf), -1), (dict(n=8193), -2), (dict(dtype=torch.float16), -2), (dict(n_seg=1 << 22), -2)])
def test_gated_descriptors_that_are_refused(dsv, change, status):
    p = dsv.GatedNorm(**{**GATED, **change})
    assert gated_fwd(dsv, p) == status and gated_bwd(dsv, p) == status and dsv.gated_norm_bwd_workspace(p) == 0


def test_gated_pointers_and_strides_that_are_refused(dsv):
    p = dsv.GatedNorm(**GATED)
    base = [ONE] * 7 + [ctypes.c_void_p(512), ONE]
    for i in range(9):
        for bad in (None, ODD):
            ptrs = list(base)
            ptrs[i] = bad
            if bad is None and i in (3, 4, 5):      # modulations may be missing
                continue
            assert gated_fwd(dsv, p, ptrs) == -1, (i, bad)
    assert gated_fwd(dsv, p, base[:8] + [ctypes.c_void_p(264)]) == -1                                                # stats off their 16 bytes
    for i in range(13):
        for bad in (None, ODD):
            ptrs = [ONE] * 13
            ptrs[i] = bad
            if bad is None and i in (3, 4, 7, 10, 11, 12):
                continue
            assert gated_bwd(dsv, p, ptrs) == -1, (i, bad)
    for names, call in ((("x", "y", "z", "h", "gate", "scale", "shift"), gated_fwd), (("x", "y", "gate", "scale", "dz", "dh", "dx", "dy", "dgate", "dscale", "dshift"), gated_bwd)):
        for name in names:
            for bad in (-128, 1 << 40):
                assert call(dsv, changed(dsv.GatedNorm(**GATED), name, bad)) == -1, name
    for name, call in (("z", gated_fwd), ("h", gated_fwd), ("dx", gated_bwd), ("dy", gated_bwd), ("dgate", gated_bwd), ("dscale", gated_bwd), ("dshift", gated_bwd)):
        assert call(dsv, changed(dsv.GatedNorm(**GATED), name, 127)) == -1, name                                     # rows on one another
    assert gated_fwd(dsv, changed(dsv.GatedNorm(**GATED), "h", 256), [ONE] * 9) == -1                                # H is X, other strides
    assert gated_bwd(dsv, changed(dsv.GatedNorm(**GATED), "dx", 256)) == -1                                          # dX is dH, other strides
    for name, value in (("kind", 2), ("kind", -1), ("post", 2), ("flags", 1)):
        assert gated_fwd(dsv, changed(dsv.GatedNorm(**GATED), name, value)) == -1, name
    # without Y: no H, gate, dY, dgate, and nothing to norm before the gate
    alone = [ONE, None, ONE, None, ONE, ONE, ONE, None, ONE]
    for i in (3, 7):
        ptrs = list(alone)
        ptrs[i] = ONE
        assert gated_fwd(dsv, p, ptrs) == -1
    assert gated_fwd(dsv, dsv.GatedNorm(**{**GATED, "post": True}), alone) == -1
    alone = [ONE, None, ONE, None, ONE, ONE, ONE, ONE, ONE, None, None, ONE, ONE]
    for i in (3, 9, 10):
        ptrs = list(alone)
        ptrs[i] = ONE
        assert gated_bwd(dsv, p, ptrs) == -1
    big = dsv.GatedNorm(**{**GATED, "tokens": 100000})
    need = dsv.gated_norm_bwd_workspace(big)
    assert need > 0
    for ws, n in ((None, need), (ONE, need - 1), (ctypes.c_void_p(264), need)):
        assert gated_bwd(dsv, big, ws=ws, ws_bytes=n) == -3
    none = dsv.GatedNorm(**{**GATED, "tokens": 0})
    assert gated_fwd(dsv, none, [None, None, ONE] + [None] * 6) == 0
    assert gated_bwd(dsv, none, [None, None, ONE] + [None] * 10, ws=None, ws_bytes=0) == 0
    with pytest.raises(dsv.DsvError):
        dsv.GatedNorm(**{**GATED, "kind": "batch"})


def test_strides_of_gated_tensors_that_are_not_there_are_not_looked_at(dsv):
    """A descriptor whose fields for NULL tensors were left at zero, or hold anything.  The calls end at a check behind that of the strides: a workspace that is
    too small."""
    forward, backward = ("x", "y", "z", "h", "gate", "scale", "shift"), ("x", "y", "gate", "scale", "dz", "dh", "dx", "dy", "dgate", "dscale", "dshift")
    big = {**GATED, "tokens": 100000}
    for left in (0, -5, 1 << 50):
        def descriptor(there, **more):
            p = dsv.GatedNorm(**{**big, **more})
            for name in forward + backward:
                if name not in there:
                    setattr(p._c, name, left)
            return p

        # no block output: its stream, gate and gradients are not there
        p = descriptor(("x", "z", "scale", "shift", "dz", "dh", "dx", "dscale", "dshift"))
        need = dsv.gated_norm_bwd_workspace(p)
        assert need == dsv.gated_norm_bwd_workspace(dsv.GatedNorm(**big)) > 0
        assert gated_bwd(dsv, p, [ONE, None, ONE, None, ONE, ONE, ONE, ONE, ONE, None, None, ONE, ONE], ws_bytes=need - 1) == -3
        # no modulation wanted but one, and nothing that comes back to h
        p = descriptor(("x", "y", "dz", "dx", "dy", "dshift"))
        assert gated_bwd(dsv, p, [ONE, ONE, ONE, None, None, ONE, ONE, None, ONE, ONE, None, None, ONE], ws_bytes=need - 1) == -3
        assert gated_bwd(dsv, p, [ONE, ONE, ONE, None, None, ONE, ONE, None, ONE, ONE, ONE, None, ONE], ws_bytes=need - 1) == -1
        # no rows at all
        p = descriptor((), tokens=0)
        assert gated_fwd(dsv, p, [None, None, ONE] + [None] * 6) == 0
        assert gated_bwd(dsv, p, [None, None, ONE] + [None] * 10, ws=None, ws_bytes=0) == 0


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
def test_the_gated_reference(kind, post):
    """Against automatic differentiation, and against differences of its own forward."""
    g = torch.Generator().manual_seed(2)
    T, n, cu = 7, 10, [0, 3, 3, 6]
    normal = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    leaves = dict(X=normal(T, n), Y=normal(T, n), gate=normal(3, n), scale=normal(3, n), shift=normal(3, n))
    dZ, dH = normal(T, n), normal(T, n)
    dZ[6], dH[6] = 0, 0                      # the row of no segment
    opts = dict(eps=1e-3, kind=kind, post=post, residual=0.7)
    out = ref.gated(leaves["X"], cu, leaves["Y"], leaves["gate"], leaves["scale"], leaves["shift"], dZ, dH, **opts)

    def normed(v):
        c = v - v.mean(1, keepdim=True) if kind == "layer" else v
        return c / (c.square().mean(1, keepdim=True) + 1e-3).sqrt()

    def loss(X, Y, gate, scale, shift):
        seg = torch.tensor([0, 0, 0, 2, 2, 2, 0])
        h = 0.7 * X + gate[seg] * (normed(Y) if post else Y)
        z = normed(h) * (1 + scale[seg]) + shift[seg]
        keep = torch.tensor([1.0] * 6 + [0.0], dtype=torch.float64)[:, None]
        return ((z * dZ + h * dH) * keep).sum()

    live = {k: v.clone().requires_grad_() for k, v in leaves.items()}
    grads = dict(zip(live, torch.autograd.grad(loss(**live), live.values())))
    for name, key in (("X", "dX"), ("Y", "dY"), ("gate", "dgate"), ("scale", "dscale"), ("shift", "dshift")):
        want = out[key][0]
        look = ~want.isnan()
        assert (grads[name] - want)[look].abs().max() < 1e-12, name
        at = tuple(int(i) for i in look.nonzero()[3])
        for step in (1e-6,):
            moved = [{k: v.clone() for k, v in leaves.items()} for _ in range(2)]
            moved[0][name][at] += step
            moved[1][name][at] -= step
            diff = (loss(**moved[0]) - loss(**moved[1])) / (2 * step)
            assert abs(float(diff) - float(want[at])) < 1e-6, name


# ---------------------------------------------------------------------------------------------- cache
def append(dsv, p, turn=None, ptrs=None):      # K, V, cu, lens, table, pos, freq, K8, V8, kscale, vscale
    return dsv.load_library().dsv_cache_append(p.c, turn.c if turn else None, *(ptrs or [ONE] * 11), None)


def attend(dsv, p, ptrs=None, ws=ONE, ws_bytes=1 << 40):      # Q, cu, lens, table, K8, V8, kscale, vscale, O, lse
    return dsv.load_library().dsv_cache_attn_fwd(p.c, *(ptrs or [ONE] * 10), ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(n_seq=0), -1), (dict(total=-1), -1), (dict(max_new=-1), -1), (dict(max_len=-1), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=7), -1), (dict(n_pages=0), -1),
    (dict(max_pages=0), -1), (dict(page=0), -1), (dict(scale=0.0), -1), (dict(scale=math.nan), -1), (dict(scale=1e31), -1), (dict(page=8), -2), (dict(page=48), -2),
    (dict(page=512), -2), (dict(d=80), -2), (dict(dtype=torch.float16), -2), (dict(max_pages=1 << 26), -2), (dict(total=1 << 29), -2), (dict(n_seq=1 << 23), -2)])
def test_cache_descriptors_that_are_refused(dsv, change, status):
    p = dsv.Cache(**{**CACHE, **change})
    assert append(dsv, p) == status and attend(dsv, p) == status and dsv.cache_attn_fwd_workspace(p) == 0


def test_launches_of_more_lanes_than_a_grid_holds_are_refused(dsv):
    """2^32 of them: pages that many sequences may touch, and blocks of many short segments."""
    assert append(dsv, dsv.Cache(**{**CACHE, **dict(Hq=1, Hkv=1, d=128, page=16, max_pages=1 << 20, n_seq=1 << 23, total=1 << 28, max_new=64)})) == -2
    assert append(dsv, dsv.Cache(**{**CACHE, **dict(Hq=1, Hkv=1, d=128, page=256, max_pages=1 << 20, n_seq=1 << 22, total=1 << 28, max_new=200)})) == -2
    assert gated_fwd(dsv, dsv.GatedNorm(**{**GATED, **dict(tokens=1 << 24, n=32, n_seg=(1 << 24) - 1)})) == -2


@pytest.mark.parametrize("change", [dict(page=256, max_pages=(1 << 22) + 1), dict(page=256, max_pages=(1 << 23) - 1), dict(page=16, max_pages=(1 << 27) - 1, max_len=(1 << 30) + 1)])
def test_caches_of_more_than_2_to_the_30_tokens_are_refused(dsv, change):
    """The kernels count keys in 32 bits, a piece of them, or a few tiles, ahead: from 2^31 - 512 tokens on (in pieces from 2^30) that passes 2^31, and a
    negative key has a page before the table."""
    p = dsv.Cache(**{**CACHE, **change})
    assert append(dsv, p) == -2 and attend(dsv, p) == -2 and dsv.cache_attn_fwd_workspace(p) == 0


@pytest.mark.parametrize("change", [dict(page=256, max_pages=1 << 22), dict(page=256, max_pages=(1 << 23) - 1, max_len=1 << 30), dict(page=16, max_pages=(1 << 27) - 1, max_len=5000)])
def test_tables_of_more_are_not_where_max_len_says_less(dsv, change):
    p = dsv.Cache(**{**CACHE, **change})
    assert dsv.cache_attn_fwd_workspace(p) > 0                                               # in pieces
    assert attend(dsv, p, ws=None, ws_bytes=0) == -3
    none = dsv.Cache(**{**CACHE, **change, "total": 0})
    assert append(dsv, none) == 0 and attend(dsv, none) == 0


def test_cache_pointers_strides_and_workspaces_that_are_refused(dsv):
    p = dsv.Cache(**CACHE)
    turn = dsv.Rotary(300, 2, 128, "bf16", 64)
    for i in range(11):
        for bad in (None, ctypes.c_void_p(258 if i in (2, 3, 4, 5, 6, 9, 10) else 264)):
            ptrs = [ONE] * 11
            ptrs[i] = bad
            assert append(dsv, p, turn, ptrs) == -1, (i, bad)
    for i in range(10):
        for bad in (None, ctypes.c_void_p(258 if i in (1, 2, 3, 6, 7, 9) else 264)):
            ptrs = [ONE] * 10
            ptrs[i] = bad
            assert attend(dsv, p, ptrs) == -1, (i, bad)
    assert append(dsv, p, dsv.Rotary(300, 2, 64, "bf16", 32)) == -1                          # another head dimension
    assert append(dsv, p, changed(dsv.Rotary(300, 2, 128, "bf16", 64), "layout", 7)) == -1
    for name in ("k", "v"):
        for strides in ((1028, 128), (-1024, 128), (1 << 41, 128), (1024, 4)):
            assert append(dsv, changed(dsv.Cache(**CACHE), name, strides)) == -1, (name, strides)
    for name in ("q", "o"):
        for strides in ((1028, 128), (-1024, 128), (1 << 41, 128), (1024, 4)):
            assert attend(dsv, changed(dsv.Cache(**CACHE), name, strides)) == -1, (name, strides)
    for strides in ((0, 128), (1024, 0), (128, 128), (136, 256)):
        assert attend(dsv, changed(dsv.Cache(**CACHE), "o", strides)) == -1                  # rows on one another
    for name, value in (("causal", 2), ("flags", 1)):
        assert append(dsv, changed(dsv.Cache(**CACHE), name, value)) == -1 and attend(dsv, changed(dsv.Cache(**CACHE), name, value)) == -1
    long = dsv.Cache(8, 8, 1, 8, 2, 128, "bf16", 2000, 64, 200, max_len=10000)
    need = dsv.cache_attn_fwd_workspace(long)
    assert need > 0
    for ws, n in ((None, need), (ONE, need - 1), (ctypes.c_void_p(264), need)):
        assert attend(dsv, long, ws=ws, ws_bytes=n) == -3
    none = dsv.Cache(**{**CACHE, "total": 0})
    assert append(dsv, none, None, [None, None, ONE, ONE, ONE, None, None, ONE, ONE, ONE, ONE]) == 0
    assert attend(dsv, none, [None] + [ONE] * 7 + [None, None], ws=None, ws_bytes=0) == 0


def test_e4m3_of_the_reference_is_torchs():
    """Every finite value is kept, and between neighbours the nearest is taken, the even one of two."""
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    every = every[every.isfinite()]
    assert torch.equal(ref.e4m3(every), every)
    up = every[every >= 0].sort().values.unique()
    x = torch.cat([(up[1:] + up[:-1]) / 2, up[1:] * 0.999, up[:-1] * 1.001 + 1e-5, -(up[1:] + up[:-1]) / 2])
    assert torch.equal(ref.e4m3(x), x.float().to(torch.float8_e4m3fn).double())
    for most in (448.0, 449.0, 1.75, 1.7500001, 1e-30, 3e38, 0.0, 2.0 ** -117 * 448):
        s = ref.page_scale(most)
        assert most <= 448 * s or s == 2.0 ** 119
        assert s == 2.0 ** -117 or most > 224 * s
