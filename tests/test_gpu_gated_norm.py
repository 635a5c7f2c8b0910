"""Gated norms on the GPU against their formulas in 64 bits: widths around every split of a row over lanes, segments of none to many rows, missing parts,
views, and runs of them together."""
import random

import pytest
import torch

import block_ref as ref
import packed_ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"
PARTS = ("Y", "gate", "scale", "shift", "dH")


def inputs(T, n, n_seg, dtype, seed=0, off=0.0):
    g = torch.Generator().manual_seed(seed)
    td = packed_ref.DTYPES[dtype]
    normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    out = dict(X=normal(T, n) * (1 + 3 * torch.rand(n, generator=g)) + off, Y=normal(T, n) + 0.2, dZ=normal(T, n), dH=normal(T, n))
    out.update(gate=normal(n_seg, n), scale=0.5 * normal(n_seg, n), shift=normal(n_seg, n))
    return {k: v.to(td) for k, v in out.items()}


def strided(x, wide):
    """x as a slice of rows `wide` elements longer, of NaN."""
    if x is None or not wide:
        return x
    big = torch.full((x.shape[0], x.shape[1] + wide), float("nan"), dtype=x.dtype, device=x.device)
    big[:, wide // 2 : wide // 2 + x.shape[1]] = x
    return big[:, wide // 2 : wide // 2 + x.shape[1]]


def check(lens, n, dtype, without=(), kind="layer", post=False, residual=1.0, eps=1e-6, behind=0, wide=0, seed=0, host=None, off=0.0):
    T, n_seg = sum(lens) + behind, len(lens)
    host = dict(inputs(T, n, n_seg, dtype, seed, off)) if host is None else host
    for k in without:
        host[k] = None
    cu = packed_ref.cu_of(lens)
    want = ref.gated(*[host["X"].double(), cu.tolist()], *[None if host[k] is None else host[k].double() for k in ("Y", "gate", "scale", "shift", "dZ", "dH")],
                     eps=eps, kind=kind, post=post, residual=float(torch.tensor(residual)), dtype=dtype)
    d = {k: None if v is None else strided(v.to(DEV), wide) for k, v in host.items()}
    p = dsv.GatedNorm(T, n, n_seg, dtype, eps, kind=kind, post=post, residual=residual)
    td = packed_ref.DTYPES[dtype]
    fill = lambda *s, t=td: torch.full(s, 7.0, dtype=t, device=DEV)  # noqa: E731
    Z, H, stats = dsv.gated_norm_fwd(p, d["X"], cu.to(DEV), d["Y"], d["gate"], d["scale"], d["shift"], Z=fill(T, n), H=None if d["Y"] is None else fill(T, n),
                                     stats=fill(T, 4, t=torch.float32))
    grads = {k: fill(n_seg, n, t=torch.float32) for k in ("dgate", "dscale", "dshift") if k != "dgate" or host["Y"] is not None}
    dX, dY, dgate, dscale, dshift = dsv.gated_norm_bwd(p, d["X"], cu.to(DEV), stats, d["dZ"], d["Y"], d["gate"], d["scale"], d["dH"], dX=fill(T, n),
                                                       dY=None if d["Y"] is None else fill(T, n), **grads)
    torch.cuda.synchronize()
    got = dict(Z=Z, H=H, stats=stats, dX=dX, dY=dY, dgate=dgate, dscale=dscale, dshift=dshift)
    for name, t in got.items():
        if name not in want or t is None:
            assert t is None and (name not in want or host["Y"] is None), name
            continue
        packed_ref.assert_within(f"{name} n={n} {dtype}", t, want[name])
        if name in ("Z", "H", "stats", "dX", "dY"):                     # rows of no segment are as they were
            assert (t[sum(lens):] == 7).all(), name
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 3, 8, 31, 64, 65, 100, 128, 255, 256, 257, 512, 520, 768, 1024, 1028, 1155, 1536, 2048, 2056, 4096, 4100, 4104, 8191, 8192])
def test_widths(n, dtype):
    check([3, 2], n, dtype)
    check([3, 2], n, dtype, kind="rms", post=True, residual=0.5)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_segments_of_no_one_and_many_rows(dtype, post, kind):
    check([0, 1, 700, 0, 33, 5, 0], 256, dtype, kind=kind, post=post, behind=9)
    check([1] * 70, 64, dtype, kind=kind, post=post)
    check([1200, 3000], 72, dtype, kind=kind, post=post, residual=-0.7)
    check([40, 0, 41], 4104, dtype, kind=kind, post=post, behind=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,n", [([9000], 128), ([4000, 1, 5000], 520), ([70000], 8), ([2000, 600], 2048), ([1100], 8192), ([3000], 1155)])
def test_segments_of_several_blocks(lens, n, dtype):
    check(lens, n, dtype, post=n < 600)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype,n", [("bf16", 5888), ("bf16", 8192), ("f32", 2560), ("f32", 4480)])
def test_wide_rows_of_several_blocks(dtype, n, kind):
    """512 lanes to a row: segments of many blocks, of one, of none; more segments than blocks are held back for."""
    check([600, 0, 3, 500], n, dtype, kind=kind, post=kind == "rms", behind=2)
    check([1] * 90 + [400], n, dtype, kind=kind, post=kind == "layer")


@pytest.mark.parametrize("n", [64, 1001])
@pytest.mark.parametrize("without", [(k,) for k in PARTS if k != "Y"] + [("gate", "scale", "shift", "dH"), ("Y", "gate"), ("Y", "gate", "scale", "shift", "dH")])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_parts_that_are_not_there(without, n, kind):
    """Two kinds of rows: many to a wave, and (rms without Y: one sum a row) a row to a block."""
    check([5, 0, 12], n, "bf16", without=without, kind=kind)
    check([5, 12], 8 * n if n == 1001 else 8000, "f32", without=without, kind=kind)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [8, 16, 6, 2048])
def test_strides(wide, dtype):
    a = check([30, 11], 512, dtype, wide=wide, post=True)
    b = check([30, 11], 512, dtype, post=True)
    if wide % 16 == 0:
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_chunks_of_one_projection_and_their_gradients_in_one_tensor():
    """shift, scale and gate as three chunks of a projection's output [n_seg, 6 n]; their gradients into chunks of one float tensor."""
    T, n, cu = 40, 128, packed_ref.cu_of([17, 23])
    h = inputs(T, n, 2, "bf16")
    mods = torch.cat([h["shift"], h["scale"], h["gate"]] * 2, 1).to(DEV)
    dmods = torch.full((2, 6 * n), 7.0, device=DEV)
    x, y, dz = (h[k].to(DEV) for k in ("X", "Y", "dZ"))
    p = dsv.GatedNorm(T, n, 2, "bf16")
    part = lambda t, i: t[:, i * n : (i + 1) * n]  # noqa: E731
    Z, H, stats = dsv.gated_norm_fwd(p, x, cu.to(DEV), y, part(mods, 5), part(mods, 4), part(mods, 3))
    dsv.gated_norm_bwd(p, x, cu.to(DEV), stats, dz, y, part(mods, 5), part(mods, 4), dgate=part(dmods, 5), dscale=part(dmods, 4), dshift=part(dmods, 3))
    want = ref.gated(h["X"].double(), cu.tolist(), *[h[k].double() for k in ("Y", "gate", "scale", "shift", "dZ")])
    for i, name in ((5, "dgate"), (4, "dscale"), (3, "dshift")):
        packed_ref.assert_within(name, part(dmods, i), want[name])
    packed_ref.assert_within("Z", Z, want["Z"])
    assert (dmods[:, : 3 * n] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    """The stream updated where it lies, and the gradient that comes back to it."""
    lens, n = [100, 31], 768
    h = {k: v.to(DEV) for k, v in inputs(131, n, 2, dtype).items()}
    cu = packed_ref.cu_of(lens).to(DEV)
    p = dsv.GatedNorm(131, n, 2, dtype, residual=0.9)
    Z, H, stats = dsv.gated_norm_fwd(p, h["X"], cu, h["Y"], h["gate"], h["scale"], h["shift"])
    dX, dY, *sums = dsv.gated_norm_bwd(p, h["X"], cu, stats, h["dZ"], h["Y"], h["gate"], h["scale"], h["dH"])
    x, dh = h["X"].clone(), h["dH"].clone()
    dX2, dY2, *sums2 = dsv.gated_norm_bwd(p, x, cu, stats, h["dZ"], h["Y"], h["gate"], h["scale"], dh, dX=dh)
    Z2, H2, stats2 = dsv.gated_norm_fwd(p, x, cu, h["Y"], h["gate"], h["scale"], h["shift"], H=x)
    assert dX2 is dh and H2 is x
    for a, b in zip((Z, H, stats, dX, dY, *sums), (Z2, H2, stats2, dX2, dY2, *sums2)):
        assert torch.equal(a, b)


def test_rows_far_from_zero_and_constant_rows():
    check([20], 512, "f32", off=1000.0)
    h = inputs(6, 128, 1, "f32")
    h["X"], h["Y"] = torch.full((6, 128), 0.5), torch.full((6, 128), 0.25)
    h["gate"] = torch.ones(1, 128)
    check([6], 128, "f32", host=h)
    check([6], 128, "f32", host=dict(h), post=True, kind="rms")


def test_no_rows_and_gradients_that_are_not_wanted():
    p = dsv.GatedNorm(0, 64, 2, "bf16")
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    cu, m = torch.zeros(3, dtype=torch.int32, device=DEV), torch.ones(2, 64, dtype=torch.bfloat16, device=DEV)
    Z, H, stats = dsv.gated_norm_fwd(p, x, cu, x, m, m, m)
    _, _, *sums = dsv.gated_norm_bwd(p, x, cu, stats, x, x, m, m, dgate=torch.full((2, 64), 7.0, device=DEV))
    assert all((s == 0).all() for s in sums)
    h = {k: v.to(DEV) for k, v in inputs(50, 64, 1, "bf16").items()}
    p, cu = dsv.GatedNorm(50, 64, 1, "bf16"), packed_ref.cu_of([50]).to(DEV)
    Z, H, stats = dsv.gated_norm_fwd(p, h["X"], cu, h["Y"], None, None, h["shift"])
    dX, dY, dgate, dscale, dshift = dsv.gated_norm_bwd(p, h["X"], cu, stats, h["dZ"], h["Y"])
    assert dgate is None and dscale is None and dshift is None and torch.equal(dX, dY)
    only = torch.full((1, 64), 7.0, device=DEV)
    assert dsv.gated_norm_bwd(p, h["X"], cu, stats, h["dZ"], h["Y"], dshift=only)[2:] == (None, None, only)
    assert (only - h["dZ"].float().sum(0)).abs().max() < 1e-4


@pytest.mark.parametrize("seed", range(12))
def test_any_shape(seed):
    r = random.Random(seed)
    n = r.choice([r.randint(1, 300), 64 * r.randint(1, 40), r.randint(300, 3000)])
    lens = [r.choice([0, 1, r.randint(1, 80)]) for _ in range(r.choice([1, 2, 7, 90]))]
    lens[0] = lens[0] or 1
    gone = r.choice([(), (), ("gate",), ("scale", "shift"), ("dH",), ("Y", "gate")])
    check(lens, n, r.choice(["bf16", "f32"]), without=gone, kind=r.choice(["layer", "rms"]), post="Y" not in gone and r.random() < 0.5, residual=r.choice([1.0, 0.3]),
          behind=r.choice([0, 5]), wide=r.choice([0, 0, 16, 5]), seed=seed)


@pytest.mark.parametrize("n", [64, 65])
def test_many_segments(n):
    g = torch.Generator().manual_seed(3)
    check(torch.randint(0, 3, (5000,), generator=g).tolist(), n, "bf16")


def test_rows_behind_4_gb():
    """Rows that lie 2^31 elements and more apart."""
    T, n, apart = 3, 512, 2 ** 31 + 64
    h = {k: v.to(DEV) for k, v in inputs(T, n, 1, "bf16").items()}
    far = torch.empty(2 * apart + n, dtype=torch.bfloat16, device=DEV).as_strided((T, n), (apart, 1))
    cu = packed_ref.cu_of([T]).to(DEV)
    p = dsv.GatedNorm(T, n, 1, "bf16")
    args = (cu, h["Y"], h["gate"], h["scale"], h["shift"])
    Z, H, stats = dsv.gated_norm_fwd(p, h["X"], *args)
    want = dsv.gated_norm_bwd(p, h["X"], cu, stats, h["dZ"], h["Y"], h["gate"], h["scale"], h["dH"])
    far.copy_(h["X"])
    for a, b in zip(dsv.gated_norm_fwd(p, far, *args), (Z, H, stats)):
        assert torch.equal(a, b)
    for a, b in zip(dsv.gated_norm_bwd(p, far, cu, stats, h["dZ"], h["Y"], h["gate"], h["scale"], h["dH"]), want):
        assert torch.equal(a, b)
    dsv.gated_norm_fwd(p, h["X"], *args, H=far)
    assert torch.equal(far, H)


def test_lengths_that_make_no_sense_stay_inside():
    """Entries of cu that do not ascend or point behind the tensor: no answer, but nothing outside the tensors is touched."""
    T, n = 300, 64
    h = {k: v.to(DEV) for k, v in inputs(T, n, 4, "bf16").items()}
    p = dsv.GatedNorm(T, n, 4, "bf16")
    for cu in ([0, 200, 100, 5000, 300], [-7, 2 ** 31 - 1, -(2 ** 31), 0, 12], [300, 299, 0, 300, 1], [0, 0, 0, 0, 2 ** 30]):
        c = torch.tensor(cu, dtype=torch.int32, device=DEV)
        guard = torch.full((T + 64, n), 7.0, dtype=torch.bfloat16, device=DEV)
        Z, H, stats = dsv.gated_norm_fwd(p, h["X"], c, h["Y"], h["gate"], h["scale"], h["shift"], Z=guard[32 : 32 + T])
        stats.nan_to_num_(0.0)
        dsv.gated_norm_bwd(p, h["X"], c, stats, h["dZ"], h["Y"], h["gate"], h["scale"], h["dH"])
        torch.cuda.synchronize()
        assert (guard[:32] == 7).all() and (guard[32 + T :] == 7).all()


def test_runs_replays_and_other_streams_are_equal_bit_for_bit():
    lens, n = [2500, 1, 0, 3000], 256
    T = sum(lens)
    h = {k: v.to(DEV) for k, v in inputs(T, n, 4, "bf16").items()}
    cu = packed_ref.cu_of(lens).to(DEV)
    p = dsv.GatedNorm(T, n, 4, "bf16", post=True)
    ws = torch.empty(dsv.gated_norm_bwd_workspace(p), dtype=torch.uint8, device=DEV)
    bf = lambda: torch.empty(T, n, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    out = [bf(), bf(), torch.empty(T, 4, device=DEV), bf(), bf()] + [torch.empty(4, n, device=DEV) for _ in range(3)]

    def step(cu=cu, stream=None):
        dsv.gated_norm_fwd(p, h["X"], cu, h["Y"], h["gate"], h["scale"], h["shift"], *out[:3], stream=stream)
        dsv.gated_norm_bwd(p, h["X"], cu, out[2], h["dZ"], h["Y"], h["gate"], h["scale"], h["dH"], *out[3:], workspace=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    eager = [x.clone() for x in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, eager))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        for x in out:
            x.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
    other = packed_ref.cu_of([1, 5000, 500, 0]).to(DEV)
    step(other)
    torch.cuda.synchronize()
    want = [x.clone() for x in out]
    cu.copy_(other)                                     # the graph replays on what cu holds then
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refused_by_the_binding():
    h = {k: v.to(DEV) for k, v in inputs(10, 64, 2, "bf16").items()}
    p, cu = dsv.GatedNorm(10, 64, 2, "bf16"), packed_ref.cu_of([4, 6]).to(DEV)
    ok = dict(Y=h["Y"], gate=h["gate"], scale=h["scale"], shift=h["shift"])
    for bad in (dict(Y=h["Y"].float()), dict(Y=h["Y"][:5]), dict(gate=h["gate"][:1]), dict(scale=h["scale"].cpu()), dict(shift=h["shift"].t()), dict(Y=h["Y"].t().contiguous().t())):
        with pytest.raises(dsv.DsvError):
            dsv.gated_norm_fwd(p, h["X"], cu, **{**ok, **bad})
    for x, c in ((h["X"].cpu(), cu), (h["X"], cu.cpu()), (h["X"], cu.long()), (h["X"], cu[:2]), (h["X"], None)):
        with pytest.raises(dsv.DsvError):
            dsv.gated_norm_fwd(p, x, c, **ok)
    with pytest.raises(dsv.DsvError):
        dsv.gated_norm_fwd(p, h["X"], cu, None, h["gate"])
