"""Rotary positions on the GPU against their formula in 64 bits: every layout, whole and partial heads, pairs in eights and not, views, far and negative positions."""
import math
import random

import pytest
import torch

import block_ref as ref
import packed_ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"
LAYOUTS = ["interleaved", "halves", "axis_halves"]


def inputs(tokens, heads, d, axes, dtype, seed=0, first=0):
    g = torch.Generator().manual_seed(seed)
    X, dY = (torch.randn(tokens, heads, d, generator=g).to(packed_ref.DTYPES[dtype]) for _ in range(2))
    pos = torch.randint(-40, 3000, (tokens, axes), generator=g).int()
    pos[:, 0] += first
    return X, dY, pos


def check(tokens, heads, d, pairs, pattern, dtype, layout="token", gain=1.0, first=0, freq=None, seed=0):
    X, dY, pos = inputs(tokens, heads, d, len(pairs), dtype, seed, first)
    freq = ref.freqs(pairs) if freq is None else freq
    p = dsv.Rotary(tokens, heads, d, dtype, pairs, layout=pattern, gain=gain)
    gain = float(torch.tensor(gain))                                        # as the descriptor holds it
    x, dy, dpos, dfreq = packed_ref.laid_out(X.to(DEV), layout), packed_ref.laid_out(dY.to(DEV), layout), pos.to(DEV), freq.to(DEV)
    Y, dX = dsv.rotary_fwd(p, x, dpos, dfreq), dsv.rotary_bwd(p, dy, dpos, dfreq)
    torch.cuda.synchronize()
    packed_ref.assert_within("Y", Y, ref.rotary(X.double(), pos, freq, pairs, pattern, gain, dtype=dtype))
    packed_ref.assert_within("dX", dX, ref.rotary(dY.double(), pos, freq, pairs, pattern, gain, back=True, dtype=dtype))
    rot = 2 * sum(pairs)
    assert torch.equal(Y[..., rot:].cpu(), X[..., rot:]) and torch.equal(dX[..., rot:].cpu(), dY[..., rot:])
    return Y, dX


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pattern", LAYOUTS)
@pytest.mark.parametrize("d,pairs", [(128, [64]), (128, [16, 24, 24]), (128, [16, 16]), (64, [16, 8, 8]), (64, [3, 2, 5]), (128, [48]), (128, [21, 22, 21]), (48, [24]), (80, [8, 16]),
                                     (2, [1]), (5, [1, 1]), (96, [0, 20, 4]), (16, [1]), (256, [100, 28])])
def test_pairs_of_a_head(d, pairs, pattern, dtype):
    check(37, 3, d, pairs, pattern, dtype)


@pytest.mark.parametrize("pattern", LAYOUTS)
@pytest.mark.parametrize("tokens,heads", [(1, 1), (1, 40), (2, 7), (129, 1), (4099, 2), (600, 32)])
def test_sizes(tokens, heads, pattern):
    check(tokens, heads, 128, [16, 24, 24], pattern, "bf16")
    check(tokens, heads, 64, [7, 2], pattern, "f32")


@pytest.mark.parametrize("layout", ["head", "slice"])
@pytest.mark.parametrize("pairs", [[16, 24, 24], [5, 6, 7]])
def test_views(layout, pairs):
    a = check(301, 6, 128, pairs, "axis_halves", "bf16", layout)
    b = check(301, 6, 128, pairs, "axis_halves", "bf16")
    assert torch.equal(a[0].contiguous(), b[0].contiguous()) and torch.equal(a[1].contiguous(), b[1].contiguous())


@pytest.mark.parametrize("first", [1_200_000, 2_147_000_000, -2_147_000_000])
def test_positions_far_out(first):
    """Angles of 10^9 radians, where 32 bits hold none at all."""
    check(50, 2, 64, [32], "halves", "f32", first=first)
    check(50, 2, 128, [16, 24, 24], "interleaved", "bf16", first=first)


def test_frequencies_scaled_for_long_contexts():
    freq, gain = dsv.rotary_freqs(48, 10000.0, "parts", 8, original=4096)
    check(300, 4, 128, [48], "halves", "bf16", gain=gain, freq=freq)
    check(300, 4, 128, [48], "interleaved", "f32", gain=gain, freq=freq)


def test_rows_off_their_16_bytes():
    X, _, pos = inputs(40, 1, 128, 1, "bf16")
    wide = torch.zeros(40, 1, 131, dtype=torch.bfloat16, device=DEV)
    x = wide[:, :, 1:129]
    x.copy_(X)
    p = dsv.Rotary(40, 1, 128, "bf16", [64], layout="halves")
    Y = dsv.rotary_fwd(p, x, pos.to(DEV), ref.freqs([64]).to(DEV))
    packed_ref.assert_within("Y", Y, ref.rotary(X.double(), pos, ref.freqs([64]), [64], "halves"))


@pytest.mark.parametrize("pairs", [[48], [5, 6, 7]])
@pytest.mark.parametrize("pattern", LAYOUTS)
def test_in_place_in_a_fused_projection_and_nothing_beside(pairs, pattern):
    """Q and K of a fused projection turned where they lie, as one call; V behind them is not touched.  Then back, which undoes it."""
    T, Hq, Hkv, d = 130, 4, 2, 128
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(DEV)
    old = qkv.clone()
    pos = torch.randint(0, 1000, (T, len(pairs)), generator=g).int()
    p = dsv.Rotary(T, Hq + Hkv, d, "f32", pairs, layout=pattern)
    qk, freq = qkv[:, : Hq + Hkv], ref.freqs(pairs).to(DEV)
    apart = dsv.rotary_fwd(p, qk, pos.to(DEV), freq)
    assert dsv.rotary_fwd(p, qk, pos.to(DEV), freq, Y=qk) is qk
    assert torch.equal(qk, apart) and torch.equal(qkv[:, Hq + Hkv :], old[:, Hq + Hkv :])
    packed_ref.assert_within("Y", qk, ref.rotary(old[:, : Hq + Hkv].double().cpu(), pos, ref.freqs(pairs), pairs, pattern, dtype="f32"))
    dsv.rotary_bwd(p, qk, pos.to(DEV), freq, dX=qk)
    # two turns, each 6 + pi / 2 + 3 half steps of 2^-24 of two values, which are up to sqrt(2) times the largest, and a rounding: 63 of them
    assert (qkv - old).abs().max() < 64 * 2.0 ** -24 * float(old.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pattern", LAYOUTS)
@pytest.mark.parametrize("pairs", [[3], [11], [8], [40, 5]])
def test_channels_that_are_not_turned_are_copied_bit_for_bit(pairs, pattern, dtype):
    """Zeros of both signs, infinities and NaN in them, also next to pairs that are turned and in the same 16 bytes."""
    X, _, pos = inputs(20, 3, 128, len(pairs), dtype)
    rot = 2 * sum(pairs)
    odd = torch.tensor([-0.0, 0.0, math.inf, -math.inf, math.nan, 1e-40, 3e38], dtype=X.dtype)
    X[..., rot:] = odd[torch.arange(128 - rot) % len(odd)]
    p = dsv.Rotary(20, 3, 128, dtype, pairs, layout=pattern, gain=1.25)
    freq = ref.freqs(pairs)
    Y = dsv.rotary_fwd(p, X.to(DEV), pos.to(DEV), freq.to(DEV)).cpu()
    whole = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(Y[..., rot:].contiguous().view(whole), X[..., rot:].contiguous().view(whole))
    value, bound = ref.rotary(X.double(), pos, freq, pairs, pattern, 1.25, dtype=dtype)
    packed_ref.assert_within("Y", Y[..., :rot], (value[..., :rot], bound[..., :rot]))


@pytest.mark.parametrize("seed", range(12))
def test_any_shape(seed):
    r = random.Random(seed)
    d = r.choice([r.randint(2, 200), 64, 128, 16 * r.randint(1, 16)])
    pairs = [r.randint(0, d // 6) for _ in range(r.randint(1, 3))]
    pairs[0] = pairs[0] or 1
    check(r.choice([1, 3, 70, 513]), r.choice([1, 2, 5, 16, 33]), d, pairs, r.choice(LAYOUTS), r.choice(["bf16", "f32"]), r.choice(["token", "head", "slice"]),
          gain=r.choice([1.0, 1.2]), first=r.choice([0, 10 ** 6]), seed=seed)


@pytest.mark.parametrize("pairs", [[64], [5]])
def test_rows_behind_4_gb(pairs):
    T, H, d, apart = 2, 3, 128, 2 ** 31 + 64
    X, _, pos = inputs(T, H, d, 1, "bf16")
    far = torch.empty(apart + H * d, dtype=torch.bfloat16, device=DEV).as_strided((T, H, d), (apart, d, 1))
    far.copy_(X)
    p = dsv.Rotary(T, H, d, "bf16", pairs)
    want = dsv.rotary_fwd(p, X.to(DEV), pos.to(DEV), ref.freqs(pairs).to(DEV))
    dsv.rotary_fwd(p, far, pos.to(DEV), ref.freqs(pairs).to(DEV), Y=far)
    assert torch.equal(far, want)


def test_streams_graphs_and_no_tokens():
    T, H, d = 500, 8, 128
    X, dY, pos = inputs(T, H, d, 3, "bf16")
    x, freq, dpos = X.to(DEV), ref.freqs([16, 24, 24]).to(DEV), pos.to(DEV)
    p = dsv.Rotary(T, H, d, "bf16", [16, 24, 24], layout="axis_halves")
    want = dsv.rotary_fwd(p, x, dpos, freq)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = dsv.rotary_fwd(p, x, dpos, freq, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dsv.rotary_fwd(p, x, dpos, freq, Y=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsv.rotary_fwd(p, x, dpos, freq, Y=out)
    for shift in (0, 7, -3):                                                     # positions move between replays
        moved = dpos + shift
        keep = dpos.clone()
        dpos.copy_(moved)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dsv.rotary_fwd(p, x, moved, freq))
        dpos.copy_(keep)
    none = dsv.Rotary(0, H, d, "bf16", [64])
    assert dsv.rotary_fwd(none, torch.empty(0, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(0, 1, dtype=torch.int32, device=DEV), ref.freqs([64]).to(DEV)).shape == (0, H, d)


def test_refused_by_the_binding():
    X, _, pos = inputs(8, 2, 64, 1, "bf16")
    p = dsv.Rotary(8, 2, 64, "bf16", [32])
    x, dpos, freq = X.to(DEV), pos.to(DEV), ref.freqs([32]).to(DEV)
    for args in ((X, dpos, freq), (x, pos, freq), (x, dpos.long(), freq), (x, dpos, freq.float()), (x, dpos[:4], freq), (x.float(), dpos, freq), (x[:, :1], dpos, freq),
                 (x.transpose(1, 2), dpos, freq), (x, dpos, freq[:16]), (x, None, freq), (x, dpos, None)):
        with pytest.raises(dsv.DsvError):
            dsv.rotary_fwd(p, *args)
    assert math.isfinite(float(dsv.rotary_fwd(p, x, dpos, freq).float().sum()))
