"""The 8-bit cache on the GPU: what an append leaves in it, value by value, and attention over it against 64 bits; odd lengths, pages that end inside a tile, pools
full of NaN where nothing was written, and both together as a sampler runs them."""
import math
import random

import pytest
import torch

import block_ref as ref
import packed_ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def rows(T, H, d, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, H, d, generator=g) * size).to(packed_ref.DTYPES[dtype])


def check_append(new, old, Hkv, d, page, dtype, pairs=None, pattern="halves", layout="token", grow=1.5, seed=0, K=None, V=None, spare=3):
    lens, T = [a + b for a, b in zip(new, old)], sum(new)
    table, n_pages = ref.pages_for(lens, page, seed, spare)
    before = {}
    for i, name in enumerate("KV"):
        before[name] = ref.quantised(rows(sum(old), Hkv, d, "f32", seed + 10 + i), old, table, n_pages, page)
    K = rows(T, Hkv, d, dtype, seed + 20, grow) if K is None else K
    V = rows(T, Hkv, d, dtype, seed + 21, grow) if V is None else V
    p = dsv.Cache(len(new), T, max(new), Hkv, Hkv, d, dtype, n_pages, page, table.shape[1])
    K8, V8, ks, vs = (t.to(DEV) for t in (before["K"][0], before["V"][0], before["K"][1], before["V"][1]))
    turn, want_k, off_k, kw = None, K.double(), torch.zeros(K.shape, dtype=torch.float64), {}
    if pairs:
        turn = dsv.Rotary(T, Hkv, d, dtype, pairs, layout=pattern)
        g = torch.Generator().manual_seed(seed + 30)
        pos = torch.randint(0, 5000, (T, len(pairs)), generator=g).int()
        want_k, off_k = ref.rotary(K.double(), pos, ref.freqs(pairs), pairs, pattern, in_32=True)
        kw = dict(rotary=turn, pos=pos.to(DEV), freq=ref.freqs(pairs).to(DEV))
    dsv.cache_append(p, packed_ref.laid_out(K.to(DEV), layout), packed_ref.laid_out(V.to(DEV), layout), packed_ref.cu_of(new).to(DEV), ints(lens), table.to(DEV),
                     K8.view(E4M3), V8, ks, vs, **kw)
    torch.cuda.synchronize()
    for name, pool, scale, want, off in (("K", K8, ks, want_k, off_k), ("V", V8, vs, V.double(), torch.zeros(V.shape, dtype=torch.float64))):
        read = lambda v, s: (v.cpu().view(E4M3).double(), s.cpu().double())  # noqa: E731
        ref.check_append(read(*before[name]), read(pool, scale), want, off, new, lens, table, page)
    return K8, V8, ks, vs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_append_pages(d, page, dtype):
    """Sequences that begin a page, go on within one, end at its end, cross several; one that gets nothing."""
    check_append([1, page, page - 1, 5, 0, 3 * page + 7], [0, 0, 1, page - 2, page + 3, 2 * page - 1], 3, d, page, dtype)
    check_append([1] * 7, [0, 1, page - 1, page, page + 1, 5 * page, 7], 2, d, page, dtype, pairs=[d // 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pattern", ["interleaved", "halves", "axis_halves"])
@pytest.mark.parametrize("pairs", [[32], [16, 8, 8], [24], [3, 2, 5], [16, 16]])
def test_append_turned(pairs, pattern, dtype):
    check_append([40, 3], [5, 0], 2, 64, 32, dtype, pairs=pairs, pattern=pattern)
    check_append([90, 1], [100, 63], 5, 128, 64, dtype, pairs=pairs, pattern=pattern)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs,pattern", [([64], "halves"), ([57], "axis_halves"), ([29, 3, 7], "axis_halves"), ([61], "interleaved"), ([9], "halves")])
@pytest.mark.parametrize("page", [128, 256])
def test_append_turned_to_large_pages(page, pairs, pattern, dtype):
    check_append([700, 1, 255], [100, 255, 3], 3, 128, page, dtype, pairs=pairs, pattern=pattern)


def test_append_of_many_sequences():
    """More than one step of the search for a page's sequence, most of them without a token."""
    g = torch.Generator().manual_seed(9)
    new = (torch.rand(5000, generator=g) < 0.05).long().tolist()
    check_append(new, torch.randint(0, 40, (5000,), generator=g).tolist(), 1, 64, 16, "bf16", pairs=[32])
    check_append([3 * x for x in new[:700]], torch.randint(0, 40, (700,), generator=g).tolist(), 1, 64, 16, "f32")


@pytest.mark.parametrize("seed", range(12))
def test_append_of_any_shape(seed):
    r = random.Random(seed)
    d, n = r.choice([64, 128]), r.choice([1, 2, 5, 9])
    page, pairs = r.choice([16, 32, 64, 128, 256]), [r.randint(1, d // 6) for _ in range(r.randint(1, 3))]
    new = [r.choice([0, 1, r.randint(1, 400)]) for _ in range(n)]
    new[0] = new[0] or 1
    check_append(new, [r.choice([0, r.randint(0, 500)]) for _ in range(n)], r.choice([1, 2, 3, 5]), d, page, r.choice(["bf16", "f32"]), pairs=r.choice([None, pairs, [d // 2], [8, 8]]),
                 pattern=r.choice(["interleaved", "halves", "axis_halves"]), layout=r.choice(["token", "head", "slice"]), grow=r.choice([0.1, 1.0, 30.0]), seed=seed)


@pytest.mark.parametrize("layout", ["head", "slice"])
def test_append_views(layout):
    a = check_append([100, 20], [7, 0], 3, 128, 32, "bf16", pairs=[64], layout=layout)
    b = check_append([100, 20], [7, 0], 3, 128, 32, "bf16", pairs=[64])
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("grow", [1e-3, 1.0, 300.0, 1e6, 1e-30])
def test_append_to_begun_pages_of_other_sizes(grow):
    """New tokens far smaller than the page's (its scale stays), and far larger (its values move, into the subnormal range and to zero)."""
    check_append([3, 20], [10, 17], 2, 64, 32, "f32", grow=grow)


def test_append_of_zeros_and_of_the_ends_of_the_range():
    T = 20
    zero = torch.zeros(T, 1, 64)
    check_append([T], [0], 1, 64, 16, "f32", K=zero, V=zero)
    x = rows(T, 1, 64, "f32", 3)
    x[0], x[1, 0, 0], x[5] = 0.0, 3e38, 1e-38
    y = x.clone()
    y[1, 0, 0], y[2, 0, 3] = 448.0 * 4, -448.0 * 4                    # whole powers: the scale is 4, not 8
    check_append([T], [0], 1, 64, 16, "f32", K=x, V=y)


def test_append_of_values_that_are_no_numbers():
    """They are NaN in the cache; the page's scale and its other values are what they are without them."""
    T, H, d, page = 20, 2, 64, 16
    clean = rows(T, H, d, "f32", 5)
    bad = clean.clone()
    bad[3, 0, 7], bad[4, 1, 9], bad[18, 0, 0] = math.nan, math.inf, -math.inf
    holes = clean.clone()
    holes[3, 0, 7] = holes[4, 1, 9] = holes[18, 0, 0] = 0
    table, n_pages = ref.pages_for([T], page)
    out = []
    for x in (bad, holes):
        p = dsv.Cache(1, T, T, H, H, d, "f32", n_pages, page, table.shape[1])
        K8, V8 = (torch.zeros(n_pages, H, page, d, dtype=torch.uint8, device=DEV) for _ in range(2))
        ks, vs = (torch.zeros(n_pages, H, device=DEV) for _ in range(2))
        dsv.cache_append(p, x.to(DEV), x.to(DEV), ints([0, T]), ints([T]), table.to(DEV), K8, V8, ks, vs)
        out.append([t.cpu() for t in (K8, V8, ks, vs)])
    for a, b in zip(out[0][2:], out[1][2:]):
        assert torch.equal(a, b)
    for a, b in zip(out[0][:2], out[1][:2]):
        nan = a.view(E4M3).float().isnan()
        assert int(nan.sum()) == 3 and torch.equal(a[~nan], b[~nan]) and (b[nan] == 0).all()


def test_append_with_tables_and_lengths_that_make_no_sense_stays_inside():
    T, H, d, page, n_pages = 50, 2, 64, 16, 6
    K = rows(T, H, d, "bf16", 1).to(DEV)
    p = dsv.Cache(3, T, T, H, H, d, "bf16", n_pages, page, 4)
    for cu, lens, table in (([0, 20, 40, 50], [20, 20, 10], [[0, -1, 2 ** 31 - 1, 6], [-(2 ** 31), 3, 1, 1], [6, 6, 6, 6]]), ([0, 20, 40, 50], [5, -3, 2 ** 31 - 1], [[0, 1, 2, 3]] * 3),
                            ([30, -5, 2 ** 31 - 1, 4], [64, 64, 64], [[0, 1, 2, 3], [4, 5, 0, 1], [2, 3, 4, 5]])):
        pools = [torch.full((n_pages + 2, H, page, d), 9, dtype=torch.uint8, device=DEV) for _ in range(2)]
        scales = [torch.ones(n_pages + 2, H, device=DEV) for _ in range(2)]
        dsv.cache_append(p, K, K, ints(cu), ints(lens), ints(table), *[x[1:-1] for x in pools], *[x[1:-1] for x in scales])
        torch.cuda.synchronize()
        for x in pools:
            assert (x[0] == 9).all() and (x[-1] == 9).all()
        for x in scales:
            assert (x[0] == 1).all() and (x[-1] == 1).all()


# ---------------------------------------------------------------------------------------------- attention
def make_cache(lens, Hkv, d, page, seed=0):
    """A cache whose unwritten places are NaN, scales of unused pages too, and its table's unused entries nonsense."""
    table, n_pages = ref.pages_for(lens, page, seed)
    g = torch.Generator().manual_seed(seed + 1)
    basis = torch.randn(d // 2, d, generator=g) / math.sqrt(d // 2)
    K = torch.randn(sum(lens), Hkv, d // 2, generator=g) @ basis
    V = torch.randn(sum(lens), Hkv, d, generator=g) * torch.exp(torch.randn(sum(lens), Hkv, 1, generator=g))
    K8, ks = ref.quantised(K, lens, table, n_pages, page)
    V8, vs = ref.quantised(V, lens, table, n_pages, page)
    Kw, Vw = ref.widened(K8, ks, lens, table, page), ref.widened(V8, vs, lens, table, page)
    return table, n_pages, K8, V8, ks, vs, Kw, Vw, basis


def check_attend(new, lens, Hq, Hkv, d, page, dtype, causal=True, layout="token", behind=0, max_len=None, seed=0):
    table, n_pages, K8, V8, ks, vs, Kw, Vw, basis = make_cache(lens, Hkv, d, page, seed)
    g = torch.Generator().manual_seed(seed + 2)
    T, scale = sum(new) + behind, 1.3 / math.sqrt(d)
    Q = (torch.randn(T, Hq, d // 2, generator=g) @ basis).to(packed_ref.DTYPES[dtype])
    p = dsv.Cache(len(new), T, max(new), Hq, Hkv, d, dtype, n_pages, page, table.shape[1], scale=scale, causal=causal, max_len=max_len)
    O = torch.full((T, Hq, d), 7.0, dtype=Q.dtype, device=DEV)
    lse = torch.full((Hq, T), 7.0, device=DEV)
    O, lse = dsv.cache_attn_fwd(p, packed_ref.laid_out(Q.to(DEV), layout), packed_ref.cu_of(new).to(DEV), ints(lens), table.to(DEV), K8.to(DEV).view(E4M3), V8.to(DEV),
                                ks.to(DEV), vs.to(DEV), O=O, lse=lse)
    torch.cuda.synchronize()
    scale32 = float(torch.tensor(scale))
    want = packed_ref.attention(Q.double(), Kw, Vw, packed_ref.cu_of(new), packed_ref.cu_of(lens), scale32, causal, dtype=dtype)
    packed_ref.assert_within("O", O, want["O"])
    packed_ref.assert_within("lse", lse, want["lse"])
    assert (O[sum(new):] == 7).all() and (lse[:, sum(new):] == 7).all()
    return O, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_pages(causal, d, page, dtype):
    """One token and a few of each; lengths that end a page, begin one, leave one short, and none at all."""
    check_attend([1, 1, 1, 1, 1, 1], [1, page, page + 1, 3 * page - 1, 0, 300], 4, 2, d, page, dtype, causal)
    check_attend([5, 1, 40, 0, 3], [page + 5, 2 * page, 40, 77, 700], 6, 2, d, page, dtype, causal, behind=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (7, 1), (16, 2), (40, 1), (9, 3)])
def test_attend_heads(Hq, Hkv, dtype):
    check_attend([1, 1], [513, 100], Hq, Hkv, 128, 64, dtype)
    check_attend([33, 20], [120, 20], Hq, Hkv, 64, 16, dtype, behind=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_tiles_of_many_rows(causal, dtype):
    """Blocks of 128 rows: queries of one and of several tiles, more queries than keys (the first see nothing), ends inside tiles."""
    check_attend([300, 129], [300, 1000], 2, 1, 128, 64, dtype, causal)
    check_attend([200, 260], [90, 191], 4, 2, 64, 32, dtype, causal, behind=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[6000], [5000, 1, 300, 2049], [2048, 4096]])
def test_attend_in_pieces(lens, dtype):
    """Long caches of few streams: the key axis in pieces that are joined, some of them past the end of the shorter ones."""
    p = dsv.Cache(len(lens), len(lens), 1, 4, 2, 128, dtype, 400, 64, 100, max_len=max(lens))
    assert dsv.cache_attn_fwd_workspace(p) > 0
    a = check_attend([1] * len(lens), lens, 4, 2, 128, 64, dtype, max_len=max(lens))
    b = check_attend([1] * len(lens), lens, 4, 2, 128, 64, dtype)                 # sized by what the table holds
    for x, y in zip(a, b):
        assert (x - y).abs().max() < 0.05
    check_attend([40] + [3] * (len(lens) - 1), lens, 4, 2, 64, 16, dtype, causal=False, max_len=max(lens))


@pytest.mark.parametrize("layout", ["head", "slice"])
def test_attend_views(layout):
    a = check_attend([5, 30], [100, 64], 4, 2, 64, 32, "bf16", layout=layout)
    b = check_attend([5, 30], [100, 64], 4, 2, 64, 32, "bf16")
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("seed", range(16))
def test_attend_of_any_shape(seed):
    r = random.Random(100 + seed)
    n, Hkv = r.choice([1, 2, 5, 9]), r.choice([1, 2, 3])
    new = [1] * n if r.random() < 0.4 else [r.choice([0, 1, r.randint(1, 300)]) for _ in range(n)]
    new[0] = new[0] or 1
    most = r.choice([100, 1500, 3000])
    check_attend(new, [r.choice([0, 1, r.randint(1, most)]) for _ in range(n)], Hkv * r.choice([1, 2, 4, 7]), Hkv, r.choice([64, 128]), r.choice([16, 32, 64, 128, 256]),
                 r.choice(["bf16", "f32"]), r.random() < 0.6, layout=r.choice(["token", "head", "slice"]), behind=r.choice([0, 3]), max_len=r.choice([None, most]), seed=seed)


def test_pages_behind_4_gb():
    """A pool of more than 2^32 bytes: the same tokens into its first pages and into its last, the same bytes there and the same attention over them."""
    H, d, page, T = 8, 128, 256, 300
    n_pages = 2 ** 32 // (H * page * d) + 4
    K, V, Q = (rows(T, h, d, "bf16", i).to(DEV) for i, h in enumerate((H, H, 16)))
    cu, lens = ints([0, T]), ints([T])
    K8, V8 = (torch.zeros(n_pages, H, page, d, dtype=torch.uint8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(n_pages, H, device=DEV) for _ in range(2))
    p = dsv.Cache(1, T, T, 16, H, d, "bf16", n_pages, page, 2, scale=0.1)
    got = []
    for first in (0, n_pages - 2):
        table = ints([[first, first + 1]])
        dsv.cache_append(p, K, V, cu, lens, table, K8, V8, ks, vs)
        got.append((*dsv.cache_attn_fwd(p, Q, cu, lens, table, K8, V8, ks, vs), K8[first : first + 2], V8[first : first + 2], ks[first : first + 2], vs[first : first + 2]))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert got[0][2].any() and not K8[2 : n_pages - 2 : 997].any()


def test_attend_many_streams():
    g = torch.Generator().manual_seed(4)
    lens = torch.randint(0, 200, (150,), generator=g).tolist()
    check_attend([1] * 150, lens, 4, 2, 64, 16, "bf16")


def test_every_value_of_e4m3_at_every_scale_is_widened_exactly():
    """Attention over one key returns its V: all 254 numbers, at scales from the least to the largest, as fp32 and as bf16 hold them."""
    numbers = torch.arange(256, dtype=torch.uint8)
    numbers = numbers[~numbers.view(E4M3).float().isnan()]
    d, page = 128, 16
    byte = torch.zeros(2 * d, dtype=torch.uint8)
    byte[: len(numbers)] = numbers
    for e in (-117, -100, -30, -1, 0, 1, 30, 100, 119):
        V8 = torch.full((2, 1, page, d), 0x7F, dtype=torch.uint8)
        V8[0, 0, 0], V8[1, 0, 0] = byte[:d], byte[d:]
        K8, ones = torch.zeros_like(V8), torch.ones(2, 1, device=DEV)
        scale = torch.full((2, 1), 2.0 ** e, device=DEV)
        for dtype in ("bf16", "f32"):
            p = dsv.Cache(2, 2, 1, 1, 1, d, dtype, 2, page, 1)
            Q = torch.ones(2, 1, d, dtype=packed_ref.DTYPES[dtype], device=DEV)
            O, lse = dsv.cache_attn_fwd(p, Q, ints([0, 1, 2]), ints([1, 1]), ints([[0], [1]]), K8.to(DEV), V8.to(DEV), ones, scale)
            want = byte.view(E4M3).float() * 2.0 ** e
            assert torch.equal(O.float().cpu().reshape(-1), want), (e, dtype)
            assert (lse == 0).all()


def test_attend_with_tables_and_lengths_that_make_no_sense_stays_inside():
    H, d, page, n_pages = 2, 64, 16, 6
    K8 = torch.zeros(n_pages, H, page, d, dtype=torch.uint8, device=DEV)
    ks = torch.ones(n_pages, H, device=DEV)
    Q = rows(50, 4, d, "bf16", 1).to(DEV)
    for most in (1, 50):
        p = dsv.Cache(3, 50, most, 4, H, d, "bf16", n_pages, page, 4)
        for cu, lens, table in (([0, 1, 2, 3], [64, 64, 64], [[0, -1, 2 ** 31 - 1, 6], [-(2 ** 31), 3, 1, 1], [6, 6, 6, 6]]), ([0, 20, 40, 50], [5, -3, 2 ** 31 - 1], [[0, 1, 2, 3]] * 3),
                                ([30, -5, 2 ** 31 - 1, 4], [64, 64, 64], [[0, 1, 2, 3]] * 3)):
            guard = torch.full((114, 4, d), 7.0, dtype=torch.bfloat16, device=DEV)
            dsv.cache_attn_fwd(p, Q, ints(cu), ints(lens), ints(table), K8, K8, ks, ks, O=guard[32:82])
            torch.cuda.synchronize()
            assert (guard[:32] == 7).all() and (guard[82:] == 7).all()


def test_refused_by_the_binding():
    table, n_pages, K8, V8, ks, vs, *_ = make_cache([40], 2, 64, 16)
    table, K8, V8, ks, vs = (t.to(DEV) for t in (table, K8, V8, ks, vs))
    p = dsv.Cache(1, 3, 3, 4, 2, 64, "bf16", n_pages, 16, table.shape[1])
    Q, cu, lens = rows(3, 4, 64, "bf16", 1).to(DEV), ints([0, 3]), ints([40])
    good = [Q, cu, lens, table, K8, V8, ks, vs]
    dsv.cache_attn_fwd(p, *good)
    for i, bad in ((0, Q.float()), (0, Q[:2]), (0, Q.cpu()), (1, cu.long()), (1, cu[:1]), (2, lens.cpu()), (3, table[:, :1]), (4, K8.float()), (4, K8[:1]), (5, V8.transpose(2, 3)),
                   (6, ks.double()), (7, vs[:1]), (7, None), (3, None)):
        args = list(good)
        args[i] = bad
        with pytest.raises(dsv.DsvError):
            dsv.cache_attn_fwd(p, *args)
    K = rows(3, 2, 64, "bf16", 2).to(DEV)
    turn = dsv.Rotary(3, 2, 64, "bf16", 32)
    for kw in (dict(rotary=turn), dict(rotary=turn, pos=ints([[1]] * 3)), dict(rotary=turn, pos=ints([[1]] * 2), freq=ref.freqs([32]).to(DEV)),
               dict(rotary=turn, pos=ints([[1]] * 3), freq=ref.freqs([32]))):
        with pytest.raises(dsv.DsvError):
            dsv.cache_append(p, K, K, cu, lens, table, K8, V8, ks, vs, **kw)


# ---------------------------------------------------------------------------------------------- together
def test_runs_replays_and_graphs_that_share_a_workspace():
    """Append and attention captured together, on lengths that move on the device from replay to replay; a second graph on the same workspace between."""
    n, Hq, Hkv, d, page = 3, 4, 2, 128, 64
    lens0 = [700, 63, 1500]
    room = [x + 10 for x in lens0]
    table, n_pages = ref.pages_for(room, page)
    K8, ks = ref.quantised(rows(sum(lens0), Hkv, d, "f32", 1), lens0, table, n_pages, page)
    V8, vs = ref.quantised(rows(sum(lens0), Hkv, d, "f32", 2), lens0, table, n_pages, page)
    pool = [t.to(DEV) for t in (K8, V8, ks, vs)]
    table = table.to(DEV)
    p = dsv.Cache(n, n, 1, Hq, Hkv, d, "bf16", n_pages, page, table.shape[1], scale=0.1, max_len=1600)
    turn, freq = dsv.Rotary(n, Hkv, d, "bf16", 64), ref.freqs([64]).to(DEV)
    ws = torch.empty(dsv.cache_attn_fwd_workspace(p), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    cu, lens, pos = ints([0, 1, 2, 3]), ints(lens0), ints([[0]] * 3)
    K, V, Q = (torch.empty(n, h, d, dtype=torch.bfloat16, device=DEV) for h in (Hkv, Hkv, Hq))
    O, lse, O2, lse2 = (torch.empty(n, Hq, d, dtype=torch.bfloat16, device=DEV), torch.empty(Hq, n, device=DEV), torch.empty(n, Hq, d, dtype=torch.bfloat16, device=DEV),
                        torch.empty(Hq, n, device=DEV))

    def token(i):
        for k, t in enumerate((K, V, Q)):
            t.copy_(rows(n, t.shape[1], d, "bf16", 100 * i + k))

    def step(pool, O, lse, advance=True):
        if advance:
            lens.add_(1)
            pos.copy_(lens[:, None] - 1)
        dsv.cache_append(p, K, V, cu, lens, table, *pool, rotary=turn, pos=pos, freq=freq)
        dsv.cache_attn_fwd(p, Q, cu, lens, table, *pool, O=O, lse=lse, workspace=ws)

    start = [t.clone() for t in pool]
    eager = []
    for i in range(4):
        token(i)
        step(pool, O, lse)
        torch.cuda.synchronize()
        eager.append((O.clone(), lse.clone()))
    after = [t.clone() for t in pool]
    other = [t.clone() for t in start]

    def reset(to):
        for a, b in zip(to, start):
            a.copy_(b)
        lens.copy_(ints(lens0))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        reset(pool)
        step(pool, O, lse)
    torch.cuda.current_stream().wait_stream(side)
    reset(pool)
    graph, graph2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pool, O, lse)
    with torch.cuda.graph(graph2):
        step(other, O2, lse2, advance=False)
    for i in range(4):
        token(i)
        ws.fill_(255)
        graph.replay()
        graph2.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, eager[i][0]) and torch.equal(lse, eager[i][1]) and torch.equal(O2, O) and torch.equal(lse2, lse), i
    for a, b, c in zip(pool, after, other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(c.view(torch.uint8), b.view(torch.uint8))


def test_other_streams():
    lens, new = [300, 20], [3, 20]
    table, n_pages, K8, V8, ks, vs, *_ = make_cache([297, 0], 2, 64, 16)
    table, n_pages = ref.pages_for(lens, 16)
    args = [t.to(DEV) for t in (table,)]
    K, Q = rows(23, 2, 64, "bf16", 1).to(DEV), rows(23, 4, 64, "bf16", 2).to(DEV)
    p = dsv.Cache(2, 23, 20, 4, 2, 64, "bf16", n_pages, 16, table.shape[1], scale=0.2)
    got = []
    for stream in (None, torch.cuda.Stream()):
        K8, V8 = (torch.full((n_pages, 2, 16, 64), 0x31, dtype=torch.uint8, device=DEV) for _ in range(2))
        ks, vs = (torch.ones(n_pages, 2, device=DEV) for _ in range(2))
        cu, ln = packed_ref.cu_of(new).to(DEV), ints(lens)
        torch.cuda.synchronize()
        dsv.cache_append(p, K, K, cu, ln, *args, K8, V8, ks, vs, stream=stream)
        O, lse = dsv.cache_attn_fwd(p, Q, cu, ln, *args, K8, V8, ks, vs, stream=stream)
        torch.cuda.synchronize()
        got.append((K8, V8, ks, vs, O, lse))
    assert all(torch.equal(a, b) for a, b in zip(*got))
