"""Attention over the 8-bit cache in blocks of 128 rows (calls of many queries), against 64 bits: what tests/test_gpu_cache.py, whose calls all run in blocks of 32,
does not reach."""
import pytest
import torch

import block_ref as ref
import packed_ref
from cache_calls import BEHIND_4_GB, LARGE_TILES, NONSENSE, any_large
from test_gpu_cache import check_attend, ints, make_cache, rows

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("call", LARGE_TILES, ids=lambda c: f"{sum(c[0])}-{max(c[1])}-{c[2]}x{c[3]}-d{c[4]}-{c[6]}")
def test_calls_of_many_rows(call, causal):
    check_attend(*call, causal, behind=2, max_len=max(call[1]))


@pytest.mark.parametrize("layout", ["head", "slice"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views(dtype, layout):
    call = next(c for c in LARGE_TILES if c[4:] == (64, 32, dtype))
    a, b = check_attend(*call, layout=layout), check_attend(*call)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("seed", range(8))
def test_any_shape(seed):
    call, causal, layout, behind = any_large(seed)
    check_attend(*call, causal, layout=layout, behind=behind, seed=seed)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tables_and_lengths_that_make_no_sense_stay_inside(dtype):
    n_seq, T, most, H, _, d, page, max_pages = NONSENSE
    n_pages = 6
    K8 = torch.zeros(n_pages, H, page, d, dtype=torch.uint8, device=DEV)
    ks = torch.ones(n_pages, H, device=DEV)
    Q = rows(T, H, d, dtype, 1).to(DEV)
    low, high = -(2 ** 31), 2 ** 31 - 1
    p = dsv.Cache(n_seq, T, most, H, H, d, dtype, n_pages, page, max_pages)
    tables = [[[0, -1, high, 6] * 10, [low, 3, 1, 1] * 10, [6, 6, 6, 6] * 10], [[high] * 40, [low] * 40, [0, 1, 2, 3] * 10]]
    for cu, lens in (([0, 200, 400, 700], [640, 640, 640]), ([0, 200, 400, 700], [5, -3, high]), ([300, -5, high, 4], [640, 641, 1]), ([0, 700, 0, 700], [low, 100, 639])):
        for table in tables:
            guard = torch.full((T + 64, H, d), 7.0, dtype=Q.dtype, device=DEV)
            dsv.cache_attn_fwd(p, Q, ints(cu), ints(lens), ints(table), K8, K8, ks, ks, O=guard[32 : 32 + T])
            torch.cuda.synchronize()
            assert (guard[:32] == 7).all() and (guard[32 + T :] == 7).all()


def test_pages_behind_4_gb():
    """The same tokens in a pool's first pages and behind 2^32 bytes of it: the same attention over them."""
    new, lens, H, _, d, page, dtype = BEHIND_4_GB
    table, n_pages, K8, V8, ks, vs, Kw, Vw, _ = make_cache(lens, H, d, page)
    first = 2 ** 32 // (H * page * d) + 1
    pools = [torch.zeros(first + n_pages, H, page, d, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(first + n_pages, H, device=DEV) for _ in range(2)]
    Q, cu = rows(sum(new), H, d, dtype, 5).to(DEV), packed_ref.cu_of(new).to(DEV)
    p = dsv.Cache(2, sum(new), max(new), H, H, d, dtype, first + n_pages, page, table.shape[1], scale=0.1)
    got = []
    for at in (0, first):
        for pool, x in zip(pools, (K8, V8)):
            pool[at : at + n_pages] = x.to(DEV)
        for s, x in zip(scales, (ks, vs)):
            s[at : at + n_pages] = x.to(DEV)
        got.append(dsv.cache_attn_fwd(p, Q, cu, ints(lens), (table + at).to(DEV), *pools, *scales))
        for pool in pools:
            pool[at : at + n_pages] = 0x7F
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and got[0][0].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_runs_and_replays_are_equal_bit_for_bit(dtype):
    """In pieces, on a workspace full of NaN; lengths that change between replays."""
    new, lens, Hq, Hkv, d, page, _ = next(c for c in LARGE_TILES if c[5] == 128 and c[6] == dtype)
    table, n_pages, K8, V8, ks, vs, *_ = make_cache(lens, Hkv, d, page)
    args = [t.to(DEV) for t in (table, K8, V8, ks, vs)]
    Q, cu, ln = rows(sum(new), Hq, d, dtype, 5).to(DEV), packed_ref.cu_of(new).to(DEV), ints(lens)
    p = dsv.Cache(len(new), sum(new), max(new), Hq, Hkv, d, dtype, n_pages, page, table.shape[1], scale=0.1, max_len=max(lens))
    ws = torch.empty(dsv.cache_attn_fwd_workspace(p), dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    other = ints([x // 2 for x in lens])
    want = [dsv.cache_attn_fwd(p, Q, cu, x, *args) for x in (ln, other)]
    O, lse = (torch.empty_like(t) for t in want[0])
    held = ln.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dsv.cache_attn_fwd(p, Q, cu, held, *args, O=O, lse=lse, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dsv.cache_attn_fwd(p, Q, cu, held, *args, O=O, lse=lse, workspace=ws)
    for i, x in enumerate((ln, other, ln)):
        held.copy_(x)
        ws.fill_(255)
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])
