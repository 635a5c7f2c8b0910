"""Attention over packed sequences on the GPU against its formulas in 64 bits: lengths of 0, 1 and around every tile, causal or not, shared
heads, both types and head dimensions, layouts, pieces of the long axis, rows outside every sequence, streams and graphs."""
import math

import pytest
import torch

import packed_ref as ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


class Case:
    def __init__(self, lens_q, lens_k, Hq, Hkv, d, dtype, causal=False, layout="token", seed=0, scale=None, spare_q=0, spare_k=0, slack=0):
        self.cu_q, self.cu_k = ref.cu_of(lens_q), ref.cu_of(lens_k)
        tq, tk = sum(lens_q) + spare_q, sum(lens_k) + spare_k
        self.scale = scale or 2 / math.sqrt(d)
        self.dtype, self.causal, self.layout = dtype, causal, layout
        self.host = ref.attention_inputs(tq, tk, Hq, Hkv, d, dtype, seed)
        self.p = dsv.Packed(len(lens_q), tq, tk, max(lens_q) + slack, max(lens_k) + slack, Hq, Hkv, d, dtype, self.scale, causal=causal)
        self.Q, self.K, self.V, self.dO = (ref.laid_out(x.to(DEV), layout) for x in self.host)
        self.dcu = self.cu_q.to(DEV), self.cu_k.to(DEV)

    def want(self, grad=True, tail=True):
        Q, K, V, dO = (x.double() for x in self.host)
        return ref.attention(Q, K, V, self.cu_q, self.cu_k, self.scale, self.causal, dO if grad else None, self.dtype, tail)

    def run(self, grad=True, tail=True, **kw):
        t = torch.empty(self.Q.shape, dtype=self.Q.dtype, device=DEV) if tail and self.dtype == "bf16" else None
        O, lse = dsv.packed_attn_fwd(self.p, self.Q, self.K, self.V, *self.dcu, O_tail=t)
        out = {"O": O, "lse": lse}
        if grad:
            out["dQ"], out["dK"], out["dV"] = dsv.packed_attn_bwd(self.p, self.Q, self.K, self.V, *self.dcu, O, lse, self.dO, O_tail=t)
        torch.cuda.synchronize()
        return out

    def check(self, grad=True, tail=True):
        out, want = self.run(grad, tail), self.want(grad, tail)
        for n in out:
            ref.assert_within(n, out[n], want[n])
        return out


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 0, 127, 128, 129, 17]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_around_every_tile(dtype, d, causal):
    Case(EDGES, EDGES, 2, 2, d, dtype, causal).check()
    Case(EDGES, EDGES[::-1], 2, 1, d, dtype, causal).check()      # causal: sequences with more queries than keys, some with none


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 1), ("bf16", 64, 4), ("f32", 64, 1), ("f32", 128, 7), ("bf16", 128, 3)])
@pytest.mark.parametrize("causal", [False, True])
def test_calls_of_many_rows(dtype, d, group, causal):
    """Tiles of 128 rows and keys: enough heads and tokens to fill the chip."""
    Hkv = 32
    lens = [300, 129, 0, 511, 1, 128]
    rows = sum(lens) * group
    assert (rows // 128 + 1) * Hkv >= 256 and sum(lens) // len(lens) > 64 and (sum(lens) // 128 + 1) * Hkv >= 256
    Case(lens, lens, Hkv * group, Hkv, d, dtype, causal).check()
    if group == 1:
        Case([640, 511, 0, 77], [65, 700, 300, 1], Hkv, Hkv, d, dtype, causal).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,Hq,Hkv", [(128, 4, 1), (64, 6, 6), (128, 14, 2)])
def test_single_queries_against_long_caches(dtype, d, Hq, Hkv):
    """Keys in pieces, joined; sequences that end inside a piece, at its end, and before the others' second one."""
    lens_k = [2500, 1, 256, 257, 0, 512, 1999, 31]
    c = Case([1] * len(lens_k), lens_k, Hq, Hkv, d, dtype, True, slack=1000)
    assert dsv.packed_attn_fwd_workspace(c.p) > 0
    c.check()
    Case([1], [3001], Hq, Hkv, d, dtype, False).check()
    Case([3, 1, 40], [1500, 900, 20], Hq, Hkv, d, dtype, True).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_queries_against_few_keys(dtype):
    """The rows of the key-major step in pieces."""
    c = Case([2000, 700, 1], [77, 13, 120], 3, 3, 128, dtype)
    assert dsv.packed_attn_bwd_workspace(c.p) > 2 * 210 * 3 * 128 * 4
    c.check()
    Case([1900, 33], [40, 33], 8, 1, 64, dtype, True).check()


@pytest.mark.parametrize("layout", ["head", "slice"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_layouts(layout, dtype, d):
    out = Case([70, 200], [70, 200], 4, 2, d, dtype, True, layout).check()
    plain = Case([70, 200], [70, 200], 4, 2, d, dtype, True).run()
    for n in out:
        assert torch.equal(out[n].contiguous(), plain[n].contiguous()), n


def test_head_major_memory_is_one_sequence_of_all_heads():
    """[B, H, L, d], the library's own layout, beside dsv_sparse_attn_fwd that keeps every key."""
    B, H, L, d = 2, 3, 200, 128
    g = torch.Generator().manual_seed(1)
    Q, K, V = (torch.randn(B, H, L, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(3))
    p = dsv.Packed(1, L, L, L, L, B * H, B * H, d, "bf16", 0.1)
    cu = torch.tensor([0, L], dtype=torch.int32, device=DEV)
    O = torch.empty_like(Q)
    rows = lambda x: x.view(B * H, L, d).transpose(0, 1)  # noqa: E731
    _, lse = dsv.packed_attn_fwd(p, rows(Q), rows(K), rows(V), cu, cu, O=rows(O))
    sp = dsv.Problem(B, H, L, d, 16, "bf16", [L] * H, 0.1)
    idx = torch.arange(L, dtype=torch.int32, device=DEV).repeat(B * H * L)
    Os, lses = dsv.sparse_attn_fwd(sp, Q, K, V, idx)
    # both round O once, and weights by 2^-8 at most: within two steps of either bound
    assert (O.float() - Os.float()).abs().max() <= 4 * 2.0 ** -8 * V.float().abs().max()
    assert (lse.view(B, H, L) - lses).abs().max() < 1e-4


def test_without_the_tail():
    Case([5, 60, 200], [5, 60, 200], 2, 2, 128, "bf16", True).check(tail=False)


def test_the_tail_is_what_rounding_took():
    c = Case([130], [200], 2, 2, 64, "bf16")
    t = torch.empty(c.Q.shape, dtype=torch.bfloat16, device=DEV)
    O, _ = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O_tail=t)
    assert (t.float().abs() <= 2.0 ** -8 * O.float().abs()).all() and (t != 0).any()
    O2, _ = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu)
    assert torch.equal(O, O2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many", [False, True])
def test_rows_of_no_sequence(dtype, many):
    """Not written, and NaN in them reaches nothing: rows behind the last sequence and between cut ones."""
    H = 32 if many else 2
    lens = [200, 333, 90, 500] if many else [40, 77, 1]
    c = Case(lens, lens, H, H, 64, dtype, True, spare_q=50, spare_k=70)
    for x, used in ((c.Q, sum(lens)), (c.K, sum(lens)), (c.V, sum(lens)), (c.dO, sum(lens))):
        x[used:] = float("nan")
    outs = dict(O=torch.full_like(c.Q, 7), lse=torch.full((H, c.Q.shape[0]), 7.0, device=DEV))
    dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, **outs)
    grads = dict(dQ=torch.full_like(c.Q, 7), dK=torch.full_like(c.K, 7), dV=torch.full_like(c.V, 7))
    O = outs["O"].clone()
    O[sum(lens):] = float("nan")
    dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, outs["lse"], c.dO, **grads)
    want = c.want(tail=False)
    for n, x in {**outs, **grads}.items():
        ref.assert_within(n, x, want[n])
        rest = x[:, sum(lens):] if n == "lse" else x[sum(lens):]
        assert (rest == 7).all(), n


def test_sequences_longer_than_the_limits_and_ends_behind_the_tensors():
    """Nothing outside the tensors is touched, and the sequences that keep to the limits come out right."""
    lens = [60, 50, 40]
    c = Case(lens, lens, 2, 2, 64, "bf16")
    want = c.want()
    c.p = dsv.Packed(3, 150, 150, 50, 50, 2, 2, 64, "bf16", c.scale)          # the first one is longer than 50
    out = c.run()
    for n in out:
        v, b = (x.clone() for x in want[n])
        (v[:, :60] if n == "lse" else v[:60]).fill_(float("nan"))
        ref.assert_within(n, out[n], (v, b))
    c.p = dsv.Packed(3, 150, 150, 60, 60, 2, 2, 64, "bf16", c.scale)
    c.dcu = (torch.tensor([0, 60, 110, 1000], dtype=torch.int32, device=DEV), torch.tensor([0, 60, 110, 2 ** 31 - 1], dtype=torch.int32, device=DEV))
    out = c.run()
    for n in out:
        ref.assert_within(n, out[n], want[n])                                  # cut at the tensors' ends: the same lengths
    c.dcu = tuple(torch.tensor([0, 60, -5, 150], dtype=torch.int32, device=DEV) for _ in range(2))
    out = c.run()
    for n in out:
        v, b = (x.clone() for x in want[n])
        (v[:, 60:] if n == "lse" else v[60:]).fill_(float("nan"))
        # the third one now begins at 0 and ends at 150: cut to 60 of the same rows
        (v[:, :60] if n == "lse" else v[:60]).fill_(float("nan"))
        ref.assert_within(n, torch.nan_to_num(out[n].float()), (v, b))


def test_many_sequences():
    """More than the 64 that one step of the search looks at."""
    g = torch.Generator().manual_seed(9)
    lens = torch.randint(0, 12, (333,), generator=g).tolist()
    Case(lens, lens, 2, 1, 64, "bf16", True).check()
    Case([1] * 4200, torch.randint(0, 4, (4200,), generator=g).tolist(), 1, 1, 64, "f32", True).check()


def test_shared_inputs_of_many_heads():
    """K and V of one head, broadcast by a stride of zero: gradients come out head by head."""
    c = Case([100], [90], 4, 4, 64, "bf16")
    one = [x[:, :1].clone() for x in c.host[1:3]]
    c.host[1], c.host[2] = (x.expand(-1, 4, -1).contiguous() for x in one)
    c.K, c.V = (x.to(DEV).expand(-1, 4, -1) for x in one)
    c.check()


def test_peaked_and_flat_weights():
    for scale in (1e-6, 3.0):
        Case([65, 200], [65, 200], 2, 2, 128, "f32", True, scale=scale).check()
    c = Case([40], [40], 1, 1, 64, "bf16", scale=30.0)
    c.check()


def test_runs_are_equal_bit_for_bit():
    for c in (Case([900, 50], [900, 50], 4, 2, 128, "bf16", True), Case([1, 1], [2000, 300], 8, 2, 128, "bf16")):
        a, b = c.run(), c.run()
        for n in a:
            assert torch.equal(a[n], b[n]), n


def test_another_stream_and_poisoned_workspaces():
    c = Case([1, 30], [1500, 900], 4, 2, 128, "bf16", True)
    a = c.run()
    ws = torch.full((max(dsv.packed_attn_fwd_workspace(c.p), dsv.packed_attn_bwd_workspace(c.p)),), 255, dtype=torch.uint8, device=DEV)   # NaN patterns
    t = torch.empty(c.Q.shape, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    O, lse = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O_tail=t, workspace=ws, stream=side)
    with torch.cuda.stream(side):
        ws.fill_(255)
    dQ, dK, dV = dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, lse, c.dO, O_tail=t, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for n, x in dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV).items():
        assert torch.equal(x, a[n]), n


def test_a_captured_step_replays_on_other_lengths():
    lens = [30, 100, 70]
    c = Case(lens, lens, 4, 2, 64, "bf16", True, slack=200)
    other = Case([120, 10, 70], [120, 10, 70], 4, 2, 64, "bf16", True, slack=200)
    c.p = dsv.Packed(3, 200, 200, 200, 200, 4, 2, 64, "bf16", c.scale, causal=True)
    other.p = c.p
    eager, eager_other = c.run(), other.run()
    t = torch.empty(c.Q.shape, dtype=torch.bfloat16, device=DEV)
    out = {n: torch.zeros_like(x) for n, x in eager.items()}
    ws = torch.empty(max(dsv.packed_attn_fwd_workspace(c.p), dsv.packed_attn_bwd_workspace(c.p)), dtype=torch.uint8, device=DEV)

    def step():
        dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O=out["O"], lse=out["lse"], O_tail=t, workspace=ws)
        dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, out["O"], out["lse"], c.dO, dQ=out["dQ"], dK=out["dK"], dV=out["dV"], O_tail=t, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        now, expect = (c, eager) if rep % 2 == 0 else (other, eager_other)
        for a, b in zip(c.dcu, now.dcu if rep % 2 else (c.cu_q, c.cu_k)):
            a.copy_(b)
        for x in out.values():
            x.zero_()
        scratch = torch.randn(1 << 16, device=DEV).sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert math.isfinite(float(scratch))
        for n in out:      # the inputs of both cases are the same: one seed
            assert torch.equal(out[n], expect[n]), (rep, n)


@pytest.mark.parametrize("dtype,d,Hq,Hkv,causal", [("bf16", 128, 4, 4, False), ("bf16", 128, 4, 4, True), ("bf16", 64, 8, 2, True), ("f32", 64, 4, 2, True),
                                                   ("f32", 128, 3, 3, False), ("bf16", 64, 4, 4, False)])
def test_large_tiles_in_pieces(dtype, d, Hq, Hkv, causal):
    """Tiles of 128 rows that see the long axis in pieces, the pieces of short sequences and those that no row sees among them."""
    lens = [2100, 300, 1, 190] if causal else [2300]
    c = Case(lens, lens, Hq, Hkv, d, dtype, causal)
    assert dsv.packed_attn_fwd_workspace(c.p) >= 2 * sum(lens) * Hq * d * 4
    assert dsv.packed_attn_bwd_workspace(c.p) >= 2 * sum(lens) * Hq * d * 4 + sum(lens) * Hq * 8
    out = c.check(tail=False)
    # nothing is read of the workspace that this call has not written
    ws = torch.full((max(dsv.packed_attn_fwd_workspace(c.p), dsv.packed_attn_bwd_workspace(c.p)),), 255, dtype=torch.uint8, device=DEV)
    O, lse = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, workspace=ws)
    ws.fill_(255)
    dQ, dK, dV = dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, lse, c.dO, workspace=ws)
    for n, x in dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV).items():
        assert torch.equal(x, out[n]), n


@pytest.mark.parametrize("causal", [False, True])
def test_pieces_of_unequal_sides(causal):
    """More queries than keys and more keys than queries, large tiles, pieces; causal: queries that see no key, keys seen by all."""
    for lens_q, lens_k in (([1500, 700], [2600, 300]), ([2600, 300], [1500, 700])):
        c = Case(lens_q, lens_k, 4, 2, 64, "bf16", causal)
        assert dsv.packed_attn_fwd_workspace(c.p) > 0
        c.check()


@pytest.mark.parametrize("d,group", [(128, 2), (128, 8), (128, 16), (128, 32), (64, 2), (64, 16), (64, 32), (128, 5), (64, 6)])
@pytest.mark.parametrize("layout", ["token", "head"])
def test_groups_of_shared_heads(d, group, layout):
    """As many heads to a group as a load brings rows, fewer, more and no divisor of it; tiles that end inside a token's heads."""
    Hkv = 16 if group < 8 else 4
    lens = [430, 1, 130, 77]
    Case(lens, lens, Hkv * group, Hkv, d, "bf16", True, layout).check()


def _wide(x, width):
    """x [T, H, d] in rows of `width` elements."""
    T, H, d = x.shape
    return torch.empty(T * width, dtype=x.dtype, device=x.device)[: T * width].view(T, width)[:, : H * d].unflatten(1, (H, d)).copy_(x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_behind_four_gigabytes(dtype):
    """A long cache of wide rows, and its gradients in such rows; then as many queries."""
    T, width = 70001, 1 << 15
    for lens_q, lens_k in (([1], [T]), ([T], [40])):
        c = Case(lens_q, lens_k, 1, 1, 64, dtype, causal=lens_q == [1])
        assert T * width * c.Q.element_size() > 1 << 32
        if lens_k[0] == T:
            c.K, c.V = _wide(c.K, width), _wide(c.V, width)
            more = dict(dK=_wide(c.K, width), dV=_wide(c.V, width))
        else:
            c.Q, c.dO = _wide(c.Q, width), _wide(c.dO, width)
            more = dict(dQ=_wide(c.Q, width))
        O, lse = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O=None if lens_k[0] == T else _wide(c.Q, width))
        dQ, dK, dV = dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, lse, c.dO, **more)
        torch.cuda.synchronize()
        want = c.want(tail=False)
        for n, x in dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV).items():
            ref.assert_within(n, x, want[n])
        del c, O, dQ, dK, dV, more
        torch.cuda.empty_cache()


def test_two_graphs_share_a_workspace():
    """Replayed in turn with eager calls between; every call finds the workspace as the one before left it."""
    a = Case([1, 1, 1], [1500, 700, 33], 8, 2, 128, "bf16", True)
    b = Case([900], [900], 4, 4, 64, "bf16")
    size = max(f(c.p) for c in (a, b) for f in (dsv.packed_attn_fwd_workspace, dsv.packed_attn_bwd_workspace))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    graphs, outs, eager = [], [], [c.run(tail=False) for c in (a, b)]
    for c, e in zip((a, b), eager):
        out = {n: torch.zeros_like(x) for n, x in e.items()}

        def step(c=c, out=out):
            dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O=out["O"], lse=out["lse"], workspace=ws)
            dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, out["O"], out["lse"], c.dO, dQ=out["dQ"], dK=out["dK"], dV=out["dV"], workspace=ws)

        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
        outs.append(out)
    for rep in range(3):
        for g, out, c, e in zip(graphs, outs, (a, b), eager):
            for x in out.values():
                x.zero_()
            if rep:
                ws.fill_(255)
            g.replay()
            again = c.run(tail=False)
            for n in out:
                assert torch.equal(out[n], e[n]) and torch.equal(again[n], e[n]), (rep, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_keys_or_no_queries_at_all(dtype):
    c = Case([5, 0, 130], [0, 0, 0], 4, 2, 64, dtype, True)
    out = c.run()
    assert (out["O"] == 0).all() and (out["lse"] == -math.inf).all() and (out["dQ"] == 0).all() and out["dK"].shape == (0, 2, 64)
    c = Case([0, 0], [3, 200], 4, 2, 64, dtype)
    dK, dV = torch.full_like(c.K, 7), torch.full_like(c.V, 7)
    O, lse = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu)
    dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, lse, c.dO, dK=dK, dV=dV)
    assert O.shape == (0, 4, 64) and (dK == 0).all() and (dV == 0).all()


@pytest.mark.parametrize("dtype,side", [("bf16", "keys"), ("bf16", "queries"), ("f32", "keys"), ("f32", "queries")])
def test_the_widest_rows(dtype, side):
    """128 rows of just under 4 GB: the last 32-bit offsets inside a tile, for heads of their own and shared ones."""
    width = (1 << 25) // ref.DTYPES[dtype].itemsize - 16
    for Hq, T in ((2, 131), (4, 130)):
        c = Case([T], [T], Hq, 2, 128, dtype, True)
        more = {}
        if side == "keys":
            c.K, c.V = _wide(c.K, width), _wide(c.V, width)
        else:
            c.Q, c.dO = _wide(c.Q, width), _wide(c.dO, width)
            more = dict(O=_wide(c.Q, width))
        O, lse = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, **more)
        dQ, dK, dV = (torch.full(x.shape, float("nan"), dtype=x.dtype, device=DEV) for x in (c.Q, c.K, c.V))
        dsv.packed_attn_bwd(c.p, c.Q, c.K, c.V, *c.dcu, O, lse, c.dO, dQ=dQ, dK=dK, dV=dV)
        want = c.want(tail=False)
        for n, x in dict(O=O, lse=lse, dQ=dQ, dK=dK, dV=dV).items():
            ref.assert_within(n, x, want[n])
        del c, O, more
        torch.cuda.empty_cache()


def test_more_rows_than_one_axis_of_a_grid_takes():
    """17 million queries: the kernels with a wave to a few rows need a second axis.  64 bits on the GPU, over three keys."""
    T, nk, d = (1 << 24) + 1000, 3, 64
    torch.manual_seed(3)
    Q, dO = (torch.randn(T, 1, d, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    K, V = (torch.randn(nk, 1, d, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    cu = [torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (T, nk)]
    p = dsv.Packed(1, T, nk, T, nk, 1, 1, d, "bf16", 0.125)
    O, lse = dsv.packed_attn_fwd(p, Q, K, V, *cu)
    dQ, dK, dV = dsv.packed_attn_bwd(p, Q, K, V, *cu, O, lse, dO)
    k, v = K[:, 0].double(), V[:, 0].double()
    for lo in range(0, T, 1 << 22):
        q, do = Q[lo : lo + (1 << 22), 0].double(), dO[lo : lo + (1 << 22), 0].double()
        x = 0.125 * q @ k.t().contiguous()
        P = torch.softmax(x, 1)
        o = P @ v
        ds = P * (do @ v.t().contiguous() - (do * o).sum(1, keepdim=True))
        # O: its rounding and the weights', 2^-8 of the values each; dQ: O's rounding in Delta (sum |dO O|) beside the result's own
        part = slice(lo, lo + q.shape[0])
        assert ((O[part, 0].double() - o).abs() <= 2.0 ** -8 * o.abs() + 2.0 ** -7 * P @ v.abs()).all()
        assert (lse[0, part].double() - torch.logsumexp(x, 1)).abs().max() < 1e-4      # (d + 4) 2^-24 of scale sum |q k|, below 100 / 8
        off = 2.0 ** -7 * (do.abs() * (o.abs() + P @ v.abs())).sum(1, keepdim=True)
        dq, tol = 0.125 * ds @ k, 0.125 * (2.0 ** -8 * ds.abs() + P * off) @ k.abs()
        assert ((dQ[part, 0].double() - dq).abs() <= tol + 2.0 ** -8 * dq.abs()).all()
    assert dK.isfinite().all() and dV.isfinite().all()
