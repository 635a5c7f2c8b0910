"""Packed attention on the GPU: roundings that it says it keeps, in norm; rows that are not numbers; long sequences among single
rows; sums over its longest row axis."""
import math

import pytest
import torch

import packed_ref as ref
import packed_roundings as rnd
from test_gpu_packed import DEV, Case, dsv

pytestmark = pytest.mark.gpu

# the form of a call follows from rows, heads and sequences: tiles of 32 rows for few of them, of 128 for many
FORMS = [(rnd.FEW_KEYS, 64, 4, 2, 2), (rnd.FEW_KEYS, 128, 4, 4, 2), (rnd.MANY_ROWS, 64, 32, 32, 2), (rnd.MANY_ROWS, 128, 32, 32, 8), (rnd.MANY_ROWS, 128, 64, 32, 2)]


@pytest.mark.parametrize("lens,d,Hq,Hkv,peak", FORMS)
def test_gradients_keep_the_bits_they_are_said_to_keep(lens, d, Hq, Hkv, peak):
    """dS as two words in dQ, Delta by all bits of O: without either the errors pass these bounds, as the same roundings in 64 bits do."""
    c = Case(lens, lens, Hq, Hkv, d, "bf16", True, seed=21, scale=peak / math.sqrt(d))
    want = {n: v for n, (v, _) in c.want().items()}
    got = c.run()
    off = {n: rnd.off(got[n], want[n]) for n in ("O", "dQ", "dK", "dV")}
    assert off["dQ"] < rnd.DQ_MOST and off["dK"] < rnd.DK_MOST and off["dV"] < rnd.DV_MOST, off
    without = c.run(tail=False)
    assert rnd.off(without["dQ"], want["dQ"]) > 1.2 * off["dQ"], off


@pytest.mark.parametrize("lens_q,lens_k,Hq,Hkv", [([1 + i % 40 for i in range(64)], [1 + i % 32 for i in range(64)], 4, 2),    # tiles of 32 rows, a wave to 32 keys
                                                  ([200, 129, 300], [64, 33, 50], 64, 64)])                                     # of 128 rows and 64 keys
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["token", "head", "slice"])
def test_the_output_and_its_tail_are_the_average_by_the_rounded_weights(lens_q, lens_k, Hq, Hkv, d, layout):
    """All keys of a row in one tile: the weights are 2^(s - max), rounded.  O and its tail together hold 16 bits of their average, 2^-17 of it
    in norm.  A weight is rounded the other way where its score's error in 32 bits takes it over the middle of a step: 3e-6 (24 steps of 2^-24 times the score's
    size, 20) either side of the middles of steps of 2^-8 at least, one in 600, and each moves the average by 2^-8 of that weight's share at most: 1.7e-4."""
    c = Case(lens_q, lens_k, Hq, Hkv, d, "bf16", layout=layout, seed=5)
    tail = torch.full(c.Q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    O, _ = dsv.packed_attn_fwd(c.p, c.Q, c.K, c.V, *c.dcu, O_tail=tail)
    Q, K, V, dO = (x.double() for x in c.host)
    want = torch.zeros_like(Q)
    for s in range(len(lens_q)):
        a, b = slice(int(c.cu_q[s]), int(c.cu_q[s + 1])), slice(int(c.cu_k[s]), int(c.cu_k[s + 1]))
        for h in range(Hq):
            x = c.scale * (Q[a, h] @ K[b, h // (Hq // Hkv)].T)
            w = rnd.bf16(torch.exp(x - x.amax(1, keepdim=True)))
            want[a, h] = w @ V[b, h // (Hq // Hkv)] / w.sum(1, keepdim=True)
    assert rnd.off(O.double() + tail.double(), want) < 5e-4
    assert rnd.off(O, want) > 1e-3                       # what the tail holds
    assert (tail.float().abs() <= 2.0 ** -8 * O.float().abs()).all()


NAN = [
    dict(lens_q=[40, 50], lens_k=[40, 50], Hq=4, Hkv=2, d=64),                              # tiles of 32 rows
    dict(lens_q=[1] * 4, lens_k=[2500, 1200, 31, 700], Hq=4, Hkv=2, d=128),                 # and in pieces
    dict(lens_q=[1, 1], lens_k=[20000, 300], Hq=4, Hkv=2, d=128),                           # more than eight
    dict(lens_q=[300, 129, 511, 128], lens_k=[300, 129, 511, 128], Hq=32, Hkv=32, d=64),    # tiles of 128 rows
    dict(lens_q=[2300, 190], lens_k=[2300, 190], Hq=4, Hkv=4, d=128),                       # and in pieces
    dict(lens_q=[2300, 190], lens_k=[2300, 190], Hq=4, Hkv=2, d=64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("form", range(len(NAN)))
@pytest.mark.parametrize("where", ["query", "key", "infinite score"])
def test_scores_that_are_no_numbers_are_not_taken_for_no_keys(form, dtype, causal, where):
    """A row with such a score has no O, no lse and no gradient that is a number, and so have the keys it sees; other sequences and heads keep
    theirs bit for bit, other rows of its tile (sums are rescaled for all of a wave's rows at once) within the bounds."""
    c = Case(dtype=dtype, causal=causal, seed=form, **NAN[form])
    clean = c.run()
    g, Hkv = c.p.Hq // c.p.Hkv, c.p.Hkv
    s = 1                                                # the sequence, K/V head and row or key of it
    a, b = slice(int(c.cu_q[s]), int(c.cu_q[s + 1])), slice(int(c.cu_k[s]), int(c.cu_k[s + 1]))
    nq, nk, hk = a.stop - a.start, b.stop - b.start, Hkv - 1
    i, j = nq - 1 - nq // 3, nk // 3
    rows = torch.zeros(c.p.total_q, c.p.Hq, dtype=torch.bool, device=DEV)                   # that see such a score
    if where == "key":
        c.K[b.start + j, hk, 5] = float("nan")
        rows[a.start + (max(0, j - (nk - nq)) if causal else 0) : a.stop, hk * g : (hk + 1) * g] = True
    else:
        if where == "query":
            c.Q[a.start + i, hk * g, 5] = float("nan")
        else:
            c.Q[a.start + i, hk * g] = 1e25
            c.K[b.start + j, hk] = 1e25
        rows[a.start + i, hk * g] = True
    seen = torch.zeros(c.p.total_k, Hkv, dtype=torch.bool, device=DEV)                      # keys that such a row sees
    last = (nq - 1 if where == "key" else i) + nk - nq if causal else nk - 1
    assert not causal or j <= last
    seen[b.start : b.start + last + 1, hk] = True
    mine, mine_k = torch.zeros_like(rows), torch.zeros_like(seen)                           # the sequence and heads that it is among
    mine[a, hk * g : (hk + 1) * g], mine_k[b, hk] = True, True
    got = c.run()
    assert got["lse"].t()[rows].isnan().all()
    for n in ("O", "dQ"):
        assert got[n][rows].isnan().all(), n
        assert torch.equal(got[n][~mine], clean[n][~mine]), n
    for n in ("dK", "dV"):
        assert not got[n][seen].isfinite().any(), n
        assert torch.equal(got[n][~mine_k], clean[n][~mine_k]), n
    assert torch.equal(got["lse"].t()[~mine], clean["lse"].t()[~mine])
    if where == "query" or where == "key" and causal:    # rows that do not see it
        want = c.want(grad=False)                        # from the inputs as they were
        for n in ("O", "lse"):
            value, bound = want[n]
            value[rows.t().cpu() if n == "lse" else rows.cpu()] = float("nan")
            ref.assert_within(n, got[n], (value, bound))


@pytest.mark.parametrize("dtype,causal,Hq,Hkv", [("bf16", False, 8, 8), ("bf16", True, 8, 2), ("f32", True, 4, 4)])
def test_a_long_sequence_among_single_rows(dtype, causal, Hq, Hkv):
    """A prompt among new tokens of other streams, first, last and in the middle of them."""
    for at in (0, 40, 80):
        lens_q = [1] * 80
        lens_k = [1 + 37 * i % 300 for i in range(80)]
        lens_q.insert(at, 1500)
        lens_k.insert(at, 1700)
        Case(lens_q, lens_k, Hq, Hkv, 128, dtype, causal, seed=at).check()


def test_sums_over_seventeen_million_rows():
    """dK and dV of three keys, in pieces of a quarter of a million rows: one of 64 left out, taken twice or from another place is 2^-6 of the sums,
    where rounding the results is 2^-8 at most and the other roundings, random over so many rows, leave less than a quarter of that (the sums of a
    piece in 32 bits: 2^14 steps of half of 2^-24 if all went one way)."""
    T, nk, d = (1 << 24) + 1000, 3, 64
    torch.manual_seed(4)
    late = (1 + 0.25 * torch.arange(T, device=DEV) / T)[:, None, None]                             # the pieces' shares are unlike
    Q = (late * (0.5 + 0.5 * torch.randn(T, 1, d, device=DEV))).to(torch.bfloat16)
    dO = (late * (torch.randn(d, device=DEV) + torch.randn(T, 1, d, device=DEV))).to(torch.bfloat16)
    K, V = (torch.randn(nk, 1, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    cu = [torch.tensor([0, n], dtype=torch.int32, device=DEV) for n in (T, nk)]
    p = dsv.Packed(1, T, nk, T, nk, 1, 1, d, "bf16", 0.125)
    O, lse = dsv.packed_attn_fwd(p, Q, K, V, *cu)
    _, dK, dV = dsv.packed_attn_bwd(p, Q, K, V, *cu, O, lse, dO)
    k, v = K[:, 0].double(), V[:, 0].double()
    sum_k, sum_v, shares = torch.zeros_like(k), torch.zeros_like(v), []
    for lo in range(0, T, 1 << 21):
        q, do = Q[lo : lo + (1 << 21), 0].double(), dO[lo : lo + (1 << 21), 0].double()
        P = torch.softmax(0.125 * q @ k.t().contiguous(), 1)
        ds = P * (do @ v.t().contiguous() - (do * (P @ v)).sum(1, keepdim=True))
        part_k, part_v = 0.125 * ds.t().contiguous() @ q, P.t().contiguous() @ do
        sum_k += part_k
        sum_v += part_v
        shares.append((part_k, part_v))
    for name, got, want, at in (("dK", dK, sum_k, 0), ("dV", dV, sum_v, 1)):
        for share in shares[:-1]:                        # of like parts: eighths, within a factor of two
            assert share[at].norm() > want.norm() / 16, name
        assert rnd.off(got[:, 0], want) < 2.0 ** -8 + 2.0 ** -10, name
