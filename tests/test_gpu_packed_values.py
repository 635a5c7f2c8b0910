"""Packed attention on the GPU: roundings that it says it keeps, in norm; sums over its longest row axis."""
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
