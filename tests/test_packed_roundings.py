"""The bounds on gradients of packed attention, in norm, tell its roundings from ones that it does not make.  CPU only."""
import math

import pytest

import packed_ref as ref
import packed_roundings as rnd


@pytest.mark.parametrize("d,group,lens,peak", [(64, 1, rnd.FEW_KEYS, 2), (128, 2, rnd.FEW_KEYS, 2), (64, 1, rnd.MANY_ROWS, 2), (128, 1, rnd.MANY_ROWS, 8)])
def test_bounds_tell_the_roundings_apart(d, group, lens, peak):
    cu = ref.cu_of(lens)
    Q, K, V, dO = (x.double() for x in ref.attention_inputs(sum(lens), sum(lens), 2 * group, 2, d, "bf16", 21))
    scale = peak / math.sqrt(d)
    want = {n: v for n, (v, _) in ref.attention(Q, K, V, cu, cu, scale, True, dO).items()}

    def off(**kw):
        got = rnd.step(Q, K, V, dO, cu, cu, scale, True, **kw)
        return {n: rnd.off(got[n], want[n]) for n in ("dQ", "dK", "dV")}

    kept = off()
    assert kept["dQ"] < rnd.DQ_MOST and kept["dK"] < rnd.DK_MOST and kept["dV"] < rnd.DV_MOST, kept
    assert off(words=1)["dQ"] > rnd.DQ_MOST
    without = off(tail=False)
    assert without["dQ"] > 1.2 * kept["dQ"] and without["dQ"] > rnd.DQ_MOST and without["dK"] > rnd.DK_MOST, without
