"""The weights of bf16 attention over the 8-bit cache in blocks of 32 rows: two bf16 words each, so that O is off by little but its own rounding."""
import math

import pytest
import torch

import packed_ref
from test_gpu_cache import ints, make_cache

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


@pytest.mark.parametrize("new,lens,Hq,Hkv,d,page", [([1] * 5, [3000, 700, 513, 90, 1], 8, 2, 128, 64), ([1, 1], [6000, 2047], 14, 2, 64, 128), ([9, 33, 1], [400, 1500, 77], 4, 4, 128, 16),
                                                    ([5, 2], [20, 2500], 6, 3, 64, 256)])
def test_weights_are_not_rounded_to_one_word(new, lens, Hq, Hkv, d, page):
    """Scores, sums and exponentials have the bounds of the fp32 call (the products of bf16 are exact in 32 bits for both).  A weight is within 2^-8 of its first
    word and what that leaves within 2^-8 of the second: 2^-16 of sum p |v|.  O itself is rounded once, 2^-8 of the result.  (One word alone: 2^-8 of sum p |v|.)"""
    table, n_pages, K8, V8, ks, vs, Kw, Vw, basis = make_cache(lens, Hkv, d, page, 3)
    g, T, scale = torch.Generator().manual_seed(5), sum(new), 0.5 / math.sqrt(d)
    Q = (torch.randn(T, Hq, d // 2, generator=g) @ basis).to(torch.bfloat16)
    p = dsv.Cache(len(new), T, max(new), Hq, Hkv, d, "bf16", n_pages, page, table.shape[1], scale=scale)
    cu = packed_ref.cu_of(new)
    O, lse = dsv.cache_attn_fwd(p, Q.to(DEV), cu.to(DEV), ints(lens), table.to(DEV), *(t.to(DEV) for t in (K8, V8, ks, vs)))
    args = (cu, packed_ref.cu_of(lens), float(torch.tensor(scale)), True)
    want = packed_ref.attention(Q.double(), Kw, Vw, *args, dtype="f32")
    value, bound = want["O"]
    sizes = packed_ref.attention(Q.double(), Kw, Vw.abs(), *args, dtype="f32")["O"][0]
    off = bound + 2.0 ** -16 * sizes
    packed_ref.assert_within("O", O, (value, off + 2.0 ** -8 * (value.abs() + off)))
    packed_ref.assert_within("lse", lse, want["lse"])
