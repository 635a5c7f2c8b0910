"""The step of packed attention in 64 bits with the roundings to bf16 that the library makes, each of them to be left out or made twice: what its
gradients are off by, in norm, tells whether it keeps what it says it keeps.  Plain torch on the CPU; nothing of the package is used.

Let r be what rounding to bf16 is off by in norm: half a step is 2^-8 at the bottom of a binade, so r <= 2^-8 / sqrt(3) = 2.26e-3, and 1.66e-3
for values spread over their binades.  Roundings that do not know of each other add as squares.
  dQ: its own; and Delta by O's weights, delta Delta_i = sum_j eps_ij dS_ij, which reaches dQ_i by scale times the average of K, below the whole
      of it: at most sqrt(2) r = 2.35e-3.  dS as one word: sqrt(3) r = 2.87e-3 where a row sees few keys.
  dK: its own, Delta's, and dS as one word: at most sqrt(3) r = 2.87e-3.
  dV: its own and that of the weights, sqrt(2) r = 2.35e-3.
Delta by O alone is off by sum_c eps_c dO_c O_c besides, which has nothing of dS in it: where a row sees one key, dS is 0 and this is not."""
import torch

DQ_MOST, DK_MOST, DV_MOST = 2.4e-3, 3e-3, 2.4e-3

# lengths of causal sequences: rows that see one to 24 keys, where roundings of O and dS weigh most; sequences that fill tiles of 128 rows
FEW_KEYS = [1 + i % 24 for i in range(96)]
MANY_ROWS = [300, 129, 511, 128]


def bf16(x):
    return x.float().to(torch.bfloat16).double()


def off(got, want):
    """|got - want| / |want| in norm, over the values that are numbers in `want`."""
    got, want = got.detach().double().cpu(), want.cpu()
    look = ~want.isnan()
    return float((got - want)[look].norm() / want[look].norm())


def step(Q, K, V, dO, cu_q, cu_k, scale, causal, tail=True, words=2):
    """{name: value} of O, O_tail, dQ, dK, dV; `words` of dS in dQ's product, Delta by O and its tail or by O alone."""
    g, out = Q.shape[1] // K.shape[1], {n: torch.zeros_like(x) for n, x in (("O", Q), ("O_tail", Q), ("dQ", Q), ("dK", K), ("dV", V))}
    for s in range(len(cu_q) - 1):
        a, b = slice(int(cu_q[s]), int(cu_q[s + 1])), slice(int(cu_k[s]), int(cu_k[s + 1]))
        nq, nk = a.stop - a.start, b.stop - b.start
        if nk == 0 or nq == 0:
            continue
        for h in range(Q.shape[1]):
            q, k, v, do = Q[a, h], K[b, h // g], V[b, h // g], dO[a, h]
            x = scale * (q @ k.T)
            if causal:
                x = x.masked_fill(torch.arange(nk)[None] > torch.arange(nq)[:, None] + nk - nq, -torch.inf)
            top = x.amax(1, keepdim=True)
            top = torch.where(top.isinf(), 0.0, top)
            w = bf16(torch.exp(x - top))
            whole = w.sum(1, keepdim=True)
            o = torch.where(whole > 0, w @ v / whole.clamp(min=1e-300), 0.0)
            out["O"][a, h] = bf16(o)
            out["O_tail"][a, h] = bf16(o - bf16(o))
            e = torch.exp(x - top)
            p = e / e.sum(1, keepdim=True).clamp(min=1e-300)
            kept = bf16(o) + (bf16(o - bf16(o)) if tail else 0.0)
            ds = p * (do @ v.T - (do * kept).sum(1, keepdim=True))
            one = bf16(ds)
            out["dQ"][a, h] = scale * ((one + (bf16(ds - one) if words == 2 else 0.0)) @ k)
            out["dK"][b, h // g] += scale * (one.T @ q)
            out["dV"][b, h // g] += bf16(p).T @ do
    for n in ("dQ", "dK", "dV"):
        out[n] = bf16(out[n])
    return out
