"""Attention over packed sequences and layer norm from their formulas in 64 bits, with element-wise bounds on what a kernel that rounds
where the library says it does may be off by.  Plain torch on the CPU; nothing of the package is used.

u is half a step of the storage type (bf16 2^-8, fp32 2^-24), e = 2^-24 half a step of the 32-bit sums."""
import math

import torch

E = 2.0 ** -24
TINY = 2.0 ** -126
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def cu_of(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32)


def attention(Q, K, V, cu_q, cu_k, scale, causal, dO=None, dtype="bf16", tail=True):
    """Q [T, Hq, d] .. in float64 holding storage-type values.  {name: (value, bound)} for O, lse and, with dO, dQ, dK, dV; rows of no
    sequence are NaN in the values.

    Bounds, per query row: a score is a sum of d products, e_s = (d + 4) e scale sum |q k|; its exponential, against a maximum or the
    lse held in 32 bits, is off by w = 2 e_s + 4 e (|s| + |lse|) + 8 e relatively.  Weights enter the sums over keys as storage-type
    values (u), sums of n terms in 32 bits add n e.  dS = p (dP - Delta): w of p, (d + 4) e sum |dO v| of dP, and of Delta what O is off by
    -- u^2 of itself with the tail, u without, and the weights' part -- against |dO|.  A weight, a dS or a product of them below 2^-126, the
    least normal number of both types, may be taken for zero: 2^-126 more for each, against what it multiplies."""
    u = HALF_STEP[dtype]
    Hq, Hkv, d = Q.shape[1], K.shape[1], Q.shape[2]
    g = Hq // Hkv
    nan = float("nan")
    val = {"O": torch.full_like(Q, nan), "lse": torch.full((Hq, Q.shape[0]), nan, dtype=torch.float64)}
    bnd = {"O": torch.zeros_like(Q), "lse": torch.zeros((Hq, Q.shape[0]), dtype=torch.float64)}
    if dO is not None:
        for n, x in (("dQ", Q), ("dK", K), ("dV", V)):
            val[n], bnd[n] = torch.full_like(x, nan), torch.zeros_like(x)
    for s in range(len(cu_q) - 1):
        qa, qb, ka, kb = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        nq, nk = qb - qa, kb - ka
        if dO is not None:
            for n in ("dK", "dV"):
                val[n][ka:kb] = 0
        for h in range(Hq):
            q, k, v = Q[qa:qb, h], K[ka:kb, h // g], V[ka:kb, h // g]
            x = scale * (q @ k.T)
            if causal:
                seen = torch.arange(nk)[None] <= torch.arange(nq)[:, None] + nk - nq
            else:
                seen = torch.ones(nq, nk, dtype=torch.bool)
            x = x.masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(x, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            lse0 = torch.where(lse.isinf(), 0.0, lse)
            p = torch.exp(x - lse0[:, None])
            O = p @ v
            es = (d + 4) * E * scale * (q.abs() @ k.abs().T)
            w = 2 * es + 4 * E * (x.masked_fill(~seen, 0).abs() + lse0.abs()[:, None]) + 8 * E
            mass = (p * (w + u + nk * E) + TINY) @ v.abs() + nk * TINY
            val["O"][qa:qb, h], val["lse"][h, qa:qb] = O, lse
            off_O = mass + 4 * E * O.abs()
            bnd["O"][qa:qb, h] = u * O.abs() + off_O
            bnd["lse"][h, qa:qb] = (p * w).sum(1) + (nk + 8) * E + 2 * E * lse0.abs()
            if dO is None:
                continue
            do = dO[qa:qb, h]
            dp = do @ v.T
            delta = (do * O).sum(1, keepdim=True)
            ds = p * (dp - delta)
            off_delta = (do.abs() * (off_O + (u * u if tail else u) * O.abs())).sum(1, keepdim=True) + (d + 4) * E * (do.abs() * O.abs()).sum(1, keepdim=True)
            off_ds = (w + u + 4 * E) * ds.abs() + TINY * (1 + (dp - delta).abs()) + p * ((d + 4) * E * (do.abs() @ v.abs().T) + off_delta)
            sums = ds.abs() + off_ds
            val["dQ"][qa:qb, h] = scale * (ds @ k)
            bnd["dQ"][qa:qb, h] = scale * ((off_ds + nk * E * sums) @ k.abs() + nk * TINY) + (u + 2 * E) * val["dQ"][qa:qb, h].abs()
            n_rows = nq * g
            val["dK"][ka:kb, h // g] += scale * (ds.T @ q)
            bnd["dK"][ka:kb, h // g] += scale * ((off_ds + n_rows * E * sums).T @ q.abs() + nq * TINY)
            val["dV"][ka:kb, h // g] += p.T @ do
            bnd["dV"][ka:kb, h // g] += (p * (w + u + n_rows * E) + TINY).T @ do.abs() + nq * TINY
    if dO is not None:
        for n in ("dK", "dV"):
            bnd[n] += (u + 2 * E) * val[n].nan_to_num().abs()
    return {n: (val[n], bnd[n]) for n in val}


def norm(X, gamma, beta, eps, dY=None, dtype="bf16"):
    """{name: (value, bound)} of Y, mean, rstd and, with dY, dX, dgamma, dbeta; X [tokens, heads, n] float64.

    The mean is off by n e mean|x|, a difference from it by that and e of itself, the variance relatively by (n + 8) e plus twice
    what the mean's error makes of it (it enters squared and crosswise), 1 / sqrt by half of that and 2 e."""
    u, n, rows = HALF_STEP[dtype], X.shape[2], X.shape[0] * X.shape[1]
    gam = torch.ones(n, dtype=torch.float64) if gamma is None else gamma
    bet = torch.zeros(n, dtype=torch.float64) if beta is None else beta
    mu = X.mean(2, keepdim=True)
    c = X - mu
    var = c.square().mean(2, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    xh = c * r
    off_mu = (n + 2) * E * X.abs().mean(2, keepdim=True)
    off_c = off_mu + 2 * E * c.abs()
    off_var = (n + 8) * E * var + 2 * (c.abs() * off_c).mean(2, keepdim=True) + off_c.square().mean(2, keepdim=True)
    rel_r = off_var * r * r + 4 * E          # d(1/sqrt t) = t^(-3/2) dt / 2; twice that covers the second order of small variances
    off_xh = r * off_c * (1 + rel_r) + xh.abs() * rel_r + 2 * E * xh.abs()
    y = xh * gam + bet
    out = {"Y": (y, u * y.abs() + gam.abs() * off_xh + 4 * E * ((xh * gam).abs() + bet.abs())),
           "mean": (mu[..., 0], off_mu[..., 0] + E * mu[..., 0].abs()), "rstd": (r[..., 0], (r * rel_r)[..., 0])}
    if dY is None:
        return out
    g = dY * gam
    m1, m2 = g.mean(2, keepdim=True), (g * xh).mean(2, keepdim=True)
    dx = r * (g - m1 - xh * m2)
    off_m1 = (n + 4) * E * g.abs().mean(2, keepdim=True)
    off_m2 = (n + 4) * E * (g * xh).abs().mean(2, keepdim=True) + (g.abs() * off_xh).mean(2, keepdim=True)
    off_dx = r * (4 * E * (g.abs() + m1.abs() + (xh * m2).abs()) + off_m1 + xh.abs() * off_m2 + off_xh * (m2.abs() + off_m2)) + dx.abs() * (rel_r + 2 * E)
    out["dX"] = (dx, u * dx.abs() + off_dx)
    out["dgamma"] = ((dY * xh).sum((0, 1)), ((rows + 4) * E * (dY * xh).abs() + dY.abs() * off_xh).sum((0, 1)))
    out["dbeta"] = (dY.sum((0, 1)), (rows * E * dY.abs()).sum((0, 1)))
    return out


def assert_within(name, got, want):
    """got within want's bound of want's value, element by element; NaN in the value: not looked at; infinities have to agree."""
    value, bound = want
    got = got.detach().double().cpu()
    assert got.shape == value.shape, f"{name}: {tuple(got.shape)} for {tuple(value.shape)}"
    look = ~value.isnan()
    inf = look & value.isinf()
    assert torch.equal(got[inf], value[inf]), f"{name}: infinities"
    look &= ~inf
    assert got[look].isfinite().all(), f"{name}: {int((~got[look].isfinite()).sum())} values are not finite"
    err, tol = (got - value).abs()[look], bound[look]
    bad = err > tol
    if bad.any():
        worst = int((err / tol.clamp(min=1e-300)).argmax())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} out of bounds; worst {err[worst]:.3e} for {tol[worst]:.3e} at value {value[look][worst]:.3e}")


# ---------------------------------------------------------------------------------------------- inputs
def laid_out(x, layout, more=2):
    """x [T, H, d] as a view: as it is, head by head, or a slice of wider rows."""
    if layout == "head":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "slice":
        wide = torch.full((x.shape[0], x.shape[1] + more, x.shape[2]), float("nan"), dtype=x.dtype, device=x.device)
        wide[:, 1 : 1 + x.shape[1]] = x
        return wide[:, 1 : 1 + x.shape[1]]
    return x


def attention_inputs(total_q, total_k, Hq, Hkv, d, dtype, seed=0):
    """Values of the storage type, on the CPU in that type: Q and K share directions, so that weights are uneven."""
    g = torch.Generator().manual_seed(seed)
    basis = torch.randn(d // 2, d, generator=g) / math.sqrt(d // 2)
    Q = torch.randn(total_q, Hq, d // 2, generator=g) @ basis
    K = torch.randn(total_k, Hkv, d // 2, generator=g) @ basis
    V, dO = torch.randn(total_k, Hkv, d, generator=g), torch.randn(total_q, Hq, d, generator=g)
    return [x.to(DTYPES[dtype]) for x in (Q, K, V, dO)]
