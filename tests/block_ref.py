"""Rotary positions, gated norms and the 8-bit cache from their formulas in 64 bits, with element-wise bounds on what a kernel that rounds where the
library says it does may be off by.  Plain torch on the CPU; nothing of the package is used.

u is half a step of the storage type (bf16 2^-8, fp32 2^-24), E = 2^-24 half a step of the 32-bit sums (packed_ref)."""
import math

import torch

from packed_ref import DTYPES, E, HALF_STEP, TINY


# ---------------------------------------------------------------------------------------------- rotary
def pairs_of(pairs, layout):
    """[(lo, hi, coordinate)] of every pair, by hand."""
    out, done = [], 0
    total = sum(pairs)
    for axis, n in enumerate(pairs):
        for i in range(n):
            if layout == "interleaved":
                out.append((2 * (done + i), 2 * (done + i) + 1, axis))
            elif layout == "halves":
                out.append((done + i, total + done + i, axis))
            else:
                out.append((2 * done + i, 2 * done + n + i, axis))
        done += n
    return out


def rotary(X, pos, freq, pairs, layout, gain=1.0, back=False, dtype="bf16", in_32=False):
    """(value, bound) of X [tokens, heads, d] float64 turned.  in_32: the bound before the last rounding to the storage type.

    An angle is formed in 64 bits (three roundings of it, 2^-51 of it in all), brought within half a turn and rounded to 32 bits (2^-26 turns at
    most), its sine and cosine are good to 4 E, the gain's product to E; a result is two products and a sum, 3 E of their sizes."""
    lo, hi, axis = (torch.tensor(v) for v in zip(*pairs_of(pairs, layout)))
    t = pos.double()[:, axis] * freq
    c, s = gain * torch.cos(t)[:, None], gain * torch.sin(t)[:, None]
    if back:
        s = -s
    off = (abs(gain) * (2 * math.pi * 2.0 ** -26 + t.abs() * 2.0 ** -51 + 6 * E))[:, None]
    y, bound = X.clone(), torch.zeros_like(X)
    a, b = X[:, :, lo], X[:, :, hi]
    y[:, :, lo], y[:, :, hi] = a * c - b * s, a * s + b * c
    sizes = off * (a.abs() + b.abs()) + 3 * E * ((a * c).abs() + (b * s).abs())
    bound[:, :, lo], bound[:, :, hi] = sizes, off * (a.abs() + b.abs()) + 3 * E * ((a * s).abs() + (b * c).abs())
    if not in_32:
        bound += HALF_STEP[dtype] * (y.abs() + bound) * (bound > 0) + TINY
    return y, bound


def freqs(pairs, base=10000.0):
    return torch.cat([base ** (-torch.arange(n, dtype=torch.float64) / max(1, n)) for n in pairs])


# ---------------------------------------------------------------------------------------------- gated norm
def _normed(v, off, eps, rms, n):
    """(normed, r, bound of normed, relative bound of r) of rows v that are off by `off` already: as packed_ref.norm has it."""
    if rms:
        c, off_c = v, off
        mu, off_mu = torch.zeros_like(v[:, :1]), torch.zeros_like(v[:, :1])
    else:
        mu = v.mean(1, keepdim=True)
        off_mu = (n + 2) * E * v.abs().mean(1, keepdim=True) + off.mean(1, keepdim=True)
        c = v - mu
        off_c = off + off_mu + 2 * E * c.abs()
    var = c.square().mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    off_var = (n + 8) * E * var + 2 * (c.abs() * off_c).mean(1, keepdim=True) + off_c.square().mean(1, keepdim=True)
    rel = off_var * r * r + 4 * E
    return c * r, r, r * off_c * (1 + rel) + (c * r).abs() * (rel + 2 * E), rel, mu, off_mu


def _back(w, off_w, xh, off_xh, r, rel, rms, n):
    """(r (w - mean w - xh mean(w xh)), its bound)."""
    m1 = torch.zeros_like(w[:, :1]) if rms else w.mean(1, keepdim=True)
    off_m1 = torch.zeros_like(m1) if rms else (n + 4) * E * w.abs().mean(1, keepdim=True) + off_w.mean(1, keepdim=True)
    m2 = (w * xh).mean(1, keepdim=True)
    off_m2 = (n + 4) * E * (w * xh).abs().mean(1, keepdim=True) + (w.abs() * off_xh + off_w * xh.abs() + off_w * off_xh).mean(1, keepdim=True)
    g = r * (w - m1 - xh * m2)
    off = r * (off_w + off_m1 + xh.abs() * off_m2 + off_xh * (m2.abs() + off_m2) + 4 * E * (w.abs() + m1.abs() + (xh * m2).abs()))
    return g, off * (1 + rel) + g.abs() * (rel + 2 * E)


def gated(X, cu, Y=None, gate=None, scale=None, shift=None, dZ=None, dH=None, eps=1e-6, kind="layer", post=False, residual=1.0, dtype="bf16"):
    """{name: (value, bound)} of Z, H, stats and, with dZ, of dX, dY, dgate, dscale, dshift; everything float64, rows of no segment NaN."""
    u8, rms = HALF_STEP[dtype], kind == "rms"
    T, n = X.shape
    n_seg = len(cu) - 1
    seg = torch.full((T,), -1)
    for i in range(n_seg):
        seg[int(cu[i]):int(cu[i + 1])] = i
    here = seg >= 0
    at = seg.clamp(min=0)

    def rows(m, fill):
        return torch.full((T, n), fill, dtype=torch.float64) if m is None else m[at]

    g, m, t = rows(gate, 1.0), rows(scale, 0.0), rows(shift, 0.0)
    zero = torch.zeros_like(X)
    if Y is None:
        u, off_u, ry, rel_y, mu_y, off_mu_y = zero, zero, None, None, None, None
    elif post:
        u, ry, off_u, rel_y, mu_y, off_mu_y = _normed(Y, zero, eps, rms, n)
    else:
        u, off_u = Y, zero
    h = residual * X + g * u
    off_h = g.abs() * off_u + 4 * E * ((residual * X).abs() + (g * u).abs())
    xh, r, off_xh, rel, mu, off_mu = _normed(h, off_h, eps, rms, n)
    z = xh * (1 + m) + t
    out = {"Z": (z, u8 * z.abs() + (1 + m).abs() * off_xh + 4 * E * ((1 + m.abs()) * xh.abs() + t.abs()) + TINY)}
    if Y is not None:
        out["H"] = (h, u8 * h.abs() + off_h + TINY)
    none = torch.zeros(T, 1, dtype=torch.float64)
    has = Y is not None and post
    out["stats"] = (torch.cat([mu, r, mu_y if has else none, ry if has else none], 1),
                    torch.cat([off_mu + E * mu.abs(), r * rel, off_mu_y + E * mu_y.abs() if has else none, ry * rel_y if has else none], 1))
    if dZ is not None:
        dh0 = zero if dH is None else dH
        w = dZ * (1 + m)
        off_w = 3 * E * dZ.abs() * (1 + m.abs())
        dh, off_dh = _back(w, off_w, xh, off_xh, r, rel, rms, n)
        dh = dh + dh0
        off_dh = off_dh + 2 * E * (dh.abs() + dh0.abs())
        dx = residual * dh
        out["dX"] = (dx, u8 * dx.abs() + abs(residual) * off_dh + E * dx.abs() + TINY)
        v = g * dh
        off_v = g.abs() * off_dh + 2 * E * v.abs()
        if Y is not None:
            dy, off_dy = _back(v, off_v, u, off_u, ry, rel_y, rms, n) if post else (v, off_v)
            out["dY"] = (dy, u8 * dy.abs() + off_dy + TINY)
        terms = {"dgate": (dh * u, off_dh * u.abs() + dh.abs() * off_u), "dscale": (dZ * xh, dZ.abs() * off_xh), "dshift": (dZ, zero)}
        for name, (x, off) in terms.items():
            val, bnd = torch.zeros(n_seg, n, dtype=torch.float64), torch.zeros(n_seg, n, dtype=torch.float64)
            for i in range(n_seg):
                a, b = int(cu[i]), int(cu[i + 1])
                val[i] = x[a:b].sum(0)
                bnd[i] = ((b - a + 4) * E * x[a:b].abs() + off[a:b]).sum(0) + TINY
            out[name] = (val, bnd)
    for name in ("Z", "H", "stats", "dX", "dY"):
        if name in out:
            out[name][0][~here] = float("nan")
    return out


# ---------------------------------------------------------------------------------------------- cache
def e4m3(x):
    """The nearest of the values with three bits behind the leading one, exponents -6 (below it the same step) to 8, up to 448; the even one of two."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def page_scale(most):
    """The least power of two s with most <= 448 s, from 2^-117 to 2^119."""
    if most == 0:
        return 2.0 ** -117
    e = -117
    while most > 448 * 2.0 ** e and e < 119:
        e += 1
    return 2.0 ** e


def check_append(before, after, rows, off, new, lens, table, page):
    """before, after: (values float64 [pages, H, page, d], scales [pages, H]); rows [T, H, d] float64, off by `off`.  Every value and scale has to be what
    some row within the bound gives; what no sequence reached has to be as it was."""
    (v0, s0), (v1, s1) = before, after
    want, a = v0.clone(), 0
    touched = torch.zeros(v0.shape[0], dtype=torch.bool)
    for i, n in enumerate(new):
        at, end = lens[i] - n, lens[i]
        while at < end:
            pg, begun = int(table[i, at // page]), at % page
            k = min(page - begun, end - at)
            touched[pg] = True
            for h in range(v0.shape[1]):
                x, o = rows[a : a + k, h], off[a : a + k, h]
                held = float(s0[pg, h]) if begun else 0.0
                sizes = x.abs()
                may = {max(held, page_scale(float((sizes - o).clamp(min=0).max()))), max(held, page_scale(float((sizes + o).max())))}
                s = float(s1[pg, h])
                assert s in may, (pg, h, s, may)
                lo, hi = e4m3((x - o) / s), e4m3((x + o) / s)
                got = v1[pg, h, begun : begun + k]
                assert ((got >= lo) & (got <= hi)).all(), (pg, h)
                want[pg, h, begun : begun + k] = got
                if begun:
                    want[pg, h, :begun] = e4m3(v0[pg, h, :begun] * (held / s))
            a, at = a + k, at + k
    same = (want == v1) | (want.isnan() & v1.isnan())
    assert same.all(), f"{int((~same).sum())} values of the cache are not what they were, or not what they should be moved to"
    keep = ~touched
    assert torch.equal(s0[keep].nan_to_num(-1), s1[keep].nan_to_num(-1))


def quantised(rows, lens, table, n_pages, page, fill=None):
    """Rows [T, H, d] of all streams in turn as the cache holds them: (uint8 [pages, H, page, d], float [pages, H]); `fill`: the byte everywhere else."""
    H, d = rows.shape[1:]
    pool, scale = torch.full((n_pages, H, page, d), 0x7F if fill is None else fill, dtype=torch.uint8), torch.full((n_pages, H), float("nan"))
    a = 0
    for i, n in enumerate(lens):
        for at in range(0, n, page):
            k = min(page, n - at)
            pg = int(table[i, at // page])
            for h in range(H):
                x = rows[a + at : a + at + k, h].double()
                s = page_scale(float(x.abs().max()))
                scale[pg, h] = s
                pool[pg, h, :k] = e4m3(x / s).float().to(torch.float8_e4m3fn).view(torch.uint8)
        a += n
    return pool, scale


def widened(pool, scale, lens, table, page):
    """Rows [T, H, d] float64 that the cache stands for."""
    v = pool.view(torch.float8_e4m3fn).double() * scale.double()[:, :, None, None]
    out = []
    for i, n in enumerate(lens):
        pages = table[i, : -(-n // page)].long()
        out.append(v[pages].transpose(1, 2).reshape(-1, v.shape[1], v.shape[3])[:n])
    return torch.cat(out) if out else torch.zeros(0, v.shape[1], v.shape[3], dtype=torch.float64)


def pages_for(lens, page, seed=0, spare=1, garbage=-12345):
    """(table int32 [n_seq, max_pages], pages in all): pages handed out in no order, entries past the last page `garbage`."""
    counts = [-(-n // page) for n in lens]
    order = torch.randperm(sum(counts) + spare, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(lens), max(max(counts), 1) + 1), garbage, dtype=torch.int32)
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at : at + n].int()
        at += n
    return table, sum(counts) + spare
