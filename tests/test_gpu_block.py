"""Rotary positions, gated norms, the cache and both kinds of attention together: a DiT block's training step with its gradients, and the same block as a
sampler runs it, a frame and a token at a time."""
import math

import pytest
import torch

import block_ref as ref
import packed_ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


def grid_positions(f, h, w):
    return torch.stack(torch.meshgrid(torch.arange(f), torch.arange(h), torch.arange(w), indexing="ij"), -1).reshape(-1, 3).int()


def test_a_block_step_of_two_clips():
    """norm -> q, k, v -> q, k turned -> attention -> gate, residual, norm, and back: every gradient against automatic differentiation in 64 bits, with
    full attention and with sparse attention that keeps every key (of one clip)."""
    H, d, pairs, scale = 2, 64, [16, 8, 8], 0.125
    n = H * d
    clips = [(2, 4, 8), (1, 5, 6)]
    lens = [f * h * w for f, h, w in clips]
    T, cu = sum(lens), packed_ref.cu_of(lens)
    pos = torch.cat([grid_positions(*c) for c in clips])
    g = torch.Generator().manual_seed(7)
    normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x0, W, mods, dZ, dH = normal(T, n), normal(n, 3 * n) / math.sqrt(n), 0.5 * normal(2, 5 * n), normal(T, n), normal(T, n)
    freq = ref.freqs(pairs)

    # 64 bits
    leaves = [t.double().requires_grad_() for t in (x0, W, mods)]
    x, w, m = leaves
    seg = torch.repeat_interleave(torch.arange(2), torch.tensor(lens))
    part = lambda i: m[seg, i * n : (i + 1) * n]  # noqa: E731
    normed = lambda v: torch.nn.functional.layer_norm(v, (n,), eps=1e-6)  # noqa: E731
    qkv = ((normed(x) * (1 + part(0)) + part(1)) @ w).reshape(T, 3 * H, d)
    lo, hi, axis = (torch.tensor(v) for v in zip(*ref.pairs_of(pairs, "axis_halves")))
    t = pos.double()[:, axis] * freq
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    qk = qkv[:, : 2 * H]
    a, b = qk[..., lo], qk[..., hi]
    qk = torch.zeros_like(qk).index_copy(2, lo, a * c - b * s).index_copy(2, hi, a * s + b * c)
    scores = scale * torch.einsum("ihd,jhd->hij", qk[:, :H], qk[:, H:])
    scores = scores.masked_fill(seg[:, None] != seg[None], -math.inf)
    y = torch.einsum("hij,jhd->ihd", torch.softmax(scores, 2), qkv[:, 2 * H :]).reshape(T, n)
    h = x + part(2) * y
    z = normed(h) * (1 + part(3)) + part(4)
    want = torch.autograd.grad((z * dZ.double()).sum() + (h * dH.double()).sum(), leaves)

    # the library; products by torch
    X, Wd, M, dz, dh, P, F, CU = (v.to(DEV) for v in (x0, W, mods, dZ, dH, pos, freq, cu))
    part = lambda t, i: t[:, i * n : (i + 1) * n]  # noqa: E731
    gn = dsv.GatedNorm(T, n, 2, "f32")
    rot = dsv.Rotary(T, 2 * H, d, "f32", pairs, layout="axis_halves")
    Z1, _, st1 = dsv.gated_norm_fwd(gn, X, CU, scale=part(M, 0), shift=part(M, 1))
    qkv = (Z1 @ Wd).reshape(T, 3 * H, d)
    dsv.rotary_fwd(rot, qkv[:, : 2 * H], P, F, Y=qkv[:, : 2 * H])
    Q, K, V = qkv[:, :H], qkv[:, H : 2 * H], qkv[:, 2 * H :]
    p = dsv.Packed(2, T, T, max(lens), max(lens), H, H, d, "f32", scale)
    O, lse = dsv.packed_attn_fwd(p, Q, K, V, CU, CU)

    def rest(O, dO_of):
        Y = O.reshape(T, n)
        Z, Hs, st = dsv.gated_norm_fwd(gn, X, CU, Y, part(M, 2), part(M, 3), part(M, 4))
        dM = torch.empty(2, 5 * n, device=DEV)
        dx, dY, *_ = dsv.gated_norm_bwd(gn, X, CU, st, dz, Y, part(M, 2), part(M, 3), dh.clone(), dgate=part(dM, 2), dscale=part(dM, 3), dshift=part(dM, 4))
        dqkv = torch.empty(T, 3 * H, d, device=DEV)
        dO_of(dY.reshape(T, H, d), dqkv)
        dsv.rotary_bwd(rot, dqkv[:, : 2 * H], P, F, dX=dqkv[:, : 2 * H])
        dqkv = dqkv.reshape(T, 3 * n)
        dsv.gated_norm_bwd(gn, X, CU, st1, dqkv @ Wd.t(), scale=part(M, 0), dH=dx, dX=dx, dscale=part(dM, 0), dshift=part(dM, 1))
        return dx, Z1.t() @ dqkv, dM

    def full(dO, dqkv):
        dsv.packed_attn_bwd(p, Q, K, V, CU, CU, O, lse, dO, dQ=dqkv[:, :H], dK=dqkv[:, H : 2 * H], dV=dqkv[:, 2 * H :])

    sparse = dsv_sparse(lens[0], H, d, scale)
    heads = lambda t: t[: lens[0]].transpose(0, 1).contiguous()[None]  # noqa: E731
    idx = torch.arange(lens[0], dtype=torch.int32, device=DEV).repeat(H * lens[0])
    Os, lses = dsv.sparse_attn_fwd(sparse, heads(Q), heads(K), heads(V), idx)
    O2 = O.clone()
    O2[: lens[0]] = Os[0].transpose(0, 1)

    def mixed(dO, dqkv):
        full(dO, dqkv)
        got = dsv.sparse_attn_bwd(sparse, heads(Q), heads(K), heads(V), idx, Os, lses, heads(dO))
        for i, t in enumerate(got):
            dqkv[: lens[0], i * H : (i + 1) * H] = t[0].transpose(0, 1)

    for got in (rest(O, full), rest(O2, mixed)):
        for name, a, b in zip(("dX", "dW", "dmods"), got, want):
            # sums of at most 128 * 94 terms of size one in 32 bits, through six steps: 1e-4 of the largest is over a hundred times 2^-24 of their root
            assert (a.double().cpu() - b).abs().max() < 1e-4 * max(1.0, float(b.abs().max())), name


def dsv_sparse(L, H, d, scale):
    return dsv.Problem(1, H, L, d, 16, "f32", [L] * H, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("frame", [24, 1])
def test_a_sampler_a_frame_or_a_token_at_a_time(dtype, frame):
    """Three streams of unlike lengths make 96 tokens each, `frame` at a time: norm, projections, q turned, k turned into the cache, attention over it, gate and
    norm.  Every step's attention is that of the cache's own values in 64 bits, within the packed attention's bounds; and what the whole cache holds at the end
    is what the keys and values were, to half a step of e4m3 and the moves to larger scales."""
    n_seq, steps, Hq, Hkv, d, page = 3, 96 // frame, 4, 2, 64, 32
    n, td, u = Hq * d, packed_ref.DTYPES[dtype], packed_ref.HALF_STEP[dtype]
    pairs, lens = [16, 8, 8], [0, 40, 7]
    T = n_seq * frame
    room = [x + 96 for x in lens]
    table, n_pages = ref.pages_for(room, page)
    g = torch.Generator().manual_seed(3)
    W = (torch.randn(n, (Hq + 2 * Hkv) * d, generator=g) / math.sqrt(n)).to(td).to(DEV)
    mods = (0.5 * torch.randn(n_seq, 3 * n, generator=g)).to(td).to(DEV)
    start = [rows_of(sum(lens), Hkv, d, g) for _ in range(2)]
    K8, ks = ref.quantised(start[0], lens, table, n_pages, page)
    V8, vs = ref.quantised(start[1], lens, table, n_pages, page)
    pool = [t.to(DEV) for t in (K8, V8, ks, vs)]
    cu = packed_ref.cu_of([frame] * n_seq)
    CU, TB, F = cu.to(DEV), table.to(DEV), ref.freqs(pairs).to(DEV)
    gn = dsv.GatedNorm(T, n, n_seg := n_seq, dtype)
    held = [[start[i][sum(lens[:s]) : sum(lens[: s + 1])].double() for s in range(n_seq)] for i in range(2)]
    x = torch.randn(T, n, generator=g).to(td).to(DEV)
    scale = 0.125
    for step in range(steps):
        now = [b + (step + 1) * frame for b in lens]
        L = torch.tensor(now, dtype=torch.int32, device=DEV)
        pos = torch.cat([grid_positions(200, 4, 6)[m - frame : m] for m in now]).to(DEV)
        part = lambda i: mods[:, i * n : (i + 1) * n]  # noqa: E731
        z, _, _ = dsv.gated_norm_fwd(gn, x, CU, scale=part(0), shift=part(1))
        qkv = (z @ W).reshape(T, Hq + 2 * Hkv, d)
        Q, K, V = qkv[:, :Hq], qkv[:, Hq : Hq + Hkv], qkv[:, Hq + Hkv :]
        p = dsv.Cache(n_seq, T, frame, Hq, Hkv, d, dtype, n_pages, page, table.shape[1], scale=scale, causal=False)
        dsv.cache_append(p, K, V, CU, L, TB, *pool, rotary=dsv.Rotary(T, Hkv, d, dtype, pairs, layout="axis_halves"), pos=pos, freq=F)
        dsv.rotary_fwd(dsv.Rotary(T, Hq, d, dtype, pairs, layout="axis_halves"), Q, pos, F, Y=Q)
        O, lse = dsv.cache_attn_fwd(p, Q, CU, L, TB, *pool)
        kt, _ = ref.rotary(K.double().cpu(), pos.cpu(), ref.freqs(pairs), pairs, "axis_halves")
        for s in range(n_seq):
            rows = slice(s * frame, (s + 1) * frame)
            held[0][s], held[1][s] = torch.cat([held[0][s], kt[rows]]), torch.cat([held[1][s], V[rows].double().cpu()])
        if step % 16 == 0 or step == steps - 1:
            kv = [ref.widened(pool[i].cpu(), pool[2 + i].cpu(), now, table, page) for i in range(2)]
            want = packed_ref.attention(Q.double().cpu(), *kv, cu, packed_ref.cu_of(now), scale, False, dtype=dtype)
            packed_ref.assert_within("O", O, want["O"])
            packed_ref.assert_within("lse", lse, want["lse"])
        x = dsv.gated_norm_fwd(gn, x, CU, O.reshape(T, n), part(2), part(0), part(1))[1]
    for i in range(2):
        got, want = ref.widened(pool[i].cpu(), pool[2 + i].cpu(), now, table, page), torch.cat(held[i])
        # a page's scale s has its largest value above 224 s, if it never moved; a move rounds those below 2^-6 s once more, by 2^-10 s at most; at most eight moves
        most = want.abs().max()
        assert ((got - want).abs() <= (2.0 ** -4 + u) * want.abs() + 9 * 2.0 ** -10 * most / 224 + 1e-5 * most).all()


def rows_of(T, H, d, g):
    return torch.randn(T, H, d, generator=g)
