"""Attention over packed sequences and layer norm: the calls they are measured by, their plain forms and 64-bit references.

Every case is one pass as a training loop or a sampler of a video DiT makes it: attention of clips packed one behind
another (to themselves, to a caption, to a cache of earlier tokens), its training step, and the norms in front of it.
Shapes are those of workloads/configs.py with as many heads as keep a plain pass short, and odd ones beside them.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"
EPS = 1e-5


def listed():
    return [
        # one new token per stream of an autoregressive sampler, against caches of very different lengths
        dict(name="decode_caches", kind="attn", dtype="bf16", Hq=16, Hkv=4, d=128, causal=True, layout="token",
             lens_q="1,1,1,1,1,1,1,1,1,1,1,1", lens_k="16001,9320,7777,5200,4096,3111,2048,1560,1023,512,77,1"),
        # the smallest block in use (8 x 8 x 16 latent, fp32) and a shorter clip behind it: latency counts
        dict(name="small_f32", kind="attn", dtype="f32", Hq=2, Hkv=2, d=64, causal=False, layout="token",
             lens_q="1024,700", lens_k="1024,700"),
        # video tokens of four clips to their captions
        dict(name="cross_captions", kind="attn", dtype="bf16", Hq=16, Hkv=16, d=64, causal=False, layout="token",
             lens_q="20280,8192,4096,1560", lens_k="77,226,120,512"),
        # clips of three sizes in one batch, full attention forward
        dict(name="clips_forward", kind="attn", dtype="bf16", Hq=4, Hkv=4, d=128, causal=False, layout="qkv",
             lens_q="20280,8192,4096", lens_k="20280,8192,4096"),
        # the smallest block's training step
        dict(name="small_step_f32", kind="attn_step", dtype="f32", Hq=2, Hkv=2, d=64, causal=False, layout="head",
             lens_q="1024", lens_k="1024"),
        # a clip whose size is no power of two (13 x 30 x 52) through a training step
        dict(name="clip_step", kind="attn_step", dtype="bf16", Hq=4, Hkv=4, d=128, causal=False, layout="qkv",
             lens_q="20280", lens_k="20280"),
        # causal clips of ragged lengths whose heads share K and V, training step
        dict(name="causal_shared_step", kind="attn_step", dtype="bf16", Hq=8, Hkv=2, d=128, causal=True, layout="token",
             lens_q="8191,4100,1560,333,64,1", lens_k="8191,4100,1560,333,64,1"),
        # one layer of an ordinary clip (16 x 32 x 64 latent), full attention, training step, the library's head-major layout
        dict(name="video_step", kind="attn_step", dtype="bf16", Hq=4, Hkv=4, d=128, causal=False, layout="head",
             lens_q="32768", lens_k="32768"),
        # a few rows of an odd width
        dict(name="norm_few_rows", kind="norm", dtype="f32", rows=77, heads=1, n=1155, affine=True),
        # the norm of every head's query rows, read in place from the fused projection's output
        dict(name="query_norm_step", kind="norm_step", dtype="bf16", rows=32768, heads=16, n=128, affine=True, layout="qkv"),
        # a block's norm over the model's width, training step
        dict(name="block_norm_step", kind="norm_step", dtype="bf16", rows=32768, heads=1, n=2048, affine=True),
        # the same in fp32 at a width that is no power of two, long clip
        dict(name="block_norm_f32", kind="norm_step", dtype="f32", rows=20280, heads=1, n=1536, affine=True),
    ]


def _ints(text):
    return [int(x) for x in text.split(",")]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.35:
        c = dict(kind=rng.choice(["norm", "norm_step", "norm_step"]), dtype=rng.choice(["bf16", "bf16", "f32"]), affine=rng.random() < 0.75)
        if rng.random() < 0.4:      # rows of heads
            c["n"], c["heads"] = rng.choice([64, 128]), rng.randint(1, 16)
            c["rows"] = _log_int(rng, 1, 40000)
            c["layout"] = rng.choice(["token", "qkv", "head"])
        else:
            c["n"], c["heads"] = _log_int(rng, 16, 8192), 1
            if rng.random() < 0.5:
                c["n"] = max(64, c["n"] // 64 * 64)
            c["rows"] = _log_int(rng, 1, max(2, min(40000, 60_000_000 // c["n"])))
        return c
    c = dict(kind=rng.choice(["attn", "attn_step"]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), d=rng.choice([64, 128, 128]),
             causal=rng.random() < 0.5, layout=rng.choice(["token", "qkv", "head"]))
    c["Hkv"] = rng.choice([1, 2, 3, 4, 8])
    c["Hq"] = c["Hkv"] * rng.choice([1, 1, 2, 4, 7])
    most = {"f32": 2e8, "bf16": 1e9}[c["dtype"]]     # pairs of the padded batch
    form = rng.choice(["self", "self", "cross", "decode", "append"])
    n = rng.choice([1, 1, 2, 3, 5, 8, 16]) if form != "decode" else rng.choice([1, 2, 8, 24, 64])
    if form == "self":
        top = int(math.sqrt(most / (n * c["Hq"])))
        lk = [_log_int(rng, 1, min(top, 30000)) for _ in range(n)]
        lq = list(lk)
    elif form == "cross":
        lk = [_log_int(rng, 1, 600) for _ in range(n)]
        top = int(most / (n * c["Hq"] * max(lk)))
        lq = [_log_int(rng, 1, min(top, 20000)) for _ in range(n)]
        c["causal"] = False
    elif form == "decode":
        top = int(most / (n * c["Hq"]))
        lk = [_log_int(rng, 1, min(top, 20000)) for _ in range(n)]
        lq = [1] * n
        c["kind"] = "attn"
    else:                            # a piece of new tokens behind a cache; a cache that was cut leaves the first of them no key
        lq = [_log_int(rng, 1, 400) for _ in range(n)]
        top = int(most / (n * c["Hq"] * max(lq)))
        lk = [_log_int(rng, 1, min(top, 12000)) for _ in range(n)]
    if form != "decode" and n > 2 and rng.random() < 0.3:
        lk[rng.randrange(n)] = 0     # a sequence of no keys
    if max(lk) < 32:                 # one key in every sequence and no gradient would reach Q and K
        lk[0] = 32 + lk[0]
        lq[0] = lk[0] if form == "self" else lq[0]
    if c["layout"] == "qkv" and lq != lk:
        c["layout"] = "token"
    c["lens_q"], c["lens_k"] = ",".join(map(str, lq)), ",".join(map(str, lk))
    return c


# ---------------------------------------------------------------------------------------------- inputs
def _laid_out(x, layout, more):
    """x [T, H, d] as a view of the memory the layout names: as it is, head by head, or a slice of rows that hold `more` heads as well."""
    if layout == "head":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "qkv":
        wide = torch.zeros(x.shape[0], x.shape[1] + more, x.shape[2], dtype=x.dtype, device=x.device)
        wide[:, : x.shape[1]] = x
        return wide[:, : x.shape[1]]
    return x.contiguous()


def _cu(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEVICE)


def _attn_inputs(case, seed):
    """Q and K on a basis of 64 (32) directions shared by all heads plus noise, so that scores spread as trained ones do; V and dO white."""
    g = torch.Generator(device=DEVICE).manual_seed(1000003 * (seed + 1))
    Hq, Hkv, d, td = case["Hq"], case["Hkv"], case["d"], DTYPES[case["dtype"]]
    lq, lk = _ints(case["lens_q"]), _ints(case["lens_k"])

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    rank = 64 if d == 128 else 32
    basis = normal(rank, d) / math.sqrt(rank)
    Q = (normal(sum(lq), Hq, rank) @ basis + 0.1 * normal(sum(lq), Hq, d)).to(td)
    K = (normal(sum(lk), Hkv, rank) @ basis + 0.1 * normal(sum(lk), Hkv, d)).to(td)
    V, dO = normal(sum(lk), Hkv, d).to(td), normal(sum(lq), Hq, d).to(td)
    return Q, K, V, dO


def _norm_inputs(case, seed):
    """Activations with a few large channels, off zero; weights near one."""
    g = torch.Generator(device=DEVICE).manual_seed(1000003 * (seed + 1) + 1)
    rows, heads, n, td = case["rows"], case["heads"], case["n"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    channel = 1 + 4 * (torch.rand(n, generator=g, device=DEVICE) < 0.02)
    X = (normal(rows, heads, n) * channel + 0.3 * normal(n)).to(td)
    dY = normal(rows, heads, n).to(td)
    gamma, beta = ((1 + 0.1 * normal(n)).to(td), (0.1 * normal(n)).to(td)) if case["affine"] else (None, None)
    return X, dY, gamma, beta


def prepare(case, seed):
    s = {k: case[k] for k in case}
    if case["kind"].startswith("norm"):
        X, s["dY"], s["gamma"], s["beta"] = _norm_inputs(case, seed)
        s["X"] = _laid_out(X, case.get("layout", "token"), 2 * case["heads"])
        return s
    lq, lk = _ints(case["lens_q"]), _ints(case["lens_k"])
    s["n_seq"], s["max_q"], s["max_k"] = len(lq), max(lq), max(lk)
    s["cu_q"], s["cu_k"] = _cu(lq), _cu(lk)
    Q, K, V, s["dO"] = _attn_inputs(case, seed)
    layout, Hq, Hkv = case["layout"], case["Hq"], case["Hkv"]
    s["Q"], s["K"], s["V"] = _laid_out(Q, layout, 2 * Hkv), _laid_out(K, layout, Hq + Hkv), _laid_out(V, layout, Hq + Hkv)
    s["scale"] = _scale(case)
    return s


def _scale(case):
    return 2.0 / math.sqrt(case["d"])


# ---------------------------------------------------------------------------------------------- plain forms
def _pad(x, cu, most):
    """x [T, H, d] by sequences, fp32 [n_seq, H, most, d], zero behind their ends."""
    pos = torch.arange(most, device=x.device)
    at = (cu[:-1, None] + pos).clamp(max=x.shape[0] - 1).long()
    there = pos < (cu[1:] - cu[:-1])[:, None]
    return (x.float()[at] * there[:, :, None, None]).transpose(1, 2).contiguous()


def _pack(x, cu, total):
    """The inverse of _pad: [n_seq, H, most, ...] back to [total, H, ...]."""
    t = torch.arange(total, device=x.device)
    seq = torch.bucketize(t, cu[1:].long(), right=True)
    return x.transpose(1, 2)[seq, t - cu.long()[seq]]


def _plain_attention(s, grad):
    Hq, Hkv, d, scale, td = s["Hq"], s["Hkv"], s["d"], s["scale"], DTYPES[s["dtype"]]
    n, mq, mk, group = s["n_seq"], s["max_q"], s["max_k"], s["Hq"] // s["Hkv"]
    cu_q, cu_k = s["cu_q"], s["cu_k"]
    nq, nk = cu_q[1:] - cu_q[:-1], cu_k[1:] - cu_k[:-1]
    q = _pad(s["Q"], cu_q, mq).reshape(n, Hkv, group * mq, d)
    k, v = _pad(s["K"], cu_k, mk), _pad(s["V"], cu_k, mk)
    i, j = torch.arange(mq, device=q.device)[None, :, None], torch.arange(mk, device=q.device)[None, None, :]
    seen = (j < nk[:, None, None]) & ((j <= i + (nk - nq)[:, None, None]) if s["causal"] else (i >= 0))
    p = (q @ k.transpose(2, 3).contiguous()).mul_(scale)
    p.view(n, Hkv, group, mq, mk).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(3, keepdim=True).clamp(min=-3e38)      # rows that see no key: every weight exp(-inf)
    p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    lse = top + total.log()
    p.div_(total.clamp(min=1e-38))

    def rows(x, last):
        return _pack(x.reshape((n, Hq, mq) + last), cu_q, s["Q"].shape[0])

    out = [rows(p @ v, (d,)).to(td), rows(lse, ()).transpose(0, 1).contiguous()]
    if grad:
        do = _pad(s["dO"], cu_q, mq).reshape(n, Hkv, group * mq, d)
        dv = p.transpose(2, 3) @ do
        ds = do @ v.transpose(2, 3).contiguous()
        ds.sub_((p * ds).sum(3, keepdim=True)).mul_(p).mul_(scale)
        total_k = s["K"].shape[0]
        out += [rows(ds @ k, (d,)).to(td), _pack(ds.transpose(2, 3) @ q, cu_k, total_k).to(td), _pack(dv, cu_k, total_k).to(td)]
    return out


def _plain_norm(s, grad):
    td, x = DTYPES[s["dtype"]], s["X"].float()
    mean = x.mean(2, keepdim=True)
    rstd = ((x - mean).square().mean(2, keepdim=True) + EPS).rsqrt()
    xh = (x - mean) * rstd
    gamma = s["gamma"].float() if s["affine"] else 1.0
    y = xh * gamma + (s["beta"].float() if s["affine"] else 0.0)
    out = [y.to(td), mean[:, :, 0], rstd[:, :, 0]]
    if grad:
        dy = s["dY"].float()
        g = dy * gamma
        dx = rstd * (g - g.mean(2, keepdim=True) - xh * (g * xh).mean(2, keepdim=True))
        out += [dx.to(td)] + ([(dy * xh).sum((0, 1)), dy.sum((0, 1))] if s["affine"] else [])
    return out


# ---------------------------------------------------------------------------------------------- one pass
def _own_attention(s, grad):
    import paper_2502_07590_amd as dsv
    p = dsv.Packed(s["n_seq"], s["Q"].shape[0], s["K"].shape[0], s["max_q"], s["max_k"], s["Hq"], s["Hkv"], s["d"], s["dtype"], s["scale"],
                   causal=s["causal"])
    if not grad:
        return list(dsv.packed_attn_fwd(p, s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"]))
    tail = torch.empty(s["Q"].shape, dtype=s["Q"].dtype, device=s["Q"].device) if s["dtype"] == "bf16" else None
    O, lse = dsv.packed_attn_fwd(p, s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], O_tail=tail)
    return [O, lse, *dsv.packed_attn_bwd(p, s["Q"], s["K"], s["V"], s["cu_q"], s["cu_k"], O, lse, s["dO"], O_tail=tail)]


def _own_norm(s, grad):
    import paper_2502_07590_amd as dsv
    p = dsv.Norm(s["rows"], s["n"], s["dtype"], EPS, heads=s["heads"])
    y, mean, rstd = dsv.layer_norm_fwd(p, s["X"], s["gamma"], s["beta"])
    if not grad:
        return [y, mean, rstd]
    dX, dgamma, dbeta = dsv.layer_norm_bwd(p, s["X"], s["gamma"], mean, rstd, s["dY"])
    return [y, mean, rstd, dX] + ([dgamma, dbeta] if s["affine"] else [])


def run(s):
    grad = s["kind"].endswith("_step")
    if own:
        return _own_norm(s, grad) if s["kind"].startswith("norm") else _own_attention(s, grad)
    return _plain_norm(s, grad) if s["kind"].startswith("norm") else _plain_attention(s, grad)


# ---------------------------------------------------------------------------------------------- floors
def _pairs(case):
    """(query, key) pairs that are not masked, over all query heads."""
    total = 0
    for nq, nk in zip(_ints(case["lens_q"]), _ints(case["lens_k"])):
        if not case["causal"]:
            total += nq * nk
        else:                        # query i sees min(nk, max(0, i + 1 + nk - nq)) keys
            first = max(0, nq - nk)  # queries that see nothing
            rows = nq - first
            total += rows * nk - rows * (rows - 1) // 2
    return total * case["Hq"]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    grad = case["kind"].endswith("_step")
    if case["kind"].startswith("norm"):
        rows, n = case["rows"] * case["heads"], case["n"]
        weights = n if case["affine"] else 0
        fwd = {"bytes": 2 * rows * n * es + 8 * rows + 2 * weights * es, "flops": 8 * rows * n}
        if not grad:
            return fwd
        return {"bytes": fwd["bytes"] + rows * n * es * 2 + 8 * weights, "flops": fwd["flops"] + 12 * rows * n}   # x once, dY once, dX once
    q, k = sum(_ints(case["lens_q"])) * case["Hq"] * case["d"] * es, sum(_ints(case["lens_k"])) * case["Hkv"] * case["d"] * es
    lse = 4 * sum(_ints(case["lens_q"])) * case["Hq"]
    if not grad:
        return {"bytes": 2 * q + 2 * k + lse, "flops": 4 * case["d"] * _pairs(case)}
    return {"bytes": 4 * q + 4 * k + lse, "flops": 14 * case["d"] * _pairs(case)}


# ---------------------------------------------------------------------------------------------- 64-bit references
def _exact_attention(case, seed):
    Q, K, V, dO = (x.double() for x in _attn_inputs(case, seed))
    grad, group, scale = case["kind"].endswith("_step"), case["Hq"] // case["Hkv"], _scale(case)
    O, dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    lse = torch.full((case["Hq"], Q.shape[0]), -math.inf, dtype=torch.float64, device=DEVICE)
    a = b = 0
    for nq, nk in zip(_ints(case["lens_q"]), _ints(case["lens_k"])):
        for h in range(case["Hq"] if nk else 0):
            k, v = K[b : b + nk, h // group], V[b : b + nk, h // group]
            step = max(1, (1 << 28) // nk)
            for i0 in range(0, nq, step):
                at = slice(a + i0, a + min(nq, i0 + step))
                q, do = Q[at, h], dO[at, h]
                x = scale * (q @ k.T)
                if case["causal"]:
                    last = torch.arange(i0, i0 + q.shape[0], device=DEVICE) + nk - nq
                    x = torch.where(torch.arange(nk, device=DEVICE)[None] <= last[:, None], x, -math.inf)
                lse[h, at] = torch.logsumexp(x, 1)
                p = torch.exp(x - torch.where(lse[h, at].isinf(), 0.0, lse[h, at])[:, None])
                O[at, h] = p @ v
                if grad:
                    dp = do @ v.T
                    ds = p * (dp - (do * O[at, h]).sum(1, keepdim=True))
                    dQ[at, h] = scale * (ds @ k)
                    dK[b : b + nk, h // group] += scale * (ds.T @ q)
                    dV[b : b + nk, h // group] += p.T @ do
        a, b = a + nq, b + nk
    return [O, lse] + ([dQ, dK, dV] if grad else [])


def _exact_norm(case, seed):
    X, dY, gamma, beta = _norm_inputs(case, seed)
    x, dy, one = X.double(), dY.double(), torch.ones(case["n"], dtype=torch.float64, device=DEVICE)
    gamma, beta = (gamma.double(), beta.double()) if case["affine"] else (one, 0 * one)
    var, mean = torch.var_mean(x, 2, correction=0, keepdim=True)
    sd = torch.sqrt(var + EPS)
    xh = (x - mean) / sd
    out = [gamma * xh + beta, mean[:, :, 0], 1 / sd[:, :, 0]]
    if case["kind"].endswith("_step"):
        g = gamma * dy
        out.append((g - g.mean(2, keepdim=True) - xh * (g * xh).mean(2, keepdim=True)) / sd)
        out += [(xh * dy).sum((0, 1)), dy.sum((0, 1))] if case["affine"] else []
    return out


def exact(case, seed):
    return _exact_norm(case, seed) if case["kind"].startswith("norm") else _exact_attention(case, seed)
