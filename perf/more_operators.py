"""Rotary positions, gated norms with modulation, and an 8-bit paged cache with the attention that reads it: the calls they are measured by,
their plain forms and 64-bit references.

Every case is one pass as a block of a video DiT makes it, in a training step (positions and norms around its attention) or in a sampler that
makes a video piece by piece (new tokens go into a cache of earlier ones and attend to it).  Shapes are those of workloads/configs.py and
of perf/operators.py, and odd ones beside them.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"
EPS = 1e-6
E4M3 = torch.float8_e4m3fn
CACHES = "16001,9320,7777,5200,4096,3111,2048,1560,1023,512,77,1"


def listed():
    return [
        # Q and K of the smallest block in use (8 x 8 x 16 latent, fp32): latency counts
        dict(name="turn_small_f32", kind="rotary", dtype="f32", tokens=1024, heads=4, d=64, pairs="16,8,8", pattern="interleaved", layout="token",
             grid="8,8,16", first=0, scaling=1.0),
        # Q and K of an ordinary clip (16 x 32 x 64 latent), both where the fused projection left them, and their gradients on the way back
        dict(name="turn_video_step", kind="rotary_step", dtype="bf16", tokens=32768, heads=32, d=128, pairs="16,24,24", pattern="axis_halves", layout="qkv",
             grid="16,32,64", first=0, scaling=1.0),
        # a piece of a long stream, one coordinate, three quarters of each head, positions far out and slowed down
        dict(name="turn_long_stream", kind="rotary", dtype="bf16", tokens=9320, heads=7, d=128, pairs="48", pattern="halves", layout="token",
             grid="9320", first=1200000, scaling=8.0),
        # a sampler's step: one new token of each stream, each with its own modulation
        dict(name="gate_tokens", kind="norm", dtype="bf16", lens="1,1,1,1,1,1,1,1,1,1,1,1", n=2048, form="layer", post=False, residual=1.0),
        # a block's norm over four clips of one batch, training step
        dict(name="gate_clips_step", kind="norm_step", dtype="bf16", lens="20280,8192,4096,200", n=2048, form="layer", post=False, residual=1.0),
        # norms on both sides of the block, every frame of a clip (13 x 30 x 52) with a modulation of its own, fp32
        dict(name="gate_frames_f32", kind="norm_step", dtype="f32", lens=",".join(["1560"] * 13), n=1536, form="rms", post=True, residual=0.5),
        # one new token of each stream into caches of very different lengths
        dict(name="append_tokens", kind="append", dtype="bf16", Hkv=4, d=128, page=64, pairs="64", pattern="halves", new="1,1,1,1,1,1,1,1,1,1,1,1",
             old="16000,9319,7776,5199,4095,3110,2047,1559,1022,511,76,0"),
        # clips of three sizes go into their caches at once, two of them behind earlier tokens
        dict(name="append_clips", kind="append", dtype="bf16", Hkv=16, d=128, page=64, pairs="16,24,24", pattern="axis_halves", new="20280,8192,4096", old="0,1000,77"),
        # one new token of each of a few streams against their caches
        dict(name="read_tokens", kind="cached", dtype="bf16", Hq=16, Hkv=4, d=128, page=64, causal=True, new="1,1,1,1,1,1,1,1,1,1,1,1", lens=CACHES),
        # many streams of long caches, more heads than a power of two to each of the cache
        dict(name="read_streams", kind="cached", dtype="bf16", Hq=14, Hkv=2, d=128, page=128, causal=True, new=",".join(["1"] * 64),
             lens=",".join(str(2047 + (997 * i) % 17951) for i in range(64))),
        # the next frame (30 x 52) of two streams against the frames before and itself
        dict(name="read_frames", kind="cached", dtype="bf16", Hq=8, Hkv=2, d=128, page=64, causal=False, new="1560,1560", lens="21840,7800"),
        # fp32, short odd caches in the smallest pages, a few tokens at a time, one stream that is not there
        dict(name="read_odd_f32", kind="cached", dtype="f32", Hq=6, Hkv=2, d=64, page=16, causal=True, new="7,1,0,33,2", lens="1023,77,0,40,512"),
    ]


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(xs):
    return ",".join(map(str, xs))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_pairs(rng, d):
    """Pairs of channels turned by one coordinate or by three, over the whole head or a part of it."""
    rot = rng.choice([d, d, d // 2, d // 4 * 3, rng.randint(3, d // 2) * 2]) // 2
    if rng.random() < 0.5:
        return str(rot)
    if rng.random() < 0.5:
        return {64: "16,8,8", 128: "16,24,24"}[d]
    a = rng.randint(1, rot - 2)
    b = rng.randint(1, rot - a - 1)
    return _text([a, b, rot - a - b])


def _draw_rotary(rng):
    c = dict(kind=rng.choice(["rotary", "rotary_step"]), dtype=rng.choice(["bf16", "bf16", "f32"]), d=rng.choice([64, 128, 128]), heads=rng.choice([1, 2, 3, 4, 7, 8, 16, 32]),
             pattern=rng.choice(["interleaved", "halves", "axis_halves"]), layout=rng.choice(["token", "qkv", "head"]))
    c["pairs"] = _draw_pairs(rng, c["d"])
    most = 60_000_000 // (c["heads"] * c["d"])
    if "," in c["pairs"]:
        f, h = _log_int(rng, 1, 32), _log_int(rng, 1, 48)
        w = _log_int(rng, 1, max(1, min(64, most // (f * h))))
        c["grid"], c["tokens"] = _text([f, h, w]), f * h * w
    else:
        c["tokens"] = _log_int(rng, 1, min(most, 40000))
        c["grid"] = str(c["tokens"])
    c["first"], c["scaling"] = rng.choice([0, 0, 77, 30000, 2000000]), rng.choice([1.0, 1.0, 4.0, 32.0])
    return c


def _draw_norm(rng):
    c = dict(kind=rng.choice(["norm", "norm_step", "norm_step"]), dtype=rng.choice(["bf16", "bf16", "f32"]), form=rng.choice(["layer", "layer", "rms"]),
             post=rng.random() < 0.4, residual=rng.choice([1.0, 1.0, 0.7071]))
    c["n"] = _log_int(rng, 32, 8192)
    if rng.random() < 0.6:
        c["n"] = max(64, c["n"] // 64 * 64)
    top = max(2, min(32000, 40_000_000 // c["n"]))
    if rng.random() < 0.3:      # frames of one length
        k = rng.randint(1, 32)
        lens = [_log_int(rng, 1, max(1, top // k))] * k
    else:
        k = rng.choice([1, 2, 3, 5, 8, 16, 64])
        lens = [_log_int(rng, 1, max(1, top // k)) for _ in range(k)]
        if k > 2 and rng.random() < 0.5:
            lens[rng.randrange(k)] = 0
    c["lens"] = _text(lens)
    return c


def _draw_append(rng):
    c = dict(kind="append", dtype=rng.choice(["bf16", "bf16", "f32"]), Hkv=rng.choice([1, 2, 3, 4, 8, 16]), d=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 64, 128, 256]),
             pattern=rng.choice(["interleaved", "halves", "axis_halves"]))
    c["pairs"] = rng.choice(["0", _draw_pairs(rng, c["d"]), _draw_pairs(rng, c["d"])])
    k = rng.choice([1, 2, 3, 8, 24])
    most = min(20000, 30_000_000 // (c["Hkv"] * c["d"] * k))
    new = [1] * k if rng.random() < 0.4 else [_log_int(rng, 1, most) for _ in range(k)]
    if k > 2 and max(new) > 1 and rng.random() < 0.4:
        new[rng.randrange(k)] = 0
    c["new"], c["old"] = _text(new), _text([rng.choice([0, _log_int(rng, 1, most)]) for _ in range(k)])
    return c


def _draw_cached(rng):
    c = dict(kind="cached", dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), Hkv=rng.choice([1, 2, 3, 4, 8]), d=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 64, 128, 256]),
             causal=rng.random() < 0.6)
    c["Hq"] = c["Hkv"] * rng.choice([1, 1, 2, 4, 7])
    k = rng.choice([1, 2, 3, 8, 24])
    cells = 100_000_000 // (k * c["Hkv"] * c["d"])      # keys of a stream that the plain form widens at once
    if rng.random() < 0.5:
        lens, new = [_log_int(rng, 32, min(20000, cells)) for _ in range(k)], [1] * k
    else:
        new = [_log_int(rng, 2, 1600) for _ in range(k)]
        most = {"f32": 5e7, "bf16": 3e8}[c["dtype"]]
        lens = [_log_int(rng, 32, max(64, min(20000, cells, int(most / (k * c["Hq"] * max(new)))))) for _ in range(k)]
    if k > 2 and rng.random() < 0.4:
        lens[rng.randrange(k)] = 0                      # a stream of no tokens yet: its queries see nothing
    c["new"], c["lens"] = _text(new), _text(lens)
    return c


def draw(rng):
    return rng.choice([_draw_rotary, _draw_norm, _draw_append, _draw_cached, _draw_cached])(rng)


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed, kind):
    return torch.Generator(device=DEVICE).manual_seed(1000003 * (seed + 1) + kind)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


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


def _freqs(pairs, factor):
    """Angles a position of every pair: each coordinate its own falling series; slow ones slowed down by `factor`, fast ones kept, a ramp between."""
    out = []
    for n in pairs:
        f = 10000.0 ** (-torch.arange(n, dtype=torch.float64, device=DEVICE) / n)
        keep = ((f * 4096 / (2 * math.pi) - 1) / 31).clamp(0, 1)
        out.append(f * (keep + (1 - keep) / factor))
    return torch.cat(out)


def _gain(factor):
    return 0.1 * math.log(factor) + 1.0


def _grid_positions(grid, first):
    axes = [torch.arange(n, device=DEVICE) for n in grid]
    at = torch.stack(torch.meshgrid(*axes, indexing="ij"), -1).reshape(-1, len(grid))
    at[:, 0] += first
    return at.to(torch.int32)


def _rotary_inputs(case, seed):
    """Rows as a projection leaves them, and what comes back from the scores."""
    g, td = _generator(seed, 0), DTYPES[case["dtype"]]
    shape = (case["tokens"], case["heads"], case["d"])
    X, dY = _normal(g, *shape).to(td), _normal(g, *shape).to(td)
    pairs = _ints(case["pairs"])
    return X, dY, _grid_positions(_ints(case["grid"]), case["first"] + seed % 1000), _freqs(pairs, case["scaling"])


def _norm_inputs(case, seed):
    """A residual stream with a few large channels, a block's output, modulations of size one as six chunks of one projection's output."""
    g, td, lens, n = _generator(seed, 1), DTYPES[case["dtype"]], _ints(case["lens"]), case["n"]
    rows = sum(lens)
    channel = 1 + 4 * (torch.rand(n, generator=g, device=DEVICE) < 0.02)
    X = (_normal(g, rows, n) * channel + 0.3 * _normal(g, n)).to(td)
    Y, dZ, dH = ((_normal(g, rows, n) * s).to(td) for s in (0.7, 1.0, 1.0))
    mods = (0.5 * _normal(g, len(lens), 6 * n)).to(td)
    return X, Y, dZ, dH, mods


def _pages(lens, page, seed):
    """(table, pages in all): pages handed out in no order, room for one token more than there is."""
    counts = [n // page + 1 for n in lens]
    order = torch.randperm(sum(counts), generator=torch.Generator().manual_seed(seed), dtype=torch.int64)
    table = torch.zeros(len(lens), max(counts), dtype=torch.int32)
    at = 0
    for i, n in enumerate(counts):
        table[i, :n] = order[at : at + n]
        at += n
    return table.to(DEVICE), sum(counts)


def _fill(rows, lens, table, n_pages, page):
    """Rows [tokens, heads, d] of all streams in turn, as an 8-bit cache holds them: (values, scales), one power of two a page and head."""
    H, d = rows.shape[1:]
    pool = torch.zeros(n_pages, page, H, d, device=DEVICE)
    a = 0
    for i, n in enumerate(lens):
        at = torch.arange(n, device=DEVICE)
        pool[table[i, at // page].long(), at % page] = rows[a : a + n]
        a += n
    scale = _scale_of(pool.abs().amax((1, 3)))
    values = (pool / scale[:, None, :, None]).to(E4M3).transpose(1, 2).contiguous()
    return values, scale


def _scale_of(most):
    """The least power of two s with most <= 448 s (of a page of zeros: the least there is)."""
    m, e = torch.frexp(most)
    e = torch.where(most > 0, e - 9 + (m > 0.875).int(), -117)
    return torch.ldexp(torch.ones_like(most), e.clamp(-117, 119))


def _cache_rows(g, tokens, H, d, basis):
    """Keys on a basis shared with the queries plus noise, so that scores spread as trained ones do; values white."""
    return _normal(g, tokens, H, basis.shape[0]) @ basis + 0.1 * _normal(g, tokens, H, d), _normal(g, tokens, H, d)


def _basis(g, d):
    rank = 64 if d == 128 else 32
    return _normal(g, rank, d) / math.sqrt(rank)


def _append_inputs(case, seed):
    g, td, d, H, page = _generator(seed, 2), DTYPES[case["dtype"]], case["d"], case["Hkv"], case["page"]
    new, old = _ints(case["new"]), _ints(case["old"])
    basis = _basis(g, d)
    s = {}
    s["table"], n_pages = _pages([a + b for a, b in zip(new, old)], page, seed)
    K, V = _cache_rows(g, sum(old), H, d, basis)
    s["K8"], s["kscale"] = _fill(K, old, s["table"], n_pages, page)
    s["V8"], s["vscale"] = _fill(V, old, s["table"], n_pages, page)
    K, V = _cache_rows(g, sum(new), H, d, basis)
    s["K"], s["V"] = (1.5 * K).to(td), (1.5 * V).to(td)
    s["cu"], s["n_seq"] = _cu(new), len(new)
    s["lens"] = torch.tensor([a + b for a, b in zip(new, old)], dtype=torch.int32, device=DEVICE)
    axes = len(_ints(case["pairs"]))
    where = torch.cat([torch.arange(b, a + b) for a, b in zip(new, old)]).to(DEVICE)
    s["pos"] = (where[:, None] if axes == 1 else torch.stack([where // 1560, where // 52 % 30, where % 52], 1)).to(torch.int32).contiguous()
    s["freq"] = _freqs(_ints(case["pairs"]), 1.0)
    return s


def _cached_inputs(case, seed):
    g, td, d, H, page = _generator(seed, 3), DTYPES[case["dtype"]], case["d"], case["Hkv"], case["page"]
    new, lens = _ints(case["new"]), _ints(case["lens"])
    basis = _basis(g, d)
    s = {}
    s["table"], n_pages = _pages(lens, page, seed)
    K, V = _cache_rows(g, sum(lens), H, d, basis)
    s["K8"], s["kscale"] = _fill(K, lens, s["table"], n_pages, page)
    s["V8"], s["vscale"] = _fill(V, lens, s["table"], n_pages, page)
    s["Q"] = _cache_rows(g, sum(new), case["Hq"], d, basis)[0].to(td)
    s["cu"], s["n_seq"] = _cu(new), len(new)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    s["max_new"], s["max_len"] = max(new), max(lens)
    return s


def _scale(case):
    return 2.0 / math.sqrt(case["d"])


def prepare(case, seed):
    s = {k: case[k] for k in case}
    if case["kind"].startswith("rotary"):
        X, dY, s["pos"], s["freq"] = _rotary_inputs(case, seed)
        s["X"], s["dY"] = _laid_out(X, case["layout"], case["heads"] // 2), dY
    elif case["kind"].startswith("norm"):
        s["X"], s["Y"], s["dZ"], s["dH"], mods = _norm_inputs(case, seed)
        n = case["n"]
        s["shift"], s["scale"], s["gate"] = (mods[:, i * n : (i + 1) * n] for i in range(3))
        s["n_seg"], s["cu"] = mods.shape[0], _cu(_ints(case["lens"]))
    elif case["kind"] == "append":
        s.update(_append_inputs(case, seed))
    else:
        s.update(_cached_inputs(case, seed))
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _channels(pairs, pattern, device):
    """The two channels of every pair, and the coordinate that turns it."""
    total = sum(pairs)
    i = torch.arange(total, device=device)
    ends = torch.tensor(pairs, device=device).cumsum(0)
    axis = torch.bucketize(i, ends, right=True)
    if pattern == "interleaved":
        return 2 * i, 2 * i + 1, axis
    if pattern == "halves":
        return i, i + total, axis
    n = torch.tensor(pairs, device=device)[axis]
    low = i + (ends - torch.tensor(pairs, device=device))[axis]      # earlier axes hold two channels a pair
    return low, low + n, axis


def _plain_turn(x, pos, freq, pairs, pattern, gain, back=False):
    """fp32 [tokens, heads, d]; the angles in 64 bits."""
    lo, hi, axis = _channels(pairs, pattern, x.device)
    t = pos.double()[:, axis] * freq
    c, s = (gain * torch.cos(t)).float()[:, None], (gain * torch.sin(t)).float()[:, None]
    if back:
        s = -s
    y = x.float().clone()
    a, b = y[:, :, lo], y[:, :, hi]
    y[:, :, lo] = a * c - b * s
    y[:, :, hi] = a * s + b * c
    return y


def _plain_rotary(s, grad):
    td, pairs, gain = DTYPES[s["dtype"]], _ints(s["pairs"]), _gain(s["scaling"])
    out = [_plain_turn(s["X"], s["pos"], s["freq"], pairs, s["pattern"], gain).to(td)]
    return out + ([_plain_turn(s["dY"], s["pos"], s["freq"], pairs, s["pattern"], gain, back=True).to(td)] if grad else [])


def _plain_normed(x, form):
    """(normed, 1 / deviation) of rows."""
    c = x - x.mean(1, keepdim=True) if form == "layer" else x
    r = (c.square().mean(1, keepdim=True) + EPS).rsqrt()
    return c * r, r


def _plain_norm_back(w, xh, r, form):
    back = w - xh * (w * xh).mean(1, keepdim=True)
    return r * (back - w.mean(1, keepdim=True) if form == "layer" else back)


def _by_segment(x, seg, n_seg):
    """Sums of the rows of each segment: long ones, in 64 bits, as the product with who belongs where."""
    member = (seg[None] == torch.arange(n_seg, device=x.device)[:, None]).double()
    return (member @ x.double()).float()


def _plain_norm(s, grad):
    td, form, a = DTYPES[s["dtype"]], s["form"], s["residual"]
    x, y = s["X"].float(), s["Y"].float()
    seg = torch.bucketize(torch.arange(x.shape[0], device=x.device), s["cu"][1:].long(), right=True)
    gate, scale, shift = (s[k].float()[seg] for k in ("gate", "scale", "shift"))
    u, ry = _plain_normed(y, form) if s["post"] else (y, None)
    h = a * x + gate * u
    xh, r = _plain_normed(h, form)
    out = [(xh * (1 + scale) + shift).to(td), h.to(td)]
    if grad:
        dz = s["dZ"].float()
        dh = s["dH"].float() + _plain_norm_back(dz * (1 + scale), xh, r, form)
        dy = _plain_norm_back(gate * dh, u, ry, form) if s["post"] else gate * dh
        out += [(a * dh).to(td), dy.to(td)] + [_by_segment(v, seg, s["n_seg"]) for v in (dh * u, dz * xh, dz)]
    return out


def _plain_append_one(rows, values, scale, pg, slot, first_pg, first_slot, begun):
    """Rows [T, H, d] (fp32) to places (pg, slot) of the cache; first_pg, first_slot: where each stream that gets any goes on."""
    most = torch.zeros_like(scale).index_reduce_(0, pg, rows.abs().amax(2), "amax")
    fresh = torch.zeros_like(scale)
    fresh[pg] = _scale_of(most)[pg]
    before = scale[first_pg].clone()
    old = torch.where(begun[:, None], before, torch.zeros_like(before))
    scale[pg] = fresh[pg]
    now = torch.maximum(fresh[first_pg], old)
    scale[first_pg] = now
    raw = values.view(torch.uint8)
    kept = values.view(torch.uint8)[first_pg].view(E4M3)
    moved = (kept.float() * (old / now)[:, :, None, None]).to(E4M3)
    there = torch.arange(kept.shape[2], device=rows.device)[None, None, :, None] < first_slot[:, None, None, None]
    raw[first_pg] = torch.where(there, moved.view(torch.uint8), kept.view(torch.uint8))
    q = (rows / scale[pg][:, :, None]).clamp(-448, 448).to(E4M3)
    raw[pg, :, slot] = q.view(torch.uint8)


def _plain_append(s):
    cu, page = s["cu"].long(), s["page"]
    count = cu[1:] - cu[:-1]
    some = count > 0
    start = s["lens"].long() - count
    t = torch.arange(s["K"].shape[0], device=cu.device)
    seq = torch.bucketize(t, cu[1:], right=True)
    place = start[seq] + t - cu[seq]
    pg, slot = s["table"].long()[seq, place // page], place % page
    start, table = start[some], s["table"].long()[some]
    first_pg = table.gather(1, (start // page)[:, None])[:, 0]
    first_slot = start % page
    pairs = _ints(s["pairs"])
    k = _plain_turn(s["K"], s["pos"], s["freq"], pairs, s["pattern"], 1.0) if pairs != [0] else s["K"].float()
    _plain_append_one(k, s["K8"], s["kscale"], pg, slot, first_pg, first_slot, first_slot > 0)
    _plain_append_one(s["V"].float(), s["V8"], s["vscale"], pg, slot, first_pg, first_slot, first_slot > 0)
    return [s["K8"], s["V8"], s["kscale"], s["vscale"]]


def _widened(values, scale, table, most):
    """fp32 [n_seq, H, most, d] of the pages of every stream in turn."""
    x = values.view(torch.uint8)[table].view(E4M3).float() * scale[table][..., None, None]
    n, pages, H, page, d = x.shape
    return x.transpose(1, 2).reshape(n, H, pages * page, d)[:, :, :most]


def _plain_cached(s):
    Hq, Hkv, d, td, n = s["Hq"], s["Hkv"], s["d"], DTYPES[s["dtype"]], s["n_seq"]
    mq, mk, group = s["max_new"], max(1, s["max_len"]), Hq // Hkv
    cu, total = s["cu"].long(), s["Q"].shape[0]
    nq, nk = cu[1:] - cu[:-1], s["lens"].long()
    pos = torch.arange(mq, device=cu.device)
    at = (cu[:-1, None] + pos).clamp(max=total - 1)
    q = (s["Q"].float()[at] * (pos < nq[:, None])[:, :, None, None]).transpose(1, 2).reshape(n, Hkv, group * mq, d)
    table = s["table"].long()
    k, v = _widened(s["K8"], s["kscale"], table, mk), _widened(s["V8"], s["vscale"], table, mk)
    i, j = pos[None, :, None], torch.arange(mk, device=cu.device)[None, None, :]
    seen = (j < nk[:, None, None]) & ((j <= i + (nk - nq)[:, None, None]) if s["causal"] else (i >= 0))
    p = (q @ k.transpose(2, 3).contiguous()).mul_(_scale(s))
    p.view(n, Hkv, group, mq, mk).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(3, keepdim=True).clamp(min=-3e38)      # rows that see no key: every weight exp(-inf)
    p.sub_(top).exp_()
    whole = p.sum(3, keepdim=True)
    t = torch.arange(total, device=cu.device)
    seq = torch.bucketize(t, cu[1:], right=True)

    def rows(x, last):
        return x.reshape((n, Hq, mq) + last).transpose(1, 2)[seq, t - cu[seq]]

    O = (p @ v).div_(whole.clamp(min=1e-38))
    return [rows(O, (d,)).to(td), rows(top + whole.log(), ()).transpose(0, 1).contiguous()]


# ---------------------------------------------------------------------------------------------- one pass
def _own_rotary(s, grad):
    import paper_2502_07590_amd as dsv
    p = dsv.Rotary(s["tokens"], s["heads"], s["d"], s["dtype"], _ints(s["pairs"]), layout=s["pattern"], gain=_gain(s["scaling"]))
    out = [dsv.rotary_fwd(p, s["X"], s["pos"], s["freq"])]
    return out + ([dsv.rotary_bwd(p, s["dY"], s["pos"], s["freq"])] if grad else [])


def _own_norm(s, grad):
    import paper_2502_07590_amd as dsv
    p = dsv.GatedNorm(s["X"].shape[0], s["n"], s["n_seg"], s["dtype"], EPS, kind=s["form"], post=s["post"], residual=s["residual"])
    Z, H, stats = dsv.gated_norm_fwd(p, s["X"], s["cu"], s["Y"], s["gate"], s["scale"], s["shift"])
    if not grad:
        return [Z, H]
    return [Z, H, *dsv.gated_norm_bwd(p, s["X"], s["cu"], stats, s["dZ"], s["Y"], s["gate"], s["scale"], dH=s["dH"])]


def _own_cache(s, total, most, Hq):
    import paper_2502_07590_amd as dsv
    return dsv, dsv.Cache(s["n_seq"], total, most, Hq, s["Hkv"], s["d"], s["dtype"], s["K8"].shape[0], s["page"], s["table"].shape[1], scale=_scale(s),
                          causal=s.get("causal", False), max_len=s.get("max_len"))


def _own_append(s):
    total = s["K"].shape[0]
    dsv, p = _own_cache(s, total, total, s["Hkv"])
    pairs = _ints(s["pairs"])
    turn = dsv.Rotary(total, s["Hkv"], s["d"], s["dtype"], pairs, layout=s["pattern"]) if pairs != [0] else None
    dsv.cache_append(p, s["K"], s["V"], s["cu"], s["lens"], s["table"], s["K8"], s["V8"], s["kscale"], s["vscale"], rotary=turn, pos=s["pos"], freq=s["freq"])
    return [s["K8"], s["V8"], s["kscale"], s["vscale"]]


def _own_cached(s):
    dsv, p = _own_cache(s, s["Q"].shape[0], s["max_new"], s["Hq"])
    return list(dsv.cache_attn_fwd(p, s["Q"], s["cu"], s["lens"], s["table"], s["K8"], s["V8"], s["kscale"], s["vscale"]))


def run(s):
    grad = s["kind"].endswith("_step")
    if s["kind"].startswith("rotary"):
        return _own_rotary(s, grad) if own else _plain_rotary(s, grad)
    if s["kind"].startswith("norm"):
        return _own_norm(s, grad) if own else _plain_norm(s, grad)
    if s["kind"] == "append":
        return _own_append(s) if own else _plain_append(s)
    return _own_cached(s) if own else _plain_cached(s)


# ---------------------------------------------------------------------------------------------- floors
def _seen(case):
    """(query, key) pairs that are not masked, over all query heads."""
    total = 0
    for nq, nk in zip(_ints(case["new"]), _ints(case["lens"])):
        if not case["causal"]:
            total += nq * nk
        else:                        # query i sees min(nk, max(0, i + 1 + nk - nq)) keys
            rows = min(nq, nk)       # those that see any
            total += rows * nk - rows * (rows - 1) // 2
    return total * case["Hq"]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    grad = case["kind"].endswith("_step")
    if case["kind"].startswith("rotary"):
        cells, pairs = case["tokens"] * case["heads"], sum(_ints(case["pairs"]))
        once = {"bytes": 2 * cells * case["d"] * es, "flops": 6 * cells * pairs}
        own_ = 4 * case["tokens"] * len(_ints(case["pairs"])) + 8 * pairs
        return {"bytes": once["bytes"] * (2 if grad else 1) + own_, "flops": once["flops"] * (2 if grad else 1)}
    if case["kind"].startswith("norm"):
        lens, n = _ints(case["lens"]), case["n"]
        rows = sum(lens)
        fwd = {"bytes": 4 * rows * n * es + 3 * len(lens) * n * es, "flops": (16 if case["post"] else 10) * rows * n}
        if not grad:
            return fwd
        return {"bytes": fwd["bytes"] + 4 * rows * n * es + 12 * len(lens) * n, "flops": fwd["flops"] + (32 if case["post"] else 20) * rows * n}
    cells = case["Hkv"] * case["d"]
    if case["kind"] == "append":
        total = sum(_ints(case["new"]))
        begun = sum(b % case["page"] for a, b in zip(_ints(case["new"]), _ints(case["old"])) if a)    # their scale has to be looked at, and may grow
        return {"bytes": 2 * total * cells * (es + 1) + 2 * begun * cells, "flops": total * cells * 6}
    q = sum(_ints(case["new"])) * case["Hq"]
    pages = sum(-(-n // case["page"]) for n in _ints(case["lens"]))
    return {"bytes": 2 * sum(_ints(case["lens"])) * cells + 2 * q * case["d"] * es + 4 * q + pages * (4 + 8 * case["Hkv"]), "flops": 4 * case["d"] * _seen(case)}


# ---------------------------------------------------------------------------------------------- 64-bit references
def _exact_turn(x, pos, freq, pairs, pattern, back=False):
    """Every pair a complex number, times a unit one."""
    y, done = x.clone(), 0
    for axis, n in enumerate(pairs):
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos[:, axis, None].double() * freq[done : done + n])[:, None]
        turn = turn.conj() if back else turn
        if pattern == "interleaved":
            lo, hi = slice(2 * done, 2 * (done + n), 2), slice(2 * done + 1, 2 * (done + n), 2)
        elif pattern == "halves":
            lo, hi = slice(done, done + n), slice(sum(pairs) + done, sum(pairs) + done + n)
        else:
            lo, hi = slice(2 * done, 2 * done + n), slice(2 * done + n, 2 * (done + n))
        z = torch.complex(x[..., lo], x[..., hi]) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        done += n
    return y


def _exact_rotary(case, seed):
    X, dY, pos, freq = _rotary_inputs(case, seed)
    pairs, gain = _ints(case["pairs"]), _gain(case["scaling"])
    rot = 2 * sum(pairs)

    def whole(x, back):
        y = _exact_turn(x.double(), pos, freq, pairs, case["pattern"], back)
        y[..., :rot] *= gain
        return y

    return [whole(X, False)] + ([whole(dY, True)] if case["kind"].endswith("_step") else [])


def _exact_norm(case, seed):
    X, Y, dZ, dH, mods = (t.double() for t in _norm_inputs(case, seed))
    n, lens, grad = case["n"], _ints(case["lens"]), case["kind"].endswith("_step")
    leaves = [X, Y] + [mods[:, i * n : (i + 1) * n].clone() for i in (2, 1, 0)]
    leaves = [t.requires_grad_(grad) for t in leaves]
    x, y, gate, scale, shift = leaves
    each = torch.tensor(lens, device=DEVICE)

    def normed(v):
        if case["form"] == "rms":
            return v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
        var, mean = torch.var_mean(v, -1, correction=0, keepdim=True)
        return (v - mean) / (var + EPS).sqrt()

    h = case["residual"] * x + gate.repeat_interleave(each, 0) * (normed(y) if case["post"] else y)
    z = normed(h) * (1 + scale.repeat_interleave(each, 0)) + shift.repeat_interleave(each, 0)
    if not grad:
        return [z, h]
    return [z.detach(), h.detach(), *torch.autograd.grad((z * dZ).sum() + (h * dH).sum(), leaves)]


def _exact_e4m3(x):
    """The nearest value of three bits behind the leading one, exponents from -6, the even one of two."""
    step = torch.ldexp(torch.ones_like(x), torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).int() - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_append(case, seed):
    s = _append_inputs(case, seed)
    page, pairs = case["page"], _ints(case["pairs"])
    K = s["K"].double() if pairs == [0] else _exact_turn(s["K"].double(), s["pos"], s["freq"], pairs, case["pattern"])
    out = []
    for rows, values, scale in ((K, s["K8"], s["kscale"]), (s["V"].double(), s["V8"], s["vscale"])):
        values, scale, a = values.double(), scale.double(), 0
        for i, (new, old) in enumerate(zip(_ints(case["new"]), _ints(case["old"]))):
            at = old
            while at < old + new:
                pg, begun = int(s["table"][i, at // page]), at % page
                n = min(page - begun, old + new - at)
                piece = rows[a : a + n]
                least = torch.exp2(torch.ceil(torch.log2(piece.abs().amax((0, 2)) / 448)))
                now = torch.maximum(least, scale[pg]) if begun else least
                values[pg, :, :begun] = _exact_e4m3(values[pg, :, :begun] * (scale[pg] / now)[:, None, None])
                values[pg, :, begun : begun + n] = _exact_e4m3(piece / now[:, None]).transpose(0, 1)
                scale[pg] = now
                a, at = a + n, at + n
        out.append((values, scale))
    return [out[0][0], out[1][0], out[0][1], out[1][1]]


def _exact_cached(case, seed):
    s = _cached_inputs(case, seed)
    Q, group, scale, page = s["Q"].double(), case["Hq"] // case["Hkv"], _scale(case), case["page"]
    O = torch.zeros_like(Q)
    lse = torch.full((case["Hq"], Q.shape[0]), -math.inf, dtype=torch.float64, device=DEVICE)
    a = 0
    for i, (nq, nk) in enumerate(zip(_ints(case["new"]), _ints(case["lens"]))):
        pages = s["table"][i, : -(-nk // page)].long()
        for h in range(case["Hkv"] if nk and nq else 0):
            k, v = ((x[pages, h].double() * y[pages, h].double()[:, None, None]).reshape(-1, case["d"])[:nk] for x, y in ((s["K8"].float(), s["kscale"]), (s["V8"].float(), s["vscale"])))
            for m in range(h * group, (h + 1) * group):
                x = scale * (Q[a : a + nq, m] @ k.T)
                if case["causal"]:
                    last = torch.arange(nq, device=DEVICE) + nk - nq
                    x = torch.where(torch.arange(nk, device=DEVICE)[None] <= last[:, None], x, -math.inf)
                total = torch.logsumexp(x, 1)
                lse[m, a : a + nq] = total
                O[a : a + nq, m] = torch.exp(x - torch.where(total.isinf(), 0.0, total)[:, None]) @ v
        a += nq
    return [O, lse]


def exact(case, seed):
    if case["kind"].startswith("rotary"):
        return _exact_rotary(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, seed)
    return _exact_append(case, seed) if case["kind"] == "append" else _exact_cached(case, seed)
