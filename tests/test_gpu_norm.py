"""Layer norm on the GPU against its formulas in 64 bits: widths around every split of a row over lanes, one to many rows, views, missing
weights, and the norm in front of both kinds of attention as a training step runs it."""
import math

import pytest
import torch

import packed_ref as ref

pytestmark = pytest.mark.gpu

dsv = pytest.importorskip("paper_2502_07590_amd")

DEV = "cuda:0"


def inputs(tokens, heads, n, dtype, seed=0, affine=True):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn(tokens, heads, n, generator=g) * (1 + 3 * torch.rand(n, generator=g)) + torch.randn(n, generator=g)
    dY = torch.randn(tokens, heads, n, generator=g)
    gamma, beta = 1 + 0.3 * torch.randn(n, generator=g), torch.randn(n, generator=g)
    td = ref.DTYPES[dtype]
    return [x.to(td) for x in (X, dY)] + ([x.to(td) for x in (gamma, beta)] if affine else [None, None])


def check(tokens, heads, n, dtype, layout="token", affine=True, eps=1e-5, seed=0, X=None):
    host = inputs(tokens, heads, n, dtype, seed, affine)
    if X is not None:
        host[0] = X
    dev = [None if x is None else x.to(DEV) for x in host]
    x, dy = ref.laid_out(dev[0], layout), ref.laid_out(dev[1], layout)
    p = dsv.Norm(tokens, n, dtype, eps, heads=heads)
    Y, mean, rstd = dsv.layer_norm_fwd(p, x, dev[2], dev[3])
    dX, dgamma, dbeta = dsv.layer_norm_bwd(p, x, dev[2], mean, rstd, dy)
    torch.cuda.synchronize()
    want = ref.norm(*[None if t is None else t.double() for t in (host[0], host[2], host[3])], eps, host[1].double(), dtype)
    got = dict(Y=Y, mean=mean, rstd=rstd, dX=dX)
    if affine:
        got.update(dgamma=dgamma, dbeta=dbeta)
    else:
        assert dgamma is None and dbeta is None
    for name, t in got.items():
        ref.assert_within(f"{name} n={n}", t, want[name])
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 31, 64, 65, 100, 128, 136, 255, 256, 257, 512, 520, 1024, 1028, 1155, 1536, 2048, 2056, 4096, 4100, 4104, 8191, 8192])
def test_widths(n, dtype):
    check(5, 1, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,n", [(1, 1, 128), (1000, 16, 128), (4099, 3, 64), (9001, 1, 256), (2500, 1, 2048), (1500, 1, 1155), (2500, 2, 32), (1100, 1, 8192)])
def test_rows_from_one_to_more_than_the_blocks_take_at_once(tokens, heads, n, dtype):
    check(tokens, heads, n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,n", [(140000, 1, 8), (45000, 3, 64), (140000, 1, 3), (17000, 1, 520), (4500, 1, 4104)])
def test_more_rows_than_either_kernel_takes_at_once(tokens, heads, n, dtype):
    """Every lane group walks: 4096 blocks of the forward, of 32 rows for the narrowest, of one for the widest."""
    check(tokens, heads, n, dtype)


@pytest.mark.parametrize("layout", ["head", "slice"])
@pytest.mark.parametrize("n", [64, 77, 128])
def test_views(layout, n):
    a = check(301, 5, n, "bf16", layout)
    b = check(301, 5, n, "bf16")
    for k in a:
        if n % 8 == 0 or k != "dgamma" and k != "dbeta":
            assert torch.equal(a[k].contiguous(), b[k].contiguous()), k


def test_rows_off_their_16_bytes():
    """A width of whole pieces whose rows begin between them: the element-wise form, the same results within the bounds."""
    tokens, n = 50, 128
    X, dY, gamma, beta = inputs(tokens, 1, n, "bf16")
    wide = torch.zeros(tokens, 1, n + 3, dtype=torch.bfloat16, device=DEV)
    x = wide[:, :, 1 : 1 + n]
    x.copy_(X)
    p = dsv.Norm(tokens, n, "bf16", 1e-5)
    Y, mean, rstd = dsv.layer_norm_fwd(p, x, gamma.to(DEV), beta.to(DEV))
    dX, dgamma, dbeta = dsv.layer_norm_bwd(p, x, gamma.to(DEV), mean, rstd, dY.to(DEV))
    want = ref.norm(X.double(), gamma.double(), beta.double(), 1e-5, dY.double())
    for name, t in dict(Y=Y, mean=mean, rstd=rstd, dX=dX, dgamma=dgamma, dbeta=dbeta).items():
        ref.assert_within(name, t, want[name])


def test_without_weights_and_with_one_of_them():
    check(40, 2, 128, "bf16", affine=False)
    check(40, 1, 1000, "f32", affine=False)
    X, dY, gamma, beta = inputs(9, 1, 64, "f32")
    p = dsv.Norm(9, 64, "f32", 1e-5)
    for g, b in ((gamma, None), (None, beta)):
        Y, mean, rstd = dsv.layer_norm_fwd(p, X.to(DEV), None if g is None else g.to(DEV), None if b is None else b.to(DEV))
        want = ref.norm(X.double(), None if g is None else g.double(), None if b is None else b.double(), 1e-5, dtype="f32")
        ref.assert_within("Y", Y, want["Y"])
    dX, dgamma, dbeta = dsv.layer_norm_bwd(p, X.to(DEV), None, mean, rstd, dY.to(DEV), dgamma=torch.empty(64, device=DEV))
    want = ref.norm(X.double(), None, None, 1e-5, dY.double(), "f32")
    for name, t in dict(dX=dX, dgamma=dgamma, dbeta=dbeta).items():
        ref.assert_within(name, t, want[name])


def test_rows_far_from_zero_and_rows_that_are_constant():
    """A mean a thousand times the spread: the variance comes from differences.  A constant row: xh is 0 and y is beta."""
    g = torch.Generator().manual_seed(5)
    check(20, 1, 512, "f32", X=1000 + torch.randn(20, 1, 512, generator=g))
    got = check(6, 1, 128, "f32", X=torch.full((6, 1, 128), 0.5))
    assert (got["mean"] == 0.5).all()


def test_no_rows():
    p = dsv.Norm(0, 64, "bf16")
    X = torch.empty(0, 1, 64, dtype=torch.bfloat16, device=DEV)
    Y, mean, rstd = dsv.layer_norm_fwd(p, X)
    gamma = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    dX, dgamma, dbeta = dsv.layer_norm_bwd(p, X, gamma, mean, rstd, X, dgamma=torch.full((64,), 7.0, device=DEV), dbeta=torch.full((64,), 7.0, device=DEV))
    assert (dgamma == 0).all() and (dbeta == 0).all()


def test_runs_and_replays_are_equal_bit_for_bit():
    tokens, heads, n = 3000, 4, 128
    X, dY, gamma, beta = (x.to(DEV) for x in inputs(tokens, heads, n, "bf16"))
    p = dsv.Norm(tokens, n, "bf16", heads=heads)
    ws = torch.empty(dsv.layer_norm_bwd_workspace(p), dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(X), torch.empty(tokens, heads, device=DEV), torch.empty(tokens, heads, device=DEV), torch.empty_like(X), torch.empty(n, device=DEV),
           torch.empty(n, device=DEV)]

    def step():
        dsv.layer_norm_fwd(p, X, gamma, beta, *out[:3])
        dsv.layer_norm_bwd(p, X, gamma, out[1], out[2], dY, *out[3:], workspace=ws)

    step()
    torch.cuda.synchronize()
    eager = [x.clone() for x in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for x in out:
            x.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_norms_in_front_of_full_and_sparse_attention():
    """A block's step: the rows of Q and K normed in place of a fused projection's output, then attention -- full, and sparse with every key
    kept -- and the gradients back through both.  The two agree with each other and with the same chain in 64 bits."""
    tokens, H, d, scale = 96, 2, 64, 0.125
    g = torch.Generator().manual_seed(11)
    qkv = torch.randn(tokens, 3 * H, d, generator=g)
    dO = torch.randn(tokens, H, d, generator=g)
    gq, bq, gk, bk = (1 + 0.2 * torch.randn(d, generator=g), 0.1 * torch.randn(d, generator=g), 1 + 0.2 * torch.randn(d, generator=g), 0.1 * torch.randn(d, generator=g))

    x = qkv.double().requires_grad_()
    w = [t.double().requires_grad_() for t in (gq, bq, gk, bk)]
    q = torch.nn.functional.layer_norm(x[:, :H], (d,), w[0], w[1], 1e-5)
    k = torch.nn.functional.layer_norm(x[:, H : 2 * H], (d,), w[2], w[3], 1e-5)
    s = scale * torch.einsum("ihd,jhd->hij", q, k)
    O = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), x[:, 2 * H :])
    grads = torch.autograd.grad((O * dO.double()).sum(), [x, *w])

    dev = qkv.to(DEV)
    Q, K, V = dev[:, :H], dev[:, H : 2 * H], dev[:, 2 * H :]
    np_ = dsv.Norm(tokens, d, "f32", 1e-5, heads=H)
    wd = [t.to(DEV) for t in (gq, bq, gk, bk)]
    Qn, mq, rq = dsv.layer_norm_fwd(np_, Q, wd[0], wd[1])
    Kn, mk, rk = dsv.layer_norm_fwd(np_, K, wd[2], wd[3])

    def back(dQn, dKn, dV):
        dx = torch.empty_like(dev)
        _, dgq, dbq = dsv.layer_norm_bwd(np_, Q, wd[0], mq, rq, dQn, dX=dx[:, :H])
        _, dgk, dbk = dsv.layer_norm_bwd(np_, K, wd[2], mk, rk, dKn, dX=dx[:, H : 2 * H])
        dx[:, 2 * H :] = dV
        return [dx, dgq, dbq, dgk, dbk]

    p = dsv.Packed(1, tokens, tokens, tokens, tokens, H, H, d, "f32", scale)
    cu = torch.tensor([0, tokens], dtype=torch.int32, device=DEV)
    Op, lse = dsv.packed_attn_fwd(p, Qn, Kn, V, cu, cu)
    packed = back(*dsv.packed_attn_bwd(p, Qn, Kn, V, cu, cu, Op, lse, dO.to(DEV)))

    head = lambda t: t.transpose(0, 1).contiguous()[None]  # noqa: E731
    sp = dsv.Problem(1, H, tokens, d, 16, "f32", [tokens] * H, scale)
    idx = torch.arange(tokens, dtype=torch.int32, device=DEV).repeat(H * tokens)
    Os, lses = dsv.sparse_attn_fwd(sp, head(Qn), head(Kn), head(V), idx)
    sparse = back(*[t[0].transpose(0, 1) for t in dsv.sparse_attn_bwd(sp, head(Qn), head(Kn), head(V), idx, Os, lses, head(dO.to(DEV)))])

    # 32-bit sums of at most 96 * 64 terms of size one, through four steps: 1e-4 is over a hundred times 2^-24 times their root
    assert (Op.double().cpu() - O).abs().max() < 1e-4 and (Os[0].transpose(0, 1).double().cpu() - O).abs().max() < 1e-4
    for name, a, b, c in zip(("dqkv", "dgamma_q", "dbeta_q", "dgamma_k", "dbeta_k"), packed, sparse, grads):
        assert (a.double().cpu() - c).abs().max() < 1e-4 * max(1.0, float(c.abs().max())), name
        assert (b.double().cpu() - c).abs().max() < 1e-4 * max(1.0, float(c.abs().max())), name
    assert math.isfinite(float(lse.sum()))
