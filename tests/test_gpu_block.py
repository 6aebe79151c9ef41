"""The transformer-block operators on the GPU against their definitions in 64 bits, element by element within the bounds that oracle/block_ops.py
derives from the arithmetic: every type, direction and activation; odd sizes; strided rows and heads; masks; empty rows; streams and graphs."""
import math

import pytest
import torch

from oracle import block_ops as O
from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
TYPES = [F16, BF16, F32]
ACTS = {"none": B.WINO_ACT_NONE, "silu": B.WINO_ACT_SILU, "gelu": B.WINO_ACT_GELU, "gelu_tanh": B.WINO_ACT_GELU_TANH}


def _rand(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def _d(t):
    return None if t is None else t.cpu().double()


def _inside(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - bound
    assert over.max() <= 0, (what, "by", over.max().item(), "at", int(over.argmax()), "error", (got - ref).abs().max().item())


def _wide(t, extra):
    """The same values as rows of a wider tensor whose other columns hold NaN."""
    big = torch.full((t.shape[0], t.shape[1] + extra), math.nan, dtype=t.dtype, device=DEV)
    big[:, :t.shape[1]] = t.to(DEV)
    return big[:, :t.shape[1]]


def _products(M, K, N, dtype, halves=1, seed=0):
    x, w = _rand((M, K), dtype, seed), _rand((halves * N, K), dtype, seed + 1, K ** -0.5)
    return x, w, _rand((halves * N,), F32, seed + 2, 0.3), _rand((M, N), dtype, seed + 3), _rand((M, N), dtype, seed + 4)


# rows, features in, features out: one token to several tiles, odd sizes, a ragged tile in every direction, long reductions (cut into ranges), whole tiles
SIZES = [(1, 8, 8), (1, 1, 1), (2, 320, 64), (5, 77, 33), (16, 1280, 40), (33, 64, 200), (64, 640, 320), (65, 128, 129), (130, 96, 256), (257, 320, 96),
         (300, 200, 136), (512, 64, 512)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_linear(M, K, N, dtype):
    x, w, b, r, _ = _products(M, K, N, dtype)
    for kind, bias, res in (("none", None, None), ("silu", b, r), ("gelu", b, None), ("gelu_tanh", None, r)):
        y = B.linear(x.to(DEV), w.to(DEV), None if bias is None else bias.to(DEV), ACTS[kind], None if res is None else res.to(DEV))
        _inside(y, *O.linear(_d(x), _d(w), _d(bias), _d(res), kind, dtype), (M, K, N, kind))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_linear_backward(M, K, N, dtype):
    x, w, b, _, dy = _products(M, K, N, dtype)
    for kind in ACTS:
        got = B.linear_backward(x.to(DEV), w.to(DEV), b.to(DEV), dy.to(DEV), ACTS[kind])
        for name, g, (ref, bound) in zip(("dx", "dw", "dbias"), got, O.linear_backward(_d(x), _d(w), _d(b), _d(dy), kind, dtype)):
            _inside(g, ref, bound, (M, K, N, kind, name))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_glu_and_backward(M, K, N, dtype):
    x, w, b, _, dh = _products(M, K, N, dtype, 2)
    for kind in ("gelu", "silu", "gelu_tanh", "none"):
        bias = None if kind == "silu" else b
        bd = None if bias is None else bias.to(DEV)
        _inside(B.glu(x.to(DEV), w.to(DEV), bd, ACTS[kind]), *O.glu(_d(x), _d(w), _d(bias), kind, dtype), (M, K, N, kind))
        got = B.glu_backward(x.to(DEV), w.to(DEV), bd, dh.to(DEV), ACTS[kind])
        for name, g, (ref, bound) in zip(("dx", "dw", "dbias"), got, O.glu_backward(_d(x), _d(w), _d(bias), _d(dh), kind, dtype)):
            _inside(g, ref, bound, (M, K, N, kind, name))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra", [8, 3])
def test_strided_rows_and_untouched_neighbours(dtype, extra):
    M, K, N = 70, 72, 88
    x, w, b, r, dy = _products(M, K, N, dtype)
    out = torch.full((M + 2, N + extra), 7.0, dtype=dtype, device=DEV)
    y = out[:M, :N]
    B.wino_linear(_wide(x, extra), w.to(DEV), b.to(DEV), y, ACTS["gelu"], _wide(r, extra), _ws(B.wino_linear_workspace_bytes(M, N, K, B.DTYPE_OF[dtype])))
    _inside(y, *O.linear(_d(x), _d(w), _d(b), _d(r), "gelu", dtype), extra)
    assert (out[M:] == 7).all() and (out[:, N:] == 7).all()
    dxo = torch.full((M, K + extra), 7.0, dtype=dtype, device=DEV)
    dw, db = torch.empty(N, K, dtype=dtype, device=DEV), torch.empty(N, device=DEV)
    ws = _ws(B.wino_linear_backward_workspace_bytes(M, N, K, B.DTYPE_OF[dtype], ACTS["silu"]))
    B.wino_linear_backward(_wide(x, extra), w.to(DEV), b.to(DEV), _wide(dy, extra), dxo[:, :K], dw, db, ACTS["silu"], ws)
    for g, (ref, bound) in zip((dxo[:, :K], dw, db), O.linear_backward(_d(x), _d(w), _d(b), _d(dy), "silu", dtype)):
        _inside(g, ref, bound, extra)
    assert (dxo[:, K:] == 7).all()
    x, w, b, _, dh = _products(M, K, N, dtype, 2)
    out.fill_(7.0)
    B.wino_glu(_wide(x, extra), w.to(DEV), b.to(DEV), y, ACTS["gelu"])
    _inside(y, *O.glu(_d(x), _d(w), _d(b), "gelu", dtype), extra)
    assert (out[M:] == 7).all() and (out[:, N:] == 7).all()


def _ws(n):
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None      # NaN in every type: what is read is written first


def test_residual_may_be_the_output():
    x, w, b, r, _ = _products(40, 64, 72, F16)
    y = r.to(DEV)
    B.wino_linear(x.to(DEV), w.to(DEV), b.to(DEV), y, ACTS["none"], y, _ws(B.wino_linear_workspace_bytes(40, 72, 64, B.WINO_F16)))
    _inside(y, *O.linear(_d(x), _d(w), _d(b), _d(r), "none", F16), "in place")


@pytest.mark.parametrize("dtype", TYPES)
def test_activations_at_the_ends_of_the_range(dtype):
    """Large, infinite and NaN pre-activations through a product with a unit matrix: no NaN that the definition does not have."""
    big = {F16: 60000.0, BF16: 1e30, F32: 1e30}[dtype]
    z = torch.tensor([[0.0, -0.0, 30.0, -30.0, 200.0, -200.0, big, -big]], dtype=dtype)
    w = torch.eye(8, dtype=dtype)
    for kind in ("silu", "gelu", "gelu_tanh"):
        y = _d(B.linear(z.to(DEV), w.to(DEV), None, ACTS[kind]))
        ref = torch.where(_d(z) > 0, _d(z), 0.0)
        assert ((y - ref).abs() <= 1e-5 + 2 * O.UNIT[dtype] * ref).all(), (kind, y)
        dx = _d(B.linear_backward(z.to(DEV), w.to(DEV), None, torch.ones_like(z).to(DEV), ACTS[kind])[0])
        slope = torch.where(_d(z) > 0, 1.0, 0.0)
        slope[0, :2] = 0.5
        assert ((dx - slope).abs() <= 1e-5 + 2 * O.UNIT[dtype]).all(), (kind, dx)
        one = torch.ones(1, 8, dtype=dtype)
        for v, want in ((math.inf, math.inf), (-math.inf, 0.0)):
            b = torch.full((8,), v, device=DEV)
            y = B.linear(one.to(DEV), w.to(DEV), b, ACTS[kind])
            assert (y == want).all(), (kind, v, y)
        assert torch.isnan(B.linear(one.to(DEV), w.to(DEV), torch.full((8,), math.nan, device=DEV), ACTS[kind])).all()


# ---- attention ------------------------------------------------------------------------------------------------------------------------
def _heads(Bn, Sq, Skv, H, Hkv, D, dtype, seed=0):
    return (_rand((Bn, Sq, H, D), dtype, seed, 1.5), _rand((Bn, Skv, Hkv, D), dtype, seed + 1), _rand((Bn, Skv, Hkv, D), dtype, seed + 2),
            _rand((Bn, Sq, H, D), dtype, seed + 3))


def _check_attention(Bn, Sq, Skv, H, Hkv, D, dtype, lens=None, mask=None, scale=None, backward=True, seed=0):
    q, k, v, do = _heads(Bn, Sq, Skv, H, Hkv, D, dtype, seed)
    valid = torch.ones(Bn, Skv, dtype=torch.bool)
    kw = {}
    if lens is not None:
        valid &= torch.arange(Skv)[None] < torch.tensor(lens)[:, None]
        kw["kv_len"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if mask is not None:
        valid &= mask
        kw["key_mask"] = mask.to(DEV)
    c = D ** -0.5 if scale is None else scale
    what = (Bn, Sq, Skv, H, Hkv, D, str(dtype), lens)
    k, v = k.clone(), v.clone()
    kd, vd = _d(k), _d(v)
    k[~valid] = math.nan                                 # what stands at other keys is never used
    v[~valid] = math.inf
    dev = [t.to(DEV) for t in (q, k, v, do)]
    o, lse = B.attention(*dev[:3], scale=scale, with_lse=True, **kw)
    ref, rlse, bound = O.attention(_d(q), kd, vd, valid, c, dtype)
    _inside(o, ref, bound, what)
    got = lse.cpu().double()
    empty = torch.isneginf(rlse)
    assert (torch.isneginf(got) == empty).all(), what
    if not empty.all():
        s = (_d(q).abs().amax() * kd.abs().amax() * D * c).item()
        assert ((got - rlse)[~empty].abs() <= (D + 40) * O.F32 * (s + 20)).all(), what
    assert torch.equal(o, B.attention(*dev[:3], scale=scale, **kw)), what          # with and without lse, twice: the same bits
    if backward:
        grads = B.attention_backward(*dev[:3], o, lse, dev[3], scale=scale, **kw)
        for name, g, (r, e) in zip(("dq", "dk", "dv"), grads, O.attention_backward(_d(q), kd, vd, valid, c, _d(do), dtype)):
            _inside(g, r, e, what + (name,))
        for g in grads[1:]:
            assert (g[~valid.to(DEV)] == 0).all(), what
        again = B.attention_backward(*dev[:3], o, lse, dev[3], scale=scale, **kw)
        assert all(torch.equal(a, b) for a, b in zip(grads, again)), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 48, 64, 72, 80, 96, 104, 128, 136, 160])
def test_attention_head_sizes(D, dtype):
    _check_attention(2, 70, 77, 2, 2, D, dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [168, 208, 256])
def test_attention_wide_heads(D, dtype):
    _check_attention(1, 40, 100, 2, 1, D, dtype, lens=[90])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Sq,Skv", [(1, 1), (1, 2), (1, 64), (1, 65), (2, 63), (3, 129), (31, 33), (32, 64), (128, 128), (129, 1), (200, 300), (5, 1100)])
def test_attention_lengths(Sq, Skv, dtype):
    _check_attention(2, Sq, Skv, 2, 2, 40, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (6, 2), (8, 4)])
@pytest.mark.parametrize("Sq", [1, 5, 67])
def test_attention_shared_heads(H, Hkv, Sq, dtype):
    _check_attention(2, Sq, 90, H, Hkv, 64, dtype, lens=[90, 41])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Sq", [1, 50])
def test_attention_masks_and_empty_rows(Sq, dtype):
    g = torch.Generator().manual_seed(5)
    mask = torch.rand((4, 200), generator=g) < 0.5
    mask[1] = False
    mask[2, :128] = False                                # whole tiles without a key
    mask[3, 1:] = False
    _check_attention(4, Sq, 200, 2, 2, 64, dtype, mask=mask)
    _check_attention(4, Sq, 200, 2, 2, 64, dtype, lens=[0, 200, 64, 1])
    _check_attention(4, Sq, 200, 2, 2, 64, dtype, lens=[130, 150, 64, 7], mask=mask)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_many_keys_for_few_rows(dtype):
    _check_attention(2, 1, 5000, 4, 2, 64, dtype, lens=[5000, 300], backward=False)
    _check_attention(1, 2, 3001, 2, 2, 128, dtype, mask=torch.rand((1, 3001), generator=torch.Generator().manual_seed(1)) < 0.01, backward=False)
    _check_attention(2, 3, 2500, 1, 1, 40, dtype, lens=[0, 2500])


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_many_rows_for_few_keys(dtype):
    """Key gradients summed over ranges of the rows."""
    _check_attention(1, 2100, 20, 2, 1, 40, dtype)
    _check_attention(2, 1030, 130, 2, 2, 64, dtype, lens=[130, 3])


def test_attention_scale_and_lengths_out_of_range():
    _check_attention(2, 20, 50, 2, 2, 64, F16, scale=0.31)
    q, k, v, _ = (t.to(DEV) for t in _heads(3, 9, 50, 2, 2, 64, F16))
    lens = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    assert torch.equal(B.attention(q, k, v, kv_len=lens([-5, 1000, 50])), B.attention(q, k, v, kv_len=lens([0, 50, 50])))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_large_scores(dtype):
    """Scores of several hundred: the running maximum carries them; weights are one or nothing."""
    Bn, S, D = 1, 130, 64
    q, k, v, _ = _heads(Bn, S, S, 1, 1, D, dtype)
    q, k = q * 8, k * 8
    o = B.attention(q.to(DEV), k.to(DEV), v.to(DEV))
    ref, _, bound = O.attention(_d(q), _d(k), _d(v), torch.ones(Bn, S, dtype=torch.bool), D ** -0.5, dtype)
    _inside(o, ref, bound, "large scores")


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_strides_of_packed_tensors(dtype):
    """q, k, v and their gradients as slices of one packed tensor each; heads in front of positions."""
    Bn, S, H, D = 2, 75, 3, 40
    packed = torch.stack([t for t in _heads(Bn, S, S, H, H, D, dtype)[:3]], 2)           # [B,S,3,H,D]
    do = _rand((Bn, S, H, D), dtype, 9)
    gpu, grads = packed.to(DEV), torch.full(packed.shape, 7.0, dtype=dtype, device=DEV)
    q, k, v = gpu.unbind(2)
    o_hs = torch.full((Bn, H, S, D), 7.0, dtype=dtype, device=DEV)                        # [B,H,S,D], seen as [B,S,H,D]
    o, lse = o_hs.transpose(1, 2), torch.empty((Bn, H, S), device=DEV)
    dt = B.DTYPE_OF[dtype]
    B.wino_attention(q, k, v, o, lse, workspace=_ws(B.wino_attention_workspace_bytes(Bn, S, S, H, H, D, dt)))
    valid = torch.ones(Bn, S, dtype=torch.bool)
    args = [_d(t) for t in packed.unbind(2)]
    ref, _, bound = O.attention(*args, valid, D ** -0.5, dtype)
    _inside(o, ref, bound, "packed")
    do_hs = do.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
    B.wino_attention_backward(q, k, v, o, lse, do_hs, *grads.unbind(2), workspace=_ws(B.wino_attention_backward_workspace_bytes(Bn, S, S, H, H, D, dt)))
    for g, (r, e) in zip(grads.unbind(2), O.attention_backward(*args, valid, D ** -0.5, _d(do), dtype)):
        _inside(g, r, e, "packed gradients")


def test_attention_broadcast_keys():
    """One prompt for the whole batch: a batch stride of zero."""
    q, k, v, _ = (t.to(DEV) for t in _heads(3, 33, 77, 2, 2, 40, F16))
    k, v = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    assert torch.equal(B.attention(q, k, v), B.attention(q, k.contiguous(), v.contiguous()))


def test_offsets_behind_32_bits():
    step, n = 1 << 23, 300                               # 300 rows 16 MB apart: 5 GB
    buf = torch.empty((n, step), dtype=BF16, device=DEV)
    k, v = buf[:, :64], buf[:, 64:128]
    k.copy_(_rand((n, 64), BF16, 1).to(DEV))
    v.copy_(_rand((n, 64), BF16, 2).to(DEV))
    q = _rand((1, 5, 1, 64), BF16, 3).to(DEV)
    wide = B.attention(q, k.view(1, n, 1, 64), v.view(1, n, 1, 64))
    assert torch.equal(wide, B.attention(q, k.contiguous().view(1, n, 1, 64), v.contiguous().view(1, n, 1, 64)))
    w, b = _rand((40, 64), BF16, 4).to(DEV), _rand((40,), F32, 5).to(DEV)
    assert torch.equal(B.linear(k, w, b), B.linear(k.contiguous(), w, b))
    y = torch.empty((n, 40), dtype=BF16, device=DEV)
    big = torch.empty((n, step), dtype=BF16, device=DEV)[:, 128:168]
    B.wino_linear(k, w, b, big, workspace=_ws(B.wino_linear_workspace_bytes(n, 40, 64, B.WINO_BF16)))
    B.wino_linear(k, w, b, y, workspace=_ws(B.wino_linear_workspace_bytes(n, 40, 64, B.WINO_BF16)))
    assert torch.equal(big, y)


# ---- together, as a block uses them -------------------------------------------------------------------------------------------------------
def _block(x, ctx, p, save=None):
    """Attention to ctx with its projections and the skip connection, then the gated feed-forward with its own."""
    Bn, S, C = x.shape
    H = 4
    q = B.linear(x, p["q"]).view(Bn, S, H, C // H)
    kv = B.linear(ctx, p["kv"]).view(Bn, ctx.shape[1], 2, H, C // H)
    o, lse = B.attention(q, kv[:, :, 0], kv[:, :, 1], with_lse=True)
    x1 = B.linear(o.view(Bn, S, C), p["o"], p["ob"], residual=x)
    h = B.glu(x1, p["up"], p["upb"])
    y = B.linear(h, p["down"], p["downb"], residual=x1)
    if save is not None:
        save.update(q=q, kv=kv, o=o, lse=lse, x1=x1, h=h)
    return y


def _block_backward(x, ctx, p, s, dy):
    Bn, S, C = x.shape
    g = {}
    dh, g["down"], g["downb"] = B.linear_backward(s["h"], p["down"], p["downb"], dy)
    dx1, g["up"], g["upb"] = B.glu_backward(s["x1"], p["up"], p["upb"], dh)
    dx1 = dx1 + dy
    do, g["o"], g["ob"] = B.linear_backward(s["o"].view(Bn, S, C), p["o"], p["ob"], dx1)
    dkv = torch.empty_like(s["kv"])
    dq = torch.empty_like(s["q"])
    k, v = s["kv"][:, :, 0], s["kv"][:, :, 1]
    ws = torch.empty(B.wino_attention_backward_workspace_bytes(Bn, S, ctx.shape[1], 4, 4, C // 4, B.DTYPE_OF[x.dtype]), dtype=torch.uint8, device=DEV)
    B.wino_attention_backward(s["q"], k, v, s["o"], s["lse"], do.view(s["o"].shape), dq, dkv[:, :, 0], dkv[:, :, 1], workspace=ws)
    dxq, g["q"], _ = B.linear_backward(x, p["q"], None, dq.view(Bn, S, C))
    dctx, g["kv"], _ = B.linear_backward(ctx, p["kv"], None, dkv.view(Bn, -1, 2 * C))
    return dx1 + dxq, dctx, g


def _block_inputs(dtype):
    Bn, S, L, C = 2, 90, 21, 160
    w = lambda n, k, seed: _rand((n, k), dtype, seed, k ** -0.5).to(DEV)
    b = lambda n, seed: _rand((n,), F32, seed, 0.1).to(DEV)
    p = dict(q=w(C, C, 1), kv=w(2 * C, 72, 2), o=w(C, C, 3), ob=b(C, 4), up=w(8 * C, C, 5), upb=b(8 * C, 6), down=w(C, 4 * C, 7), downb=b(C, 8))
    return _rand((Bn, S, C), dtype, 9).to(DEV), _rand((Bn, L, 72), dtype, 10).to(DEV), p, _rand((Bn, S, C), dtype, 11).to(DEV)


def _block_reference(x, ctx, p, dy):
    leaves = {n: t.cpu().double().requires_grad_() for n, t in dict(p, x=x, ctx=ctx).items()}
    L = leaves
    Bn, S, C = x.shape
    q = (L["x"] @ L["q"].T).view(Bn, S, 4, C // 4).transpose(1, 2)
    k, v = ((L["ctx"] @ L["kv"].T).view(Bn, -1, 2, 4, C // 4)[:, :, i].transpose(1, 2) for i in (0, 1))
    o = torch.softmax(q @ k.transpose(2, 3) * (C // 4) ** -0.5, 3) @ v
    x1 = o.transpose(1, 2).reshape(Bn, S, C) @ L["o"].T + L["ob"] + L["x"]
    z = x1 @ L["up"].T + L["upb"]
    h = z[..., :4 * C] * torch.nn.functional.gelu(z[..., 4 * C:])
    y = h @ L["down"].T + L["downb"] + x1
    y.backward(dy.cpu().double())
    return y.detach(), {n: t.grad for n, t in leaves.items()}


@pytest.mark.parametrize("dtype", TYPES)
def test_block_forward_and_backward(dtype):
    """A chain of up to six roundings a path, each at most one unit of a tensor that the next product averages: ten units of the result's norm."""
    x, ctx, p, dy = _block_inputs(dtype)
    save = {}
    y = _block(x, ctx, p, save)
    dx, dctx, g = _block_backward(x, ctx, p, save, dy)
    ref, grads = _block_reference(x, ctx, p, dy)
    unit = max(O.UNIT[dtype], 1e-6)                      # fp32: sums of up to 1280 terms
    for name, got, want in [("y", y, ref), ("x", dx, grads["x"]), ("ctx", dctx, grads["ctx"])] + [(n, g[n], grads[n]) for n in g]:
        if got is None:
            continue
        err = ((got.cpu().double() - want).norm() / want.norm()).item()
        assert err <= 10 * unit, (name, err)


def test_block_on_another_stream_and_captured():
    x, ctx, p, dy = _block_inputs(BF16)
    save = {}
    eager = [_block(x, ctx, p, save)]
    a, b, g = _block_backward(x, ctx, p, save, dy)
    eager += [a, b] + [g[n] for n in sorted(g) if g[n] is not None]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            s2 = {}
            _block(x, ctx, p, s2)
            _block_backward(x, ctx, p, s2, dy)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s3 = {}
            out = [_block(x, ctx, p, s3)]
            a, b, g = _block_backward(x, ctx, p, s3, dy)
            out += [a, b] + [g[n] for n in sorted(g) if g[n] is not None]
    for n in range(3):
        for t in out:
            t.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(eager, out)), n
        _block(x, ctx, p)                                # the program's own work between replays
    x.copy_(_rand(tuple(x.shape), BF16, 77).to(DEV))     # new values, same graph
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], _block(x, ctx, p))


def test_long_sizes_against_float32_products():
    """Sizes of a real block (many tiles in every direction): against fp32 products of the same operands, whose own error is far below."""
    for dtype in (F16, BF16):
        M, K, N = 8192, 320, 1280
        x, w, b, _, dh = (t.to(DEV) for t in _products(M, K, N, dtype, 2))
        z = x.float() @ w.float().T + b
        u, g = z[:, :N], z[:, N:]
        a, c = torch.nn.functional.gelu(g), torch.special.ndtr(g)
        h = u * a
        got = B.glu(x, w, b)
        assert ((got.float() - h).abs() <= 1.01 * O.UNIT[dtype] * h.abs() + 2e-5 * (1 + u.abs() + g.abs())).all()
        dx, dw, db = B.glu_backward(x, w, b, dh)
        dz = torch.cat([dh.float() * a, dh.float() * u * (c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi))], 1)
        for v, ref in ((dx, dz @ w.float()), (dw, dz.T @ x.float())):
            assert ((v.float() - ref).norm() / ref.norm()).item() <= 2 * O.UNIT[dtype]
        assert ((db - dz.sum(0)).norm() / db.norm()).item() <= 1e-5
        y = B.linear(got, w[:K, :].T.contiguous().view(K, K).repeat(1, 4).contiguous(), None, residual=x)
        assert torch.isfinite(y).all()


@pytest.mark.parametrize("dtype,H,Hkv,D", [(t, H, Hkv, D) for t in TYPES
                                           for H, Hkv, D in [(64, 64, 40), (64, 64, 64), (64, 64, 72), (40, 40, 128), (40, 20, 128), (40, 40, 152), (40, 40, 200)]
                                           if t != F32 or D <= 160])
def test_attention_of_many_heads(dtype, H, Hkv, D):
    """Enough rows and keys that the backward pass's workgroups own 128 of them."""
    mask = torch.rand((2, 258), generator=torch.Generator().manual_seed(D)) < 0.9
    mask[1, 64:130] = False
    _check_attention(2, 260, 258, H, Hkv, D, dtype, lens=[258, 200], mask=mask)
