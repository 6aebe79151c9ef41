"""Calls that reach the kernels and branches which the tests by size do not: one query at every head width, the general attention kernel where the one for few
rows does not take a call, and single gradients of a product."""
import math

import pytest
import torch

from oracle import block_ops as O
from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def _rand(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def _attention(q, k, v, valid, what, **kw):
    """o and lse against 64 bits, with NaN and infinity at the keys that are not valid; returns what the GPU gave."""
    dtype, D = q.dtype, q.shape[3]
    ref, rlse, bound = O.attention(q.double(), k.double(), v.double(), valid, D ** -0.5, dtype)
    k, v = k.clone(), v.clone()
    k[~valid], v[~valid] = math.nan, math.inf
    o, lse = B.attention(q.to(DEV), k.to(DEV), v.to(DEV), with_lse=True, **kw)
    got = o.cpu().double()
    assert torch.isfinite(got).all() and ((got - ref).abs() <= bound).all(), (what, ((got - ref).abs() - bound).max().item())
    empty = torch.isneginf(rlse)
    assert (torch.isneginf(lse.cpu()) == empty).all(), what
    s = (q.double().abs().amax() * torch.where(valid[:, :, None, None], k.double(), 0.0).abs().amax() * D ** 0.5).item()
    assert ((lse.cpu().double() - rlse)[~empty].abs() <= (D + 40) * O.F32 * (s + 20)).all(), what
    return o, lse


WIDTHS = [8, 16, 24, 32, 48, 72, 80, 88, 96, 104, 136, 152, 160, 168, 208, 248, 256]


@pytest.mark.parametrize("dtype,D", [(t, D) for t in (F16, BF16, F32) for D in WIDTHS if t != F32 or D <= 160])
@pytest.mark.parametrize("Skv", [1, 31, 200, 1500])
def test_one_query_at_every_width(dtype, D, Skv):
    """At most 32 rows a key head; 1500 keys are cut into ranges that are joined.  fp32 above 128 channels goes to the general kernel with the same ranges."""
    if Skv == 1500:
        assert B.wino_attention_workspace_bytes(3, 1, Skv, 6, 2, D, B.DTYPE_OF[dtype]) > 0
    q, k, v = _rand((3, 1, 6, D), dtype, D, 1.5), _rand((3, Skv, 2, D), dtype, D + 1), _rand((3, Skv, 2, D), dtype, D + 2)
    lens = [Skv, Skv // 2, 0]
    by_length = torch.arange(Skv)[None] < torch.tensor(lens)[:, None]
    _attention(q, k, v, by_length, (D, dtype, Skv, "lengths"), kv_len=torch.tensor(lens, dtype=torch.int32, device=DEV))
    mask = torch.rand((3, Skv), generator=torch.Generator().manual_seed(D)) < 0.6
    mask[1, :Skv // 2] = False
    _attention(q, k, v, mask, (D, dtype, Skv, "mask"), key_mask=mask.to(DEV))
    q = _rand((3, 9, 6, D), dtype, D + 3, 1.5)                     # 27 rows a key head
    _attention(q, k, v, torch.ones(3, Skv, dtype=torch.bool), (D, dtype, Skv, "rows"))


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (F16, 40), (F32, 64)])
def test_one_query_whose_keys_lie_far_apart(dtype, D):
    """Rows of 2^24 elements and more: the general kernel, with up to as many ranges as the one for few rows."""
    n, step = 1100, 1 << 24
    k, v = _rand((n, D), dtype, 1), _rand((n, D), dtype, 2)
    buf = torch.empty(n * step // (2 if dtype == F32 else 1), dtype=dtype, device=DEV)              # 37 GB
    if dtype == F32:
        n = 550
        k, v = k[:n], v[:n]
    far = buf.view(-1, step)
    far[:, :D], far[:, D:2 * D] = k.to(DEV), v.to(DEV)
    q = _rand((1, 2, 3, D), dtype, 3, 1.5)
    fk, fv = far[:, :D].unflatten(1, (1, D))[None], far[:, D:2 * D].unflatten(1, (1, D))[None]
    assert fk.stride(1) == step
    near = k[None, :, None].to(DEV), v[None, :, None].to(DEV)
    ref, _, bound = O.attention(q.double(), k.double()[None, :, None], v.double()[None, :, None], torch.ones(1, n, dtype=torch.bool), D ** -0.5, dtype)
    lse = []
    for kk, vv in ((fk, fv), (fk, near[1]), (near[0], fv)):
        o, l = B.attention(q.to(DEV), kk, vv, with_lse=True)
        assert ((o.cpu().double() - ref).abs() <= bound).all()
        lse.append(l)
    assert all((l - lse[0]).abs().max() < 1e-4 for l in lse)


def _space(n):
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", [(1, 8, 8), (5, 77, 33), (300, 200, 136), (1500, 64, 72), (20000, 40, 24), (20000, 33, 17), (90, 2048, 320), (320, 90, 2048)])
@pytest.mark.parametrize("glu", [False, True])
def test_each_gradient_alone(M, K, N, dtype, glu):
    """Every set of the three gradients gives what the call for all of them gives, and writes nothing else."""
    halves = 2 if glu else 1
    x, w, b = (t.to(DEV) for t in (_rand((M, K), dtype, 1), _rand((halves * N, K), dtype, 2, K ** -0.5), _rand((halves * N,), F32, 3)))
    dy = _rand((M, N), dtype, 4).to(DEV)
    call, size, acts = ((B.wino_glu_backward, B.wino_glu_backward_workspace_bytes, [B.WINO_ACT_GELU, B.WINO_ACT_NONE]) if glu else
                        (B.wino_linear_backward, B.wino_linear_backward_workspace_bytes, [B.WINO_ACT_NONE, B.WINO_ACT_SILU]))
    for act in acts:
        n = size(M, N, K, B.DTYPE_OF[dtype], act)
        whole = [torch.empty_like(t) for t in (x, w, b)]
        call(x, w, b, dy, *whole, act, workspace=_space(n))
        if act == B.WINO_ACT_NONE and not glu:
            s = dy.double().sum(0)
            assert ((whole[2].double() - s).abs() <= (M + 2) * O.F32 * dy.double().abs().sum(0)).all()
        # (alone or in pairs a product may take other blocks: another order of its fp32 sums, n 2^-24 of the magnitudes for either, and a rounding each)
        z = x.float() @ w.float().T + b
        dz = dy.float().abs() * 1.13 if not glu else torch.cat([dy.float().abs() * z[:, N:].abs(), 1.13 * dy.float().abs() * z[:, :N].abs()], 1)
        sums = [2 * (halves * N + 2) * O.F32 * (dz @ w.float().abs()), 2 * (M + 2) * O.F32 * (dz.T @ x.float().abs()), 2 * (M + 2) * O.F32 * dz.sum(0)]
        for keep in ((0,), (1,), (2,), (0, 2), (1, 2), (0, 1)):
            some = [torch.full_like(t, math.nan) if i in keep else None for i, t in enumerate((x, w, b))]
            call(x, w, b, dy, *some, act, workspace=_space(n))
            for i in keep:
                bound = sums[i] + (2 * (O.UNIT[dtype] * whole[i].float().abs() + O.FLOOR[dtype]) if i < 2 else 0)
                over = ((some[i].float() - whole[i].float()).abs() - 1.02 * bound).max().item()
                assert over <= 0, (keep, i, act, over)           # (NaN, what was there before, is not)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M", [1, 9, 16, 17, 40, 64])
@pytest.mark.parametrize("K,N", [(5120, 1280), (5123, 136), (1288, 5120), (2048, 72)])
def test_few_rows_and_long_reductions(M, K, N, dtype):
    """Either side of the rule that leaves few rows to the tiles, with the workspace that the size call asks for and no more."""
    x, w, b, r = _rand((M, K), dtype, 1), _rand((N, K), dtype, 2, K ** -0.5), _rand((N,), F32, 3), _rand((M, N), dtype, 4)
    n = B.wino_linear_workspace_bytes(M, N, K, B.DTYPE_OF[dtype], B.WINO_ACT_SILU)
    out = torch.full((M + 1, N), 7.0, dtype=dtype, device=DEV)
    B.wino_linear(x.to(DEV), w.to(DEV), b.to(DEV), out[:M], B.WINO_ACT_SILU, r.to(DEV), _space(n) if n else None)
    ref, bound = O.linear(x.double(), w.double(), b.double(), r.double(), "silu", dtype)
    assert ((out[:M].cpu().double() - ref).abs() <= bound).all() and (out[M] == 7).all()
    w, b = _rand((2 * N, K), dtype, 5, K ** -0.5), _rand((2 * N,), F32, 6)
    ref, bound = O.glu(x.double(), w.double(), b.double(), "gelu", dtype)
    assert ((B.glu(x.to(DEV), w.to(DEV), b.to(DEV)).cpu().double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", [(3, 64, 40), (64, 5120, 320), (200, 4096, 328), (257, 320, 328), (2100, 328, 640), (300, 75, 131), (3600, 1544, 520)])
def test_residual_in_place(M, K, N, dtype):
    """The output over its own residual, in every kernel that finishes a product: bit for bit what two tensors give."""
    x, w, b, r = (_rand(s, t, i, f).to(DEV) for s, t, i, f in (((M, K), dtype, 1, 1.0), ((N, K), dtype, 2, K ** -0.5), ((N,), F32, 3, 1.0), ((M, N), dtype, 4, 1.0)))
    n = B.wino_linear_workspace_bytes(M, N, K, B.DTYPE_OF[dtype], B.WINO_ACT_GELU)
    apart, wide = torch.empty_like(r), torch.full((M, N + 16), 7.0, dtype=dtype, device=DEV)
    B.wino_linear(x, w, b, apart, B.WINO_ACT_GELU, r, _space(n) if n else None)
    wide[:, :N] = r
    B.wino_linear(x, w, b, r, B.WINO_ACT_GELU, r, _space(n) if n else None)
    B.wino_linear(x, w, b, wide[:, :N], B.WINO_ACT_GELU, wide[:, :N], _space(n) if n else None)
    assert torch.equal(r, apart) and torch.equal(wide[:, :N], apart) and (wide[:, N:] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("H,Sq", [(32, 1), (33, 1), (64, 1), (11, 3), (128, 2)])
def test_many_query_heads_of_one_key_head(H, Sq, dtype):
    """Either side of the 32 rows a key head that one wave holds, with ranges of the keys, and their gradients."""
    Bn, Skv, D = 2, 1700, 64
    q, do = _rand((Bn, Sq, H, D), dtype, 1, 1.5), _rand((Bn, Sq, H, D), dtype, 2)
    k, v = _rand((Bn, Skv, 1, D), dtype, 3), _rand((Bn, Skv, 1, D), dtype, 4)
    lens = [Skv, 900]
    valid = torch.arange(Skv)[None] < torch.tensor(lens)[:, None]
    kw = dict(kv_len=torch.tensor(lens, dtype=torch.int32, device=DEV))
    o, lse = _attention(q, k, v, valid, (H, Sq, dtype), **kw)
    got = B.attention_backward(q.to(DEV), k.to(DEV), v.to(DEV), o, lse, do.to(DEV), **kw)
    for name, g, (ref, bound) in zip(("dq", "dk", "dv"), got, O.attention_backward(q.double(), k.double(), v.double(), valid, D ** -0.5, do.double(), dtype)):
        assert ((g.cpu().double() - ref).abs() <= bound).all(), (name, H, Sq)
    assert (got[1][1, 900:] == 0).all() and (got[2][1, 900:] == 0).all()
