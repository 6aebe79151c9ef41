"""Gradients in fp16 whose size is far from one: the range of the storage type ends at 65504, and below 6e-5 its numbers lose bits.  What is rounded to it on the way
(the gradients of the scores, the softmax weights, the gradients of the pre-activations) may be larger or smaller than the results, which hold
their bound whatever the size of the incoming gradient: where that is multiplied by a power of two, so is everything but the rounding of
results that are subnormal."""
import math

import pytest
import torch

from oracle import block_ops as O
from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16 = torch.float16


def _rand(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).to(F16)


def _two_roundings(got, exact, what):
    """Finite, and the norm of the error that of two independent roundings, the result's and an operand's: sqrt 2 of the result's alone where the mantissas of
    both fill their octaves alike, up to 1.7 where a few large terms do not (then an operand's rounding weighs sqrt 1.9 times the result's)."""
    got = got.detach().cpu().double()
    assert exact.abs().max() < 65504, what
    assert torch.isfinite(got).all(), what
    one = (exact.to(F16).double() - exact).norm()
    ratio = ((got - exact).norm() / one).item()
    assert ratio <= 1.7, (what, ratio)


def _attention_gradients(q, k, v, do, scale):
    dev = [t.to(DEV) for t in (q, k, v, do)]
    o, lse = B.attention(*dev[:3], scale=scale, with_lse=True)
    got = B.attention_backward(*dev[:3], o, lse, dev[3], scale=scale)
    valid = torch.ones(k.shape[:2], dtype=torch.bool)
    want = O.attention_backward(q.double(), k.double(), v.double(), valid, scale, do.double(), F16)
    return [(n, g, w) for n, g, (w, _) in zip(("dq", "dk", "dv"), got, want)]


@pytest.mark.parametrize("D,H,Hkv,Sq,Skv", [(64, 4, 2, 300, 154), (40, 2, 2, 70, 500), (160, 2, 1, 130, 77), (256, 1, 1, 64, 64), (128, 40, 20, 260, 258)])
@pytest.mark.parametrize("power", [-13, 0, 13])
def test_attention_gradients_at_any_size_of_the_incoming_one(D, H, Hkv, Sq, Skv, power):
    q, do = _rand((2, Sq, H, D), 1), _rand((2, Sq, H, D), 4) * 2.0 ** power
    k, v = _rand((2, Skv, Hkv, D), 2), _rand((2, Skv, Hkv, D), 3)
    for n, g, w in _attention_gradients(q, k, v, do, D ** -0.5):
        _two_roundings(g, w, (n, D, power))


@pytest.mark.parametrize("S", [77, 300])
def test_gradients_of_scores_beyond_the_range(S):
    """Scores with few large weights, do near the end of the range: ds passes 65504, the gradients do not."""
    D, scale = 128, 1 / 64
    q, k, v, do = _rand((1, S, 2, D), 1, 4.0), _rand((1, S, 2, D), 2, 4.0), _rand((1, S, 2, D), 3, 2.0), _rand((1, S, 2, D), 4, 8192.0)
    qh, kh, vh, doh = (t.double().transpose(1, 2) for t in (q, k, v, do))
    p = torch.softmax(qh @ kh.transpose(2, 3) * scale, 3)
    dp = doh @ vh.transpose(2, 3)
    assert (p * (dp - (p * dp).sum(3, keepdim=True))).abs().max() > 1.2 * 65504
    for n, g, w in _attention_gradients(q, k, v, do, scale):
        _two_roundings(g, w, (n, S))


def test_small_gradients_among_many_keys():
    """1024 and more keys share a gradient of 1e-4; weights of 1e-5 and below."""
    for Sq, Skv, std in ((1024, 1024, 1e-3), (64, 40000, 1.0), (64, 40000, 1e-3)):
        q, k, v, do = _rand((1, Sq, 1, 64), 1), _rand((1, Skv, 1, 64), 2), _rand((1, Skv, 1, 64), 3), _rand((1, Sq, 1, 64), 4, std)
        for n, g, w in _attention_gradients(q, k, v, do, 0.125):
            _two_roundings(g, w, (n, Sq, Skv, std))


def test_sizes_that_change_along_the_rows_and_keys():
    """Rows of growing and of falling size one after the other: each row of dq, and each sum over the rows, keeps the bound."""
    S, D = 512, 64
    q, k, v = _rand((1, S, 2, D), 1), _rand((1, S, 2, D), 2), _rand((1, S, 2, D), 3)
    up = torch.logspace(-9, 13, S, base=2.0, dtype=torch.float64)
    for size in (up, up.flip(0)):
        do = (_rand((1, S, 2, D), 4).double() * size[None, :, None, None]).to(F16)
        for n, g, w in _attention_gradients(q, k, v, do, 0.125):
            for a, b in ((0, S),) if n != "dq" else ((i, i + 64) for i in range(0, S, 64)):
                _two_roundings(g[:, a:b], w[:, a:b], (n, a))
        big = v.clone()
        big[:, ::7] *= 2.0 ** 11                         # keys whose values, and so the gradients of whose scores, are far larger
        for n, g, w in _attention_gradients(q, k, big, (do.double() * 2.0 ** -11).to(F16), 0.125):
            _two_roundings(g, w, (n, "large values"))


def test_zero_and_infinite_gradients():
    q, k, v, do = _rand((2, 90, 2, 64), 1), _rand((2, 70, 2, 64), 2), _rand((2, 70, 2, 64), 3), _rand((2, 90, 2, 64), 4)
    zero = _attention_gradients(q, k, v, torch.zeros_like(do), 0.125)
    assert all((g == 0).all() for _, g, _ in zero)
    clean = {n: g for n, g, _ in _attention_gradients(q, k, v, do, 0.125)}
    do[1, 3] = math.inf
    bad = {n: g for n, g, _ in _attention_gradients(q, k, v, do, 0.125)}
    assert not torch.isfinite(bad["dq"][1, 3]).any() and not torch.isfinite(bad["dk"][1]).any() and not torch.isfinite(bad["dv"][1]).any()
    bad["dq"][1, 3] = clean["dq"][1, 3]
    assert torch.equal(bad["dq"], clean["dq"]) and all(torch.equal(bad[n][0], clean[n][0]) for n in ("dk", "dv"))


# ---- products ---------------------------------------------------------------------------------------------------------------------------
def _product_inputs(M, K, N, halves, std, some):
    """u and g of unit size, dx and dw of one size; a part `some` of the incoming gradient is not zero, so that sums of a large one stay in range."""
    W = (M / (halves * N * K)) ** 0.25
    x, w, b = _rand((M, K), 1, 1 / (W * K ** 0.5)), _rand((halves * N, K), 2, W), torch.randn(halves * N, generator=torch.Generator().manual_seed(3)) * 0.3
    on = torch.rand((M, N), generator=torch.Generator().manual_seed(5)) < some
    return x, w, b, torch.where(on, _rand((M, N), 4, std), torch.zeros((), dtype=F16))


def _product_gradients(glu, x, w, b, dy, act="gelu"):
    code = {"silu": B.WINO_ACT_SILU, "gelu": B.WINO_ACT_GELU, "gelu_tanh": B.WINO_ACT_GELU_TANH, "none": B.WINO_ACT_NONE}[act]
    got = (B.glu_backward if glu else B.linear_backward)(*(t.to(DEV) for t in (x, w, b, dy)), code)
    want = (O.glu_backward if glu else O.linear_backward)(x.double(), w.double(), b.double(), dy.double(), act, F16)
    return [(n, g, r) for n, g, (r, _) in zip(("dx", "dw", "dbias"), got, want)]


# every kernel that stores or takes the gradients of the pre-activations: blocks of 128 and 64, any alignment, ranges with their join, few rows
@pytest.mark.parametrize("M,K,N", [(16, 256, 128), (40, 77, 33), (300, 200, 136), (700, 640, 200), (90, 1032, 320), (1500, 515, 333), (2100, 328, 640)])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("std", [2.0 ** -18, 2.0 ** -13, 1.0, 2.0 ** 11])
def test_gradients_of_products_at_any_size_of_the_incoming_one(M, K, N, glu, std):
    x, w, b, dy = _product_inputs(M, K, N, 2 if glu else 1, std, 0.1 if std > 1 else 1.0)
    for act in ("gelu", "silu"):
        for n, g, r in _product_gradients(glu, x, w, b, dy, act):
            if n == "dbias":
                assert ((g.cpu().double() - r).norm() / r.norm()).item() < 1e-5, (act, n)
            else:
                _two_roundings(g, r, (act, n))


def test_gradients_of_preactivations_beyond_the_range():
    """du and dg pass 65504, the gradients of x and w do not; one result alone, and from a strided gradient."""
    M, K, N = 700, 2000, 136
    x, w, b, dy = _product_inputs(M, K, N, 2, 2.0 ** 13, 0.1)
    z = x.double() @ w.double().T + b.double()
    u, g = z[:, :N], z[:, N:]
    slope = torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    assert (dy.double() * u * slope).abs().max() > 65504
    (_, dx, rx), (_, dw, rw), _ = _product_gradients(True, x, w, b, dy)
    _two_roundings(dx, rx, "dx")
    _two_roundings(dw, rw, "dw")
    ws = torch.full((B.wino_glu_backward_workspace_bytes(M, N, K, B.WINO_F16, B.WINO_ACT_GELU),), 255, dtype=torch.uint8, device=DEV)
    wide = torch.full((M, N + 8), math.nan, dtype=F16, device=DEV)
    wide[:, :N] = dy.to(DEV)
    for which in (0, 1):
        out = [torch.empty_like(t.to(DEV)) for t in (x, w)]
        B.wino_glu_backward(x.to(DEV), w.to(DEV), b.to(DEV), wide[:, :N], out[0] if which == 0 else None, out[1] if which == 1 else None, None, workspace=ws)
        assert torch.equal(out[which], (dx, dw)[which])


def test_replays_follow_the_size_of_the_gradient():
    """Whether the gradients of the pre-activations are formed again is decided on the GPU: one captured call, gradients of several sizes."""
    M, K, N = 300, 200, 136
    x, w, b, dy = (t.to(DEV) for t in _product_inputs(M, K, N, 2, 1.0, 0.05))
    sizes = [dy, dy * 2.0 ** 12, dy * 2.0 ** -15, torch.zeros_like(dy)]
    want = [B.glu_backward(x, w, b, t) for t in sizes]
    out = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(B.wino_glu_backward_workspace_bytes(M, N, K, B.WINO_F16, B.WINO_ACT_GELU), dtype=torch.uint8, device=DEV)
    given = dy.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        B.wino_glu_backward(x, w, b, given, *out, workspace=ws)
    for n in (0, 1, 2, 1, 3, 0):
        given.copy_(sizes[n])
        for o in out:
            o.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, r) for o, r in zip(out, want[n])), n
        B.glu_backward(x, w, b, dy)
