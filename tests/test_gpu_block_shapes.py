"""Transformer-block operators at the sizes that reach every block shape of the matrix kernels, long attention, values that must not spread, calls side by
side.  Products are compared with fp32 products of the same operands on the GPU, element by element: both sums are within K + 2 roundings of the exact one,
relative to the sum of the magnitudes, and what is rounded to the storage type adds half a step."""
import math

import pytest
import torch

from oracle import block_ops as O
from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
GELU = B.WINO_ACT_GELU


def _rand(shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, device=DEV, generator=g) * std).to(dtype)


def _product(a, b):
    """a b^T in fp32 and the bound of two fp32 evaluations' distance"""
    a, b = a.float(), b.float()
    return a @ b.t(), 2 * (a.shape[1] + 2) * O.F32 * (a.abs() @ b.abs().t())


def _close(got, ref, bound, dtype, what):
    e = bound + O.UNIT[dtype] * (ref.abs() + bound) + O.FLOOR[dtype]
    over = ((got.float() - ref).abs() - e).max().item()
    assert math.isfinite(over) and over <= 0, (what, over)


# M, K, N: 256x256 blocks; 128x128 with two and with three stages (reduction no whole number of stages); 64x64; ranges that are joined; odd sizes throughout
SHAPES = [(3600, 1544, 4104), (8192, 320, 1280), (2100, 1032, 1280), (700, 640, 200), (200, 4096, 320), (1000, 515, 777), (90, 2048, 1280)]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_linear_and_gradients(M, K, N, dtype):
    x, w, b, dy = _rand((M, K), dtype, 1), _rand((N, K), dtype, 2, K ** -0.5), _rand((N,), F32, 3), _rand((M, N), dtype, 4)
    z, ez = _product(x, w)
    z = z + b
    ez = ez + 4 * O.F32 * (z.abs() + b.abs())
    _close(B.linear(x, w, b, residual=dy), z + dy.float(), ez + 2 * O.F32 * (z.abs() + dy.float().abs()), dtype, "linear")
    dx, dw, db = B.linear_backward(x, w, b, dy)
    _close(dx, *_product(dy, w.t()), dtype, "dx")
    _close(dw, *_product(dy.t(), x.t()), dtype, "dw")
    assert ((db - dy.double().sum(0)).abs() <= (M + 2) * O.F32 * dy.double().abs().sum(0)).all()
    # with an activation: dz, rounded for the products, is the only difference
    dx, dw, db = B.linear_backward(x, w, b, dy, GELU)
    slope = torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    dz = dy.float() * slope
    edz = dy.float().abs() * (ez + 2 * O.ACT_ERROR * (1 + z.abs())) + 4 * O.F32 * dz.abs()
    er = edz + O.UNIT[dtype] * dz.abs() + O.FLOOR[dtype]
    for got, a, e, m, name in ((dx, dz, er, w.t(), "dx"), (dw, dz.t(), er.t(), x.t(), "dw")):
        ref, bound = _product(a, m)
        _close(got, ref, bound + e @ m.float().t().abs(), dtype, "gelu " + name)
    assert ((db.double() - dz.double().sum(0)).abs() <= edz.double().sum(0) + (M + 2) * O.F32 * dz.double().abs().sum(0)).all()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", [(3600, 1544, 2048), (4096, 640, 2560), (2100, 1032, 640), (700, 640, 104), (1000, 515, 333)])
def test_glu_and_gradients(M, K, N, dtype):
    if dtype == F32 and M * K * N > 4e9:
        M //= 2
    x, w, b, dh = _rand((M, K), dtype, 1), _rand((2 * N, K), dtype, 2, K ** -0.5), _rand((2 * N,), F32, 3), _rand((M, N), dtype, 4)
    z, ez = _product(x, w)
    z = z + b
    ez = ez + 4 * O.F32 * (z.abs() + b.abs())
    u, g, eu, eg = z[:, :N], z[:, N:], ez[:, :N], ez[:, N:]
    c = torch.special.ndtr(g)
    a, slope = g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    ea, es = 1.13 * eg + O.ACT_ERROR * g.abs() + 2 * O.F32 * a.abs(), eg + 2 * O.ACT_ERROR * (1 + g.abs())
    _close(B.glu(x, w, b), u * a, u.abs() * ea + a.abs() * eu + eu * ea + 4 * O.F32 * (u * a).abs(), dtype, "h")
    dx, dw, db = B.glu_backward(x, w, b, dh)
    f = dh.float()
    dz = torch.cat([f * a, f * u * slope], 1)
    edz = torch.cat([f.abs() * ea, f.abs() * (u.abs() * es + slope.abs() * eu + eu * es)], 1) + 6 * O.F32 * dz.abs()
    er = edz + O.UNIT[dtype] * dz.abs() + O.FLOOR[dtype]
    for got, p, e, m, name in ((dx, dz, er, w.t(), "dx"), (dw, dz.t(), er.t(), x.t(), "dw")):
        ref, bound = _product(p, m)
        _close(got, ref, bound + e @ m.float().t().abs(), dtype, name)
    assert ((db.double() - dz.double().sum(0)).abs() <= edz.double().sum(0) + (M + 2) * O.F32 * dz.double().abs().sum(0)).all()
    for kw in ((True, False), (False, True)):            # either gradient alone, and neither
        ws = torch.empty(B.wino_glu_backward_workspace_bytes(M, N, K, B.DTYPE_OF[dtype], GELU), dtype=torch.uint8, device=DEV)
        gx, gw = torch.empty_like(x) if kw[0] else None, torch.empty_like(w) if kw[1] else None
        B.wino_glu_backward(x, w, b, dh, gx, gw, None, GELU, ws)
        for got, name in ((gx, "dx"), (gw, "dw")):
            if got is not None:
                p, e, m = (dz, er, w.t()) if name == "dx" else (dz.t(), er.t(), x.t())
                ref, bound = _product(p, m)
                _close(got, ref, bound + e @ m.float().t().abs(), dtype, name + " alone")


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", [(5, 72, 40), (200, 72, 136), (70, 200, 72), (200, 75, 131), (2100, 1032, 1280)])
def test_what_is_not_finite_stays_in_its_row(M, K, N, dtype):
    """A row of infinities and NaN, also behind the end of the reduction where other rows begin, reaches its own results only."""
    x, w, dy = _rand((M, K), dtype, 1), _rand((N, K), dtype, 2), _rand((M, N), dtype, 3)
    clean = B.linear(x, w)
    bad, worse = x.clone(), w.clone()
    bad[1], bad[3, K - 1] = math.nan, math.inf
    y = B.linear(bad, w)
    keep = [i for i in range(M) if i not in (1, 3)]
    assert torch.equal(y[keep], clean[keep]) and not torch.isfinite(y[1]).any()
    worse[2] = math.inf
    y = B.linear(x, worse)
    keep = [i for i in range(N) if i != 2]
    assert torch.equal(y[:, keep], clean[:, keep])
    dx, _, _ = B.linear_backward(x, w, None, dy)
    dybad = dy.clone()
    dybad[1] = math.nan
    gx = B.linear_backward(x, w, None, dybad)[0]
    keep = [i for i in range(M) if i != 1]
    assert torch.equal(gx[keep], dx[keep])
    gw = B.linear_backward(bad, w, None, torch.where(torch.isfinite(bad).all(1, keepdim=True), dy, 0.0))[1]
    assert torch.isnan(gw).all()                         # 0 x NaN is NaN: it may not be hidden either


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("D,S,keys", [(64, 1500, 1300), (40, 700, 2100), (128, 600, 900)])
def test_long_attention(D, S, keys, dtype):
    c = torch.Generator().manual_seed(D)
    q, do = (torch.randn((1, S, 2, D), generator=c).to(dtype) for _ in range(2))
    k, v = (torch.randn((1, keys, 1, D), generator=c).to(dtype) for _ in range(2))
    valid = torch.ones(1, keys, dtype=torch.bool)
    g = [t.to(DEV) for t in (q, k, v, do)]
    o, lse = B.attention(*g[:3], with_lse=True)
    d = [t.double() for t in (q, k, v)]
    ref, rlse, bound = O.attention(*d, valid, D ** -0.5, dtype)
    assert ((o.cpu().double() - ref).abs() <= bound).all()
    assert ((lse.cpu().double() - rlse).abs() <= 1e-4).all()
    for name, got, (r, e) in zip("qkv", B.attention_backward(*g[:3], o, lse, g[3]), O.attention_backward(*d, valid, D ** -0.5, do.double(), dtype)):
        assert ((got.cpu().double() - r).abs() <= e).all(), name


def test_gradients_of_attention_lose_nothing_to_the_rounding_of_o():
    """Two roundings a path (the gradient of the scores, the result): the error's norm is that of two, not of three."""
    for dtype in (F16, BF16):
        c = torch.Generator().manual_seed(3)
        q, do = (torch.randn((2, 300, 4, 64), generator=c).to(dtype) for _ in range(2))
        k, v = (torch.randn((2, 154, 4, 64), generator=c).to(dtype) for _ in range(2))
        g = [t.to(DEV) for t in (q, k, v, do)]
        o, lse = B.attention(*g[:3], with_lse=True)
        want = O.attention_backward(q.double(), k.double(), v.double(), torch.ones(2, 154, dtype=torch.bool), 0.125, do.double(), dtype)
        for name, got, (r, _) in zip("qkv", B.attention_backward(*g[:3], o, lse, g[3]), want):
            one = ((r.to(dtype).double() - r).norm() / r.norm()).item()            # what the result's own rounding makes
            assert ((got.cpu().double() - r).norm() / r.norm()).item() <= 1.5 * one, name


def test_two_streams_side_by_side():
    """Calls that overlap in time with a workspace each."""
    M, K, N = 200, 4096, 320                             # the reduction is cut: both calls use their workspace
    jobs = []
    for i in range(2):
        x, w = _rand((M, K), BF16, 10 + i), _rand((N, K), BF16, 20 + i, K ** -0.5)
        q, kv = _rand((2, 4, 4, 64), BF16, 30 + i), _rand((2, 6000, 2, 64), BF16, 40 + i)
        jobs.append((x, w, q, kv, B.linear(x, w), B.attention(q, kv, kv)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = [[], []]
    need = B.wino_linear_workspace_bytes(M, N, K, B.WINO_BF16), B.wino_attention_workspace_bytes(2, 4, 6000, 4, 2, 64, B.WINO_BF16)
    assert min(need) > 0
    spaces = [[torch.empty(n, dtype=torch.uint8, device=DEV) for n in need] for _ in range(2)]
    results = [(torch.empty((M, N), dtype=BF16, device=DEV), torch.empty_like(jobs[0][2])) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (x, w, q, kv, _, _) in enumerate(jobs):
            B.wino_linear(x, w, None, results[i][0], workspace=spaces[i][0], stream=streams[i])
            B.wino_attention(q, kv, kv, results[i][1], workspace=spaces[i][1], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(results[i][0], jobs[i][4]) and torch.equal(results[i][1], jobs[i][5])


def test_captured_calls_share_no_workspace_and_replay():
    """Two graphs, each with its own workspace, replayed in turn with eager work between them."""
    M, K, N = 200, 4096, 320
    x, w = _rand((M, K), F16, 1), _rand((N, K), F16, 2, K ** -0.5)
    q, kv = _rand((2, 4, 4, 64), F16, 3), _rand((2, 6000, 2, 64), F16, 4)
    want = B.linear(x, w), B.attention(q, kv, kv)
    graphs = []
    for _ in range(2):
        ws = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in
              (B.wino_linear_workspace_bytes(M, N, K, B.WINO_F16), B.wino_attention_workspace_bytes(2, 4, 6000, 4, 2, 64, B.WINO_F16))]
        y, o = torch.empty((M, N), dtype=F16, device=DEV), torch.empty_like(q)
        s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            B.wino_linear(x, w, None, y, workspace=ws[0])
            B.wino_attention(q, kv, kv, o, workspace=ws[1])
        graphs.append((g, y, o, ws))
    for _ in range(3):
        for g, y, o, _ in graphs:
            y.fill_(math.nan)
            o.fill_(math.nan)
            g.replay()
        B.linear(x, w)
        torch.cuda.synchronize()
        for _, y, o, _ in graphs:
            assert torch.equal(y, want[0]) and torch.equal(o, want[1])
