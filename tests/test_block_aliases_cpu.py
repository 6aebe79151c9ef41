"""Buffers of the transformer-block calls that share memory: refused on the host, before anything is launched.  Calls that are accepted as far as this goes end at
a workspace that is a byte short."""
import ctypes
import os

import pytest

from paper_2412_05781_amd import binding as B

SPACE = 0x10000000
Q, K, V, O, DO, DQ, DK, DV, LSE, LENS, MASK, WS = (SPACE * i for i in range(1, 13))
SIZES = dict(B=2, Sq=3, Skv=9000, H=4, Hkv=2, D=16)                # long enough for ranges of the keys: a workspace in both directions


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2412_05781_amd.build import build_libwino
        build_libwino()
    return B.lib()


def _need(backward):
    f = B.wino_attention_backward_workspace_bytes if backward else B.wino_attention_workspace_bytes
    n = f(*SIZES.values(), B.WINO_F16)
    assert n > 0
    return n


def _call(L, backward, ws=WS, n=None, lse=LSE, lens=LENS, mask=MASK, **data):
    a = B.wino_attention_args(*SIZES.values(), B.WINO_F16, 0.25)
    for name, at, heads, s in (("q", Q, 4, 3), ("k", K, 2, 9000), ("v", V, 2, 9000), ("o", O, 4, 3), ("d_o", DO, 4, 3), ("dq", DQ, 4, 3), ("dk", DK, 2, 9000),
                               ("dv", DV, 2, 9000)):
        setattr(a, name, B.wino_tensor(data.get(name, at), s * heads * 16, heads * 16, 16))
    a.lse, a.kv_len, a.key_mask = lse, lens, mask
    return (L.wino_attention_backward if backward else L.wino_attention)(ctypes.byref(a), ws, _need(backward) - 1 if n is None else n, None)


BYTES = dict(q=2 * 3 * 4 * 32, k=2 * 9000 * 2 * 32, v=2 * 9000 * 2 * 32, o=2 * 3 * 4 * 32)
LSE_BYTES = 2 * 4 * 3 * 4


@pytest.mark.parametrize("name,at,size", [("q", Q, BYTES["q"]), ("k", K, BYTES["k"]), ("v", V, BYTES["v"]), ("o", O, BYTES["o"]), ("kv_len", LENS, 8), ("key_mask", MASK, 18000)])
def test_lse_is_an_output_of_the_forward_call(L, name, at, size):
    for lse in (at, at + size - 4, at - LSE_BYTES + 4):
        assert _call(L, False, lse=lse) == B.WINO_ERR_ALIAS, (name, hex(lse))
    for lse in (at + size, at - LSE_BYTES):
        assert _call(L, False, lse=lse) == B.WINO_ERR_WORKSPACE, (name, hex(lse))


def test_lse_is_an_input_of_the_backward_call(L):
    assert _call(L, True) == B.WINO_ERR_WORKSPACE and _call(L, False, lse=None) == B.WINO_ERR_WORKSPACE
    for at in (DQ, DK, DV):
        assert _call(L, True, lse=at) == B.WINO_ERR_ALIAS


@pytest.mark.parametrize("backward", [False, True])
def test_workspace_of_attention_overlaps_nothing(L, backward):
    need = _need(backward)
    tensors = [(Q, BYTES["q"]), (K, BYTES["k"]), (V, BYTES["v"]), (O, BYTES["o"]), (LSE, LSE_BYTES), (LENS, 8), (MASK, 18000)]
    if backward:
        tensors += [(DO, BYTES["q"]), (DQ, BYTES["q"]), (DK, BYTES["k"]), (DV, BYTES["v"])]
    for at, size in tensors:
        for ws in (at, at + (size - 1) // 16 * 16, at - (need - 1) // 16 * 16):
            assert _call(L, backward, ws=ws, n=need) == B.WINO_ERR_ALIAS, (hex(at), hex(ws))
            assert _call(L, backward, ws=ws, n=1 << 40) == B.WINO_ERR_ALIAS, (hex(at), hex(ws))


X, W, BIAS, R, Y, DX, DW, DB = (SPACE * i for i in range(21, 29))
M, N, KK = 80, 64, 4096


def test_workspace_of_products_overlaps_nothing(L):
    need = B.wino_linear_workspace_bytes(M, N, KK, B.WINO_F16)
    assert need > 0
    call = lambda ws: L.wino_linear(X, W, BIAS, R, Y, M, N, KK, KK, N, N, B.WINO_F16, 0, ws, need, None)
    for at, size in ((X, M * KK * 2), (W, N * KK * 2), (BIAS, N * 4), (R, M * N * 2), (Y, M * N * 2)):
        for ws in (at, at + size - 16, at - (need - 1) // 16 * 16):
            assert call(ws) == B.WINO_ERR_ALIAS, (hex(at), hex(ws))


@pytest.mark.parametrize("which,halves", [("wino_linear_backward", 1), ("wino_glu_backward", 2)])
@pytest.mark.parametrize("act", [0, 2])
def test_workspace_of_product_gradients_overlaps_nothing(L, which, halves, act):
    need = getattr(B, which + "_workspace_bytes")(M, N, KK, B.WINO_F16, act)
    call = lambda ws: getattr(L, which)(X, W, BIAS, Y, DX, DW, DB, M, N, KK, KK, N, KK, B.WINO_F16, act, ws, need, None)
    w = halves * N
    for at, size in ((X, M * KK * 2), (W, w * KK * 2), (BIAS, w * 4), (Y, M * N * 2), (DX, M * KK * 2), (DW, w * KK * 2), (DB, w * 4)):
        for ws in (at, at + size - 16, at - (need - 1) // 16 * 16):
            assert call(ws) == B.WINO_ERR_ALIAS, (hex(at), hex(ws))
