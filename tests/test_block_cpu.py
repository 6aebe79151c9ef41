"""Host-side checks of the transformer-block calls that need no GPU: every refusal happens before a launch, and the sizes they ask for."""
import ctypes
import os

import pytest

from paper_2412_05781_amd import binding as B

vp = ctypes.c_void_p
X, W, Y, R, BIAS, DX, DW, DB, WS = (0x10000000 * i for i in range(1, 10))
BIG = 1 << 30


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2412_05781_amd.build import build_libwino
        build_libwino()
    return B.lib()


def _linear(L, x=X, w=W, b=BIAS, r=None, y=Y, M=4, N=8, K=16, ldx=None, ldr=None, ldy=None, dt=B.WINO_F16, act=0, ws=WS, n=BIG):
    return L.wino_linear(x, w, b, r, y, M, N, K, K if ldx is None else ldx, N if ldr is None else ldr, N if ldy is None else ldy, dt, act, ws, n, None)


def test_linear_refusals(L):
    for name in ("x", "w", "y"):
        assert _linear(L, **{name: None}) == B.WINO_ERR_NULL
    assert _linear(L, dt=3) == B.WINO_ERR_DTYPE and _linear(L, dt=-1) == B.WINO_ERR_DTYPE
    assert _linear(L, act=4) == B.WINO_ERR_VARIANT and _linear(L, act=-1) == B.WINO_ERR_VARIANT
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(M=-1), dict(ldx=15), dict(ldy=7), dict(r=R, ldr=7), dict(M=1 << 30, N=1 << 20), dict(K=1 << 29), dict(ldx=1 << 40)):
        assert _linear(L, **bad) == B.WINO_ERR_DIM, bad
    for bad in (dict(x=X + 8), dict(w=W + 2), dict(y=Y + 4), dict(r=R + 8), dict(b=BIAS + 2)):
        assert _linear(L, **bad) == B.WINO_ERR_ALIGN, bad
    for bad in (dict(y=X), dict(y=W), dict(y=X + 16), dict(y=BIAS), dict(r=Y + 16), dict(r=Y, ldr=16), dict(r=Y, ldy=16)):
        assert _linear(L, **bad) == B.WINO_ERR_ALIAS, bad
    need = B.wino_linear_workspace_bytes(80, 64, 4096, B.WINO_F16)
    assert need > 0
    assert _linear(L, M=80, N=64, K=4096, n=need - 1) == B.WINO_ERR_WORKSPACE
    assert _linear(L, M=80, N=64, K=4096, ws=None) == B.WINO_ERR_WORKSPACE
    assert _linear(L, M=80, N=64, K=4096, ws=WS + 8) == B.WINO_ERR_ALIGN


def _backward(L, which, x=X, w=W, b=BIAS, dy=Y, dx=DX, dw=DW, db=DB, M=4, N=8, K=16, ldx=None, lddy=None, lddx=None, dt=B.WINO_F16, act=2, ws=WS, n=BIG):
    return getattr(L, which)(x, w, b, dy, dx, dw, db, M, N, K, K if ldx is None else ldx, N if lddy is None else lddy, K if lddx is None else lddx, dt, act, ws, n, None)


@pytest.mark.parametrize("which", ["wino_linear_backward", "wino_glu_backward"])
def test_product_backward_refusals(L, which):
    for bad in (dict(x=None), dict(w=None), dict(dy=None), dict(dx=None, dw=None, db=None)):
        assert _backward(L, which, **bad) == B.WINO_ERR_NULL, bad
    assert _backward(L, which, dt=9) == B.WINO_ERR_DTYPE
    assert _backward(L, which, act=7) == B.WINO_ERR_VARIANT
    for bad in (dict(M=0), dict(N=-3), dict(K=0), dict(ldx=1), dict(lddy=1), dict(lddx=1), dict(N=1 << 28)):
        assert _backward(L, which, **bad) == B.WINO_ERR_DIM, bad
    for bad in (dict(x=X + 2), dict(w=W + 2), dict(dy=Y + 2), dict(dx=DX + 2), dict(dw=DW + 2), dict(db=DB + 2), dict(b=BIAS + 1), dict(ws=WS + 4)):
        assert _backward(L, which, **bad) == B.WINO_ERR_ALIGN, bad
    for bad in (dict(dx=X), dict(dw=W), dict(dx=Y), dict(db=BIAS), dict(dx=DW), dict(dw=DX + 16), dict(dw=DB)):
        assert _backward(L, which, **bad) == B.WINO_ERR_ALIAS, bad
    assert _backward(L, which, ws=None) == B.WINO_ERR_WORKSPACE and _backward(L, which, n=15) == B.WINO_ERR_WORKSPACE


def test_glu_refusals(L):
    call = lambda x=X, w=W, b=BIAS, h=Y, M=4, N=8, K=16, ldx=16, ldh=8, dt=B.WINO_F16, act=2: L.wino_glu(x, w, b, h, M, N, K, ldx, ldh, dt, act, None, 0, None)
    for bad in (dict(x=None), dict(w=None), dict(h=None)):
        assert call(**bad) == B.WINO_ERR_NULL
    assert call(dt=3) == B.WINO_ERR_DTYPE and call(act=4) == B.WINO_ERR_VARIANT
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(ldx=8), dict(ldh=4)):
        assert call(**bad) == B.WINO_ERR_DIM
    assert call(x=X + 8) == B.WINO_ERR_ALIGN and call(b=BIAS + 2) == B.WINO_ERR_ALIGN
    for bad in (dict(h=X), dict(h=W + 16 * 16 * 2 - 16), dict(h=BIAS)):                # the gate half of w counts too
        assert call(**bad) == B.WINO_ERR_ALIAS, bad


NAMES = ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")


def _args(backward=False, **kw):
    a = B.wino_attention_args(kw.get("B", 2), kw.get("Sq", 3), kw.get("Skv", 5), kw.get("H", 4), kw.get("Hkv", 2), kw.get("D", 16), kw.get("dt", B.WINO_F16),
                              kw.get("scale", 0.25))
    for i, n in enumerate(NAMES):
        heads, s = (a.Hkv, a.Skv) if n in ("k", "v", "dk", "dv") else (a.H, a.Sq)
        t = getattr(a, n)
        t.data, t.stride_b, t.stride_s, t.stride_h = 0x10000000 * (i + 1), max(1, s) * heads * a.D, heads * a.D, a.D
        for field, v in kw.get(n, {}).items():
            setattr(t, field, v)
    a.lse = kw.get("lse", 0xa0000000)
    a.kv_len, a.key_mask = kw.get("kv_len"), kw.get("key_mask")
    return ctypes.byref(a)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_refusals(L, backward):
    call = lambda ws=WS * 2, n=BIG, **kw: (L.wino_attention_backward if backward else L.wino_attention)(_args(**kw), ws, n, None)
    fn = L.wino_attention_backward if backward else L.wino_attention
    assert fn(None, WS, BIG, None) == B.WINO_ERR_NULL
    used = NAMES if backward else NAMES[:4]
    outs = ("dq", "dk", "dv") if backward else ("o",)
    for n in used:
        assert call(**{n: dict(data=None)}) == B.WINO_ERR_NULL, n
        assert call(**{n: dict(data=0xb0000008)}) == B.WINO_ERR_ALIGN, n
        for st in ("stride_b", "stride_s", "stride_h"):
            assert call(**{n: {st: -16}}) == B.WINO_ERR_DIM, (n, st)
            assert call(**{n: {st: 1 << 40}}) == B.WINO_ERR_DIM, (n, st)
            assert call(**{n: {st: 20}}) == B.WINO_ERR_ALIGN, (n, st)
            if n in outs:
                assert call(**{n: {st: 0}}) == B.WINO_ERR_DIM, (n, st)
    assert call(dt=3) == B.WINO_ERR_DTYPE
    for bad in (dict(B=0), dict(Sq=0), dict(Skv=0), dict(H=0), dict(Hkv=0), dict(H=3), dict(D=0), dict(D=12), dict(D=264), dict(D=168, dt=B.WINO_F32),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(Sq=1 << 29)):
        assert call(**bad) == B.WINO_ERR_DIM, bad
    first = 0x10000000
    for n in outs:
        assert call(**{n: dict(data=first)}) == B.WINO_ERR_ALIAS, n                     # q
        assert call(lse=0x10000000 * (NAMES.index(n) + 1)) == B.WINO_ERR_ALIAS, n
    if backward:
        assert call(lse=None) == B.WINO_ERR_NULL
        assert call(dk=dict(data=first * 8)) == B.WINO_ERR_ALIAS                        # dv
        assert call(n=16) == B.WINO_ERR_WORKSPACE and call(ws=None) == B.WINO_ERR_WORKSPACE and call(ws=WS + 8) == B.WINO_ERR_ALIGN
    else:
        long = dict(B=1, Sq=1, Skv=9000, H=1, Hkv=1, D=64)
        need = B.wino_attention_workspace_bytes(1, 1, 9000, 1, 1, 64, B.WINO_F16)
        assert need > 0 and call(n=need - 1, **long) == B.WINO_ERR_WORKSPACE and call(ws=None, **long) == B.WINO_ERR_WORKSPACE
    assert call(lse=0xa0000002) == B.WINO_ERR_ALIGN and call(kv_len=0xa1000002) == B.WINO_ERR_ALIGN


def test_packed_arguments_are_the_struct():
    assert B._ATTENTION_ARGS.size == ctypes.sizeof(B.wino_attention_args)
    import torch
    q, k = torch.zeros(2, 3, 4, 16), torch.zeros(2, 5, 2, 16)
    lse, lens, mask = torch.zeros(2, 4, 3), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 5, dtype=torch.uint8)
    a = B.wino_attention_args.from_buffer_copy(B._attention(q, k, k, q, lse, lens, mask, 0.5, (q, q, k, k)))
    assert (a.B, a.Sq, a.Skv, a.H, a.Hkv, a.D, a.dtype, a.scale) == (2, 3, 5, 4, 2, 16, B.WINO_F32, 0.5)
    assert (a.lse, a.kv_len, a.key_mask) == (lse.data_ptr(), lens.data_ptr(), mask.data_ptr())
    for name in NAMES:
        t, want = getattr(a, name), k if name in ("k", "v", "dk", "dv") else q
        assert (t.data, t.stride_b, t.stride_s, t.stride_h) == (want.data_ptr(), *want.stride()[:3]), name


def test_sizes_of_bad_arguments_are_zero(L):
    assert B.wino_linear_backward_workspace_bytes(0, 8, 8, B.WINO_F16) == 0
    assert B.wino_linear_backward_workspace_bytes(8, 8, 8, 5) == 0
    assert B.wino_glu_backward_workspace_bytes(8, 8, 8, B.WINO_F16, 9) == 0
    assert B.wino_attention_backward_workspace_bytes(1, 1, 1, 1, 1, 12, B.WINO_F16) == 0
    assert B.wino_attention_workspace_bytes(1, 1, 9000, 3, 2, 64, B.WINO_F16) == 0
    assert B.wino_glu_backward_workspace_bytes(8, 8, 8, B.WINO_F16, B.WINO_ACT_GELU) >= 8 * 16 * 2


def test_binding_refuses_shapes_and_types():
    import torch
    x, w = torch.zeros(4, 16), torch.zeros(8, 16)
    for bad in (lambda: B.wino_linear(x, w, None, torch.zeros(4, 9)), lambda: B.wino_linear(x, w.half(), None, torch.zeros(4, 8)),
                lambda: B.wino_linear(x, torch.zeros(8, 15), None, torch.zeros(4, 8)), lambda: B.wino_linear(x, w, torch.zeros(8).half(), torch.zeros(4, 8)),
                lambda: B.wino_linear(x, w, torch.zeros(7), torch.zeros(4, 8)), lambda: B.wino_linear(x.t().contiguous().t(), w, None, torch.zeros(4, 8)),
                lambda: B.wino_linear(x, w, None, torch.zeros(4, 8)),                    # not on a GPU
                lambda: B.wino_glu(x, torch.zeros(7, 16), None, torch.zeros(4, 3)), lambda: B.wino_glu(x, w, None, torch.zeros(4, 8)),
                lambda: B.wino_linear_backward(x, w, None, torch.zeros(4, 8), None, torch.zeros(8, 15), None)):
        with pytest.raises(ValueError):
            bad()
    q, k = torch.zeros(2, 3, 4, 16), torch.zeros(2, 5, 2, 16)
    o = torch.zeros_like(q)
    for bad in (lambda: B.wino_attention(q, k, k[:, :4], o), lambda: B.wino_attention(q, k, k.half(), o), lambda: B.wino_attention(q, k[..., :8], k, o),
                lambda: B.wino_attention(q, k, k, o, lse=torch.zeros(2, 3, 4)), lambda: B.wino_attention(q, k, k, o, kv_len=torch.zeros(2)),
                lambda: B.wino_attention(q, k, k, o, key_mask=torch.zeros(2, 5)), lambda: B.wino_attention(q, k, k, o, key_mask=torch.zeros(2, 4, dtype=torch.bool)),
                lambda: B.wino_attention(q.transpose(2, 3).contiguous().transpose(2, 3), k, k, o), lambda: B.wino_attention(q, k, k, o)):
        with pytest.raises(ValueError):
            bad()


def test_outputs_whose_positions_meet_are_refused(L):
    """Strides that lead two positions of an output to one place, or two gradients of a packed buffer."""
    fwd = lambda **kw: L.wino_attention(_args(**kw), WS * 2, BIG, None)
    bwd = lambda **kw: L.wino_attention_backward(_args(**kw), WS * 2, 16, None)         # (accepted calls end at the workspace: nothing is launched)
    long = dict(B=2, Sq=1, Skv=9000, H=4, Hkv=2, D=64)
    assert fwd(o=dict(stride_h=8)) == B.WINO_ERR_DIM                                    # heads of 16 channels, 8 apart
    assert fwd(o=dict(stride_s=32)) == B.WINO_ERR_DIM and fwd(o=dict(stride_b=64)) == B.WINO_ERR_DIM
    assert fwd(q=dict(stride_h=8), o=dict(stride_h=8)) == B.WINO_ERR_DIM
    assert L.wino_attention(_args(q=dict(stride_h=8), **long), WS * 2, 16, None) == B.WINO_ERR_WORKSPACE       # inputs may
    for n in ("dq", "dk", "dv"):
        assert bwd(**{n: dict(stride_h=8)}) == B.WINO_ERR_DIM, n
    # one buffer [B][S][dq 4 heads | dk 2 | dv 2][16], Sq = Skv = 5
    at, row = 0x60000000, 8 * 16
    place = lambda h, **kw: dict(data=at + h * 32, stride_b=5 * row, stride_s=row, stride_h=16, **kw)
    ok = dict(Sq=5, dq=place(0), dk=place(4), dv=place(6))
    assert bwd(**ok) == B.WINO_ERR_WORKSPACE
    for bad in (dict(dk=place(3)), dict(dv=place(5)), dict(dk=place(6), dv=place(7)), dict(dv=place(7)), dict(dk=place(4 + 8))):
        assert bwd(**{**ok, **bad}) == (B.WINO_ERR_ALIAS if bad != dict(dk=place(12)) else B.WINO_ERR_WORKSPACE), bad
    assert bwd(**{**ok, "dv": dict(data=at + 6 * 32, stride_b=5 * row + 8, stride_s=row, stride_h=16)}) == B.WINO_ERR_ALIAS     # other strides
    # heads outermost: [H][B][S][D] of dq, dk and dv in turn are apart; the same heads are not
    outer = lambda first, H: dict(data=at + first * 2 * 5 * 16 * 2, stride_b=5 * 16, stride_s=16, stride_h=2 * 5 * 16)
    assert bwd(Sq=5, dq=outer(0, 4), dk=outer(4, 2), dv=outer(6, 2)) == B.WINO_ERR_WORKSPACE
    assert bwd(Sq=5, dq=outer(0, 4), dk=outer(3, 2), dv=outer(6, 2)) == B.WINO_ERR_ALIAS


def test_sizes_beyond_one_launch_are_refused(L):
    """A launch has less than 2^32 threads."""
    assert _linear(L, M=1 << 30, N=1, K=8, ldx=8) == B.WINO_ERR_DIM
    assert _linear(L, N=1 << 27, K=1) == B.WINO_ERR_DIM
    assert B.wino_linear_backward_workspace_bytes(8, 1 << 27, 8, B.WINO_F16) == 0
    assert L.wino_attention(_args(B=1 << 24, Sq=1, Skv=1, H=1, Hkv=1, D=8), None, 0, None) == B.WINO_ERR_DIM
    assert B.wino_attention_backward_workspace_bytes(1 << 20, 1 << 10, 1, 1, 1, 8, B.WINO_F16) == 0


def test_conveniences_take_any_strides():
    import torch
    x = torch.zeros(6, 16)
    assert B._flat(x[:, :8]).data_ptr() == x.data_ptr() and B._flat(x.view(2, 3, 16)).stride() == (16, 1)
    for t in (x[:1].expand(6, 16), x.t(), x[:, :1].expand(6, 16), x[:1].expand(2, 3, 16)):
        f = B._flat(t)
        assert f.stride() == (t.shape[-1], 1) and torch.equal(f, t.reshape(-1, t.shape[-1]))
    q = torch.zeros(2, 3, 4, 16)
    assert B._packed(q.transpose(1, 2)).data_ptr() == q.data_ptr()
    for t in (q.transpose(2, 3), q[:, :, :, :1].expand(2, 3, 4, 16), q.flatten()[2:2 + 2 * 3 * 3 * 16].view(2, 3, 3, 16), torch.zeros(2, 3, 4, 18)[..., :16]):
        assert B._packed(t).is_contiguous() and B._packed(t).data_ptr() % 16 == 0 and torch.equal(B._packed(t), t)
