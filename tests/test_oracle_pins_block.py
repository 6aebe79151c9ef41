"""The 64-bit definitions of the transformer-block operators against torch's own in double precision and against differences."""
import math

import pytest
import torch

from oracle import block_ops as O

D = torch.float64


def _t(*shape, seed=0):
    return torch.randn(shape, dtype=D, generator=torch.Generator().manual_seed(seed))


def _torch_act(z, kind):
    return {"none": lambda t: t, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
            "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[kind](z)


@pytest.mark.parametrize("kind", ["none", "silu", "gelu", "gelu_tanh"])
def test_products_against_autograd(kind):
    x, w, b, r, dy = _t(7, 12), _t(10, 12, seed=1), _t(10, seed=2), _t(7, 10, seed=3), _t(7, 10, seed=4)
    for t in (x, w, b):
        t.requires_grad_()
    y = _torch_act(x @ w.T + b, kind) + r
    y.backward(dy)
    with torch.no_grad():
        assert torch.allclose(O.linear(x, w, b, r, kind, torch.float32)[0], y, rtol=1e-12, atol=1e-12)
        for (v, _), t in zip(O.linear_backward(x, w, b, dy, kind, torch.float32), (x, w, b)):
            assert torch.allclose(v, t.grad, rtol=1e-11, atol=1e-12)
    for t in (x, w, b):
        t.grad = None
    z = x @ w.T + b
    h = z[:, :5] * _torch_act(z[:, 5:], kind)
    h.backward(dy[:, :5])
    with torch.no_grad():
        assert torch.allclose(O.glu(x, w, b, kind, torch.float32)[0], h, rtol=1e-12, atol=1e-12)
        for (v, _), t in zip(O.glu_backward(x, w, b, dy[:, :5], kind, torch.float32), (x, w, b)):
            assert torch.allclose(v, t.grad, rtol=1e-11, atol=1e-12)


def _case():
    q, k, v, do = _t(3, 5, 4, 8), _t(3, 6, 2, 8, seed=1), _t(3, 6, 2, 8, seed=2), _t(3, 5, 4, 8, seed=3)
    valid = torch.tensor([[1, 1, 0, 1, 0, 1], [0] * 6, [1] * 6], dtype=torch.bool)
    return q, k, v, do, valid


def test_attention_against_autograd():
    q, k, v, do, valid = _case()
    for t in (q, k, v):
        t.requires_grad_()
    bias = torch.where(valid, 0.0, -math.inf).to(D)[:, None, None, :]
    rows = [0, 2]                                        # the row without a valid key is a definition of its own
    kk, vv = (t.permute(0, 2, 1, 3).repeat_interleave(2, 1)[rows] for t in (k, v))
    s = q.permute(0, 2, 1, 3)[rows] @ kk.transpose(2, 3) * 0.3 + bias[rows]
    o = torch.softmax(s, 3) @ vv
    o.backward(do.permute(0, 2, 1, 3)[rows])
    with torch.no_grad():
        got, lse, _ = O.attention(q, k, v, valid, 0.3, torch.float32)
        assert torch.allclose(got[rows], o.permute(0, 2, 1, 3), rtol=1e-12, atol=1e-12)
        assert torch.allclose(lse[rows], torch.logsumexp(s, 3), rtol=1e-12, atol=1e-12)
        assert (got[1] == 0).all() and torch.isneginf(lse[1]).all()
        for (g, _), t in zip(O.attention_backward(q, k, v, valid, 0.3, do, torch.float32), (q, k, v)):
            assert torch.allclose(g, t.grad, rtol=1e-11, atol=1e-12)


def test_attention_against_differences():
    q, k, v, do, valid = _case()
    grads = O.attention_backward(q, k, v, valid, 0.3, do, torch.float32)
    f = lambda: (O.attention(q, k, v, valid, 0.3, torch.float32)[0] * do).sum().item()
    h = 1e-5
    for t, (g, _) in zip((q, k, v), grads):
        flat = t.view(-1)
        for i in range(0, flat.numel(), 37):
            keep = flat[i].item()
            flat[i] = keep + h
            up = f()
            flat[i] = keep - h
            slope = (up - f()) / (2 * h)
            flat[i] = keep
            assert abs(slope - g.reshape(-1)[i].item()) < 1e-7


def test_bounds_hold_for_rounded_arithmetic_and_break_for_a_wrong_element():
    """One rounding to the storage type of the exact values stays inside, an element that takes its neighbour's value does not."""
    q, k, v, do, valid = _case()
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        o, _, e = O.attention(q, k, v, valid, 0.3, dtype)
        assert ((o.to(dtype).double() - o).abs() <= e).all()
        wrong = o.clone()
        wrong[0, 0, 0, 0] = o[0, 0, 0, 1]
        assert not ((wrong - o).abs() <= e).all()
        x, w, b = _t(7, 12), _t(10, 12, seed=1), _t(10, seed=2)
        y, e = O.linear(x, w, b, None, "gelu", dtype)
        assert ((y.to(dtype).double() - y).abs() <= e).all()
        wrong = y.clone()
        wrong[3, 4] = y[3, 5]
        assert not ((wrong - y).abs() <= e).all()
