"""Transformer-block operators in 64 bits, written from their definitions: linear with an activation, the gated product, attention to another
tensor's keys, and their gradients.  Every function also gives, element by element, how far a result may be from these values when sums run in fp32
and what the interface says is rounded to the storage type is rounded there (``unit``: the largest relative error of one such rounding,
``floor``: the largest absolute one where the type's exponent ends).  torch.float64 on the CPU.
"""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
FLOOR = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
F32 = 2.0 ** -24
# The activations in fp32: distribution functions within 3e-7 (GELU's formula 1e-7, exponential and reciprocal one unit each), times |z|;
# the derivative adds |z| c'(z), of the same kind.
ACT_ERROR = 4e-7


def act(z, kind):
    """(act(z), act'(z))"""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "silu":
        c = 1 / (1 + torch.exp(-z))
        return z * c, c + z * c * (1 - c)
    if kind == "gelu":
        c = torch.special.erfc(-z * math.sqrt(0.5)) / 2                  # (small values too are right relative to themselves)
        return z * c, c + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))       # (1 + tanh t) / 2
    return z * c, c + 2 * z * c * (1 - c) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def _rounded(v, dtype):
    return UNIT[dtype] * v.abs() + FLOOR[dtype]


def _pre(x, w, b):
    """z and a bound of its error in fp32: every product and sum one rounding, in any order."""
    n = x.shape[1] + 2
    z = x @ w.T + (0 if b is None else b)
    return z, n * F32 * (x.abs() @ w.abs().T + (0 if b is None else b.abs()))


def linear(x, w, b, r, kind, dtype):
    z, ez = _pre(x, w, b)
    a, _ = act(z, kind)
    y = a if r is None else a + r
    e = 1.13 * ez + ACT_ERROR * (kind != "none") * z.abs() + 2 * F32 * (a.abs() + y.abs())       # |act'| <= 1.13
    return y, e + _rounded(y.abs() + e, dtype)


def _products(x, w, dz, ed, dtype, dx_like=None):
    """dx, dw and column sums from dz known within ed (before its rounding to the storage type, which only the products take)."""
    er = ed + _rounded(dz.abs() + ed, dtype)
    out = []
    for a, ea, m in ((dz, er, w), (dz.T, er.T, x)):
        v, n = a @ m, a.shape[1] + 2
        e = ea @ m.abs() + n * F32 * ((a.abs() + ea) @ m.abs())
        out.append((v, e + _rounded(v.abs() + e, dtype)))
    s = dz.sum(0)
    out.append((s, ed.sum(0) + (dz.shape[0] + 2) * F32 * (dz.abs() + ed).sum(0)))
    return out


def linear_backward(x, w, b, dy, kind, dtype):
    if kind == "none":
        z = dy
        return _products_exact(x, w, dy, dtype)
    z, ez = _pre(x, w, b)
    _, d = act(z, kind)
    dz = dy * d
    return _products(x, w, dz, dy.abs() * (1.0 * ez + 2 * ACT_ERROR * (1 + z.abs())) + 2 * F32 * dz.abs(), dtype)      # |act''| <= 1


def _products_exact(x, w, dz, dtype):
    out = []
    for a, m in ((dz, w), (dz.T, x)):
        v = a @ m
        e = (a.shape[1] + 2) * F32 * (a.abs() @ m.abs())
        out.append((v, e + _rounded(v.abs() + e, dtype)))
    out.append((dz.sum(0), (dz.shape[0] + 2) * F32 * dz.abs().sum(0)))
    return out


def glu(x, w, b, kind, dtype):
    n = w.shape[0] // 2
    z, ez = _pre(x, w, b)
    u, g, eu, eg = z[:, :n], z[:, n:], ez[:, :n], ez[:, n:]
    a, _ = act(g, kind)
    ea = 1.13 * eg + ACT_ERROR * (kind != "none") * g.abs()
    h = u * a
    e = u.abs() * ea + a.abs() * eu + ea * eu + 2 * F32 * h.abs()
    return h, e + _rounded(h.abs() + e, dtype)


def glu_backward(x, w, b, dh, kind, dtype):
    n = w.shape[0] // 2
    z, ez = _pre(x, w, b)
    u, g, eu, eg = z[:, :n], z[:, n:], ez[:, :n], ez[:, n:]
    a, d = act(g, kind)
    approx = ACT_ERROR * (kind != "none")
    ea, ed = 1.13 * eg + approx * g.abs(), 1.0 * eg + 2 * approx * (1 + g.abs())
    du, dg = dh * a, dh * u * d
    e = torch.cat([dh.abs() * ea + 2 * F32 * du.abs(), dh.abs() * (u.abs() * ed + d.abs() * eu + ed * eu) + 3 * F32 * dg.abs()], 1)
    return _products(x, w, torch.cat([du, dg], 1), e, dtype)


# ---- attention: q, o, do [B,Sq,H,D]; k, v [B,Skv,Hkv,D]; valid [B,Skv] -------------------------------------------------------------------
def _weights(q, k, valid, scale, group):
    """p [B,H,Sq,Skv], lse [B,H,Sq], a bound of the relative error of the weights in fp32, and the largest |s| of a row"""
    qh, kh = q.permute(0, 2, 1, 3), k.permute(0, 2, 1, 3).repeat_interleave(group, 1)
    on = valid[:, None, None, :]
    kh = torch.where(valid[:, None, :, None], kh, 0.0)
    s = qh @ kh.transpose(2, 3) * scale
    es = (q.shape[3] + 2) * F32 * scale * (qh.abs() @ kh.abs().transpose(2, 3))
    es = torch.where(on, es + 6 * F32 * s.abs(), 0.0)                   # the scores' own sums, then factor, maximum and exponent
    s = torch.where(on, s, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    e = torch.exp(s - top)
    total = e.sum(3, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p = e / torch.where(total > 0, total, 1.0)
    rel = 2 * es.amax(3, keepdim=True) + 8 * F32 * top.abs() + 16 * F32
    return p, lse, rel, total


def attention(q, k, v, valid, scale, dtype):
    """o, lse and the bound of o's error"""
    group = q.shape[2] // k.shape[2]
    p, lse, rel, total = _weights(q, k, valid, scale, group)
    vh = torch.where(valid[:, None, :, None], v.permute(0, 2, 1, 3).repeat_interleave(group, 1), 0.0)
    o = p @ vh
    n = k.shape[1] + 4
    unit = UNIT[dtype] if dtype != torch.float32 else 0.0               # the weights are operands of a matrix product in the storage type
    # their floor is relative to the largest weight, 1 before the division by a total of at least 1
    e = (p @ vh.abs()) * (rel + unit + n * F32) * 1.01 + FLOOR[dtype] * vh.abs().sum(2, keepdim=True)
    e = e + _rounded(o.abs() + e, dtype)
    return o.permute(0, 2, 1, 3), lse, e.permute(0, 2, 1, 3)


def attention_backward(q, k, v, valid, scale, do, dtype):
    """((dq, bound), (dk, bound), (dv, bound)) where o is the forward pass's result in the storage type"""
    B, Sq, H, D = q.shape
    group = H // k.shape[2]
    p, _, rel, _ = _weights(q, k, valid, scale, group)
    rel = rel + 8 * F32 * (1 + _weights(q, k, valid, scale, group)[1].nan_to_num(0, 0, 0).abs())[..., None]      # lse stored in fp32
    o, _, eo = attention(q, k, v, valid, scale, dtype)
    on = valid[:, None, :, None]
    qh, doh = q.permute(0, 2, 1, 3), do.permute(0, 2, 1, 3)
    kh, vh = (torch.where(on, t.permute(0, 2, 1, 3).repeat_interleave(group, 1), 0.0) for t in (k, v))
    unit = UNIT[dtype] if dtype != torch.float32 else 0.0
    dp = doh @ vh.transpose(2, 3)
    delta = (doh * o.permute(0, 2, 1, 3)).sum(3, keepdim=True)
    ds = p * (dp - delta)
    e_dp = (D + 2) * F32 * (doh.abs() @ vh.abs().transpose(2, 3))
    e_delta = (doh.abs() * (eo.permute(0, 2, 1, 3) + (D + 2) * F32 * o.permute(0, 2, 1, 3).abs())).sum(3, keepdim=True)
    eds = (p * (e_dp + e_delta + 2 * F32 * (dp.abs() + delta.abs())) + ds.abs() * rel) * 1.01
    eds = torch.where(valid[:, None, None, :], eds + unit * (ds.abs() + eds) + FLOOR[dtype], 0.0)
    ep = torch.where(valid[:, None, None, :], p * (rel + unit) * 1.01 + FLOOR[dtype], 0.0)

    def shared(t):                                                       # sum over the query heads of a key head
        return t.reshape(B, k.shape[2], group, t.shape[2], D).sum(2)

    out = []
    for val, err, n in ((scale * ds @ kh, scale * (eds @ kh.abs() + (k.shape[1] + 4) * F32 * (ds.abs() + eds) @ kh.abs()), 1),
                        (shared(scale * ds.transpose(2, 3) @ qh), shared(scale * (eds.transpose(2, 3) @ qh.abs() + (Sq * group + 20) * F32 * (ds.abs() + eds).transpose(2, 3) @ qh.abs())), 1),
                        (shared(p.transpose(2, 3) @ doh), shared(ep.transpose(2, 3) @ doh.abs() + (Sq * group + 20) * F32 * (p + ep).transpose(2, 3) @ doh.abs()), 1)):
        e = err + _rounded(val.abs() + err, dtype)
        out.append((val.permute(0, 2, 1, 3), e.permute(0, 2, 1, 3)))
    return out
