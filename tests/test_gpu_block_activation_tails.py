"""Activations and their derivatives where they are small: a value next to nothing is right relative to itself, not only to its largest neighbours.

Bounds, relative to the exact value: half a step of the storage type; two-byte types 1e-4 of the function itself (GELU's formula, 8.3e-5; exponential and reciprocal
2^-23 each); and z^2 2^-22 (fp32: 2^-21), the rounding of an exponent of the size of z^2, which is what one step of z itself does to such a value.  The derivative is a
difference of two such terms, of which the larger is up to 1.5 times the result for z <= -1.5."""
import pytest
import torch

from oracle import block_ops as O
from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACTS = {"silu": B.WINO_ACT_SILU, "gelu": B.WINO_ACT_GELU, "gelu_tanh": B.WINO_ACT_GELU_TANH}


def _tail(kind):
    # (the last exponent of bf16 and fp32 ends at z = -13 for GELU, at -80 for the others; gelu_tanh's is that of z^3)
    return {"silu": (-80, -2.0), "gelu": (-12, -1.5), "gelu_tanh": (-9, -1.5)}[kind]


def _inside(got, want, z, kind, dtype, times, what):
    exponent = z.square() if kind == "gelu" else z.abs() if kind == "silu" else 1.6 * z.abs() * (1 + 0.045 * z.square())
    own = 32 * O.F32 + exponent * 2.0 ** -21 if dtype == torch.float32 else 1e-4 + exponent * 2.0 ** -22
    bound = want.abs() * (O.UNIT[dtype] + times * own) * 1.01 + O.FLOOR[dtype]
    over = ((got.cpu().double() - want).abs() - bound) / want.abs()
    assert over.max() <= 0, (what, over.max().item(), "at z", z.flatten()[int(over.argmax())].item())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", list(ACTS))
@pytest.mark.parametrize("rows", [64, 512])                    # a kernel each
def test_small_values(kind, dtype, rows):
    lo, hi = _tail(kind)
    z = torch.linspace(lo, hi, rows * 8, dtype=torch.float64).view(rows, 8).to(dtype)
    w = torch.eye(8, dtype=dtype, device=DEV)
    a, slope = O.act(z.double(), kind)
    _inside(B.linear(z.to(DEV), w, None, ACTS[kind]), a, z.double(), kind, dtype, 1, "linear")
    dx, _, _ = B.linear_backward(z.to(DEV), w, None, torch.ones_like(z).to(DEV), ACTS[kind])
    _inside(dx, slope, z.double(), kind, dtype, 3, "linear, derivative")
    # gated: up rows that give 1, gate rows that give z
    x = torch.cat([z, torch.ones(rows, 8, dtype=dtype)], 1).to(DEV)
    zero = torch.zeros_like(w)
    wg = torch.cat([torch.cat([zero, w], 1), torch.cat([w, zero], 1)], 0).contiguous()
    _inside(B.glu(x, wg, None, ACTS[kind]), a, z.double(), kind, dtype, 1, "gated")
    dx, _, _ = B.glu_backward(x, wg, None, torch.ones_like(z).to(DEV), ACTS[kind])
    _inside(dx[:, :8], slope, z.double(), kind, dtype, 3, "gated, derivative by the gate")
    _inside(dx[:, 8:], a, z.double(), kind, dtype, 1, "gated, derivative by the other half")
