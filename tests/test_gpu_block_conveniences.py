"""The allocating calls of the transformer-block operators on tensors as programs have them."""
import pytest
import torch

from paper_2412_05781_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rand(*shape, dtype=torch.float16, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, device=DEV, generator=g).to(dtype)


@pytest.mark.parametrize("M", [5, 90])
def test_slices_that_start_off_a_boundary(M):
    K, N = 77, 33
    x, r, dy, dh = _rand(M + 1, K, seed=1)[1:], _rand(M + 1, N, seed=2)[1:], _rand(M + 1, N, seed=3)[1:], _rand(M + 1, N, seed=5)[1:]
    w, w2, b, b2 = _rand(N, K, seed=4), _rand(2 * N, K, seed=6), torch.randn(N, device=DEV), torch.randn(2 * N, device=DEV)
    assert all(t.data_ptr() % 16 for t in (x, r, dy, dh))
    c = [t.clone() for t in (x, r, dy, dh)]
    assert torch.equal(B.linear(x, w, b, residual=r), B.linear(c[0], w, b, residual=c[1]))
    assert torch.equal(B.glu(x, w2, b2), B.glu(c[0], w2, b2))
    for got, want in ((B.linear_backward(x, w, b, dy, B.WINO_ACT_SILU), B.linear_backward(c[0], w, b, c[2], B.WINO_ACT_SILU)),
                      (B.glu_backward(x, w2, b2, dh), B.glu_backward(c[0], w2, b2, c[3]))):
        assert all(torch.equal(g, h) for g, h in zip(got, want))
