"""What the allocating calls of the transformer-block operators do with the tensors they are given, before anything reaches a GPU."""
import pytest
import torch

from paper_2412_05781_amd import binding as B


def test_rows_that_start_off_a_boundary_are_copied():
    x = torch.arange(5 * 77, dtype=torch.float16).view(5, 77)
    assert x.data_ptr() % 16 == 0
    for t in (x[1:], x.flatten()[3:3 + 4 * 77].view(4, 77), x[:, 1:], x[2:].view(1, 3, 77)):
        assert t.data_ptr() % 16
        f = B._flat(t)
        assert f.data_ptr() % 16 == 0 and torch.equal(f, t.reshape(-1, t.shape[-1])) and f.stride(1) == 1
    assert B._flat(x[:, :70]).data_ptr() == x.data_ptr()               # at a boundary: where it is


def test_tensors_that_need_a_gradient_are_refused():
    """These calls record no history: a result without one would end a training step's gradients in silence."""
    x, w, b = torch.zeros(4, 16), torch.zeros(8, 16), torch.zeros(8)
    q, k = torch.zeros(1, 3, 2, 16), torch.zeros(1, 5, 2, 16)
    leaf = lambda t: t.clone().requires_grad_()
    calls = [lambda: B.linear(leaf(x), w, b), lambda: B.linear(x, leaf(w), b), lambda: B.linear(x, w, leaf(b)), lambda: B.linear(x, w, b, residual=leaf(torch.zeros(4, 8))),
             lambda: B.glu(leaf(x), w, b), lambda: B.glu(x, leaf(w), b), lambda: B.glu(x, w, leaf(b)), lambda: B.linear(leaf(x) * 2, w, b),
             lambda: B.attention(leaf(q), k, k), lambda: B.attention(q, leaf(k), k), lambda: B.attention(q, k, leaf(k), with_lse=True)]
    for call in calls:
        with pytest.raises(ValueError, match="_backward"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):                       # goes on to the next check
            call()
    for call in (lambda: B.linear(leaf(x).detach(), w, b), lambda: B.linear_backward(x, leaf(w), b, torch.zeros(4, 8))):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_workspace_of_few_rows_is_never_more_than_asked_for():
    """A call of few rows may take the kernel without a workspace where the size call, which does not know the strides, counted on the other one; never the reverse."""
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2412_05781_amd.build import build_libwino
        build_libwino()
    at = [0x100000000 * i for i in range(1, 5)]
    L = B.lib()
    for M in (1, 16, 33, 64):
        for K in (8, 1288, 2563, 5120, 20000):
            for N in (8, 320, 2568, 10240):
                for dt in (B.WINO_F16, B.WINO_F32):
                    need = B.wino_linear_workspace_bytes(M, N, K, dt)
                    if need:                                  # then aligned operands do need it: a byte less is refused
                        assert K > 1000
                        rc = L.wino_linear(at[0], at[1], None, None, at[2], M, N, K, (K + 7) // 8 * 8, N, N, dt, 0, at[3] * 8, need - 1, None)
                        assert rc == B.WINO_ERR_WORKSPACE or K % 8, (M, K, N, dt)
