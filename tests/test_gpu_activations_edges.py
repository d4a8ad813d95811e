"""Operators on activations in 8 bits on the GPU, at the edges of what they take: no rows, many rows, tensors that autograd saves."""
import pytest
import torch

import activations_reference as R  # noqa: F401
from test_gpu_activations import A, BF16, F32, weight_of  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fine", [False, True])
@pytest.mark.parametrize("cols,out", [(96, 32), (343, 8), (343, 21), (64, 21)])
def test_gradients_of_no_rows(A, cols, out, fine):  # noqa: F811
    """Weights that have to be laid out, and such that have not."""
    x = A.Packed8(torch.empty(0, cols, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, -(-cols // 32), dtype=torch.uint8, device="cuda"))
    w, g = weight_of(2 * out, cols, 301).cuda(), torch.empty(0, 2 * out, dtype=BF16, device="cuda")
    dx, dw = A.linear8_backward(g, x, w)
    assert dx.shape == (0, cols) and dw.shape == w.shape and not dw.any()
    gated, kept = A.gated_linear8(x, w)
    dx, dw = A.gated_linear8_backward(g[:, :out], kept, x, w, fine=fine)
    assert dx.shape == (0, cols) and dw.shape == w.shape and not dw.any()
    assert A.linear_gate8_backward(g, weight_of(2 * out, out, 302).cuda(), kept).shape == (0, 2 * out)
