"""A linear layer's gradient over one row, or of one feature out, of an odd width: what stands behind that row, here NaN, reaches nothing."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad
from tests.test_gpu_linear import buffer, outside_is_nan, whole

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("K", [1, 2, 7, 33, 63, 65, 127, 255, 257, 2047])
@pytest.mark.parametrize("M,N", [(1, 8), (8, 1), (1, 1), (1, 300), (300, 1)])
def test_gradient(M, N, K):
    """Whole numbers: sums are exact."""
    rng = np.random.default_rng(K)
    dy, x, w = whole(rng, (M, N), BF16), whole(rng, (M, K), BF16), whole(rng, (N, K), BF16)
    (dy_, _), (x_, _), (w_, _) = buffer(dy), buffer(x), buffer(w)
    dx, dx_full = buffer(torch.zeros(M, K, dtype=BF16, device="cuda"))
    dw, dw_full = buffer(torch.zeros(N, K, device="cuda"))
    kimad.kimad_linear_grad(dy_, x_, w_, dx=dx, dw=dw)
    assert torch.equal(dx, (dy.double() @ w.double()).to(BF16)) and torch.equal(dw, (dy.double().t() @ x.double()).float())
    assert outside_is_nan(dx, dx_full, 0, 0) and outside_is_nan(dw, dw_full, 0, 0)
    out, out_full = buffer(torch.zeros(M, N, device="cuda"))
    kimad.kimad_linear(x_, w_, out)
    assert torch.equal(out, (x.double() @ w.double().t()).float()) and outside_is_nan(out, out_full, 0, 0)
