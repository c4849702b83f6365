"""Weight gradients in fp32, as a round takes them, behind an activation, element by element."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F16: 2.0 ** -11, BF16: 2.0 ** -8}                              # half a step, relative


@pytest.mark.parametrize("kind", [ref.RELU, ref.GELU, ref.SILU])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("M,N,K", [(1, 40, 33), (77, 100, 65), (200, 136, 320), (1500, 520, 264)])
def test_weights_gradient(M, N, K, dtype, kind):
    """dz is rounded to the type, half a step of each term (in fp16 at least half of 2^-24); a slope's own roundings, 2^-14 of |dy| at |z| < 8, are counted beside it, a sum of M products in
    fp32 by M 2^-23 of their magnitudes, and nothing but fp32's own rounding of the result."""
    rng = np.random.default_rng(M + kind)
    dy, x, z = (torch.from_numpy(rng.normal(size=s)).cuda().to(dtype) for s in ((M, N), (M, K), (M, N)))
    d_dy, d_x, d_z = (t.double().cpu().numpy() for t in (dy, x, z))
    dz = d_dy * ref.slope(d_z, kind)
    want = dz.T @ d_x
    dw = torch.full((N, K), float("nan"), device="cuda")
    kimad.kimad_linear_grad(dy, x, None, z=z, act=kind, dw=dw)
    off = HALF[dtype] * np.abs(dz) + 2.0 ** -14 * np.abs(d_dy) + (2.0 ** -25 if dtype == F16 else 0)
    bound = (off + M * 2.0 ** -23 * np.abs(dz)).T @ np.abs(d_x)
    bound += 2.0 ** -24 * (np.abs(want) + bound)
    assert (np.abs(dw.double().cpu().numpy() - want) <= bound).all()
