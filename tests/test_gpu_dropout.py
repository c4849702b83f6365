"""Dropout from a counter-based generator, on the GPU."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def expected(x, p, seed, offset, residual=None):
    """What a product and a sum in fp32 give, rounded to the type: the same operations, so bit for bit."""
    keep, scale = ref.kept(x.numel(), p, seed, offset)
    keep = torch.from_numpy(keep).view(x.shape)
    y = torch.where(keep, x.cpu().float() * np.float32(scale), torch.zeros(()))
    return (y if residual is None else y + residual.cpu().float()).to(x.dtype)


def same(a, b):
    return torch.equal(a.cpu().nan_to_num(99.0), b.cpu().nan_to_num(99.0))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (3, 5), (1, 768), (77, 33), (5, 2048), (2049, 3)])
def test_values(rows, cols, dtype):
    x = torch.randn(rows, cols).to(dtype)
    r = torch.randn(rows, cols).to(dtype)
    for p, seed, offset in ((0.1, 1, 0), (0.5, (1 << 64) - 1, 1 << 40), (0.0, 3, 2), (1.0, 4, 5), (1e-6, 5, 5)):
        out = torch.empty(rows, cols, dtype=dtype, device="cuda")
        kimad.kimad_dropout(x.cuda(), out, p, seed, offset)
        assert same(out, expected(x, p, seed, offset))
        kimad.kimad_dropout(x.cuda(), out, p, seed, offset, residual=r.cuda())
        assert same(out, expected(x, p, seed, offset, r))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,shift", [(1, 0), (5, 1), (8, 0)])
def test_strides_and_in_place(dtype, pad, shift):
    from tests.test_gpu_linear import buffer, outside_is_nan
    x, r = torch.randn(50, 37).to(dtype), torch.randn(50, 37).to(dtype)
    want = expected(x, 0.25, 9, 1, r)
    for target in ("out", "x", "r"):
        (xb, x_full), (rb, r_full), (ob, o_full) = buffer(x.cuda(), pad, shift), buffer(r.cuda(), pad, shift), buffer(torch.zeros_like(x).cuda(), pad, shift)
        view, full = {"out": (ob, o_full), "x": (xb, x_full), "r": (rb, r_full)}[target]
        kimad.kimad_dropout(xb, view, 0.25, 9, 1, residual=rb)
        assert same(view, want) and outside_is_nan(view, full, shift, pad)


def test_what_is_dropped_is_gone():
    x = torch.tensor([[float("nan"), float("inf"), float("-inf"), 1.0] * 64])
    out = torch.empty_like(x, device="cuda")
    kimad.kimad_dropout(x.cuda(), out, 0.5, 11)
    keep, _ = ref.kept(x.numel(), 0.5, 11, 0)
    assert (out.cpu()[0][~torch.from_numpy(keep)] == 0).all() and same(out, expected(x, 0.5, 11, 0))
    kimad.kimad_dropout(x.cuda(), out, 1.0, 11)
    assert not out.any()


def test_the_gradient_is_the_same_call():
    """d (sum dy y) / dx by differences: y is linear in x, so any step does, and whole numbers make it exact."""
    x, dy = torch.arange(-40.0, 40).view(8, 10), torch.arange(80.0).view(8, 10) - 30
    out, dx = torch.empty(8, 10, device="cuda"), torch.empty(8, 10, device="cuda")
    kimad.kimad_dropout(dy.cuda(), dx, 0.5, 21, 4)
    for i in range(0, 80, 7):
        e = torch.zeros(80)
        e[i] = 1
        ends = []
        for s in (1, -1):
            kimad.kimad_dropout((x + s * e.view(8, 10)).cuda(), out, 0.5, 21, 4)
            ends.append(float((out.cpu() * dy).sum()))
        assert (ends[0] - ends[1]) / 2 == float(dx.view(-1)[i])


def test_offsets_beyond_32_bits():
    """The last of 2^32 + 70 elements, whose blocks are numbered as 64-bit counters say."""
    n = (1 << 32) + 72
    x = torch.ones(1, n, dtype=F16, device="cuda")
    kimad.kimad_dropout(x, x, 0.5, 77)
    tail = np.array([h for b in range((n - 144) // 8, n // 8) for w in ref.philox(b, 0, 77) for h in (w & 0xFFFF, w >> 16)]) >= 32768
    assert np.array_equal(x[0, -144:].cpu().numpy() == 2, tail)
    share = (x.view(-1)[:1 << 28] != 0).float().mean().item()
    assert abs(share - 0.5) < 6 * 0.5 / 2 ** 14


def test_a_recorded_call():
    x = torch.randn(33, 100, device="cuda")
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kimad.kimad_dropout(x, out, 0.3, 5, 6)
    for k in range(3):
        x.copy_(torch.randn(33, 100))
        graph.replay()
        assert same(out, expected(x, 0.3, 5, 6))
