"""Each entry of the cross entropy's G = w (p - onehot) on its own: with x the identity, z is w's transpose and dw is G's.  Logits are whole numbers, so that nothing but the softmax and
the roundings of G are seen: small probabilities beside large ones, and targets that are nearly sure."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F16: 2.0 ** -11, BF16: 2.0 ** -8}                              # half a step, relative
SPREAD = {F16: 24, BF16: 45}                                           # how far logits lie below 0


def inputs(rows, vocab, dtype, seed):
    rng = np.random.default_rng(seed)
    z = -rng.integers(0, SPREAD[dtype] + 1, (rows, vocab)).astype(np.float64)
    target = rng.integers(0, vocab, rows).astype(np.int32)
    sure = np.arange(0, rows, 2)
    z[sure, target[sure]] = rng.integers(6, 13, len(sure))
    return z, target


def true(z, target):
    d = z - z.max(1, keepdims=True)
    log_s = np.log(np.exp(d).sum(1))
    at = np.arange(len(z)), target
    G = np.exp(d - log_s[:, None])
    G[at] = np.expm1(d[at] - log_s)
    return G


def bound(G, target, dtype):
    """Two roundings to the type (e, and G); the sum of exponentials; G's argument, 64 at most, 2^-22 of it; an exponential that is too small for its format, and in fp16 G that is too
    small for the type (half its smallest step, 2^-25, over 4096).  The target's is expm1 of an argument that is off by the sum's error, rounded once.
    The sum: an exponential's argument t is off by |t| 2^-23 and it by an ulp, which weighted with exp(-t) is 2^-22 at most, in the tiles and in each of ten joins of strips, and there are
    fewer than 64 roundings on the way from a term to the sum (eight and three in a tile, two in each join): 2^-22 (1 + 10) + 2^-18 < 2^-17."""
    u, s = HALF[dtype], 2.0 ** -17
    off = np.abs(G) * (2 * u + u * u + s + 2.0 ** -15) + (2.0 ** -42 + 2.0 ** -37 if dtype == F16 else 2.0 ** -73)
    at = np.arange(len(G)), target
    off[at] = np.abs(G[at]) * (u + 2.0 ** -20) + s + 2.0 ** -37
    return off


SHAPES = [(16, 64), (64, 200), (128, 1003), (256, 3001)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_every_entry(rows, vocab, dtype):
    z, target = inputs(rows, vocab, dtype, rows)
    dw = torch.full((vocab, rows), float("nan"), device="cuda")
    kimad.kimad_linear_xent(torch.eye(rows).to(dtype).cuda(), torch.from_numpy(z.T.copy()).to(dtype).cuda(), torch.from_numpy(target).cuda(), dw=dw)
    G, got = true(z, target), dw.double().cpu().numpy().T
    off = np.abs(got - G) / bound(G, target, dtype)
    assert (off <= 1).all(), (off.max(), G.reshape(-1)[off.argmax()], got.reshape(-1)[off.argmax()])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_the_bound_tells_a_rounded_probability(rows, vocab, dtype):
    """p - 1 from a p in 16 bits, and exponentials that end at 2^-29 of the largest (2^-14 in fp16), are outside of it."""
    z, target = inputs(rows, vocab, dtype, rows)
    G = true(z, target)
    limit, at, sure = bound(G, target, dtype), (np.arange(rows), target), np.arange(0, rows, 2)
    p = torch.from_numpy(G[at] + 1).to(dtype).double().numpy()
    assert (np.abs(p - 1 - G[at]) > limit[at])[sure].mean() > 0.5
    step = 2.0 ** (-39 if dtype == BF16 else -26)
    coarse = np.round(G / step) * step
    assert (np.abs(coarse - G) > limit).any()
