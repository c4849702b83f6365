"""The cross entropy of a linear head at logits of any size, on the GPU: whole numbers, so that every logit is exact and what is seen is the softmax alone."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}             # half a step, relative

# a logit is +-8 a b, of eight products, less whole numbers of the step that fp32 has there (or of ones)
BASES = {"1e3": (1, 125), "1e6": (250, 500), "1.3e8": (4096, 4096), "8.6e9": (32768, 32768)}
SHAPES = [(3, 300), (40, 1003), (130, 1003), (600, 4099)]               # few rows and tiles of each size


def inputs(rows, vocab, base, dtype, seed):
    rng = np.random.default_rng(seed)
    a, b = BASES[base]
    step = max(1, 2 ** (int(np.log2(8 * a * b)) - 22))
    x, w = np.zeros((rows, 16)), np.zeros((vocab, 16))
    x[:, :8], w[:, :8] = a * rng.choice([-1, 1], (rows, 1)), b
    x[:, 8:10] = step * np.array([[1, 0], [0, 1], [1, 1]])[rng.integers(0, 3, rows)]
    w[:, 8:10] = -rng.integers(0, 10, (vocab, 2))
    top = (x @ w.T).argmax(1)
    target = np.where(rng.random(rows) < 0.5, top, rng.integers(0, vocab, rows)).astype(np.int32)
    weight = rng.choice([0.25, 1.0, 3.0], rows).astype(np.float32)
    return torch.from_numpy(x).to(dtype), torch.from_numpy(w).to(dtype), target, weight


def true(x, w, target, weight):
    """(loss, lse, G, d, ln s) in float64, by differences d from each row's largest logit, which are exact."""
    z = x.double().numpy() @ w.double().numpy().T
    d = z - z.max(1, keepdims=True)
    log_s = np.log(np.exp(d).sum(1))
    at = np.arange(len(target)), target
    G = np.exp(d - log_s[:, None])
    G[at] = np.expm1(d[at] - log_s)
    return weight * (log_s - d[at]), z.max(1) + log_s, G * weight[:, None], d, log_s


def call(x, w, target, weight, outs, dw_dtype=F32):
    rows, dim, vocab = *x.shape, len(w)
    new = {"loss": (rows,), "lse": (rows,), "dx": (rows, dim), "dw": (vocab, dim)}
    types = {"loss": F32, "lse": F32, "dx": x.dtype, "dw": dw_dtype}
    out = {n: torch.full(new[n], float("nan"), dtype=types[n], device="cuda") for n in outs}
    kimad.kimad_linear_xent(x.cuda(), w.cuda(), torch.from_numpy(target).cuda(), row_weight=torch.from_numpy(weight).cuda(), **out)
    return {n: t.double().cpu().numpy() for n, t in out.items()}


def sum_error(vocab):
    """Relative, of the sum of exponentials: an exponential's argument t is off by (|t| + 15) 2^-23 and it by an ulp; t exp(-t) is below one, so that all of them make
    less than 2^-19 of the sum, and adding makes 2^-24 for each of the terms at most."""
    return 2.0 ** -19 + vocab * 2.0 ** -24


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("base", BASES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_loss(rows, vocab, base, dtype):
    """The loss is ln s less an exact difference: its error does not grow with the logits, and it is never below 0 (the largest logit's own exponential is 1)."""
    x, w, target, weight = inputs(rows, vocab, base, dtype, rows)
    loss, lse, *_ = true(x, w, target, weight)
    for outs in (("loss", "lse"), ("loss", "lse", "dx")):                   # (with a gradient few rows go by tiles too)
        got = call(x, w, target, weight, outs)
        assert (got["loss"] >= 0).all()
        assert (np.abs(got["loss"] - loss) <= weight * sum_error(vocab) + 2.0 ** -22 * np.abs(loss)).all(), np.abs(got["loss"] - loss).max()
        assert (np.abs(got["lse"] - lse) <= sum_error(vocab) + 2.0 ** -23 * np.abs(lse)).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("base", BASES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_gradients(rows, vocab, base, dtype):
    """G is off by the sum of exponentials, by its own argument a (4 |a| 2^-24), by two roundings to the type (e, and G); in fp16 an exponential below 2^-14 of its strip's
    largest is off by 2^-27 of that, in bfloat16 one below 2^-29 by 2^-40, and fp16's G by half its smallest step, 2^-25, over 4096 of the largest weight.  At the
    target it is expm1 of an argument that is off by the sum's error.  Nothing of this grows with the logits."""
    x, w, target, weight = inputs(rows, vocab, base, dtype, rows + 1)
    _, _, G, d, log_s = true(x, w, target, weight)
    got = call(x, w, target, weight, ("dx", "dw"))
    u, wt = HALF[dtype], weight[:, None].astype(np.float64)
    off = np.abs(G) * (2 * u + u * u + sum_error(vocab) + 2.0 ** -20 + 2.0 ** -22 * np.abs(d - log_s[:, None]))
    off += wt * 2.0 ** -27 + wt.max() * 2.0 ** -37 if dtype == F16 else wt * 2.0 ** -40
    off[np.arange(rows), target] += weight * (sum_error(vocab) + 2.0 ** -22)
    X, W = x.double().numpy(), w.double().numpy()
    for name, want, bound, ulp in (("dx", G @ W, off @ np.abs(W) + vocab * 2.0 ** -23 * (np.abs(G) @ np.abs(W)), u),
                                   ("dw", G.T @ X, off.T @ np.abs(X) + rows * 2.0 ** -23 * (np.abs(G).T @ np.abs(X)), HALF[F32])):
        bound = bound + ulp * (np.abs(want) + bound) + 2.0 ** -24
        assert (np.abs(got[name] - want) <= bound).all(), (name, np.abs(got[name] - want).max(), bound.max())
