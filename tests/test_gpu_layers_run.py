"""A trainer's step with all of it: a residual layer (product, activation, dropout, product, residual), the head's loss, every gradient, and a worker's update of them."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_a_step():
    """Against the same step in 64 bits whose stored numbers are rounded to bfloat16 where the calls store them.  What remains: roundings that fall the other way after a
    difference in the last place of fp32 (a step, 2^-7, of few elements), e and G of the cross entropy and dz (2^-8 each, of every term); a norm
    of a gradient is off by some 3 x 2^-8 / sqrt(3) at most, and held to 2^-6."""
    rng = np.random.default_rng(0)
    T, D, F, V, p = 200, 96, 260, 1003, 0.25

    def stored(a):
        return torch.from_numpy(np.asarray(a)).to(BF16)

    def d(t):
        return t.double().cpu().numpy()

    x, w1, b1 = stored(rng.normal(size=(T, D))), stored(rng.normal(size=(F, D)) / D ** 0.5), stored(rng.normal(size=F) * 0.1)
    w2, b2, wv = stored(rng.normal(size=(D, F)) / F ** 0.5), stored(rng.normal(size=D) * 0.1), stored(rng.normal(size=(V, D)) * 2 / D ** 0.5)
    target = rng.integers(-1, V, T).astype(np.int32)
    weight = np.full(T, 1.0 / T, dtype=np.float32)
    keep, scale = ref.kept(T * F, p, 5, 17)
    keep = keep.reshape(T, F)

    # 64 bits
    a, z1 = ref.linear(d(x), d(w1), d(b1), kind=ref.GELU)
    a, z1 = d(stored(a)), d(stored(z1))
    h = d(stored(np.where(keep, a * scale, 0)))
    y = d(stored(ref.linear(h, d(w2), d(b2), d(x))[0]))
    loss, _, dy, dwv, _ = ref.xent(y, d(wv), target, weight)
    dy = d(stored(dy))
    dh, dw2, db2 = ref.linear_grad(dy, h, d(w2))
    da = d(stored(np.where(keep, d(stored(dh)) * scale, 0)))
    dx, dw1, db1 = ref.linear_grad(da, d(x), d(w1), z1, ref.GELU)
    dx = dx + dy                                                              # (the residual's)

    g = {n: t.cuda() for n, t in dict(x=x, w1=w1, b1=b1, w2=w2, b2=b2, wv=wv).items()}
    new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device="cuda")  # noqa: E731
    sizes = [V * D, F * D, F, D * F, D]
    flat = new(sum(sizes), dtype=torch.float32)                              # the gradients, back to back in fp32, as a round takes them
    gwv, gw1, gb1, gw2, gb2 = flat.split(sizes)
    ga, gz, gh, gy, gdy, gdh, gda, gdx = new(T, F), new(T, F), new(T, F), new(T, D), new(T, D), new(T, F), new(T, F), new(T, D)
    gloss = new(T, dtype=torch.float32)
    kimad.kimad_linear(g["x"], g["w1"], ga, bias=g["b1"], act=kimad.KIMAD_ACT_GELU, z=gz)
    kimad.kimad_dropout(ga, gh, p, 5, 17)
    kimad.kimad_linear(gh, g["w2"], gy, bias=g["b2"], residual=g["x"])
    kimad.kimad_linear_xent(gy, g["wv"], torch.from_numpy(target).cuda(), loss=gloss, dx=gdy, dw=gwv.view(V, D), row_weight=torch.from_numpy(weight).cuda())
    kimad.kimad_linear_grad(gdy, gh, g["w2"], dx=gdh, dw=gw2.view(D, F), db=gb2)
    kimad.kimad_dropout(gdh, gda, p, 5, 17)
    kimad.kimad_linear_grad(gda, g["x"], g["w1"], z=gz, act=kimad.KIMAD_ACT_GELU, dx=gdx, dw=gw1.view(F, D), db=gb1)
    gdx += gdy
    for name, got, want in (("loss", gloss, loss), ("wv", gwv, dwv), ("w2", gw2, dw2), ("b2", gb2, db2), ("w1", gw1, dw1), ("b1", gb1, db1), ("x", gdx, dx)):
        off = np.linalg.norm(d(got).reshape(-1) - want.reshape(-1)) / np.linalg.norm(want)
        assert off <= 2.0 ** -6, (name, off)

    # and the worker's update of them in 4 bits
    starts = torch.tensor(np.cumsum([0] + sizes), dtype=torch.int64, device="cuda")
    est, words = torch.zeros_like(flat), kimad.kimad_mx4_update_words(len(sizes), flat.numel())
    codes, scales = new(words, 64, dtype=torch.uint8), new(words, dtype=torch.int32)
    kimad.kimad_mx4_compress_ef(flat, est, starts, codes, scales)
    assert (est - flat).norm() < 0.2 * flat.norm()
