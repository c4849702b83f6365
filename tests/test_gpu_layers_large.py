"""Layers in front of a loss whose matrices pass 2^32 bytes or elements: rows at their ends, against the same rows on their own."""
import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def whole(gen, *shape):
    return torch.randint(-4, 5, shape, generator=gen, device="cuda").to(BF16)


def test_linear_and_its_gradient_beyond_32_bits():
    """Whole numbers, so that every sum is exact: out of 8.7e9 bytes, z and dz of 4.4e9."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    M, N, K = 66000, 33000, 16
    x, w = whole(gen, M, K), whole(gen, N, K)
    out, z = torch.empty(M, N, device="cuda"), torch.empty(M, N, dtype=BF16, device="cuda")
    kimad.kimad_linear(x, w, out, act=kimad.KIMAD_ACT_RELU, z=z)
    some = torch.cat([torch.arange(0, 5), torch.arange(32530, 32550), torch.arange(65060, 65100), torch.arange(M - 300, M)]).cuda()
    true = x[some].double() @ w.double().t()
    assert torch.equal(out[some], true.clamp(min=0).float()) and torch.equal(z[some], true.to(BF16))
    del out
    dy = whole(gen, 1, N).expand(M, N).contiguous()
    dx, dw, db = torch.empty(M, K, dtype=BF16, device="cuda"), torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    kimad.kimad_linear_grad(dy, x, w, z=z, act=kimad.KIMAD_ACT_RELU, dx=dx, dw=dw, db=db)
    dz = torch.where(z[some] > 0, dy[some], 0).double()
    assert torch.equal(dx[some], (dz @ w.double()).to(BF16))
    for lo, hi in ((0, 300), (N - 300, N)):
        dz = torch.where(z[:, lo:hi] > 0, dy[:, lo:hi], 0).double()
        assert torch.equal(dw[lo:hi], (dz.t() @ x.double()).float()) and torch.equal(db[lo:hi], dz.sum(0).float())


def test_cross_entropy_of_a_head_beyond_32_bits():
    """4.8e9 bytes of weights.  All but the last 1000 of them are zeros, whose logits are 0: lse is known from those and the number of the others."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    rows, vocab, dim, tail = 40, 4_000_000, 600, 1000
    x = torch.randn(rows, dim, generator=gen, device="cuda").to(BF16)
    w = torch.zeros(vocab, dim, dtype=BF16, device="cuda")
    w[-tail:] = (torch.randn(tail, dim, generator=gen, device="cuda") * 0.5).to(BF16)
    target = torch.arange(vocab - rows, vocab, device="cuda", dtype=torch.int32)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(vocab, dim, device="cuda")
    kimad.kimad_linear_xent(x, w, target, loss=loss, lse=lse, dx=dx, dw=dw)
    z = x.double() @ w[-tail:].double().t()
    true = torch.logsumexp(torch.cat([z, torch.full((rows, 1), float(np.log(vocab - tail)), device="cuda", dtype=torch.float64)], 1), 1)
    picked = z.gather(1, (target.long() - (vocab - tail))[:, None])[:, 0]
    # a logit is off by 600 x 2^-23 of some 300, lse by that and four million roundings of sums of sums, 2^-24 each at most
    assert (lse - true).abs().max() < 0.03 and (loss - (true - picked)).abs().max() < 0.06
    G = torch.exp(z - true[:, None])
    G[torch.arange(rows, device="cuda"), target.long() - (vocab - tail)] = torch.expm1(picked - true)
    # (each G off by lse's error and two roundings of 2^-8; a norm of sums of such terms by no more than the terms' own)
    assert (dw[-tail:] - G.t() @ x.double()).norm() < 0.05 * (G.t() @ x.double()).norm()
    assert (dx - G @ w[-tail:].double()).norm() < 0.05 * (G @ w[-tail:].double()).norm()
    head = torch.exp(-true)[:, None] * x.double()                              # every zero weight's gradient
    # The last of them may share its 32 or 64 columns, over which exp(z - m) is kept in 16 bits, with others.  Kept is an fp16 number of 2^15 exp(z - m): below
    # 2^-29 it is off by half an fp16 subnormal step, 2^-25 2^-15 = 2^-40, times the largest probability of those columns.  (Its true entries are 1e-14 here.)
    near = torch.cat([torch.zeros(rows, 1, device="cuda", dtype=torch.float64), z[:, :64 - (vocab - tail) % 64]], 1).amax(1)
    kept = (2.0 ** -40 * torch.exp(near - true) * x.double().norm(dim=1)).sum()
    for at, more in ((0, 0), (1_999_999, 0), (vocab - tail - 1, kept)):
        assert (dw[at] - head.sum(0)).norm() < 0.05 * head.norm() + more
