"""Operators whose offsets pass 32 bits: rows far apart, and buffers of more than 4 GiB."""
import numpy as np
import pytest

from tests import operators_reference as ref

pytestmark = pytest.mark.gpu


def _kimad():
    import paper_2312_08053_amd as kimad
    return kimad


def _far_rows(rows, cols, dtype, fill=None):
    """A matrix whose rows are more than 2^31 elements apart."""
    import torch
    ld = (1 << 31) + 7
    buf = torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda")
    m = torch.as_strided(buf, (rows, cols), (ld, 1))
    if fill is not None:
        m.copy_(fill)
    return m


def test_quantised_and_read_back_from_and_to_rows_far_apart():
    import torch
    kimad = _kimad()
    near = torch.randn(3, 333, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).cuda()
    far = _far_rows(3, 333, torch.bfloat16, near)
    want = kimad.mx4_empty(3, 333) + kimad.mx4_empty(333, 3)
    got = kimad.mx4_empty(3, 333) + kimad.mx4_empty(333, 3)
    kimad.kimad_mx4_quantise(near, *want)
    kimad.kimad_mx4_quantise(far, *got)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    kimad.kimad_mx4_dequantise(got[0], got[1], far)
    back = torch.empty_like(near)
    kimad.kimad_mx4_dequantise(got[0], got[1], back)
    assert torch.equal(far, back)


def test_distillation_of_rows_far_apart():
    import torch
    kimad = _kimad()
    gen = torch.Generator().manual_seed(1)
    for rows, vocab in ((2, 70001), (2, 3000)):
        near = (3 * torch.randn(rows, vocab, generator=gen)).to(torch.bfloat16).cuda()
        far = _far_rows(rows, vocab, torch.bfloat16, near)
        idx = torch.stack([torch.randperm(vocab, generator=gen)[:20] for _ in range(rows)]).int().cuda()
        val = torch.randn(rows, 20, generator=gen).cuda()
        out = []
        for z in (near, far):
            loss, stats = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
            kimad.kimad_distill(z, idx, val, 1.0, loss=loss, stats=stats)
            kimad.kimad_distill(z, idx, val, 1.0, grad=z)
            out.append((loss, stats, z))
        # (a row may begin elsewhere within 16 bytes: other threads add other elements, the sums agree to their rounding)
        assert torch.allclose(out[0][0], out[1][0], rtol=1e-5) and torch.allclose(out[0][1], out[1][1], rtol=1e-5)
        assert torch.allclose(out[0][2].float(), out[1][2].float(), rtol=2.0 ** -7, atol=1e-9)
        del far, out


def test_product_of_codes_beyond_four_gibibytes():
    import torch
    kimad = _kimad()
    M, N, K = 40000, 70, 262144                                     # 5.2 GB of codes
    gen = torch.Generator(device="cuda").manual_seed(2)
    a = torch.randint(0, 256, (M, K // 2), dtype=torch.uint8, generator=gen, device="cuda")
    b = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, generator=gen, device="cuda")
    one = 0x7F7F7F7F                                                # every scale 1
    sa = torch.full((K // 128, M), one, dtype=torch.int32, device="cuda")
    sb = torch.full((K // 128, N), one, dtype=torch.int32, device="cuda")
    out = torch.empty(M, N, device="cuda")
    kimad.kimad_mx4_matmul(a, sa, b, sb, K, out)
    table = torch.tensor(np.concatenate([ref.MAGNITUDES, -ref.MAGNITUDES]), device="cuda")

    def values(codes):
        return table[torch.stack([codes & 15, codes >> 4], -1).view(codes.shape[0], -1).long()]

    rows = torch.tensor([0, 1, 20000, 32767, 32768, 39998, 39999])
    want = values(a[rows.cuda()]) @ values(b).t().contiguous()
    # products of halves are multiples of a quarter, and their sums stay far below 2^22: exact in fp32, in any order
    assert torch.equal(out[rows.cuda()].double(), want)
    few = torch.empty(N, 3, device="cuda")
    kimad.kimad_mx4_matmul(b, sb, a[-3:], sa[:, -3:].contiguous(), K, few)
    assert torch.equal(few, out[-3:].t())


@pytest.mark.parametrize("M, N, K", [(256, 65536, 256), (250, 65500, 256), (200, 20000, 128), (100, 1000, 1024)])
def test_product_into_rows_far_apart(M, N, K):
    import torch
    kimad = _kimad()
    gen = torch.Generator(device="cuda").manual_seed(6)
    a, sa = kimad.mx4_empty(M, K)
    b, sb = kimad.mx4_empty(N, K)
    kimad.kimad_mx4_quantise(torch.randn(M, K, generator=gen, device="cuda"), a, sa)
    kimad.kimad_mx4_quantise(torch.randn(N, K, generator=gen, device="cuda"), b, sb)
    for dtype in (torch.float32, torch.bfloat16):
        near = torch.empty(M, N, dtype=dtype, device="cuda")
        kimad.kimad_mx4_matmul(a, sa, b, sb, K, near)
        ld = 1 << 24                                                # 256 rows: 17 GB in 32 bits
        buf = torch.full((M * ld,), -77.0, dtype=dtype, device="cuda")
        far = torch.as_strided(buf, (M, N), (ld, 1))
        kimad.kimad_mx4_matmul(a, sa, b, sb, K, far)
        assert torch.equal(far, near)                               # (the same sums in the same order)
        assert bool((buf.view(M, ld)[:, N:] == -77.0).all())
        del buf, far


def test_update_of_more_than_two_to_the_thirty_entries():
    import torch
    kimad = _kimad()
    d, tail = (1 << 30) + 4003, 5003
    starts = torch.tensor([0, 77, (1 << 30) - 1000, d], dtype=torch.int64, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = torch.randn(d, generator=gen, device="cuda")
    h, hat, x = (torch.zeros(d, device="cuda") for _ in range(3))
    assert d - ((1 << 30) - 1000) == tail
    words = kimad.kimad_mx4_update_words(3, d)
    codes, scales = torch.empty(words, 64, dtype=torch.uint8, device="cuda"), torch.empty(words, dtype=torch.int32, device="cuda")
    kimad.kimad_mx4_compress_ef(g, h, starts, codes, scales)
    kimad.kimad_mx4_server_apply([(codes, scales)], [hat], [1.0], starts, d, x, 1.0)
    assert torch.equal(h, hat) and torch.equal(x, -hat)
    # the last layer alone, and the first
    for lo, n in ((d - tail, tail), (0, 77)):
        one = torch.zeros(n, device="cuda")
        w1 = kimad.kimad_mx4_update_words(1, n)
        c1, s1 = torch.empty(w1, 64, dtype=torch.uint8, device="cuda"), torch.empty(w1, dtype=torch.int32, device="cuda")
        kimad.kimad_mx4_compress_ef(g[lo:lo + n].clone(), one, torch.tensor([0, n], dtype=torch.int64, device="cuda"), c1, s1)
        assert torch.equal(one, h[lo:lo + n])
