"""Quantisation to microscaled 4-bit floats and back, and the product of two such matrices, against 64-bit references."""
import numpy as np
import pytest

from tests import operators_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ("float32", "float16", "bfloat16")


def _kimad():
    import paper_2312_08053_amd as kimad
    return kimad


def _host(t):
    """float64 values of a device tensor."""
    return t.cpu().double().numpy()


def _words(scales):
    return scales.cpu().numpy().view(np.uint32)


def _matrix(rows, cols, kind, seed, ld=None, offset=0):
    """A matrix of the type inside a larger buffer: rows `ld` apart, beginning `offset` elements into it."""
    import torch
    rng = np.random.default_rng(seed)
    ld = cols if ld is None else ld
    x = rng.normal(0, 1, (rows, cols)) * np.exp(rng.normal(0, 1.5, (1, cols)))
    if kind == "float16":
        x = np.clip(x, -6e4, 6e4)
    buf = torch.full((offset + rows * ld + 64,), float("nan"), dtype=getattr(torch, kind), device="cuda")
    m = torch.as_strided(buf, (rows, cols), (ld, 1), offset)
    m.copy_(torch.from_numpy(x).to(getattr(torch, kind)))
    return m


def _quantise(x, rows_form=True, columns_form=False):
    import torch
    kimad = _kimad()
    R, C = x.shape
    out = []
    for want, (r, c) in ((rows_form, (R, C)), (columns_form, (C, R))):
        if not want:
            out += [None, None]
            continue
        codes, scales = kimad.mx4_empty(r, c)
        codes.fill_(0xEE)
        scales.fill_(-1)
        out += [codes, scales]
    kimad.kimad_mx4_quantise(x, *out)
    torch.cuda.synchronize()
    return out


def _assert_form(codes, scales, want, what):
    got_codes, got_bytes = ref.mx4_unpack(codes.cpu().numpy(), _words(scales))
    want_codes, want_bytes = ref.mx4_quantise(want)
    assert np.array_equal(got_bytes, want_bytes), what
    assert np.array_equal(ref.without_minus_zero(got_codes), ref.without_minus_zero(want_codes)), what


SHAPES = [(1, 1), (1, 31), (2, 32), (1, 33), (3, 127), (16, 128), (17, 129), (33, 64), (128, 128), (129, 257), (200, 40), (5, 700), (1, 8321), (260, 3)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rows_and_columns_are_quantised_by_the_definition(rows, cols, kind):
    x = _matrix(rows, cols, kind, rows * 1000 + cols)
    codes, scales, codes_t, scales_t = _quantise(x, True, True)
    _assert_form(codes, scales, _host(x), "rows")
    _assert_form(codes_t, scales_t, _host(x).T, "columns")
    alone = _quantise(x, True, False)
    assert np.array_equal(alone[0].cpu().numpy(), codes.cpu().numpy()) and np.array_equal(_words(alone[1]), _words(scales))
    columns = _quantise(x, False, True)
    assert np.array_equal(columns[2].cpu().numpy(), codes_t.cpu().numpy()) and np.array_equal(_words(columns[3]), _words(scales_t))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("offset", [0, 1, 3, 8])
def test_rows_may_begin_anywhere(kind, offset):
    x = _matrix(35, 203, kind, offset, ld=203 + 2 * offset + 1, offset=offset)
    codes, scales, codes_t, scales_t = _quantise(x, True, True)
    _assert_form(codes, scales, _host(x), "rows")
    _assert_form(codes_t, scales_t, _host(x).T, "columns")
    alone = _quantise(x)
    assert np.array_equal(alone[0].cpu().numpy(), codes.cpu().numpy())


@pytest.mark.parametrize("kind", TYPES)
def test_zeros_ties_extremes_and_what_is_not_finite(kind):
    import torch
    dt = getattr(torch, kind)
    info = torch.finfo(dt)
    x = torch.zeros(8, 256, dtype=torch.float64)
    x[0, :32] = -0.0
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.5, 6.0, 7.0, 7.9375, 4.0])
    x[1, :12], x[1, 32:44] = ties, -ties * 2.0 ** -6
    x[2, 0], x[2, 33] = info.max, -info.max
    tiny = info.smallest_normal
    x[3, :32] = torch.arange(32) * (tiny / 8)                       # down among the subnormal numbers of the type
    x[3, 32:40] = info.smallest_normal * info.eps
    x[4, 5], x[4, 40] = float("inf"), float("-inf")
    x[5, 7], x[5, 63] = float("nan"), 1.0
    x[6, 100:120] = 1.0
    x[7, 255] = float("nan")
    x = x.to(dt).cuda()
    codes, scales, codes_t, scales_t = _quantise(x, True, True)
    _assert_form(codes, scales, _host(x), "rows")
    _assert_form(codes_t, scales_t, _host(x).T, "columns")
    out = torch.empty(8, 256, dtype=torch.float32, device="cuda")
    _kimad().kimad_mx4_dequantise(codes, scales, out)
    want = ref.mx4_values(*ref.mx4_quantise(_host(x)))
    assert np.array_equal(_host(out), want, equal_nan=True)
    assert np.isnan(want[4, :64]).all() and np.isnan(want[5, :32]).all() and not np.isnan(want[5, 32:]).any()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows,cols,ld,offset", [(1, 1, 1, 0), (20, 131, 131, 0), (20, 131, 160, 3), (3, 9000, 9001, 1), (40, 64, 64, 2)])
def test_reading_back(rows, cols, ld, offset, kind):
    import torch
    x = _matrix(rows, cols, "float32", cols)
    codes, scales, _, _ = _quantise(x)
    dt = getattr(torch, kind)
    buf = torch.full((offset + rows * ld + 64,), 77.0, dtype=dt, device="cuda")
    out = torch.as_strided(buf, (rows, cols), (ld, 1), offset)
    _kimad().kimad_mx4_dequantise(codes, scales, out)
    values = ref.mx4_values(*ref.mx4_quantise(_host(x)))[:, :cols]
    # exact in float32 and bfloat16; float16 rounds what lies among its subnormal numbers, to nearest
    want = values if kind != "float16" else values.astype(np.float16).astype(np.float64)
    assert np.array_equal(_host(out), want)
    untouched = np.ones(buf.numel(), dtype=bool)
    for r in range(rows):
        untouched[offset + r * ld:offset + r * ld + cols] = False
    assert (buf.float().cpu().numpy()[untouched] == 77.0).all()


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(seed):
    rng = np.random.default_rng(100 + seed)
    rows, cols = int(np.exp(rng.uniform(0, 6))), int(np.exp(rng.uniform(0, 6)))
    x = _matrix(rows, cols, TYPES[seed % 3], seed, ld=cols + int(rng.integers(0, 9)), offset=int(rng.integers(0, 9)))
    codes, scales, codes_t, scales_t = _quantise(x, True, True)
    _assert_form(codes, scales, _host(x), "rows")
    _assert_form(codes_t, scales_t, _host(x).T, "columns")


# ---- the product -----------------------------------------------------------------------------------------------------------

def _operand(rows, K, seed, spread=6):
    """A quantised matrix in stored form (device) and its values."""
    import torch
    rng = np.random.default_rng(seed)
    words = -(-K // 128)
    codes = rng.integers(0, 16, (rows, 128 * words))
    codes[:, K:] = 0
    byte = rng.integers(127 - spread, 127 + spread, (rows, 4 * words))
    byte[:, -(-K // 32):] = 0
    packed, scale = ref.mx4_pack(codes, byte)
    return (torch.from_numpy(packed).cuda(), torch.from_numpy(scale.view(np.int32)).cuda()), ref.mx4_values(codes, byte)


def _product_close(out, a, b, K, kind):
    """Sums of K products in fp32: every addition rounds by at most 2^-24 of what it gives, which is at most the sum of the products'
    magnitudes; the matrix instruction may cut terms of one call against the largest (2^-23 each); the result is rounded once more."""
    with np.errstate(all="ignore"):
        want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    half = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[kind]
    bound = (K + 128) * 2.0 ** -23 * size + half * np.abs(want) * 1.0001
    if kind == "float16":
        bound = bound + 2.0 ** -25
        limit = 65504.0 * (1 + 2.0 ** -12)
        out, want = np.where(np.abs(want) > limit - bound, 0, out), np.where(np.abs(want) > limit - bound, 0, want)
    assert np.array_equal(np.isnan(out), np.isnan(want))
    bad = np.abs(out - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:3], out[bad][:3], want[bad][:3], bound[bad][:3])


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 100, 513), (2, 33, 64), (3, 200, 1000), (5, 1, 300), (8, 64, 4096), (16, 129, 700), (17, 63, 129),
            (31, 300, 130), (64, 64, 128), (65, 65, 640), (77, 130, 513), (100, 260, 2048), (128, 128, 256), (129, 257, 385), (256, 256, 1024),
            (300, 517, 900), (513, 130, 200), (40, 40, 9000), (1, 3000, 200), (260, 1, 260), (384, 512, 512), (16, 20, 20000)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(M, N, K):
    import torch
    kind = TYPES[(M + N + K) % 3]
    (a, sa), av = _operand(M, K, M)
    (b, sb), bv = _operand(N, K, 7 * N + 1)
    out = torch.full((M, N), 99.0, dtype=getattr(torch, kind), device="cuda")
    _kimad().kimad_mx4_matmul(a, sa, b, sb, K, out)
    _product_close(_host(out), av, bv, K, kind)


def _large_operand(rows, K, seed):
    """The same for sizes that only the device multiplies in 64 bits: random codes, scales that keep sums within a float16."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    words = -(-K // 128)
    packed = torch.randint(0, 256, (rows, 64 * words), dtype=torch.uint8, generator=gen)
    full = K // 2
    packed[:, full + K % 2:] = 0
    if K % 2:
        packed[:, full] &= 15
    byte = torch.randint(122, 128, (rows, 4 * words), dtype=torch.int64, generator=gen)
    byte[:, -(-K // 32):] = 0
    scale = (byte.view(rows, words, 4) << torch.tensor([0, 8, 16, 24])).sum(-1).to(torch.int32).t().contiguous()
    packed, byte = packed.cuda(), byte.cuda()
    magnitudes = torch.tensor(ref.MAGNITUDES, device="cuda")
    codes = torch.stack([packed & 15, packed >> 4], -1).view(rows, -1).long()
    sign = torch.where(codes >= 8, -1.0, 1.0).double()
    return (packed, scale.cuda()), sign * magnitudes[codes & 7] * (2.0 ** (byte - 127).double()).repeat_interleave(32, 1)


# sizes at which workgroups go through several tiles, of each tile's size, with rows and columns left over and without, words even and odd
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,N,K", [(8192, 5632, 768), (8200, 5641, 600), (4200, 4200, 260), (6000, 2050, 129), (3000, 2900, 100), (2049, 4100, 1300), (512, 768, 16384)])
def test_product_over_several_tiles_a_workgroup(M, N, K, kind):
    import torch
    (a, sa), av = _large_operand(M, K, 1)
    (b, sb), bv = _large_operand(N, K, 2)
    out = torch.full((M, N), 99.0, dtype=getattr(torch, kind), device="cuda")
    _kimad().kimad_mx4_matmul(a, sa, b, sb, K, out)
    bt, bt_size = bv.t().contiguous(), bv.abs().t().contiguous()
    want, size = av @ bt, av.abs() @ bt_size
    half = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[kind]
    bad = (out.double() - want).abs() > (K + 128) * 2.0 ** -23 * size + half * want.abs() * 1.0001
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (20, 33, 260), (130, 140, 400), (257, 300, 1100)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (5, 1), (8, 0)])
def test_product_into_rows_of_a_larger_buffer(M, N, K, kind, pad, offset):
    import torch
    (a, sa), av = _operand(M, K, 3)
    (b, sb), bv = _operand(N, K, 4)
    ld = N + pad
    buf = torch.full((offset + M * ld + 64,), 55.0, dtype=getattr(torch, kind), device="cuda")
    out = torch.as_strided(buf, (M, N), (ld, 1), offset)
    _kimad().kimad_mx4_matmul(a, sa, b, sb, K, out)
    _product_close(_host(out), av, bv, K, kind)
    untouched = np.ones(buf.numel(), dtype=bool)
    for r in range(M):
        untouched[offset + r * ld:offset + r * ld + N] = False
    assert (buf.float().cpu().numpy()[untouched] == 55.0).all()


@pytest.mark.parametrize("M,N,K", [(1, 64, 512), (40, 70, 300), (300, 300, 600)])
def test_a_block_that_stands_for_nan_spoils_its_row_alone(M, N, K):
    import torch
    (a, sa), av = _operand(M, K, 5)
    (b, sb), bv = _operand(N, K, 6)
    words = _words(sb).copy()
    words[1, 3] |= 0xFF00                                          # second block of word 1 of B's row 3
    sb = torch.from_numpy(words.view(np.int32)).cuda()
    bv = bv.copy()
    bv[3, 160:192] = np.nan
    out = torch.empty(M, N, device="cuda")
    _kimad().kimad_mx4_matmul(a, sa, b, sb, K, out)
    _product_close(_host(out), av, bv, K, "float32")
    assert np.isnan(_host(out)[:, 3]).all()


@pytest.mark.parametrize("M,N,K", [(1, 2000, 4096), (16, 300, 8192), (100, 90, 16384), (300, 200, 4000)])
def test_product_with_and_without_workspace_and_again(M, N, K):
    import torch
    kimad = _kimad()
    (a, sa), av = _operand(M, K, 11)
    (b, sb), bv = _operand(N, K, 12)
    out, again, alone = (torch.empty(M, N, device="cuda") for _ in range(3))
    kimad.kimad_mx4_matmul(a, sa, b, sb, K, out)
    kimad.kimad_mx4_matmul(a, sa, b, sb, K, again)
    kimad.kimad_mx4_matmul(a, sa, b, sb, K, alone, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    _product_close(_host(out), av, bv, K, "float32")
    _product_close(_host(alone), av, bv, K, "float32")
    assert np.array_equal(_host(out), _host(again))


def test_products_of_nothing():
    import torch
    kimad = _kimad()
    a, sa = kimad.mx4_empty(5, 0)
    b, sb = kimad.mx4_empty(7, 0)
    out = torch.full((5, 7), 3.0, device="cuda")
    kimad.kimad_mx4_matmul(a, sa, b, sb, 0, out)
    assert (_host(out) == 0).all()
    a, sa = kimad.mx4_empty(0, 64)
    (b, sb), _ = _operand(7, 64, 0)
    kimad.kimad_mx4_matmul(a, sa, b, sb, 64, torch.empty(0, 7, device="cuda"))
    codes, scales = kimad.mx4_empty(0, 10)
    kimad.kimad_mx4_quantise(torch.empty(0, 10, device="cuda"), codes, scales)


def test_product_on_another_stream_and_in_a_graph():
    import torch
    kimad = _kimad()
    x, y = _matrix(48, 640, "bfloat16", 1), _matrix(200, 640, "bfloat16", 2)
    forms = [kimad.mx4_empty(48, 640), kimad.mx4_empty(200, 640)]
    out = torch.zeros(48, 200, device="cuda")

    def work():
        kimad.kimad_mx4_quantise(x, *forms[0])
        kimad.kimad_mx4_quantise(y, *forms[1])
        kimad.kimad_mx4_matmul(*forms[0], *forms[1], 640, out)

    work()
    torch.cuda.synchronize()
    want = _host(out)
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    assert np.array_equal(_host(out), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(3):
        x.mul_(2.0)
        graph.replay()
        assert np.array_equal(_host(out), want * 2.0 ** (turn + 1))


def test_workspace_that_the_product_makes_stays_its_own_on_a_given_stream():
    import torch
    kimad = _kimad()
    M, N, K = 100, 90, 16384
    forms = [kimad.mx4_empty(M, K), kimad.mx4_empty(N, K)]
    kimad.kimad_mx4_quantise(_matrix(M, K, "bfloat16", 1), *forms[0])
    kimad.kimad_mx4_quantise(_matrix(N, K, "bfloat16", 2), *forms[1])
    nbytes = kimad.kimad_mx4_matmul_workspace_bytes(M, N, K)
    assert nbytes > 0
    want, out = torch.empty(M, N, device="cuda"), torch.zeros(M, N, device="cuda")
    kimad.kimad_mx4_matmul(*forms[0], *forms[1], K, want)
    big = torch.randn(4096, 4096, device="cuda")
    for handle in (False, True):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                busy = big @ big                                     # some milliseconds in front of the call
        kimad.kimad_mx4_matmul(*forms[0], *forms[1], K, out, stream=side.cuda_stream if handle else side)
        others = [torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        out.zero_()
        torch.cuda.synchronize()
        del others, busy


# whole rounds of large tiles and some rows beyond: those go by a second launch, of small tiles or of few rows
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,N,K", [(16404, 4096, 1024), (16385, 4096, 520), (16700, 4090, 1100), (33200, 2041, 900)])
def test_product_with_rows_beyond_whole_rounds(M, N, K, kind):
    test_product_over_several_tiles_a_workgroup(M, N, K, kind)


# about where products of few rows go by tiles instead, with sums shared out and not
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,N,K", [(12, 32000, 2048), (16, 32000, 2048), (32, 32001, 2048), (18, 50257, 768), (32, 50257, 768), (24, 16390, 4096), (32, 8192, 8192), (33, 8191, 8192), (64, 2048, 5632)])
def test_product_of_few_rows_by_many(M, N, K, kind):
    test_product_over_several_tiles_a_workgroup(M, N, K, kind)


@pytest.mark.parametrize("M,N", [(1, 1), (33, 70), (300, 70), (1000, 5)])
def test_a_product_over_no_columns_is_zeros_at_every_size(M, N):
    import torch
    kimad = _kimad()
    a, sa = kimad.mx4_empty(M, 0)
    b, sb = kimad.mx4_empty(N, 0)
    out = torch.full((M, N), 3.0, device="cuda")
    kimad.kimad_mx4_matmul(a, sa, b, sb, 0, out)
    assert (_host(out) == 0).all()


def test_every_rounding_case_at_scales_down_to_the_smallest_and_up_to_the_largest():
    """All magnitudes, all ties and the numbers next to them, with both signs, through the conversions along rows, along columns, and of an update."""
    import torch
    kimad = _kimad()
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    blocks = []
    for byte in (0, 1, 2, 23, 126, 127, 128, 251, 252):
        scale = np.ldexp(1.0, byte - 127)
        at = (ties * scale).astype(np.float32)
        assert (at.astype(np.float64) == ties * scale).all()
        v = np.concatenate([at, np.nextafter(at, np.float32(0)), np.nextafter(at, np.float32(np.inf)), (ref.MAGNITUDES * scale).astype(np.float32),
                            (np.array([5.5, 7.0, 7.9375]) * scale).astype(np.float32)])
        blocks += [v, -v]
        assert ref.mx4_block(v.astype(np.float64))[1] == byte
    x = np.stack(blocks)                                           # [18, 32]
    codes, scales, _, _ = _quantise(torch.from_numpy(x).cuda())
    _assert_form(codes, scales, x.astype(np.float64), "rows")
    _, _, codes_t, scales_t = _quantise(torch.from_numpy(np.ascontiguousarray(x.T)).cuda(), False, True)
    _assert_form(codes_t, scales_t, x.astype(np.float64), "columns")
    out = torch.empty(18, 32, device="cuda")
    kimad.kimad_mx4_dequantise(codes, scales, out)
    assert np.array_equal(_host(out), ref.mx4_values(*ref.mx4_quantise(x.astype(np.float64)))[:, :32])
    g, d = torch.from_numpy(x.reshape(-1)).cuda(), x.size
    h, words = torch.zeros(d, device="cuda"), kimad.kimad_mx4_update_words(1, d)
    up = torch.empty(words, 64, dtype=torch.uint8, device="cuda"), torch.empty(words, dtype=torch.int32, device="cuda")
    kimad.kimad_mx4_compress_ef(g, h, torch.tensor([0, d], device="cuda"), *up)
    want_codes, want_bytes, want_h = ref.update(x.reshape(-1), np.zeros(d, np.float32), np.array([0, d]))
    got_codes, got_bytes = ref.mx4_unpack(up[0].cpu().numpy(), _words(up[1])[None, :])
    assert np.array_equal(got_bytes, want_bytes) and np.array_equal(ref.without_minus_zero(got_codes), ref.without_minus_zero(want_codes))
    assert np.array_equal(h.cpu().numpy(), want_h)
