"""A linear layer with its epilogue, and its gradient, on the GPU.  With whole numbers as inputs every fp32 sum is exact, so that a result is the true one rounded
once, bit for bit; with real ones the bounds below count roundings."""
import itertools

import numpy as np
import pytest
import torch

import paper_2312_08053_amd as kimad
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}             # half a step, relative
# few rows; one, several and many tiles of each size; parts of a sum; odd sizes, which are laid out anew
SHAPES = [(1, 1, 1), (1, 100, 513), (3, 17, 8), (16, 64, 2048), (17, 33, 300), (32, 1000, 264), (33, 1, 8), (33, 65, 64), (64, 64, 72), (40, 7, 2000), (128, 129, 136),
          (257, 255, 192), (300, 520, 77), (64, 256, 8192), (700, 1100, 513), (2049, 1025, 320), (1, 5000, 64), (5000, 1, 64), (4096, 2304, 256)]


def whole(rng, shape, dtype, most=4):
    return torch.from_numpy(rng.integers(-most, most + 1, shape).astype(np.float32)).cuda().to(dtype)


def buffer(x, pad=0, shift=0):
    """x in a buffer of NaN whose rows are `pad` longer and begin `shift` elements into it, and the whole buffer."""
    rows, cols = x.shape
    full = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = full[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view, full


def outside_is_nan(view, full, shift, pad):
    rows, cols = view.shape
    mask = torch.ones_like(full, dtype=torch.bool)
    mask[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = False
    return bool(full[mask].isnan().all())


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (F16, F32), (F16, F16), (BF16, F32)])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_sums_of_whole_numbers(M, N, K, dtype, out_dtype):
    rng = np.random.default_rng(M + 1000 * N + K)
    x, w, b, r = whole(rng, (M, K), dtype), whole(rng, (N, K), dtype), whole(rng, (N,), dtype), whole(rng, (M, N), dtype)
    z = x.double() @ w.double().t() + b.double()
    out, kept = torch.empty(M, N, dtype=out_dtype, device="cuda"), torch.empty(M, N, dtype=dtype, device="cuda")
    kimad.kimad_linear(x, w, out, bias=b, residual=r, z=kept)
    assert torch.equal(out, (z + r.double()).to(out_dtype)) and torch.equal(kept, z.to(dtype))
    kimad.kimad_linear(x, w, out, act=kimad.KIMAD_ACT_RELU)
    assert torch.equal(out, (z - b.double()).clamp(min=0).to(out_dtype))


@pytest.mark.parametrize("M,N,K", [(5, 77, 100), (100, 77, 104), (130, 200, 513), (300, 513, 256)])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (24, 1), (3, 5)])
def test_strides_and_addresses(M, N, K, pad, shift):
    """Rows of padded buffers that begin anywhere; what stands between them is NaN, reaches nothing and stays."""
    rng = np.random.default_rng(M + pad)
    x, w, r = whole(rng, (M, K), BF16), whole(rng, (N, K), BF16), whole(rng, (M, N), BF16)
    b = whole(rng, (N,), BF16)
    want = x.double() @ w.double().t() + b.double()
    (x, _), (w, _), (r, _) = buffer(x, pad, shift), buffer(w, pad, shift), buffer(r, pad, shift)
    for dtype in (BF16, F32):
        out, out_full = buffer(torch.zeros(M, N, dtype=dtype, device="cuda"), pad, shift)
        z, z_full = buffer(torch.zeros(M, N, dtype=BF16, device="cuda"), pad, shift)
        kimad.kimad_linear(x, w, out, bias=b, residual=r, z=z)
        assert torch.equal(out, (want + r.double()).to(dtype)) and torch.equal(z, want.to(BF16))
        assert outside_is_nan(out, out_full, shift, pad) and outside_is_nan(z, z_full, shift, pad)
    # the residual in place
    r_before = r.clone()
    kimad.kimad_linear(x, w, r, bias=b, residual=r)
    assert torch.equal(r, (want + r_before.double()).to(BF16))


VALUES = [0.0, -0.0, 1.0, -1.0, 0.5, -2.5, 3.0, -5.0, 8.0, -10.0, 20.0, -20.0, 60.0, -60.0, 1e4, -1e4, 2.0 ** -10, -2.0 ** -12, float("inf"), float("-inf"), float("nan")]


@pytest.mark.parametrize("M", [1, 70])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kind", [ref.RELU, ref.GELU, ref.SILU])
def test_activations(kind, dtype, M):
    """z is one number times one: exact.  The exponential's argument a is off by a few roundings of 2^-24, times |a| in the result, which matters up to |a| = 88; then the
    exponential, a sum, a quotient and a product, an ulp each: (8 |a| + 16) 2^-24."""
    v = torch.tensor(VALUES, dtype=dtype)
    x, w = torch.zeros(M, 8, dtype=dtype), torch.zeros(len(v), 8, dtype=dtype)
    x[:, 0], w[:, 0] = 1, v
    w[~v.isfinite(), 1:] = 0
    bias = torch.where(v.isfinite(), torch.zeros_like(v), v)
    w[~v.isfinite()] = 0
    out = torch.empty(M, len(v), device="cuda")
    z = torch.empty(M, len(v), dtype=dtype, device="cuda")
    kimad.kimad_linear(x.cuda(), w.cuda(), out, bias=bias.cuda(), act=kind, z=z)
    zd = v.double().numpy()
    with np.errstate(all="ignore"):
        want = ref.act(zd, kind)
        a = np.minimum(np.abs(2 * ref.C * (zd + 0.044715 * zd ** 3) if kind == ref.GELU else zd), 88.0)
    got = out.cpu().double().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.broadcast_to(np.isnan(want), got.shape)) and (got[:, zd == np.inf] == np.inf).all()
    assert (np.abs(got - want)[:, fine] <= ((8 * a + 16) * 2.0 ** -24 * np.abs(want) + 2.0 ** -120)[fine]).all(), (got[0], want)
    assert torch.equal(z.cpu().nan_to_num(7.0), v.expand(M, -1).nan_to_num(7.0))
    # the slope, by the gradient with regard to the bias of one row of ones
    db = torch.empty(len(v), device="cuda")
    dy = torch.ones(1, len(v), dtype=dtype, device="cuda")
    kimad.kimad_linear_grad(dy, None, None, z=z[:1], act=kind, db=db)
    with np.errstate(all="ignore"):
        want = ref.slope(zd, kind)
        inner = 2 * ref.C * (1 + 3 * 0.044715 * zd * zd) if kind == ref.GELU else np.ones_like(zd)
        s = ref._sigmoid(2 * ref.C * (zd + 0.044715 * zd ** 3) if kind == ref.GELU else zd)
        # (1 - s loses s's last places where s is near one: 2^-24 times |z| inner)
        bound = (8 * a + 32) * 2.0 ** -24 * (np.abs(want) + np.abs(zd) * inner * np.minimum(s, 1 - s + 2.0 ** -24) + np.abs(zd) * inner * s * (a < 40))
    got = db.cpu().double().numpy()
    fine = np.isfinite(zd)
    assert np.isnan(got[-1]) and got[VALUES.index(float("inf"))] == 1 and got[VALUES.index(float("-inf"))] == 0
    assert (np.abs(got - want)[fine] <= bound[fine] + 2.0 ** -120).all(), (got, want, bound)


@pytest.mark.parametrize("kind", [ref.NONE, ref.GELU, ref.SILU])
@pytest.mark.parametrize("M,N,K", [(2, 50, 700), (100, 130, 513), (600, 700, 1024)])
def test_real_numbers(M, N, K, kind):
    """A sum of K products in fp32 is off by at most K 2^-23 of the sum of their magnitudes (twice the bound for roundings to nearest); gelu's and silu's slopes are at
    most 1.13, and their own roundings as above with |a| <= 88."""
    rng = np.random.default_rng(K)
    x, w = torch.from_numpy(rng.normal(size=(M, K))).cuda().to(BF16), torch.from_numpy(rng.normal(size=(N, K)) / K ** 0.5).cuda().to(BF16)
    want, z = ref.linear(x.double().cpu().numpy(), w.double().cpu().numpy(), kind=kind)
    size = (x.double().abs() @ w.double().abs().t()).cpu().numpy()
    for dtype in (F32, BF16):
        out = torch.empty(M, N, dtype=dtype, device="cuda")
        kimad.kimad_linear(x, w, out, act=kind)
        bound = 1.13 * K * 2.0 ** -23 * size + 720 * 2.0 ** -24 * np.abs(want)
        bound += HALF[dtype] * (np.abs(want) + bound) + 2.0 ** -120
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("dtype,dw_dtype", [(BF16, F32), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("M,N,K", [s for s in SHAPES if s != (4096, 2304, 256)] + [(5000, 300, 200), (129, 64, 4096)])
def test_gradient_of_whole_numbers(M, N, K, dtype, dw_dtype):
    rng = np.random.default_rng(M + 1000 * N + K)
    dy, x, w = whole(rng, (M, N), dtype), whole(rng, (M, K), dtype), whole(rng, (N, K), dtype)
    z = whole(rng, (M, N), dtype)
    for kind in (ref.NONE, ref.RELU):
        dx, dw, db = torch.empty(M, K, dtype=dtype, device="cuda"), torch.empty(N, K, dtype=dw_dtype, device="cuda"), torch.empty(N, device="cuda")
        kimad.kimad_linear_grad(dy, x, w, z=z, act=kind, dx=dx, dw=dw, db=db)
        dz = dy.double() if kind == ref.NONE else torch.where(z > 0, dy, 0).double()
        assert torch.equal(dx, (dz @ w.double()).to(dtype)), kind
        assert torch.equal(dw, (dz.t() @ x.double()).to(dw_dtype)), kind
        assert torch.equal(db, dz.sum(0).float()), kind


@pytest.mark.parametrize("M,N,K", [(5, 77, 100), (100, 77, 104), (130, 200, 513), (300, 513, 256)])
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (24, 1)])
def test_gradient_of_strided_rows(M, N, K, pad, shift):
    rng = np.random.default_rng(M + pad)
    dy, x, w, z = whole(rng, (M, N), F16), whole(rng, (M, K), F16), whole(rng, (N, K), F16), whole(rng, (M, N), F16)
    for kind in (ref.NONE, ref.RELU):
        dz = dy.double() if kind == ref.NONE else torch.where(z > 0, dy, 0).double()
        (dy_, _), (x_, _), (w_, _), (z_, _) = (buffer(t, pad, shift) for t in (dy, x, w, z))
        dx, dx_full = buffer(torch.zeros(M, K, dtype=F16, device="cuda"), pad, shift)
        dw, dw_full = buffer(torch.zeros(N, K, device="cuda"), pad, shift)
        db = torch.empty(N, device="cuda")
        kimad.kimad_linear_grad(dy_, x_, w_, z=z_, act=kind, dx=dx, dw=dw, db=db)
        assert torch.equal(dx, (dz @ w.double()).to(F16)) and torch.equal(dw, (dz.t() @ x.double()).float()) and torch.equal(db, dz.sum(0).float())
        assert outside_is_nan(dx, dx_full, shift, pad) and outside_is_nan(dw, dw_full, shift, pad)


@pytest.mark.parametrize("kind", [ref.GELU, ref.SILU])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_gradient_through_an_activation(dtype, kind):
    """dz is rounded to the type: half a step of each term; a slope's own roundings, 2^-14 of |dy| at |z| < 8, are counted beside it."""
    M, N, K = 200, 136, 320
    rng = np.random.default_rng(kind)
    dy, x, w, z = (torch.from_numpy(rng.normal(size=s)).cuda().to(dtype) for s in ((M, N), (M, K), (N, K), (M, N)))
    d = [t.double().cpu().numpy() for t in (dy, x, w, z)]
    want = ref.linear_grad(*d, kind)
    dx, dw, db = torch.empty(M, K, dtype=dtype, device="cuda"), torch.empty(N, K, dtype=dtype, device="cuda"), torch.empty(N, device="cuda")
    kimad.kimad_linear_grad(dy, x, w, z=z, act=kind, dx=dx, dw=dw, db=db)
    dz = np.abs(d[0] * ref.slope(d[3], kind))
    off = HALF[dtype] * dz + 2.0 ** -14 * np.abs(d[0])
    for got, true, bound in ((dx, want[0], (off + N * 2.0 ** -23 * dz) @ np.abs(d[2])), (dw, want[1], (off + M * 2.0 ** -23 * dz).T @ np.abs(d[1]))):
        bound = bound + HALF[dtype] * (np.abs(true) + bound)
        assert (np.abs(got.double().cpu().numpy() - true) <= bound).all()
    assert (np.abs(db.double().cpu().numpy() - want[2]) <= (2.0 ** -14 * np.abs(d[0]) + M * 2.0 ** -24 * dz).sum(0)).all()


def test_each_gradient_alone():
    rng = np.random.default_rng(0)
    M, N, K = 140, 100, 72
    dy, x, w, z = whole(rng, (M, N), BF16), whole(rng, (M, K), BF16), whole(rng, (N, K), BF16), whole(rng, (M, N), BF16)
    dz = torch.where(z > 0, dy, 0).double()
    want = {"dx": (dz @ w.double()).to(BF16), "dw": (dz.t() @ x.double()).to(BF16), "db": dz.sum(0).float()}
    for some in itertools.chain.from_iterable(itertools.combinations(want, k) for k in (1, 2, 3)):
        out = {n: torch.full_like(want[n], float("nan")) for n in some}
        kimad.kimad_linear_grad(dy, x if "dw" in some else None, w if "dx" in some else None, z=z, act=ref.RELU, **out)
        assert all(torch.equal(out[n], want[n]) for n in some), some


def test_sums_over_nothing():
    nan = float("nan")
    x, w = torch.empty(5, 0, dtype=BF16, device="cuda"), torch.empty(7, 0, dtype=BF16, device="cuda")
    b, r = torch.arange(7, device="cuda").to(BF16) - 3, torch.ones(5, 7, dtype=BF16, device="cuda")
    for dtype in (BF16, F32):
        out = torch.full((5, 7), nan, dtype=dtype, device="cuda")
        kimad.kimad_linear(x, w, out, bias=b, residual=r, act=ref.RELU)
        assert torch.equal(out, (b.double().clamp(min=0) + r.double()).to(dtype))
    # no rows: the sums over rows are 0
    dw, db = torch.full((7, 8), nan, device="cuda"), torch.full((7,), nan, device="cuda")
    kimad.kimad_linear_grad(torch.empty(0, 7, dtype=BF16, device="cuda"), torch.empty(0, 8, dtype=BF16, device="cuda"), torch.empty(7, 8, dtype=BF16, device="cuda"),
                            dx=torch.empty(0, 8, dtype=BF16, device="cuda"), dw=dw, db=db)
    assert not dw.any() and not db.any()
    # no features out
    dx = torch.full((5, 8), nan, dtype=BF16, device="cuda")
    kimad.kimad_linear_grad(torch.empty(5, 0, dtype=BF16, device="cuda"), None, torch.empty(0, 8, dtype=BF16, device="cuda"), dx=dx)
    assert not dx.any()


def test_streams_and_graphs():
    """On a stream of its own behind other work there, and recorded: replayed on new inputs, with eager calls between the replays."""
    rng = np.random.default_rng(1)
    M, N, K = 200, 333, 4000                                               # parts of a sum, and operands laid out anew
    x, w, b = whole(rng, (M, K), BF16), whole(rng, (N, K), BF16), whole(rng, (N,), BF16)
    x2, w2 = buffer(x, 1)[0], buffer(w, 1)[0]
    out, out2 = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    dy = whole(rng, (M, N), BF16)
    dw, dw2 = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
    dx, dx2 = torch.empty(M, K, dtype=BF16, device="cuda"), torch.empty(M, K, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            big = big @ big * 1e-4
        x2.add_(1)
    kimad.kimad_linear(x2, w2, out, bias=b, stream=side)
    kimad.kimad_linear_grad(dy, x2, w2, dx=dx, dw=dw, stream=side)
    side.synchronize()
    x = x + 1

    def true():
        return (x.double() @ w.double().t() + b.double()).float(), (dy.double() @ w.double()).to(BF16), (dy.double().t() @ x.double()).float()

    for got, want in zip((out, dx, dw), true()):
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kimad.kimad_linear(x2, w2, out, bias=b)
        kimad.kimad_linear_grad(dy, x2, w2, dx=dx, dw=dw)
    for k in range(4):
        x, w = whole(rng, (M, K), BF16), whole(rng, (N, K), BF16)
        x2.copy_(x), w2.copy_(w), dy.copy_(whole(rng, (M, N), BF16))
        for t in (out, dx, dw):
            t.fill_(float("nan"))
        graph.replay()
        kimad.kimad_linear(x2, w2, out2, bias=b)
        kimad.kimad_linear_grad(dy, x2, w2, dx=dx2, dw=dw2)
        torch.cuda.synchronize()
        for got, eager, want in zip((out, dx, dw), (out2, dx2, dw2), true()):
            assert torch.equal(got, want) and torch.equal(eager, want), k
