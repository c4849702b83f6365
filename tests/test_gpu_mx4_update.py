"""The update of a round in 4 bits: a worker's side and the server's, bit for bit against the definition."""
import numpy as np
import pytest

from tests import operators_reference as ref

pytestmark = pytest.mark.gpu


def _kimad():
    import paper_2312_08053_amd as kimad
    return kimad


def _starts(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)


def _device(a, shift):
    """A float32 array on the device, `shift` elements into its allocation, with guards on both sides."""
    import torch
    buf = torch.full((len(a) + shift + 64,), 123.0, device="cuda")
    buf[shift:shift + len(a)] = torch.from_numpy(a)
    return buf, buf[shift:shift + len(a)]


def _bits(t):
    return t.cpu().numpy().view(np.uint32)


def _equal(got, want):
    """Equal bit for bit, any NaN like any other, both zeros alike."""
    got, want = np.asarray(got), np.asarray(want)
    return np.array_equal(got, want, equal_nan=True)


LAYERS = [[1], [127], [128], [129], [1, 1, 1, 1], [300, 5, 0, 0, 77, 128, 256, 1], [0, 10, 0], [127, 1, 128, 1, 127], [20000], [3000, 40001, 2, 5000],
          [3] * 700, [2] * 1500, [64] * 1030 + [5000]]


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("sizes", LAYERS, ids=lambda s: f"{len(s)}_{sum(s)}")
def test_update_and_server_copy(sizes, shift):
    import torch
    kimad = _kimad()
    rng = np.random.default_rng(len(sizes) + shift)
    starts = _starts(sizes)
    d, L = int(starts[-1]), len(sizes)
    scale = np.repeat(10.0 ** rng.uniform(-5, -1, L), sizes)
    g, h = ((rng.standard_t(3, d) * scale * f).astype(np.float32) for f in (1.0, 0.5))
    hat = (rng.normal(0, 1, d) * scale).astype(np.float32)
    x = rng.normal(0, 0.02, d).astype(np.float32)
    if d > 40:
        h[7] = g[7]                                                # nothing to send there
    words = kimad.kimad_mx4_update_words(L, d)
    assert words == d // 128 + L
    (g_buf, gd), (h_buf, hd), (hat_buf, hatd), (x_buf, xd) = (_device(a, s) for a, s in ((g, shift), (h, shift), (hat, (shift + 1) % 4), (x, shift)))
    codes = torch.full((words + 1, 64), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((words + 1,), -1, dtype=torch.int32, device="cuda")
    st = torch.from_numpy(starts).cuda()
    status = torch.full((1,), -99, dtype=torch.int32, device="cuda")
    kimad.kimad_mx4_compress_ef(gd, hd, st, codes, scales, status)
    want_codes, want_bytes, want_h = ref.update(g, h, starts)
    assert int(status.item()) == 0
    got_codes, got_bytes = ref.mx4_unpack(codes[:words].cpu().numpy().reshape(words, 64), _bits(scales)[:words][None, :])
    assert np.array_equal(got_bytes, want_bytes)
    assert np.array_equal(ref.without_minus_zero(got_codes), ref.without_minus_zero(want_codes))
    assert (codes[words] == 0xEE).all() and int(scales[words]) == -1
    assert np.array_equal(_bits(hd), want_h.view(np.uint32)), "estimator"
    assert np.array_equal(_bits(gd), g.view(np.uint32))
    # the server: the same addition, then the model's step
    gamma, w = 0.37, 0.83
    kimad.kimad_mx4_server_apply([(codes, scales)], [hatd], [w], st, d, xd, gamma, status)
    sent = ref.decode_update(want_codes, want_bytes, starts).astype(np.float32)
    want_hat = hat + sent
    want_x = (x.astype(np.float64) - gamma * (w * want_hat.astype(np.float64))).astype(np.float32)
    assert int(status.item()) == 0
    assert _equal(_bits(hatd), want_hat.view(np.uint32)), "server's copy"
    assert _equal(_bits(xd), want_x.view(np.uint32)), "model"
    for buf, s in ((g_buf, shift), (h_buf, shift), (hat_buf, (shift + 1) % 4), (x_buf, shift)):
        assert (buf[:s] == 123.0).all() and (buf[s + d:] == 123.0).all()


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 11, 16])
@pytest.mark.parametrize("with_model", [True, False])
def test_server_with_several_workers(M, with_model):
    import torch
    kimad = _kimad()
    rng = np.random.default_rng(M)
    sizes = [5000, 3, 260, 0, 9001]
    starts = _starts(sizes)
    d, L = int(starts[-1]), len(sizes)
    words = d // 128 + L
    st = torch.from_numpy(starts).cuda()
    updates, hats, want = [], [], []
    for m in range(M):
        c, b, _ = ref.update(rng.normal(0, 1, d).astype(np.float32), np.zeros(d, np.float32), starts)
        packed, _ = ref.mx4_pack(c, b)
        updates.append((torch.from_numpy(packed).cuda(), torch.from_numpy(_scale_words(b)).cuda()))
        u = rng.normal(0, 1, d).astype(np.float32)
        hats.append(torch.from_numpy(u.copy()).cuda())
        want.append(u + ref.decode_update(c, b, starts).astype(np.float32))
    x = rng.normal(0, 1, d).astype(np.float32)
    xd = torch.from_numpy(x.copy()).cuda() if with_model else None
    weights = rng.uniform(0, 1, M)
    kimad.kimad_mx4_server_apply(updates, hats, weights, st, d, xd, 0.01)
    for m in range(M):
        assert np.array_equal(_bits(hats[m]), want[m].view(np.uint32)), m
    if with_model:
        total = np.zeros(d)
        for m in range(M):
            total = total + weights[m] * want[m].astype(np.float64)
        assert np.array_equal(_bits(xd), (x.astype(np.float64) - 0.01 * total).astype(np.float32).view(np.uint32))


def _scale_words(byte):
    b = byte.astype(np.uint32)
    return (b[:, 0] | b[:, 1] << 8 | b[:, 2] << 16 | b[:, 3] << 24).view(np.int32)


def test_what_is_not_finite_stays_in_its_block():
    import torch
    kimad = _kimad()
    d = 1000
    starts = _starts([d])
    rng = np.random.default_rng(5)
    g, h = rng.normal(0, 1, d).astype(np.float32), np.zeros(d, np.float32)
    g[40], g[300], g[999] = np.inf, np.nan, -np.inf
    gd, hd, st = torch.from_numpy(g).cuda(), torch.from_numpy(h.copy()).cuda(), torch.from_numpy(starts).cuda()
    words = kimad.kimad_mx4_update_words(1, d)
    codes, scales = torch.empty(words, 64, dtype=torch.uint8, device="cuda"), torch.empty(words, dtype=torch.int32, device="cuda")
    kimad.kimad_mx4_compress_ef(gd, hd, st, codes, scales)
    _, _, want = ref.update(g, h, starts)
    assert np.isnan(want).sum() == 32 + 32 + 8
    assert _equal(hd.cpu().numpy(), want)
    hat = torch.zeros(d, device="cuda")
    kimad.kimad_mx4_server_apply([(codes, scales)], [hat], [1.0], st, d)
    assert _equal(hat.cpu().numpy(), want)


@pytest.mark.parametrize("starts", [[0, 10, 5, 100], [1, 10, 50, 100], [0, 10, 50, 99], [0, 10, 50, 101], [0, 1 << 40, 50, 100]])
def test_starts_that_do_not_fit_are_reported_and_nothing_is_written(starts):
    import torch
    kimad = _kimad()
    d = 100
    g, h, hat, x = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    st = torch.tensor(starts, dtype=torch.int64, device="cuda")
    words = kimad.kimad_mx4_update_words(3, d)
    codes, scales = torch.full((words, 64), 7, dtype=torch.uint8, device="cuda"), torch.full((words,), 7, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kimad.kimad_mx4_compress_ef(g, h, st, codes, scales, status)
    assert int(status.item()) == -10 and not h.any() and (codes == 7).all() and (scales == 7).all()
    status.zero_()
    kimad.kimad_mx4_server_apply([(codes, scales)], [hat], [1.0], st, d, x, 1.0, status)
    assert int(status.item()) == -10 and not hat.any() and not x.any()


def test_rounds_in_a_row_bring_the_estimator_to_the_gradient():
    """With g fixed, every round sends what the last one's rounding lost: the error falls by at least the worst case of a block
    (a rounding error of 1/4 of an element at most 2 of 8 parts of the largest) and worker and server stay equal."""
    import torch
    kimad = _kimad()
    d = 10007
    g = torch.randn(d, generator=torch.Generator().manual_seed(1)).cuda()
    h, hat = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    st = torch.tensor([0, 4001, d], dtype=torch.int64, device="cuda")
    words = kimad.kimad_mx4_update_words(2, d)
    codes, scales = torch.empty(words, 64, dtype=torch.uint8, device="cuda"), torch.empty(words, dtype=torch.int32, device="cuda")
    last = float((g - h).abs().max())
    for _ in range(6):
        kimad.kimad_mx4_compress_ef(g, h, st, codes, scales)
        kimad.kimad_mx4_server_apply([(codes, scales)], [hat], [1.0], st, d)
        now = float((g - h).abs().max())
        # the largest error of a block is at most 2 s (a value of 8 s sent as 6 s), s at most a quarter of its largest element
        assert now <= last / 2 + 1e-6
        last = now
        assert torch.equal(h, hat)


def test_update_recorded_into_a_graph():
    import torch
    kimad = _kimad()
    d = 5000
    st = torch.tensor([0, 1234, d], dtype=torch.int64, device="cuda")
    g, x = torch.randn(d, device="cuda"), torch.zeros(d, device="cuda")
    words = kimad.kimad_mx4_update_words(2, d)
    codes, scales = torch.empty(words, 64, dtype=torch.uint8, device="cuda"), torch.empty(words, dtype=torch.int32, device="cuda")
    h, hat = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")

    def work(h, hat, x):
        kimad.kimad_mx4_compress_ef(g, h, st, codes, scales)
        kimad.kimad_mx4_server_apply([(codes, scales)], [hat], [0.5], st, d, x, 0.1)

    graph = torch.cuda.CUDAGraph()
    work(h, hat, x)
    for t in (h, hat, x):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        work(h, hat, x)
    h2, hat2, x2 = (torch.zeros(d, device="cuda") for _ in range(3))
    for _ in range(3):
        graph.replay()
        work(h2, hat2, x2)
        torch.cuda.synchronize()
        assert torch.equal(h, h2) and torch.equal(hat, hat2) and torch.equal(x, x2)
        g.add_(0.25)


def _apart(n, shift, gen, scale):
    """Normal values times `scale`, `shift` elements into an allocation of their own."""
    import torch
    out = torch.empty(n + 8, device="cuda")[shift:shift + n]
    out.copy_(torch.randn(n, generator=gen, device="cuda") * scale)
    return out


# Layers on cache lines and buffers too large for the cache (384 MiB) go by nontemporal accesses; the same values an element further go by ordinary ones.
@pytest.mark.parametrize("M", [1, 3])
def test_large_sets_on_cache_lines_give_what_they_give_off_them(M):
    import torch
    kimad = _kimad()
    sizes = [32 * 5, 0, 128 * 1000, 32, 50_400_000, 32 * 77, 96 + 37]                 # the last word is partly filled
    starts = _starts(sizes)
    d, L = int(starts[-1]), len(sizes)
    assert (starts[:-1] % 32 == 0).all() and 8 * d > 384 << 20
    words = kimad.kimad_mx4_update_words(L, d)
    st = torch.from_numpy(starts).cuda()
    gen = torch.Generator(device="cuda").manual_seed(17 + M)
    scale = torch.repeat_interleave(torch.tensor([1.0, 1.0, 1e-3, 4.0, 0.1, 1e-5, 2.0], device="cuda"), torch.tensor(sizes, device="cuda"))
    g, h, x = (_apart(d, 0, gen, scale * f) for f in (1.0, 0.5, 0.1))
    hats = [_apart(d, 0, gen, scale) for _ in range(M)]
    for t in (g, h, x, *hats):
        assert t.data_ptr() % 128 == 0
    g[5], g[d - 1], g[3_000_000] = float("inf"), float("nan"), -float("inf")

    def off(t):
        return torch.empty(d + 8, device="cuda")[1:1 + d].copy_(t)

    g0, h0 = g[:400].cpu().numpy(), h[:400].cpu().numpy()
    tail = int(starts[-2])
    g1, h1 = g[tail:].cpu().numpy(), h[tail:].cpu().numpy()
    copies = off(g), off(h), off(x), [off(t) for t in hats]
    sent = []
    for gd, hd in ((g, h), copies[:2]):
        codes = torch.full((words, 64), 0xEE, dtype=torch.uint8, device="cuda")
        scales = torch.full((words,), -1, dtype=torch.int32, device="cuda")
        status = torch.full((1,), -99, dtype=torch.int32, device="cuda")
        kimad.kimad_mx4_compress_ef(gd, hd, st, codes, scales, status)
        assert int(status.item()) == 0
        sent.append((codes, scales))
    assert torch.equal(sent[0][0], sent[1][0]) and torch.equal(sent[0][1], sent[1][1])
    assert torch.equal(h.view(torch.int32), copies[1].clone().view(torch.int32))
    # the first layers and the last one by the definition
    _, _, want = ref.update(g0, h0, np.array([0, 160, 160, 400]))
    assert _equal(h[:160].cpu().numpy(), want[:160]) and _equal(h[160:384].cpu().numpy(), want[160:384])
    codes_t, bytes_t, want = ref.update(g1, h1, np.array([0, len(g1)]))
    assert _equal(h[tail:].cpu().numpy(), want)
    first = tail // 128 + L - 1
    got_codes, got_bytes = ref.mx4_unpack(sent[0][0][first:].cpu().numpy(), _bits(sent[0][1])[first:][None, :])
    assert np.array_equal(got_bytes[:2], bytes_t) and np.array_equal(ref.without_minus_zero(got_codes[:2]), ref.without_minus_zero(codes_t))
    # the server, of which every worker sent the same
    weights = [(1.0 + m) / 7 for m in range(M)]
    before = [t[tail:].cpu().numpy() for t in hats], x[tail:].cpu().numpy()
    kimad.kimad_mx4_server_apply([sent[0]] * M, hats, weights, st, d, x, 0.37)
    kimad.kimad_mx4_server_apply([sent[1]] * M, copies[3], weights, st, d, copies[2], 0.37)
    for a, b in zip([x, *hats], [copies[2], *copies[3]]):
        assert torch.equal(a.view(torch.int32), b.clone().view(torch.int32))
    q = ref.mx4_values(codes_t, bytes_t).reshape(-1)[:len(g1)].astype(np.float32)
    total = np.zeros(len(g1))
    for m in range(M):
        want = before[0][m] + q
        assert _equal(hats[m][tail:].cpu().numpy(), want)
        total = total + weights[m] * want.astype(np.float64)
    assert _equal(x[tail:].cpu().numpy(), (before[1].astype(np.float64) - 0.37 * total).astype(np.float32))
