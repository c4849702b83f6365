"""What the operators beside a round refuse, before anything reaches a device (no GPU needed)."""
import ctypes as C

import pytest

import paper_2312_08053_amd as kimad

BAD, SMALL = -1, -2
P = 0x10000                                                        # an address of the right alignment; nothing reads it


def test_quantise_refuses():
    f = kimad.lib().kimad_mx4_quantise
    assert f(P, 3, 4, 4, 4, P, P, 0, 0, 0) == BAD                  # unknown type
    assert f(P, 0, 4, 8, 7, P, P, 0, 0, 0) == BAD                  # rows overlap
    assert f(P, 0, 4, 4, 4, 0, 0, 0, 0, 0) == BAD                  # nothing wanted
    assert f(P, 0, 4, 4, 4, P, 0, 0, 0, 0) == BAD                  # codes without scales
    assert f(P, 0, 4, 4, 4, P + 8, P, 0, 0, 0) == BAD              # alignment
    assert f(P, 0, 4, 4, 4, P, P + 2, 0, 0, 0) == BAD
    assert f(P + 2, 0, 4, 4, 4, P, P, 0, 0, 0) == BAD
    assert f(P + 1, 2, 4, 4, 4, P, P, 0, 0, 0) == BAD
    assert f(0, 0, 4, 4, 4, P, P, 0, 0, 0) == BAD
    assert f(P, 0, 1 << 41, 4, 4, P, P, 0, 0, 0) == BAD
    assert f(0, 0, 0, 4, 4, P, P, 0, 0, 0) == 0                    # no rows: nothing to do


def test_dequantise_refuses():
    f = kimad.lib().kimad_mx4_dequantise
    assert f(P, P, 4, 4, P, 5, 4, 0) == BAD
    assert f(P, P, 4, 4, P, 0, 3, 0) == BAD
    assert f(0, P, 4, 4, P, 0, 4, 0) == BAD
    assert f(P, P, 4, 4, 0, 0, 4, 0) == BAD
    assert f(P + 4, P, 4, 4, P, 0, 4, 0) == BAD
    assert f(P, P, 4, 4, P + 1, 1, 4, 0) == BAD
    assert f(P, P, 4, 0, P, 0, 0, 0) == 0


def test_matmul_refuses():
    f = kimad.lib().kimad_mx4_matmul
    assert f(P, P, 4, P, P, 4, 4, P, 3, 4, 0, 0, 0) == BAD
    assert f(P, P, 4, P, P, 4, 4, P, 0, 3, 0, 0, 0) == BAD
    assert f(0, P, 4, P, P, 4, 4, P, 0, 4, 0, 0, 0) == BAD
    assert f(P, P, 4, P, 0, 4, 4, P, 0, 4, 0, 0, 0) == BAD
    assert f(P, P, 4, P, P, 4, 4, 0, 0, 4, 0, 0, 0) == BAD
    assert f(P, P, 4, P + 4, P, 4, 4, P, 0, 4, 0, 0, 0) == BAD
    assert f(P, P, 4, P, P, 4, 4, P, 0, 4, P + 4, 64, 0) == BAD    # workspace alignment
    assert f(P, P, 0, P, P, 4, 4, P, 0, 4, 0, 0, 0) == 0


def test_update_and_server_refuse():
    f = kimad.lib().kimad_mx4_compress_ef
    assert f(0, P, P, 1, 4, P, P, 0, 0) == BAD
    assert f(P, 0, P, 1, 4, P, P, 0, 0) == BAD
    assert f(P, P, 0, 1, 4, P, P, 0, 0) == BAD
    assert f(P, P, P, 0, 4, P, P, 0, 0) == BAD
    assert f(P, P, P, 1, 0, P, P, 0, 0) == BAD
    assert f(P, P, P, 1, 4, 0, 0, 0, 0) == BAD
    assert f(P, P, P, 1, 4, P, 0, 0, 0) == BAD
    assert f(P + 2, P, P, 1, 4, P, P, 0, 0) == BAD
    assert kimad.kimad_mx4_update_words(3, 1000) == 10
    from paper_2312_08053_amd.binding import _Mx4Update
    s = kimad.lib().kimad_mx4_server_apply
    up, bad, hat, w = (_Mx4Update * 1)(_Mx4Update(P, P)), (_Mx4Update * 1)(_Mx4Update(P, 0)), (C.c_void_p * 1)(P), (C.c_double * 1)(1.0)
    none = (C.c_void_p * 1)(0)
    assert s(up, hat, w, 0, P, 1, 4, 0, 0.0, 0, 0) == BAD
    assert s(up, hat, w, 17, P, 1, 4, 0, 0.0, 0, 0) == BAD
    assert s(bad, hat, w, 1, P, 1, 4, 0, 0.0, 0, 0) == BAD
    assert s(up, none, w, 1, P, 1, 4, 0, 0.0, 0, 0) == BAD
    assert s(up, hat, w, 1, 0, 1, 4, 0, 0.0, 0, 0) == BAD
    assert s(up, hat, w, 1, P, 1, 4, P + 2, 0.0, 0, 0) == BAD


def test_distillation_refuses():
    f = kimad.lib().kimad_distill

    def call(logits=P, kind=0, rows=4, vocab=100, ld=100, idx=P, val=P, k=8, T=1.0, weight=0, loss=P, stats=0, grad=0, ld_grad=0, ws=0, nbytes=0):
        return f(logits, kind, rows, vocab, ld, idx, val, k, T, weight, loss, stats, grad, ld_grad, ws, nbytes, 0)

    for bad in (dict(kind=3), dict(vocab=0), dict(vocab=1 << 31, ld=1 << 31), dict(ld=99), dict(k=1025), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")),
                dict(T=float("inf")), dict(T=1e-9), dict(logits=0), dict(idx=0), dict(val=0), dict(loss=0), dict(grad=P, ld_grad=99), dict(logits=P + 2),
                dict(grad=P + 2, ld_grad=100)):
        assert call(**bad) == BAD, bad
    assert call(rows=0, logits=0) == 0
    need = kimad.kimad_distill_workspace_bytes(1, 200000, 8)
    assert need > 0
    assert call(rows=1, vocab=200000, ld=200000) == SMALL
    assert call(rows=1, vocab=200000, ld=200000, ws=P, nbytes=need - 1) == SMALL
    g = kimad.lib().kimad_distill_grad
    assert g(P, 0, 4, 100, 100, P, P, 8, 1.0, 0, 0, P, 100, 0) == BAD
    assert g(P, 0, 4, 100, 100, P, P, 8, 1.0, 0, P, 0, 100, 0) == BAD


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    x = torch.zeros(4, 100)
    codes, scales = kimad.mx4_empty(4, 100, "cpu")
    with pytest.raises(ValueError):
        kimad.kimad_mx4_quantise(x.t(), codes, scales, stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_mx4_quantise(torch.zeros(4, 200), codes, scales, stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_mx4_quantise(torch.zeros(100), codes, scales, stream=0)
    with pytest.raises(TypeError):
        kimad.kimad_mx4_quantise(x.double(), codes, scales, stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_mx4_matmul(codes, scales, codes, scales, 200, torch.zeros(4, 4), stream=0)
    idx, val = torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    with pytest.raises(ValueError):
        kimad.kimad_distill(x, idx[:3], val, 1.0, loss=torch.zeros(4), stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_distill(x, idx, val, 1.0, loss=torch.zeros(3), stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_distill(x, idx.long(), val, 1.0, loss=torch.zeros(4), stream=0)
    with pytest.raises(ValueError):
        kimad.kimad_distill(x, idx, val, 1.0, grad=torch.zeros(4, 99), stream=0)


def test_the_binding_refuses_host_memory():
    import torch
    x, idx, val = torch.zeros(4, 128), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    codes, scales = kimad.mx4_empty(4, 128, "cpu")
    starts, flat = torch.tensor([0, 512]), torch.zeros(512)
    up = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    for call in (lambda: kimad.kimad_mx4_quantise(x, codes, scales, stream=0),
                 lambda: kimad.kimad_mx4_dequantise(codes, scales, x, stream=0),
                 lambda: kimad.kimad_mx4_matmul(codes, scales, codes, scales, 128, torch.zeros(4, 4), stream=0),
                 lambda: kimad.kimad_distill(x, idx, val, 1.0, loss=torch.zeros(4), stream=0),
                 lambda: kimad.kimad_distill_grad(x, idx, val, 1.0, torch.zeros(4, 2), torch.zeros(4, 128), stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat, flat.clone(), starts, *up, stream=0),
                 lambda: kimad.kimad_mx4_server_apply([up], [flat], [1.0], starts, 512, stream=0)):
        with pytest.raises(ValueError, match="device tensors are wanted"):
            call()


def test_the_workspace_of_any_product_is_told():
    for K in (0, 1, 128, 129, 5000, 1 << 25, (1 << 25) + 1):
        for M in (0, 1, 32, 33, 64, 65, 1000, 100000, 1 << 40, (1 << 40) + 1):
            for N in (0, 1, 70, 50257, 1 << 24):
                need = kimad.kimad_mx4_matmul_workspace_bytes(M, N, K)
                assert need % 4 == 0 and (need == 0 or (K > 0 and need >= 8 * M * N))


def test_more_threads_than_a_launch_holds_are_refused():
    L = kimad.lib()
    assert L.kimad_mx4_quantise(P, 0, 1 << 29, 4, 4, P, P, 0, 0, 0) == BAD
    assert L.kimad_mx4_dequantise(P, P, 1 << 29, 4, P, 0, 4, 0) == BAD
    assert L.kimad_mx4_matmul(P, P, 1 << 30, P, P, 1 << 20, 0, P, 0, 1 << 20, 0, 0, 0) == BAD
    assert L.kimad_mx4_matmul(P, P, 1 << 40, P, P, 1 << 24, 0, P, 0, 1 << 24, 0, 0, 0) == BAD
    for rows, vocab in ((1 << 30, 100), (1 << 23, 40000), (1 << 22, 65000)):
        assert L.kimad_distill(P, 0, rows, vocab, vocab, P, P, 8, 1.0, 0, P, 0, 0, 0, 0, 0, 0) == BAD, (rows, vocab)
    assert L.kimad_distill(P, 0, 1 << 20, 1 << 20, 1 << 20, P, P, 8, 1.0, 0, P, 0, 0, 0, P, 1 << 60, 0) == BAD
    assert L.kimad_distill_grad(P, 0, 1 << 25, 100, 100, P, P, 8, 1.0, 0, P, P, 100, 0) == BAD


def test_more_layers_than_the_kernels_count_are_refused():
    from paper_2312_08053_amd.binding import _Mx4Update
    L = kimad.lib()
    up, hat, w = (_Mx4Update * 1)(_Mx4Update(P, P)), (C.c_void_p * 1)(P), (C.c_double * 1)(1.0)
    for layers in (1 << 31, (1 << 32) - 256, (1 << 32) - 1):
        assert L.kimad_mx4_compress_ef(P, P, P, layers, 4, P, P, 0, 0) == BAD, layers
        assert L.kimad_mx4_server_apply(up, hat, w, 1, P, layers, 4, 0, 0.0, 0, 0) == BAD, layers


def test_a_distillation_of_no_rows_has_nothing_to_do():
    L = kimad.lib()                                                # empty tensors have no address
    assert L.kimad_distill(0, 0, 0, 100, 100, 0, 0, 8, 1.0, 0, 0, 0, 0, 0, 0, 0, 0) == 0
    assert L.kimad_distill_grad(0, 0, 0, 100, 100, 0, 0, 8, 1.0, 0, 0, 0, 100, 0) == 0
    assert L.kimad_distill(0, 3, 0, 100, 100, 0, 0, 8, 1.0, 0, 0, 0, 0, 0, 0, 0, 0) == BAD
    assert L.kimad_distill(P, 0, 1, 100, 100, P, P, 8, 1.0, 0, 0, 0, 0, 0, 0, 0, 0) == BAD


def test_arrays_that_are_not_aligned_like_their_elements_are_refused():
    from paper_2312_08053_amd.binding import _Mx4Update
    L = kimad.lib()
    names = ("idx", "val", "weight", "loss", "stats")
    for off in names:
        at = {n: P + 2 * (n == off) for n in names}
        assert L.kimad_distill(P, 0, 4, 100, 100, at["idx"], at["val"], 8, 1.0, at["weight"], at["loss"], at["stats"], 0, 0, 0, 0, 0) == BAD, off
        if off != "loss":
            assert L.kimad_distill_grad(P, 0, 4, 100, 100, at["idx"], at["val"], 8, 1.0, at["weight"], at["stats"], P, 100, 0) == BAD, off
    assert L.kimad_mx4_compress_ef(P, P, P + 4, 1, 4, P, P, 0, 0) == BAD
    assert L.kimad_mx4_compress_ef(P, P, P, 1, 4, P, P, P + 1, 0) == BAD
    up, hat, w = (_Mx4Update * 1)(_Mx4Update(P, P)), (C.c_void_p * 1)(P), (C.c_double * 1)(1.0)
    assert L.kimad_mx4_server_apply(up, hat, w, 1, P + 4, 1, 4, 0, 0.0, 0, 0) == BAD
    assert L.kimad_mx4_server_apply(up, hat, w, 1, P, 1, 4, 0, 0.0, P + 2, 0) == BAD


def test_a_quantisation_beyond_the_header_s_limits_is_refused():
    L = kimad.lib()
    for cols, rows, pairs in ((2147483520, 8388480, (P, P, P, P)), (2147483520, 8388480, (0, 0, P, P)), (67107840, 268435440, (P, P, 0, 0))):
        assert L.kimad_mx4_quantise(P, 0, 1, cols + 1, cols + 1, *pairs, 0) == BAD
        assert L.kimad_mx4_quantise(P, 0, rows + 1, 1, 1, *pairs, 0) == BAD
    assert L.kimad_mx4_dequantise(P, P, 1, 67107841, P, 0, 67107841, 0) == BAD
    assert L.kimad_mx4_dequantise(P, P, 268435441, 1, P, 0, 1, 0) == BAD


def test_the_binding_refuses_parts_of_a_quantised_matrix_that_are_none():
    import torch
    codes, scales = kimad.mx4_empty(100, 512, "cpu")
    other, other_scales = kimad.mx4_empty(70, 512, "cpu")
    out, product = torch.zeros(100, 512), torch.zeros(100, 70)
    for call in (lambda: kimad.kimad_mx4_dequantise(codes[:50], scales, out[:50], stream=0),               # scales of 100 rows
                 lambda: kimad.kimad_mx4_dequantise(codes, scales, out[:50], stream=0),
                 lambda: kimad.kimad_mx4_dequantise(codes, scales, out[:, :128], stream=0),                # fewer words a row
                 lambda: kimad.kimad_mx4_dequantise(codes.view(50, 512), scales.view(8, 50), out[:50], stream=0),
                 lambda: kimad.kimad_mx4_quantise(out[:50], codes, scales, stream=0),
                 lambda: kimad.kimad_mx4_quantise(out[:, :300], codes, scales, stream=0),
                 lambda: kimad.kimad_mx4_quantise(out, None, None, codes, scales, stream=0),                # the transpose's shape is another
                 lambda: kimad.kimad_mx4_matmul(codes, scales, other, other_scales, 128, product, stream=0),   # K of another quantisation
                 lambda: kimad.kimad_mx4_matmul(codes[:50], scales, other, other_scales, 512, product[:50], stream=0),
                 lambda: kimad.kimad_mx4_matmul(codes, scales, other, other_scales, 512, product[:, :60], stream=0)):
        with pytest.raises(ValueError, match="shapes"):
            call()
    for pairs in ((codes, None), (None, scales), (codes, scales, codes, None), (None, None, None, scales)):
        with pytest.raises(ValueError, match="together"):
            kimad.kimad_mx4_quantise(out, *pairs, stream=0)
    # as much as is wanted: what is refused then is that it is host memory
    for call in (lambda: kimad.kimad_mx4_dequantise(codes, scales, out[:, :390], stream=0),
                 lambda: kimad.kimad_mx4_dequantise(torch.zeros(90000, dtype=torch.uint8), torch.zeros(1000, dtype=torch.int32), out, stream=0),
                 lambda: kimad.kimad_mx4_matmul(codes, scales, other, other_scales, 400, product, stream=0)):
        with pytest.raises(ValueError, match="device tensors are wanted"):
            call()


def test_the_binding_refuses_other_types_of_the_same_size():
    import torch
    x, idx, val = torch.zeros(4, 128), torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 3)
    codes, scales = kimad.mx4_empty(4, 128, "cpu")
    starts, flat = torch.tensor([0, 512]), torch.zeros(512)
    up = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    whole, row, stats = torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(4, 2)
    for call in (lambda: kimad.kimad_distill(x, val, val, 1.0, loss=row, stream=0),                        # entries' numbers as floats
                 lambda: kimad.kimad_distill(x, idx, idx, 1.0, loss=row, stream=0),
                 lambda: kimad.kimad_distill(x, idx, val, 1.0, loss=whole, stream=0),
                 lambda: kimad.kimad_distill(x, idx, val, 1.0, stats=stats.int(), stream=0),
                 lambda: kimad.kimad_distill(x, idx, val, 1.0, loss=row, row_weight=whole, stream=0),
                 lambda: kimad.kimad_distill_grad(x, idx, val, 1.0, stats.int(), x.clone(), stream=0),
                 lambda: kimad.kimad_mx4_quantise(x, codes.bool(), scales, stream=0),
                 lambda: kimad.kimad_mx4_quantise(x, codes, scales.float(), stream=0),
                 lambda: kimad.kimad_mx4_dequantise(codes, scales.float(), x, stream=0),
                 lambda: kimad.kimad_mx4_matmul(codes, scales, codes.bool(), scales, 128, torch.zeros(4, 4), stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat.int(), flat, starts, *up, stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat, flat.int(), starts, *up, stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat, flat, starts.double(), *up, stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat, flat, starts, up[0].bool(), up[1], stream=0),
                 lambda: kimad.kimad_mx4_compress_ef(flat, flat, starts, up[0], up[1].float(), stream=0),
                 lambda: kimad.kimad_mx4_server_apply([up], [flat.int()], [1.0], starts, 512, stream=0),
                 lambda: kimad.kimad_mx4_server_apply([up], [flat], [1.0], starts.double(), 512, stream=0),
                 lambda: kimad.kimad_mx4_server_apply([up], [flat], [1.0], starts, 512, flat.int(), stream=0)):
        with pytest.raises(ValueError, match="contiguous elements of"):
            call()
    # whole numbers without a sign are the same numbers
    with pytest.raises(ValueError, match="device tensors are wanted"):
        kimad.kimad_mx4_compress_ef(flat, flat.clone(), starts.to(torch.uint64), up[0], up[1].view(torch.uint32), stream=0)


def test_the_binding_refuses_a_status_that_is_no_int32():
    import torch
    starts, flat = torch.tensor([0, 512]), torch.zeros(512)
    up = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    for status in (torch.zeros(1, dtype=torch.uint8), torch.zeros(0, dtype=torch.int32), torch.zeros(1), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(ValueError, match="status_out"):
            kimad.kimad_mx4_compress_ef(flat, flat.clone(), starts, *up, status, stream=0)
        with pytest.raises(ValueError, match="status_out"):
            kimad.kimad_mx4_server_apply([up], [flat], [1.0], starts, 512, None, 0.0, status, stream=0)


def test_the_binding_refuses_a_workspace_with_less_memory_than_elements_or_gaps():
    import torch
    a, sa = kimad.mx4_empty(100, 16384, "cpu")
    x, idx, val = torch.zeros(2, 70001), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    for ws in (torch.zeros(1).expand(1 << 20), torch.zeros(1 << 12, 2)[:, 0]):
        with pytest.raises(ValueError, match="workspace"):
            kimad.kimad_mx4_matmul(a, sa, a, sa, 16384, torch.zeros(100, 100), workspace=ws, stream=0)
        with pytest.raises(ValueError, match="workspace"):
            kimad.kimad_distill(x, idx, val, 1.0, loss=torch.zeros(2), workspace=ws, stream=0)


class _Elsewhere:
    """As much of a tensor as is asked where its memory is."""

    def __init__(self, device):
        self.index, self.shape, self.device, self.is_cuda = device, (4, 4), f"cuda:{device}", device >= 0

    def get_device(self):
        return self.index


def test_the_binding_refuses_memory_of_another_device(monkeypatch):
    import torch
    from paper_2312_08053_amd import binding
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    here, there = _Elsewhere(1), _Elsewhere(0)
    with pytest.raises(ValueError, match="one device"):
        binding._on_device(0, here, None, there)
    with pytest.raises(ValueError, match="current device"):
        binding._on_device(0, there, there)
    assert binding._on_device(0, here, None, here) == 0
    assert binding._on_device(0x1234, there, there) == 0x1234      # a stream of that device, for all that a handle tells
    with pytest.raises(ValueError, match="device tensors"):
        binding._on_device(0, here, _Elsewhere(-1))


def test_the_binding_takes_either_part_of_a_quantised_matrix_flat():
    import torch
    codes, scales = kimad.mx4_empty(100, 512, "cpu")
    out = torch.zeros(100, 512)
    for pair in ((codes, scales), (codes.view(-1), scales), (codes, scales.view(-1)), (codes.view(-1), scales.view(-1))):
        with pytest.raises(ValueError, match="device tensors are wanted"):       # all that is wrong with them
            kimad.kimad_mx4_dequantise(*pair, out, stream=0)
    for pair in ((codes.view(-1)[1:], scales), (codes, scales.view(-1)[1:])):
        with pytest.raises(ValueError, match="contiguous elements of"):
            kimad.kimad_mx4_dequantise(*pair, out, stream=0)
