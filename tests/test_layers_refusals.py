"""What the layers in front of a loss refuse, before anything reaches a device (no GPU needed)."""
import pytest

import paper_2312_08053_amd as kimad

OK, BAD, SMALL = 0, -1, -2
P = 0x10000                                                        # an address of the right alignment; nothing reads it
F32, F16, BF16 = 0, 1, 2
BIG = 1 << 40


def linear(x=P, ld_x=64, w=P, ld_w=64, kind=BF16, M=40, N=48, K=64, bias=0, res=0, ld_res=48, act=0, z=0, ld_z=48, out=P, out_kind=BF16, ld_out=48, ws=P, nbytes=0):
    return kimad.lib().kimad_linear(x, ld_x, w, ld_w, kind, M, N, K, bias, res, ld_res, act, z, ld_z, out, out_kind, ld_out, ws, nbytes, 0)


def linear_grad(dy=P, ld_dy=48, x=P, ld_x=64, w=P, ld_w=64, z=0, ld_z=48, kind=BF16, M=40, N=48, K=64, act=0, dx=P, ld_dx=64, dw=P, dw_kind=BF16, ld_dw=64, db=0, ws=P, nbytes=0):
    return kimad.lib().kimad_linear_grad(dy, ld_dy, x, ld_x, w, ld_w, z, ld_z, kind, M, N, K, act, dx, ld_dx, dw, dw_kind, ld_dw, db, ws, nbytes, 0)


def xent(x=P, ld_x=64, w=P, ld_w=64, kind=BF16, rows=40, vocab=100, dim=64, target=P, weight=0, loss=P, lse=0, dx=0, ld_dx=64, dw=0, dw_kind=BF16, ld_dw=64, ws=P, nbytes=0):
    return kimad.lib().kimad_linear_xent(x, ld_x, w, ld_w, kind, rows, vocab, dim, target, weight, loss, lse, dx, ld_dx, dw, dw_kind, ld_dw, ws, nbytes, 0)


def dropout(x=P, kind=F32, rows=4, cols=8, ld=8, res=0, ld_res=8, p=0.5, seed=1, offset=0, out=P, ld_out=8):
    return kimad.lib().kimad_dropout(x, kind, rows, cols, ld, res, ld_res, p, seed, offset, out, ld_out, 0)


@pytest.mark.parametrize("bad", [
    dict(kind=F32), dict(kind=3), dict(out_kind=F16), dict(out_kind=3), dict(act=4), dict(ld_x=63), dict(ld_w=63), dict(ld_out=47), dict(x=0), dict(w=0), dict(out=0),
    dict(x=P + 1), dict(w=P + 1), dict(out=P + 1), dict(out=P + 2, out_kind=F32), dict(bias=P + 1), dict(res=P + 1), dict(res=P, ld_res=47), dict(z=P + 1), dict(z=P, ld_z=47),
    dict(M=4194241), dict(ld_x=(1 << 22) + 1), dict(ld_out=(1 << 24) + 1), dict(N=(1 << 22) + 1, ld_out=1 << 23), dict(M=1 << 20, N=1 << 13, ld_out=1 << 13)])
def test_linear_refuses(bad):
    assert linear(**bad) == BAD


def test_linear_asks_for_its_workspace():
    need = kimad.lib().kimad_linear_workspace_bytes
    assert need(P, 64, P, 64, 40, 48, 64) == 0
    assert need(P, 65, P, 65, 200, 48, 65) == -(-2 * 200 * 72 // 256) * 256 + -(-2 * 48 * 72 // 256) * 256      # both laid out anew
    assert need(P + 2, 64, P, 64, 200, 48, 64) == 2 * 200 * 64                                                  # one of them
    assert need(P + 2, 65, P, 65, 32, 48, 65) == 0                                                              # few rows: read as they lie
    assert linear(x=P + 2, M=200) == SMALL and linear(x=P + 2, M=200, ws=0, nbytes=BIG) == SMALL and linear(x=P + 2, M=200, ws=P + 8, nbytes=BIG) == SMALL
    assert linear(M=0) == OK and linear(N=0) == OK and linear(M=0, x=0, out=0, w=0) == BAD and linear(M=0, x=0, out=0) == OK


@pytest.mark.parametrize("bad", [
    dict(kind=F32), dict(dw_kind=F16), dict(act=4), dict(act=1), dict(act=1, z=P + 1), dict(act=1, z=P, ld_z=47), dict(dy=0), dict(dy=P + 1), dict(ld_dy=47), dict(x=0), dict(w=0),
    dict(dx=P + 1), dict(dw=P + 1), dict(dw=P + 2, dw_kind=F32), dict(db=P + 2), dict(ld_dx=63), dict(ld_dw=63), dict(M=4194241), dict(ld_dy=(1 << 22) + 1)])
def test_linear_grad_refuses(bad):
    assert linear_grad(**bad) == BAD


def test_linear_grad_asks_for_its_workspace():
    need = kimad.lib().kimad_linear_grad_workspace_bytes
    assert need(P, 48, P, 64, P, 64, 40, 48, 64, 0, 7) == 0
    assert need(P, 48, P, 64, P, 64, 40, 48, 64, 1, 1) == 2 * 40 * 48                                           # dz
    assert need(P, 48, P, 64, P, 64, 40, 48, 64, 1, 4) == 0                                                     # the bias alone
    assert need(P, 48, P, 64, P, 64, 400, 48, 64, 0, 4) == 7 * 4 * 48 + 192                                     # sums of 64 rows each, in whole 256 bytes
    assert linear_grad(act=1, z=P) == SMALL and linear_grad(act=1, z=P, ws=P + 8, nbytes=BIG) == SMALL
    assert linear_grad(x=0, dw=0, ws=0, dx=0, w=0) == OK                                                        # nothing wanted


@pytest.mark.parametrize("bad", [
    dict(kind=F32), dict(dw=P, dw_kind=F16), dict(vocab=0), dict(vocab=(1 << 22) - 63), dict(dim=0, ld_x=64), dict(ld_x=63), dict(ld_w=63), dict(x=0), dict(w=0), dict(x=P + 1),
    dict(target=0), dict(target=P + 2), dict(weight=P + 2), dict(loss=P + 2), dict(lse=P + 2), dict(dx=P + 1), dict(dx=P, ld_dx=63), dict(dw=P + 1), dict(dw=P, ld_dw=63),
    dict(dw=P + 2, dw_kind=F32), dict(rows=4194241), dict(loss=0)])
def test_cross_entropy_refuses(bad):
    assert xent(**bad, nbytes=BIG) == BAD


def test_cross_entropy_asks_for_its_workspace():
    need = kimad.lib().kimad_linear_xent_workspace_bytes(P, 64, P, 64, BF16, 40, 100, 64, 0, BF16)
    assert need > 0
    assert xent(nbytes=need - 1) == SMALL and xent(ws=0, nbytes=need) == SMALL and xent(ws=P + 8, nbytes=need) == SMALL
    assert xent(rows=0, x=0, target=0, loss=0) == OK and kimad.lib().kimad_linear_xent_workspace_bytes(P, 64, P, 64, BF16, 0, 100, 64, 0, BF16) == 0
    # what a gradient keeps is bounded, however many rows there are: 1 GiB of exponentials, and what goes by rows
    for rows in (8192, 1 << 20):
        assert kimad.lib().kimad_linear_xent_workspace_bytes(P, 768, P, 768, BF16, rows, 50257, 768, 3, BF16) < (1 << 30) + rows * 768 * 2 + 50257 * 768 * 4 + (1 << 28)


@pytest.mark.parametrize("bad", [
    dict(kind=3), dict(x=0), dict(out=0), dict(x=P + 2), dict(out=P + 2), dict(x=P + 1, kind=BF16), dict(ld=7), dict(ld_out=7), dict(res=P, ld_res=7), dict(res=P + 2), dict(p=-0.1),
    dict(p=1.1), dict(p=float("nan")), dict(rows=1 << 20, cols=1 << 15, ld=1 << 15, ld_out=1 << 15), dict(rows=1 << 33, cols=1 << 31, ld=1 << 31, ld_out=1 << 31)])
def test_dropout_refuses(bad):
    assert dropout(**bad) == BAD


def test_dropout_of_nothing():
    assert dropout(rows=0, x=0, out=0) == OK and dropout(cols=0, x=0, out=0) == OK


def test_the_binding_refuses_what_it_cannot_pass():
    import torch
    bf, f = torch.bfloat16, torch.float32
    x, w, y = torch.zeros(4, 8, dtype=bf), torch.zeros(6, 8, dtype=bf), torch.zeros(4, 6, dtype=bf)
    for error, call in [
            (ValueError, lambda: kimad.kimad_linear(x, w, y)),                                         # host memory
            (TypeError, lambda: kimad.kimad_linear(x.float(), w.float(), y)),
            (ValueError, lambda: kimad.kimad_linear(x, w.half(), y)),
            (ValueError, lambda: kimad.kimad_linear(x, w[:, :7], y)),
            (ValueError, lambda: kimad.kimad_linear(x, w, y.half())),
            (ValueError, lambda: kimad.kimad_linear(x, w, y[:, :5])),
            (ValueError, lambda: kimad.kimad_linear(x, w, y.t())),
            (ValueError, lambda: kimad.kimad_linear(x, w, y, bias=torch.zeros(6))),
            (ValueError, lambda: kimad.kimad_linear(x, w, y, bias=torch.zeros(7, dtype=bf))),
            (ValueError, lambda: kimad.kimad_linear(x, w, y, residual=y.float())),
            (ValueError, lambda: kimad.kimad_linear(x, w, y, z=y.float())),
            (ValueError, lambda: kimad.kimad_linear_grad(y, x, w, dx=x, dw=w.half())),
            (ValueError, lambda: kimad.kimad_linear_grad(y, None, w, dw=w)),
            (ValueError, lambda: kimad.kimad_linear_grad(y, x, None, dx=x)),
            (ValueError, lambda: kimad.kimad_linear_grad(y, x, w, act=1, dx=x)),
            (ValueError, lambda: kimad.kimad_linear_grad(y, x, w, db=torch.zeros(6, dtype=bf))),
            (ValueError, lambda: kimad.kimad_linear_xent(x, w, torch.zeros(4, dtype=torch.int64), loss=torch.zeros(4))),
            (ValueError, lambda: kimad.kimad_linear_xent(x, w, torch.zeros(3, dtype=torch.int32), loss=torch.zeros(4))),
            (ValueError, lambda: kimad.kimad_linear_xent(x, w, torch.zeros(4, dtype=torch.int32), dx=x.float())),
            (TypeError, lambda: kimad.kimad_linear_xent(x.float(), w.float(), torch.zeros(4, dtype=torch.int32), loss=torch.zeros(4))),
            (ValueError, lambda: kimad.kimad_dropout(x, x.float(), 0.5, 1)),
            (ValueError, lambda: kimad.kimad_dropout(x, x, 0.5, -1)),
            (ValueError, lambda: kimad.kimad_dropout(x, x, 0.5, 1 << 64)),
            (TypeError, lambda: kimad.kimad_dropout(x.double(), x.double(), 0.5, 1))]:
        with pytest.raises(error):
            call()
