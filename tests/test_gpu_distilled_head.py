"""The operators together, as the example runs them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _values(form, rows, cols):
    import torch
    import paper_2312_08053_amd as kimad
    out = torch.empty(rows, cols, device="cuda")
    kimad.kimad_mx4_dequantise(*form, out)
    return out.double()


def test_a_head_learns_and_both_sides_agree():
    import torch
    from examples import distilled_head as ex
    torch.manual_seed(0)
    head = ex.Head(1003, 200, step=4.0)
    batch = ex.teacher_batch(300, 200, 1003, 8)
    losses = []
    for _ in range(8):
        loss, dx = head.round(*batch)
        losses.append(float(loss.sum()))
        assert torch.equal(head.h, head.server_h) and int(head.status.item()) == 0
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0], losses
    assert (loss[batch[3] == 0] == 0).all() and not dx[batch[3] == 0].any()


def test_gradients_are_those_of_the_quantised_head():
    """Loss, dX and dW against 64 bits on the quantised operands.  The logits are rounded to bfloat16 (2^-9 of the largest, some 2^-9 * 2, enters a
    probability by as much), and the rounding of dZ to bfloat16 may put an element on the other side of a 4-bit step, which moves a sum by
    up to a quarter of its block's largest element: the comparison is of whole matrices, in the 2-norm."""
    import torch
    from examples import distilled_head as ex
    torch.manual_seed(1)
    tokens, hidden, vocab = 200, 150, 900
    head = ex.Head(vocab, hidden)
    x, idx, val, weight = ex.teacher_batch(tokens, hidden, vocab, 6)
    loss, dx, dw = head.gradients(x, idx, val, weight)
    x_rows, x_cols = ex.both_forms(x)
    w_rows, w_cols = ex.both_forms(head.weights)
    T = head.temperature
    z = _values(x_rows, tokens, hidden) @ _values(w_rows, vocab, hidden).t().contiguous() / T
    p = torch.softmax(val.double() / T, 1)
    log_q = torch.log_softmax(z, 1)
    w = weight.double()
    want_loss = w * T * T * (p * (p.log() - log_q.gather(1, idx.long()))).sum(1)
    assert torch.allclose(loss.double(), want_loss, rtol=1e-2, atol=1e-6)
    dz = (w * T)[:, None] * torch.exp(log_q).scatter_add(1, idx.long(), -p)
    z_rows, z_cols = ex.both_forms(dz.to(torch.bfloat16))
    want_dx = _values(z_rows, tokens, vocab) @ _values(w_cols, hidden, vocab).t().contiguous()
    want_dw = _values(z_cols, vocab, tokens) @ _values(x_cols, hidden, tokens).t().contiguous()
    for got, want in ((dx, want_dx), (dw, want_dw)):
        assert float((got.double() - want).norm() / want.norm()) < 0.05
