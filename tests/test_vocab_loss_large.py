"""Softmax cross entropy from hidden rows (dgc_vocab_loss_*) at sizes and values far out."""
import pytest
import torch

from test_vocab_loss import _bind


@pytest.mark.gpu
def test_a_label_2_to_the_30_before_a_piece_is_a_label():
    """A vocabulary of 33 pieces of 2^25 words, the last from word 2^30 on: label 0 is 2^30 words before it.

    Both rows have the same hidden number, and only words near the vocabulary's end count, so that the rows'
    gradients differ at their labels alone.  The last words' probabilities are 1/4 each, exact in every type."""
    B = _bind()
    dt, V = torch.bfloat16, 2 ** 30 + 2 ** 25
    h, y = torch.ones(2, 1, dtype=dt, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    w, b = torch.zeros(V, 1, dtype=dt, device="cuda"), torch.full((V,), -float("inf"), dtype=dt, device="cuda")
    b[-4:], b[:2] = 0.0, -60.0
    w[-4:] = 3.0
    w[:2] = 5.0
    loss, d = torch.empty(2, device="cuda"), torch.tensor([1.0, 0.5], device="cuda")
    dh, dw, db = torch.full_like(h, 7.0), torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    B.vocab_loss_grad(h, w, y, d, loss, dh, dw, bias=b, dbias=db)
    # logits: 3 at the last four words, -55 at the labels; p = 1/4 and e^-58 / 4 (below every tolerance here)
    want = torch.tensor([[3.0 - 5.0], [0.5 * (3.0 - 5.0)]], device="cuda")
    assert torch.equal(dh.float(), want)
    for got in (dw[:, 0], db):
        assert bool((got[-4:].float() == 0.375).all())          # (1 + 0.5) / 4
        assert got[:2].tolist() == [-1.0, -0.5] and not bool(got[2:-4].any())
    assert bool(((loss.double() - (58 + 1.3862943611198906)).abs() <= 64 * 2.0 ** -22).all())
    B.tensor_check()
