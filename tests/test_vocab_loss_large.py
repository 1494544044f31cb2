"""Softmax cross entropy from hidden rows (dgc_vocab_loss_*) at sizes and values far out."""
import pytest
import torch

from test_vocab_loss import DT, _bind, _check


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


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("R,V,D", [(40, 500, 8200), (3, 270, 65536)])
def test_long_hidden_rows(R, V, D, dt):
    """Sums of many terms: the bounds count 2^-23 for each (a tensor core's additions cut off), to the longest row there is."""
    _check(R, V, D, dt, bias=True)


def test_the_workspace_is_what_the_header_says():
    """Host only.  8 bytes for 128 logits (64 in 32 bits) or a piece of the gradient, whichever is more; the rows' copy, the
    matrix's where it is in 32 bits or off 16 bytes; dh's sums; 12 bytes a row; each on 256 bytes."""
    from paper_1712_01887_b200 import binding as B
    for dtype, rows, vocab, hidden, ld in ((1, 16384, 262144, 1024, 1024), (0, 16384, 262144, 1024, 1024), (2, 1, 131072, 1024, 1024),
                                           (0, 700, 10000, 1500, 1500), (1, 33, 50021, 2048, 2048), (1, 100, 5000, 129, 130),
                                           (0, 1, 1, 1, 1), (2, 8192, 1000, 64, 64), (1, 70000, 140000, 96, 96)):
        wide, up = 6 if dtype == 0 else 2, (hidden + 7) // 8 * 8
        copies = rows * up * wide + (vocab * up * wide if dtype == 0 or ld % 8 else 0)
        logits = 8 * rows * -(-vocab // (64 if dtype == 0 else 128))
        piece = max(128 << 20, 256 * rows * wide) + 256 * rows * wide
        sums = max(4 * rows * up, 20 << 20)
        args = B.VOCAB_LOSS.pack(dtype, vocab, hidden, 0, rows, 4096, ld, 4096, ld, 0, 4096, 4096, 4096, 4096, 4096, ld, 4096, ld, 0, 0, 0)
        forward, gradient = (B._lib.dgc_vocab_loss_workspace_bytes(args, g) for g in (0, 1))
        least = logits + copies + 12 * rows
        assert least <= forward <= least + 8 * 256, (dtype, rows, vocab)
        assert least <= gradient <= max(logits, piece) + copies + sums + 12 * rows + 8 * 256, (dtype, rows, vocab)
