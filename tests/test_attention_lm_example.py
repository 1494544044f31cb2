"""The example that runs linear attention, the loss over the vocabulary and the compressed exchange together.

Tolerance of the gradient, in 32 bits: the operators' own bounds are 2.5e-5 of the sums of absolute values
(attention) and 2^-15 of them (loss), and a product of at most 100 terms adds 100 * 2^-24; together under 1e-4, for
sums of up to ten times the largest entry of a weight's gradient 1e-3 of it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    spec = importlib.util.spec_from_file_location("attention_lm", os.path.join(ROOT, "examples", "attention_lm.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_of_all_weights_against_autograd_in_64_bits():
    ex = _example()
    vocab, hidden, heads, n = 61, 24, 3, 90
    state = ex.B.State(ex.Model.numel(vocab, hidden), 1, 0.9, 0.0, 0.9)
    model = ex.Model(state, vocab, hidden, heads, seed=3, dtype=torch.float32)
    toks, labels, start = ex.batch(torch.randperm(vocab, generator=torch.Generator().manual_seed(1)), n, 5, 1)
    grad = torch.full((state.arena_len,), float("nan"), device="cuda")
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        loss = model.loss_and_grad(toks, start, labels, grad, 0.5)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before

    ws = [w.double().detach().requires_grad_() for w in model.views(model.arena)]
    q, k, v = model.split(ws[0][toks] @ ws[1].t())
    rows, S, at = [], None, set(start.tolist())
    for t in range(n):
        if t in at:
            S = torch.zeros(heads, hidden // heads, hidden // heads, dtype=torch.float64, device="cuda")
        S = model.decay.double()[:, None, None] * S + k[t, :, :, None] * v[t, :, None, :]
        rows.append(model.scale * (q[t, :, :, None] * S).sum(1).flatten())
    logits = torch.stack(rows) @ ws[2].t() + ws[3]
    on = labels >= 0
    want = torch.zeros(n, dtype=torch.float64, device="cuda")
    want[on] = -torch.log_softmax(logits, 1)[on].gather(1, labels[on].long()[:, None])[:, 0]
    (0.5 * want.sum()).backward()
    want = want.detach()
    assert float((loss - want).abs().max()) <= 1e-4 * float(1 + want.abs().max())
    for got, w in zip(model.views(grad), ws):
        assert float((got - w.grad).abs().max()) <= 1e-3 * float(w.grad.abs().max())
    ex.B.tensor_check()
    state.close()


def test_the_model_trains_and_writes():
    ex = _example()
    history, written = ex.train(steps=12, workers=2, vocab=500, hidden=64, heads=2, tokens=256, seqs=7, say=lambda *a: None)
    assert all(h == h and h < float("inf") for h in history)
    assert written.shape == (4, 10) and int(written.min()) >= 0 and int(written.max()) < 500
