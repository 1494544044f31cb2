"""The example that runs the recurrence, the lists, the loss and the compressed exchange together.

Tolerance of the gradient: in 32 bits a product sums at most 300 terms of like size (300 * 2^-24 =
2e-5 of their sum's bound), the operators add 1e-4 of their largest result (tests of their own):
2e-4 of the largest entry of each weight's gradient covers both with room for the layers' composition."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    spec = importlib.util.spec_from_file_location("distill_lm", os.path.join(ROOT, "examples", "distill_lm.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_of_all_weights_against_autograd_in_64_bits():
    ex = _example()
    vocab, hidden, n, k, T, hard = 61, 24, 90, 7, 2.0, 0.25
    state = ex.B.State(ex.Student.numel(vocab, hidden), 1, 0.9, 0.0, 0.9)
    st = ex.Student(state, vocab, hidden, seed=3, dtype=torch.float32)
    toks, start = ex.batch(vocab, n, 5, 1)
    teacher = torch.randn(n, vocab, device="cuda")
    idx, val = torch.empty(n, k, dtype=torch.int32, device="cuda"), torch.empty(n, k, device="cuda")
    ex.B.top_logits(teacher, idx, val)
    labels = idx[:, 1].contiguous()
    grad = torch.full((state.arena_len,), float("nan"), device="cuda")
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        loss = st.loss_and_grad(toks, start, idx, val, labels, grad, 0.5, T, hard)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before

    ws = [w.double().detach().requires_grad_() for w in st.views(st.arena)]
    both = ws[0][toks] @ ws[1].t()
    f, x = torch.sigmoid(both[:, :hidden]), both[:, hidden:]
    rows, cur, at = [], None, set(start.tolist())
    for t in range(n):
        if t in at:
            cur = torch.zeros(hidden, dtype=torch.float64, device="cuda")
        cur = f[t] * cur + (1 - f[t]) * x[t]
        rows.append(cur)
    s = torch.stack(rows) @ ws[2].t()
    q = torch.softmax(val.double() / T, 1)
    kl = (q * (torch.log(q) - torch.log_softmax(s / T, 1).gather(1, idx.long()))).sum(1)
    want = (1 - hard) * T * T * kl - hard * torch.log_softmax(s, 1).gather(1, labels.long()[:, None])[:, 0]
    (0.5 * want.sum()).backward()
    want = want.detach()
    assert float((loss - want).abs().max()) <= 2e-4 * float(1 + want.abs().max())
    for got, w in zip(st.views(grad), ws):
        assert float((got - w.grad).abs().max()) <= 2e-4 * float(w.grad.abs().max())
    state.close()


def test_the_student_learns_and_writes():
    ex = _example()
    history, written = ex.train(steps=40, workers=2, vocab=500, hidden=64, tokens=512, seqs=7, say=lambda *a: None)
    assert all(h == h and h < float("inf") for h in history)
    assert sum(history[-5:]) < 0.8 * sum(history[:5])          # it learns
    assert written.shape == (4, 9) and int(written.min()) >= 0 and int(written.max()) < 500
