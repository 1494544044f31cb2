"""A small recurrent language model taught by another model's top logits, its gradients compressed.

    python examples/distill_lm.py [--steps 60] [--workers 4] [--vocab 2000] [--hidden 256]

One training step, for each simulated worker: token embeddings -> one product that gives gate and
input of a gated recurrence -> the recurrence over packed sequences of uneven length -> logits;
the teacher's logits are cut down to their top entries; loss and gradient of the distillation;
backward through the recurrence; every weight's gradient lands in the worker's arena.  Then all
workers' gradients are compressed, the lists summed and the weights moved, as in any training with
this library.  At the end the student writes a few tokens, one step of the recurrence a token.

The products are torch's; data and teacher are synthetic (a fixed random bigram model).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1712_01887_b200 import binding as B  # noqa: E402


class Student:
    """Embedding [vocab, hidden], in-projection [2 hidden, hidden] (gate and input), out-projection
    [vocab, hidden]: views of one fp32 arena laid out by a compression state."""

    def __init__(self, state: B.State, vocab: int, hidden: int, seed: int = 0, dtype=torch.bfloat16):
        self.vocab, self.hidden, self.dtype = vocab, hidden, dtype
        self.shapes = [(vocab, hidden), (2 * hidden, hidden), (vocab, hidden)]
        self.offset = [int(o) for o in state.arena_offset]
        self.arena = torch.zeros(state.arena_len, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for w, std in zip(self.views(self.arena), (0.5, hidden ** -0.5, hidden ** -0.5)):
            w.copy_(torch.randn(w.shape, generator=gen, device="cuda") * std)

    @staticmethod
    def numel(vocab: int, hidden: int):
        return [vocab * hidden, 2 * hidden * hidden, vocab * hidden]

    def views(self, arena: torch.Tensor):
        return [arena[o:o + a * b].view(a, b) for o, (a, b) in zip(self.offset, self.shapes)]

    def weights(self):
        return [w.to(self.dtype) for w in self.views(self.arena)]

    def forward(self, tokens: torch.Tensor, seq_start: torch.Tensor):
        emb, w_in, w_out = self.weights()
        e = emb[tokens]
        both = e @ w_in.t()                                        # gate and input side by side
        gate, x = both[:, :self.hidden], both[:, self.hidden:]
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
        B.gated_scan_forward(gate, x, h, seq_start=seq_start, num_seqs=seq_start.numel() - 1)
        return e, gate, x, h, h @ w_out.t()

    def loss_and_grad(self, tokens, seq_start, idx, val, labels, grad_arena, scale: float, temperature: float = 2.0,
                      hard_weight: float = 0.25) -> torch.Tensor:
        """Losses of all tokens; writes scale times their sum's gradient to grad_arena."""
        _, w_in, w_out = self.weights()
        e, gate, x, h, logits = self.forward(tokens, seq_start)
        n = tokens.numel()
        loss = torch.empty(n, device="cuda")
        B.distill_loss_grad(logits, idx, val, torch.full((n,), scale, device="cuda"), loss, logits,   # over the logits
                            temperature=temperature, soft_weight=1.0 - hard_weight, hard_weight=hard_weight, labels=labels)
        g_emb, g_in, g_out = self.views(grad_arena)
        g_out.copy_(logits.t() @ h)
        d_both = torch.empty(n, 2 * self.hidden, dtype=self.dtype, device="cuda")
        B.gated_scan_backward(gate, x, h, logits @ w_out, d_both[:, :self.hidden], d_both[:, self.hidden:],
                              seq_start=seq_start, num_seqs=seq_start.numel() - 1)
        g_in.copy_(d_both.t() @ e)
        g_emb.zero_().index_add_(0, tokens, (d_both @ w_in).float())
        return loss

    def write(self, first: torch.Tensor, length: int) -> torch.Tensor:
        """`length` tokens after each of the first ones, the likeliest each time."""
        emb, w_in, w_out = self.weights()
        n = first.numel()
        state = torch.zeros(n, self.hidden, device="cuda")
        out = torch.empty(n, self.hidden, dtype=self.dtype, device="cuda")
        idx, val = torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, 1, device="cuda")
        tokens = [first]
        for _ in range(length):
            both = emb[tokens[-1]] @ w_in.t()
            B.gated_scan_step(both[:, :self.hidden], both[:, self.hidden:], state, out)
            B.top_logits(out @ w_out.t(), idx, val)
            tokens.append(idx[:, 0].long())
        return torch.stack(tokens, 1)


def batch(vocab: int, tokens: int, seqs: int, seed: int):
    """Random tokens in packed sequences of uneven length."""
    gen = torch.Generator().manual_seed(seed)
    cuts = torch.sort(torch.randint(1, tokens, (seqs - 1,), generator=gen)).values
    start = torch.cat([torch.zeros(1), cuts, torch.full((1,), tokens)]).to(torch.int32)
    return torch.randint(0, vocab, (tokens,), generator=gen).cuda(), start.cuda()


def train(steps: int = 60, workers: int = 4, vocab: int = 2000, hidden: int = 256, tokens: int = 1024, seqs: int = 12,
          k: int = 32, sparsity: float = 0.98, lr: float = 4.0, momentum: float = 0.9, say=print):
    states = [B.State(Student.numel(vocab, hidden), workers, momentum, 0.0, sparsity, seed=w) for w in range(workers)]
    student = Student(states[0], vocab, hidden)
    gen = torch.Generator(device="cuda").manual_seed(99)
    left, right = (torch.randn(vocab, 24, generator=gen, device="cuda") for _ in range(2))   # the teacher: a bigram model
    grads = [torch.zeros(states[0].arena_len, device="cuda") for _ in range(workers)]
    nnz, L = states[0].max_nnz, states[0].arena_len
    out_idx = [torch.empty(nnz, dtype=torch.int32, device="cuda") for _ in range(workers)]
    out_val = [torch.empty(nnz, device="cuda") for _ in range(workers)]
    dense = torch.empty(L, device="cuda")
    scratch = torch.empty(B.decode_workspace_bytes(workers, L), dtype=torch.uint8, device="cuda")
    idx, val = torch.empty(tokens, k, dtype=torch.int32, device="cuda"), torch.empty(tokens, k, device="cuda")
    history = []
    for step in range(steps):
        total = 0.0
        for w in range(workers):
            toks, start = batch(vocab, tokens, seqs, step * workers + w)
            B.top_logits((left[toks] @ right.t()) * 0.6, idx, val)
            loss = student.loss_and_grad(toks, start, idx, val, idx[:, 0].contiguous(), grads[w], 1.0 / (tokens * workers))
            total += loss.mean()
        B.compress_batch(states, grads, out_idx, out_val)
        B.decode_accumulate_sgd(out_idx, out_val, dense, student.arena, lr, scratch)
        history.append(float(total) / workers)
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step:4d}  loss {history[-1]:.4f}")
    B.gated_scan_check()
    written = student.write(torch.arange(4, device="cuda"), 8)
    for row in written.tolist():
        say("wrote", row)
    for s in states:
        s.close()
    return history, written


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 60), ("workers", 4), ("vocab", 2000), ("hidden", 256)):
        ap.add_argument("--" + name, type=int, default=default)
    train(**vars(ap.parse_args()))
