"""A small language model with linear attention, trained on the next token, its gradients compressed.

    python examples/attention_lm.py [--steps 60] [--workers 4] [--vocab 2000] [--hidden 256] [--heads 4]

One training step, for each simulated worker: token embeddings -> one product that gives queries, keys and
values -> linear attention with a decay for each head over packed sequences of uneven length -> the loss over the
vocabulary and its gradient, the logits never kept -> backward through the attention; every weight's
gradient lands in the worker's arena.  Then all workers' gradients are compressed, the lists summed and the
weights moved.  At the end the model reads a prompt and writes a few tokens, one step of the attention a token.

The products are torch's; the data is synthetic (each token's successor is mostly the same).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1712_01887_b200 import binding as B  # noqa: E402


class Model:
    """Embedding [vocab, hidden], in-projection [3 hidden, hidden] (queries, keys, values), output matrix
    [vocab, hidden] and bias [vocab]: views of one fp32 arena laid out by a compression state."""

    def __init__(self, state: B.State, vocab: int, hidden: int, heads: int, seed: int = 0, dtype=torch.bfloat16):
        self.vocab, self.hidden, self.heads, self.dtype = vocab, hidden, heads, dtype
        self.shapes = [(vocab, hidden), (3 * hidden, hidden), (vocab, hidden), (vocab,)]
        self.offset = [int(o) for o in state.arena_offset]
        self.arena = torch.zeros(state.arena_len, device="cuda")
        self.scale = (hidden // heads) ** -0.5
        self.decay = 1 - 2.0 ** -torch.linspace(1, 6, heads, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for w, std in zip(self.views(self.arena), (0.7, hidden ** -0.5, hidden ** -0.5, 0.0)):
            w.copy_(torch.randn(w.shape, generator=gen, device="cuda") * std)

    @staticmethod
    def numel(vocab: int, hidden: int):
        return [vocab * hidden, 3 * hidden * hidden, vocab * hidden, vocab]

    def views(self, arena: torch.Tensor):
        return [arena[o:o + torch.Size(s).numel()].view(s) for o, s in zip(self.offset, self.shapes)]

    def weights(self):
        return [w.to(self.dtype) for w in self.views(self.arena)]

    def split(self, wide: torch.Tensor):
        """Queries, keys, values [tokens, heads, dim]: slices of one product's output."""
        return [t.unflatten(1, (self.heads, -1)) for t in wide.split(self.hidden, dim=1)]

    def attend(self, q, k, v, seq_start, state=None):
        out = torch.empty(v.shape, dtype=v.dtype, device="cuda")
        B.decay_attention_forward(q, k, v, out, self.decay, seq_start=seq_start, num_seqs=seq_start.numel() - 1,
                                  s_last=state, scale=self.scale)
        return out

    def loss_and_grad(self, tokens, seq_start, labels, grad_arena, scale: float) -> torch.Tensor:
        """Losses of all tokens; writes scale times their sum's gradient to grad_arena."""
        emb, w_in, w_out, bias = self.weights()
        n = tokens.numel()
        e = emb[tokens]
        q, k, v = self.split(e @ w_in.t())
        h = self.attend(q, k, v, seq_start).flatten(1)
        loss, dh, dw, db = torch.empty(n, device="cuda"), torch.empty_like(h), torch.empty_like(w_out), torch.empty_like(bias)
        B.vocab_loss_grad(h, w_out, labels, torch.full((n,), scale, device="cuda"), loss, dh, dw, bias=bias, dbias=db)
        wide = torch.empty(n, 3 * self.hidden, dtype=self.dtype, device="cuda")
        B.decay_attention_backward(q, k, v, dh.view(v.shape), *self.split(wide), self.decay, seq_start=seq_start,
                                   num_seqs=seq_start.numel() - 1, scale=self.scale)
        g_emb, g_in, g_out, g_bias = self.views(grad_arena)
        g_in.copy_(wide.t() @ e)
        g_out.copy_(dw)
        g_bias.copy_(db)
        g_emb.zero_().index_add_(0, tokens, (wide @ w_in).float())
        return loss

    def write(self, prompts: torch.Tensor, length: int) -> torch.Tensor:
        """`length` tokens after each prompt [count, tokens], the likeliest each time."""
        emb, w_in, w_out, bias = self.weights()
        n, t = prompts.shape
        dim = self.hidden // self.heads
        state = torch.empty(n, self.heads, dim, dim, device="cuda")
        starts = torch.arange(0, n * t + 1, t, dtype=torch.int32, device="cuda")
        h = self.attend(*self.split(emb[prompts.flatten()] @ w_in.t()), starts, state).view(n, t, -1)[:, -1]
        idx, val = torch.empty(n, 1, dtype=torch.int32, device="cuda"), torch.empty(n, 1, device="cuda")
        out = torch.empty(n, self.heads, dim, dtype=self.dtype, device="cuda")
        written = [prompts]
        for step in range(length):
            B.top_logits(h @ w_out.t() + bias, idx, val)
            written.append(idx.long())
            B.decay_attention_step(*self.split(emb[idx[:, 0].long()] @ w_in.t()), state, out, self.decay, scale=self.scale)
            h = out.flatten(1)
        return torch.cat(written, 1)


def batch(successor: torch.Tensor, tokens: int, seqs: int, seed: int):
    """Packed sequences of uneven length, their labels (the last token of each has none) and offsets."""
    gen = torch.Generator().manual_seed(seed)
    vocab = successor.numel()
    cuts = torch.sort(torch.randint(1, tokens, (seqs - 1,), generator=gen)).values
    start = torch.cat([torch.zeros(1), cuts, torch.full((1,), tokens)]).to(torch.int32)
    noise, strange = torch.randint(0, vocab, (tokens,), generator=gen), torch.rand(tokens, generator=gen) < 0.2
    toks = [int(noise[0])]
    for t in range(1, tokens):
        toks.append(int(noise[t]) if strange[t] else int(successor[toks[-1]]))
    toks = torch.tensor(toks)
    labels = torch.roll(toks, -1).to(torch.int32)
    labels[(start[1:].long() - 1).clamp(min=0)] = -1
    return toks.cuda(), labels.cuda(), start.cuda()


def train(steps: int = 60, workers: int = 4, vocab: int = 2000, hidden: int = 256, heads: int = 4, tokens: int = 1024,
          seqs: int = 12, sparsity: float = 0.98, lr: float = 2.0, momentum: float = 0.9, say=print):
    states = [B.State(Model.numel(vocab, hidden), workers, momentum, 0.0, sparsity, seed=w) for w in range(workers)]
    model = Model(states[0], vocab, hidden, heads)
    successor = torch.randperm(vocab, generator=torch.Generator().manual_seed(5))
    nnz, length = states[0].max_nnz, states[0].arena_len
    grads = [torch.zeros(length, device="cuda") for _ in range(workers)]
    out_idx = [torch.empty(nnz, dtype=torch.int32, device="cuda") for _ in range(workers)]
    out_val = [torch.empty(nnz, device="cuda") for _ in range(workers)]
    dense = torch.empty(length, device="cuda")
    scratch = torch.empty(B.decode_workspace_bytes(workers, length), dtype=torch.uint8, device="cuda")
    history = []
    for step in range(steps):
        total = 0.0
        for w in range(workers):
            toks, labels, start = batch(successor, tokens, seqs, step * workers + w)
            total += model.loss_and_grad(toks, start, labels, grads[w], 1.0 / (tokens * workers)).mean()
        B.compress_batch(states, grads, out_idx, out_val)
        B.decode_accumulate_sgd(out_idx, out_val, dense, model.arena, lr, scratch)
        history.append(float(total) / workers)
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step:4d}  loss {history[-1]:.4f}")
    B.tensor_check()
    written = model.write(torch.arange(8, device="cuda").view(4, 2), 8)
    for row in written.tolist():
        say("wrote", row)
    for s in states:
        s.close()
    return history, written


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 60), ("workers", 4), ("vocab", 2000), ("hidden", 256), ("heads", 4)):
        ap.add_argument("--" + name, type=int, default=default)
    train(**vars(ap.parse_args()))
