"""How linear attention (dgc_decay_attention_*) deals its work out: parts of many chunks, packs of many sequences in the order of
their lengths, calls without a workspace.  Tolerances and reference are test_attention_ranges.py's."""
import random

import pytest
import torch

from test_attention_ranges import DT, _bind, _data, _run, _verify

ALIGNED = 1 << 20


def _need(B, dt, num_seqs, heads, dk, dv, tokens, backward, packed=False):
    """Workspace of a call whose tensors lie on 16 bytes, for parts alone (without what float16 gradients keep of dout)."""
    dk8, dv8 = (dk + 7) // 8 * 8, (dv + 7) // 8 * 8
    kd, vd = (ALIGNED, heads * dk8, dk8), (ALIGNED, heads * dv8, dv8)
    args = B.ATTENTION.pack(B.DTYPES[dt], num_seqs, heads, dk, dv, 1.0, tokens, ALIGNED if packed else 0, ALIGNED, *kd, *kd, *vd, *vd,
                            0, 0, *vd, *kd, *kd, *vd, 0, 0, 0, 0)
    kept = (tokens * heads + 255) // 256 * 256 if backward and dt == torch.float16 else 0
    return int(B._lib.dgc_decay_attention_workspace_bytes(args, backward)) - kept


@pytest.mark.gpu
@pytest.mark.parametrize("dt,lens,heads,dk,dv", [
    (torch.bfloat16, [6000], 24, 64, 64), (torch.float16, [6000], 24, 64, 64),
    (torch.bfloat16, [6001], 12, 128, 128), (torch.float16, [6001], 12, 128, 128),
    (torch.bfloat16, [3000, 0, 4100], 16, 128, 96), (torch.float16, [2999, 4101], 16, 40, 64),
    (torch.float32, [3000], 24, 64, 64)], ids=str)
def test_parts_of_many_chunks(dt, lens, heads, dk, dv):
    """Parts longer than a chunk (of 128 tokens; 32 in 32 bits), the last chunk not whole, against 64 bits."""
    B = _bind()
    for backward in (0, 1):
        need, state = _need(B, dt, len(lens), heads, dk, dv, sum(lens), backward, True), heads * dk * dv * 4 * (1 + backward)
        assert 0 < need < (sum(lens) // 256 + len(lens)) * state       # parts of more than 256 tokens
    x, s, decay = _data(lens, heads, dk, dv, dt, decays=(0.999, 1.0, 0.97, 0.5))
    _verify(_run(lens, x, s, decay, dk ** -0.5), x, s, decay, dk ** -0.5, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("seqs,heads", [(40, 5), (256, 1), (257, 1), (300, 2)])
def test_many_sequences_of_uneven_length(seqs, heads, dt):
    """More sequences and heads than the GPU runs blocks at once: the longest go first (up to 256 sequences)."""
    _bind()
    rng = random.Random(seqs)
    lens = [rng.choice([0, 1, 17, 64, 64, 127, 128, 130, 250, rng.randrange(1, 200)]) for _ in range(seqs)]
    for dim in (64, 24):
        x, s, decay = _data(lens, heads, dim, dim, dt, decays=(0.9, 1.0, 0.99))
        _verify(_run(lens, x, s, decay, 0.2), x, s, decay, 0.2, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 61])
def test_long_sequences_without_a_workspace(dt, dim, monkeypatch):
    B = _bind()
    monkeypatch.setattr(B._lib, "dgc_decay_attention_workspace_bytes", lambda args, backward: 0)
    monkeypatch.setattr(B, "_work", lambda *a: pytest.fail("a workspace was taken"))
    lens = [2500, 300]
    x, s, decay = _data(lens, 2, dim, dim, dt)
    _verify(_run(lens, x, s, decay, 0.2), x, s, decay, 0.2, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=str)
def test_rows_outside_the_sequences_stay_where_rows_are_laid_anew(dt):
    B = _bind()
    N, H, d = 300, 2, 61
    x, _, decay = _data([N], H, d, d, dt)
    q, k, v, do = x
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (v, q, k, v))
    starts = torch.tensor([20, 150, 270], dtype=torch.int32, device="cuda")
    B.decay_attention_forward(q, k, v, out, decay, seq_start=starts, num_seqs=2)
    B.decay_attention_backward(q, k, v, do, dq, dk, dv, decay, seq_start=starts, num_seqs=2)
    for t in (out, dq, dk, dv):
        assert bool((t[:20] == 7).all()) and bool((t[270:] == 7).all()) and not bool((t[20:270] == 7).all(2).any())
    B.tensor_check()


@pytest.mark.parametrize("dt", DT, ids=str)
def test_only_calls_that_gain_are_cut(dt):
    """A call of equal sequences that fill the GPU is not cut; a few long sequences are.  (Host only.)"""
    from paper_1712_01887_b200 import binding as B
    for seqs, heads in ((8, 16), (16, 8), (4, 32), (9, 16), (16, 16), (14, 8), (1, 296), (2, 148)):
        assert _need(B, dt, seqs, heads, 128, 128, seqs * 4096, 0) == 0, (seqs, heads)
    for seqs, heads in ((5, 16), (3, 16), (1, 48), (1, 40), (7, 7)):
        assert _need(B, dt, seqs, heads, 128, 128, seqs * 4096, 1) == 0, (seqs, heads)
    for seqs, heads, backward in ((1, 8, 0), (1, 8, 1), (1, 1, 1), (2, 16, 0), (1, 16, 1)):
        assert _need(B, dt, seqs, heads, 128, 128, seqs * 4096, backward) > 0, (seqs, heads)
    # whatever is cut is cut into two parts at least: one part of a sequence that is no multiple of 128 takes one state a head
    for units in range(1, 296):
        for tokens in (1025, 1500, 4097, 65537):
            need = _need(B, dt, 1, units, 64, 64, tokens, 0)
            assert need == 0 or need >= 2 * units * 64 * 64 * 4, (units, tokens)
    # packs, of which only the mean length is known, from a mean of 1024 (256 in 32 bits) on; nothing to cut, nothing cut
    mean = 256 if dt == torch.float32 else 1024
    for seqs, heads in ((8, 4), (4, 2), (32, 4)):
        assert _need(B, dt, seqs, heads, 64, 64, seqs * mean - 1, 0, True) == 0 < _need(B, dt, seqs, heads, 64, 64, seqs * mean, 0, True)
    for seqs, tokens in ((1, 0), (1, 1), (2, 0), (3, 2), (2, 100)):
        for backward in (0, 1):
            assert _need(B, dt, seqs, 4, 64, 64, tokens, backward, True) == 0
            assert tokens % seqs or _need(B, dt, seqs, 4, 64, 64, tokens, backward) == 0


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16], ids=str)
def test_rows_are_laid_anew_where_it_gains(dt):
    """Rows off 16 bytes: taken in 32-bit arithmetic as they are where a sequence is hardly more than one chunk of that.  (Host only.)"""
    from paper_1712_01887_b200 import binding as B

    def need(seqs, heads, dim, tokens, backward):
        t, n = (ALIGNED + 2, heads * dim, dim), seqs * tokens
        args = B.ATTENTION.pack(B.DTYPES[dt], seqs, heads, dim, dim, 1.0, n, 0, ALIGNED, *t * 4, 0, 0, *t * 4, 0, 0, 0, 0)
        kept = (n * heads + 255) // 256 * 256 if backward and dt == torch.float16 else 0
        return int(B._lib.dgc_decay_attention_workspace_bytes(args, backward)) - kept
    for seqs, heads, dim, tokens, backward in ((20, 12, 125, 24, 1), (200, 4, 61, 32, 0), (200, 4, 61, 32, 1), (64, 16, 61, 16, 0), (1, 12, 125, 16, 0)):
        assert need(seqs, heads, dim, tokens, backward) == 0, (seqs, heads, dim, tokens)
    for seqs, heads, dim, tokens, backward in ((20, 12, 125, 24, 0), (20, 12, 125, 35, 1), (64, 16, 61, 40, 0), (64, 16, 61, 40, 1)):
        rows = (7 if backward else 4) * seqs * tokens * heads * ((dim + 7) // 8 * 16)
        assert need(seqs, heads, dim, tokens, backward) >= rows, (seqs, heads, dim, tokens)
