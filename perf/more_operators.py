"""What is measured of linear attention with a decay for each head and of the loss over a large vocabulary.

Two operators: the attention (forward over packed sequences, forward + backward, one token a sequence) and
softmax cross entropy from hidden rows and output matrix, the logits never kept, with its gradient.  Each
case runs in a plain form (elementary torch operations in 32 bits) or, where `own` is true, through the
library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 128          # tokens of a chunk in the plain form


# --------------------------------------------------------------------------- cases

def listed():
    return [
        # serving: 64 sequences, one token each, states in a cache of 96 slots
        dict(name="step_64x16x128_bf16", op="attn_step", seqs=64, slots=96, heads=16, dk=128, dv=128, dtype="bf16"),
        # serving a few sequences, where latency counts; values wider than keys
        dict(name="step_3x8x64x96_f32", op="attn_step", seqs=3, slots=5, heads=8, dk=64, dv=96, dtype="f32"),
        # prompts of all lengths packed back to back, their states kept for the answers
        dict(name="prompts_40007x16x128_bf16", op="attn_forward", tokens=40007, seqs=37, heads=16, dk=128, dv=128,
             dtype="bf16", ragged=True, joint=True),
        # one prompt of middling length, latency counts
        dict(name="prompt_1500x8x64_f16", op="attn_forward", tokens=1500, seqs=1, heads=8, dk=64, dv=64, dtype="f16",
             ragged=False, joint=False),
        # training in full precision, the truncated batch and hidden size of the 2-layer LSTM language model: 12 heads of 125
        dict(name="train_20x35x12x125_f32", op="attn_train", tokens=700, seqs=20, heads=12, dk=125, dv=125, dtype="f32",
             ragged=False, joint=False),
        # training on utterances of uneven length, q, k and v slices of one product
        dict(name="train_25013x16x64_f16", op="attn_train", tokens=25013, seqs=32, heads=16, dk=64, dv=64, dtype="f16",
             ragged=True, joint=True),
        # training on one very long document
        dict(name="train_65536x16x128_bf16", op="attn_train", tokens=65536, seqs=1, heads=16, dk=128, dv=128,
             dtype="bf16", ragged=False, joint=False),
        # scoring of one token each of a few sequences over a large vocabulary: the output matrix is read once
        dict(name="loss_33x50021x2048_bf16", op="loss", rows=33, vocab=50021, hidden=2048, dtype="bf16", bias=False),
        # evaluation of the LSTM language model: a truncated batch in full precision, with the softmax layer's bias
        dict(name="loss_700x10000x1500_f32", op="loss", rows=700, vocab=10000, hidden=1500, dtype="f32", bias=True),
        # its training step
        dict(name="loss_grad_700x10000x1500_f32", op="loss_grad", rows=700, vocab=10000, hidden=1500, dtype="f32",
             bias=True),
        # training: loss and gradient in one call
        dict(name="loss_grad_4096x50021x1024_bf16", op="loss_grad", rows=4096, vocab=50021, hidden=1024, dtype="bf16",
             bias=False),
        # training under an autograd engine: the loss first, the gradient later
        dict(name="loss_then_grad_2047x131072x1024_f16", op="loss_two_calls", rows=2047, vocab=131072, hidden=1024,
             dtype="f16", bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _some_dim(rng, lo, hi):
    """A head's or a hidden row's length: mostly on 16 bytes, sometimes of any size."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.25 else max(lo, n // 8 * 8)


def draw(rng: random.Random):
    op = rng.choice(["attn_step", "attn_forward", "attn_train", "attn_train", "loss", "loss_grad", "loss_grad",
                     "loss_two_calls"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op.startswith("attn"):
        heads, dk = _log_int(rng, 1, 32), _some_dim(rng, 16, 128)
        dv = dk if rng.random() < 0.6 else _some_dim(rng, 16, 128)
        if op == "attn_step":
            seqs = _log_int(rng, 1, max(1, min(600, 2 ** 24 // (heads * dk * dv))))
            return dict(op=op, seqs=seqs, slots=seqs + rng.randrange(0, seqs + 3), heads=heads, dk=dk, dv=dv, dtype=dtype)
        most = 2 ** (28 if dtype != "f32" else 25) // (heads * (dk + dv))
        tokens = _log_int(rng, 1, min(70000, most))
        ragged = rng.random() < 0.5
        seqs = _log_int(rng, 1, max(1, min(200, tokens)))
        if not ragged:
            tokens = seqs * max(1, tokens // seqs)
        return dict(op=op, tokens=tokens, seqs=seqs, heads=heads, dk=dk, dv=dv, dtype=dtype, ragged=ragged,
                    joint=rng.random() < 0.5)
    hidden, vocab = _some_dim(rng, 64, 2048), _log_int(rng, 1000, 140000)
    most = min(2 ** 28 // vocab, (2 * 10 ** 11 if dtype != "f32" else 2 * 10 ** 10) // (vocab * hidden), 8192)
    return dict(op=op, rows=_log_int(rng, 1, max(1, most)), vocab=vocab, hidden=hidden, dtype=dtype,
                bias=rng.random() < 0.4)


def work(case):
    op, sz = case["op"], SIZE[case["dtype"]]
    if op.startswith("attn"):
        H, dk, dv = case["heads"], case["dk"], case["dv"]
        if op == "attn_step":
            n = case["seqs"] * H
            return {"bytes": n * (8 * dk * dv + (2 * dk + 2 * dv) * sz) + 4 * case["seqs"], "flops": 5 * n * dk * dv}
        n, states = case["tokens"] * H, case["seqs"] * H * dk * dv * 4
        if op == "attn_forward":
            return {"bytes": n * (2 * dk + 2 * dv) * sz + 2 * states, "flops": 4 * n * dk * dv}
        return {"bytes": n * (4 * dk + 4 * dv) * sz + 4 * states, "flops": 14 * n * dk * dv}   # q, k, v, do in; out, dq, dk, dv out
    R, V, D = case["rows"], case["vocab"], case["hidden"]
    b = V * sz if case["bias"] else 0
    if op == "loss":
        return {"bytes": (R + V) * D * sz + b + 8 * R, "flops": 2 * R * V * D}
    return {"bytes": 2 * (R + V) * D * sz + 2 * b + 12 * R, "flops": 6 * R * V * D}


# --------------------------------------------------------------------------- inputs

def _lengths(case, seed):
    """Lengths of a pack: most of them uneven, one of none where there is room."""
    seqs, tokens = case["seqs"], case["tokens"]
    if not case["ragged"]:
        return [tokens // seqs] * seqs
    rng = random.Random(seed * 7919 + tokens)
    weight = [rng.expovariate(1.0) + 0.05 for _ in range(seqs)]
    if seqs >= 4:
        weight[rng.randrange(seqs)] = 0.0
    total, cuts, acc = sum(weight), [0], 0.0
    for w in weight[:-1]:
        acc += w
        cuts.append(min(tokens, int(round(tokens * acc / total))))
    cuts.append(tokens)
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _decays(H):
    """From fast to slow, the last head without any where there are a few."""
    g = [1.0 - 2.0 ** -(1.0 + 9.0 * (h + 1) / H) for h in range(H)]
    if H >= 4:
        g[-1] = 1.0
    return torch.tensor(g, dtype=torch.float32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32).mul_(std)

    st = {"case": case}
    if op.startswith("attn"):
        H, dk, dv = case["heads"], case["dk"], case["dv"]
        st["decay"], st["scale"] = _decays(H), dk ** -0.5
        if op == "attn_step":
            S = case["seqs"]
            st["q"], st["k"], st["v"] = (normal(S, H, d).to(dt) for d in (dk, dk, dv))
            st["state"] = normal(case["slots"], H, dk, dv)
            st["slots"] = torch.randperm(case["slots"], generator=gen, device="cuda")[:S].to(torch.int32)
            st["out"] = torch.empty(S, H, dv, dtype=dt, device="cuda")
            return st
        N, S = case["tokens"], case["seqs"]

        def three(fill):         # one product's output, cut in three, or three tensors
            if case["joint"]:
                whole = torch.empty(N, H * (2 * dk + dv), dtype=dt, device="cuda")
                parts = whole.split([H * dk, H * dk, H * dv], dim=1)
                parts = [p.unflatten(1, (H, d)) for p, d in zip(parts, (dk, dk, dv))]
            else:
                parts = [torch.empty(N, H, d, dtype=dt, device="cuda") for d in (dk, dk, dv)]
            if fill:
                for p in parts:
                    p.copy_(normal(*p.shape))
            return parts

        st["q"], st["k"], st["v"] = three(True)
        lens = _lengths(case, seed)
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + n)
        st["seqs"] = S
        st["seq_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        st["packed"] = st["seq_start"] if case["ragged"] else None
        # where the chunks of each sequence lie (the plain form's plan)
        at, seq, nth = [], [], []
        for s, n in enumerate(lens):
            for c in range((n + CHUNK - 1) // CHUNK):
                at.append((starts[s] + c * CHUNK, min(CHUNK, n - c * CHUNK)))
                seq.append(s)
                nth.append(c)
        first, size = torch.tensor(at, device="cuda").view(-1, 2).unbind(1)
        place = torch.arange(CHUNK, device="cuda")
        there = place < size[:, None]
        st["chunks"] = dict(at=torch.where(there, first[:, None] + place, 0), there=there, size=size,
                            seq=torch.tensor(seq, device="cuda"), nth=torch.tensor(nth, device="cuda"))
        st["s0"] = normal(S, H, dk, dv, std=0.5)
        st["out"] = torch.empty(N, H, dv, dtype=dt, device="cuda")
        st["s_last"] = torch.empty(S, H, dk, dv, device="cuda")
        if op == "attn_train":
            # 16-bit floats of a narrow range come with a loss scale, as such training does
            st["dout"], st["ds_last"] = normal(N, H, dv, std=0.1).to(dt), normal(S, H, dk, dv, std=0.1)
            st["dq"], st["dk"], st["dv"] = three(False)
            st["ds0"] = torch.empty_like(st["s0"])
        return st

    R, V, D = case["rows"], case["vocab"], case["hidden"]
    st["hidden"] = normal(R, D).to(dt)
    st["weight"] = normal(V, D, std=2.0 * D ** -0.5).to(dt)      # logits of spread 2
    st["bias"] = normal(V).to(dt) if case["bias"] else None
    st["labels"] = torch.randint(0, V, (R,), generator=gen, device="cuda", dtype=torch.int32)
    if R >= 4:
        st["labels"][R // 2] = -1                                # a padding token
    st["loss"], st["stats"] = torch.empty(R, device="cuda"), torch.empty(R, 2, device="cuda")
    if op != "loss":
        scale = 4096.0 if case["dtype"] == "f16" else 1.0
        st["dloss"] = torch.rand(R, generator=gen, device="cuda").add_(0.5).mul_(scale / R)
        st["dhidden"], st["dweight"] = torch.empty_like(st["hidden"]), torch.empty_like(st["weight"])
        st["dbias"] = torch.empty_like(st["bias"]) if case["bias"] else None
    return st


# --------------------------------------------------------------------------- plain forms

def _walk(st, q, k, v, s_in, late, w_k):
    """Decayed linear attention in chunks, 32 bits: rows (not scaled) and the states after each sequence.
    `late`: from the last token to the first, as gradients go (what comes in is not decayed before the first use).
    w_k: factor of the keys on their way to the state and to the rows."""
    ch, lg = st["chunks"], torch.log2(st["decay"])
    at, size, seq, nth = ch["at"], ch["size"], ch["seq"], ch["nth"]
    if not len(at):
        return torch.zeros_like(v), s_in.clone()
    there = ch["there"][:, :, None, None]
    qc, kc, vc = (torch.where(there, x[at], 0).transpose(1, 2) for x in (q, k, v))       # [chunks, heads, C, dim]
    kc = kc * w_k
    place = torch.arange(CHUNK, device=q.device)
    away = place[:, None] - place[None, :]
    away = -away if late else away
    D = torch.where(away >= 0, torch.exp2(away.clamp(min=0) * lg[:, None, None]), 0)      # [heads, C, C]
    rows = ((qc @ kc.transpose(2, 3)) * D) @ vc
    n = size[:, None, None]
    if late:     # the state that comes from behind the chunk, and what goes out before it
        to_row, from_row = n - 1 - place, place + 1
    else:
        to_row, from_row = place + 1 + 0 * n, n - 1 - place
    to_row = torch.exp2(to_row.clamp(min=0) * lg[:, None])                                # [chunks, heads, C]
    from_row = torch.exp2(from_row.clamp(min=0) * lg[:, None])
    local = (kc * from_row[..., None]).transpose(2, 3) @ vc                               # [chunks, heads, dk, dv]
    # the states before each chunk and after each sequence: sums over the chunks that go before, a product
    # (of a sequence's chunks only the last is not whole)
    total = torch.zeros(st["seqs"], dtype=torch.long, device=q.device).index_add_(0, seq, size)
    begin = nth * CHUNK
    gap = begin[None, :] - (begin + size)[:, None] if late else begin[:, None] - (begin + size)[None, :]
    joined = (seq[:, None] == seq[None, :]) & (gap >= 0)
    W = torch.where(joined, torch.exp2(gap.clamp(min=0) * lg[:, None, None]), 0)          # [heads, chunks, chunks]
    flat = local.flatten(2).transpose(0, 1)
    before = total[seq] - begin - size if late else begin
    s = (W @ flat).transpose(0, 1).view_as(local) + s_in[seq] * torch.exp2(before[:, None] * lg)[..., None, None]
    rows = rows + (qc @ s) * to_row[..., None]
    behind = begin if late else total[seq] - begin - size
    last = s_in * torch.exp2(total[:, None] * lg)[..., None, None]
    last = last.index_add(0, seq, local * torch.exp2(behind[:, None] * lg)[..., None, None])
    y = torch.zeros(q.shape[0], *rows.shape[1:2], rows.shape[3], device=q.device)
    y[at[ch["there"]]] = rows.transpose(1, 2)[ch["there"]]
    return y, last


def _attn_plain(st):
    c, dt = st["scale"], st["q"].dtype
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    out, s_last = _walk(st, q, k, v, st["s0"], False, 1.0)
    out = (c * out).to(dt)
    if st["case"]["op"] == "attn_forward":
        return out, s_last
    do = st["dout"].float()
    dq, _ = _walk(st, do, v, k, st["s0"].transpose(2, 3), False, 1.0)
    dv, ds0 = _walk(st, k, q, do, st["ds_last"], True, c)
    dk, _ = _walk(st, v, do, q, st["ds_last"].transpose(2, 3), True, c)
    return out, s_last, (c * dq).to(dt), dk.to(dt), dv.to(dt), ds0


def _step_plain(st):
    q, k, v, at = st["q"].float(), st["k"].float(), st["v"].float(), st["slots"].long()
    s = st["state"][at] * st["decay"][:, None, None] + k[..., :, None] * v[..., None, :]
    st["state"][at] = s
    out = st["scale"] * (q[..., :, None] * s).sum(2)
    return out.to(st["q"].dtype), st["state"]


def _loss_plain(st):
    op, dt = st["case"]["op"], st["hidden"].dtype
    h, w = st["hidden"].float(), st["weight"].float()
    l = h @ w.t()
    if st["bias"] is not None:
        l += st["bias"].float()
    labelled = (st["labels"] >= 0) & (st["labels"] < l.shape[1])
    y = torch.where(labelled, st["labels"], 0).long()[:, None]
    m = l.amax(1, keepdim=True)
    own_logit = torch.gather(l, 1, y) - m
    p = l.sub_(m).exp_()
    total = p.sum(1, keepdim=True)
    loss = torch.where(labelled, (torch.log(total) - own_logit)[:, 0], 0.0)
    if op == "loss":
        return loss
    weight = torch.where(labelled, st["dloss"], 0.0)[:, None]
    g = p.mul_(weight / total)
    g.scatter_add_(1, y, -weight)
    grads = (g @ w).to(dt), (g.t() @ h).to(dt)
    if st["bias"] is not None:
        grads += (g.sum(0).to(dt),)
    return (loss,) + grads


# --------------------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        if op == "attn_step":
            return _step_plain(st)
        return _attn_plain(st) if op.startswith("attn") else _loss_plain(st)
    from paper_1712_01887_b200 import binding as B
    if op == "attn_step":
        B.decay_attention_step(st["q"], st["k"], st["v"], st["state"], st["out"], st["decay"], slots=st["slots"],
                               scale=st["scale"])
        return st["out"], st["state"]
    if op.startswith("attn"):
        how = dict(seq_start=st["packed"], num_seqs=st["seqs"], s0=st["s0"], scale=st["scale"])
        B.decay_attention_forward(st["q"], st["k"], st["v"], st["out"], st["decay"], s_last=st["s_last"], **how)
        if op == "attn_forward":
            return st["out"], st["s_last"]
        B.decay_attention_backward(st["q"], st["k"], st["v"], st["dout"], st["dq"], st["dk"], st["dv"], st["decay"],
                                   ds_last=st["ds_last"], ds0=st["ds0"], **how)
        return st["out"], st["s_last"], st["dq"], st["dk"], st["dv"], st["ds0"]
    data = st["hidden"], st["weight"], st["labels"]
    if op == "loss":
        B.vocab_loss_forward(*data, st["loss"], bias=st["bias"])
        return st["loss"]
    grads = dict(bias=st["bias"], dbias=st["dbias"])
    if op == "loss_grad":
        B.vocab_loss_grad(*data, st["dloss"], st["loss"], st["dhidden"], st["dweight"], **grads)
    else:
        B.vocab_loss_forward(*data, st["loss"], st["stats"], bias=st["bias"])
        B.vocab_loss_backward(*data, st["stats"], st["dloss"], st["dhidden"], st["dweight"], **grads)
    return (st["loss"], st["dhidden"], st["dweight"]) + ((st["dbias"],) if case["bias"] else ())


# --------------------------------------------------------------------------- the definition in 64 bits

def _exact_attn(st):
    """One token after the other, the sequences side by side."""
    c, g = st["scale"], st["decay"].double()[:, None, None]
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    a, b = st["seq_start"][:-1].long(), st["seq_start"][1:].long()
    lens = (b - a).tolist()
    order = sorted(range(len(lens)), key=lambda s: -lens[s])            # the longest first: step t has the first few
    live = [0] * (max(lens) + 1)
    for n in lens:
        for_t = n - 1
        live[for_t] += 1 if n else 0
    for t in range(len(live) - 2, -1, -1):
        live[t] += live[t + 1]
    rank = torch.tensor(order, device="cuda")
    begin = a[rank]
    s = st["s0"].double()[rank].contiguous()
    train = st["case"]["op"] == "attn_train"
    out = torch.zeros_like(v)
    if train:
        do, dq, dk, dv = st["dout"].double(), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(max(lens)):
        n = live[t]
        at, part = begin[:n] + t, s[:n]
        part.mul_(g).add_(k[at][..., :, None] * v[at][..., None, :])
        out[at] = c * (q[at][..., None, :] @ part)[..., 0, :]
        if train:
            dq[at] = c * (part @ do[at][..., :, None])[..., 0]
    s_last = torch.empty_like(s)
    s_last[rank] = s
    if not train:
        return out, s_last
    e = st["ds_last"].double()[rank].contiguous()
    for t in range(max(lens) - 1, -1, -1):
        n = live[t]
        at, part = begin[:n] + t, e[:n]
        part.add_(c * q[at][..., :, None] * do[at][..., None, :])
        dv[at] = (k[at][..., None, :] @ part)[..., 0, :]
        dk[at] = (part @ v[at][..., :, None])[..., 0]
        part.mul_(g)
    ds0 = torch.empty_like(e)
    ds0[rank] = e
    return out, s_last, dq, dk, dv, ds0


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "attn_step":
        at, g = st["slots"].long(), st["decay"].double()
        state = st["state"].double()
        state[at] = torch.einsum("h,rhkv->rhkv", g, state[at]) + torch.einsum("rhk,rhv->rhkv", st["k"].double(), st["v"].double())
        return st["scale"] * torch.einsum("rhk,rhkv->rhv", st["q"].double(), state[at]), state
    if op.startswith("attn"):
        return _exact_attn(st)
    h, w = st["hidden"].double(), st["weight"].double()
    dh, dw, loss = torch.zeros_like(h), torch.zeros_like(w), torch.zeros(h.shape[0], dtype=torch.float64, device="cuda")
    db = torch.zeros(w.shape[0], dtype=torch.float64, device="cuda")
    for r in range(0, h.shape[0], 512):
        rows = slice(r, r + 512)
        logits = torch.mm(h[rows], w.t())
        if case["bias"]:
            logits += st["bias"].double()
        logp = torch.log_softmax(logits, 1)
        on = torch.nonzero(st["labels"][rows] >= 0).flatten()
        y = st["labels"][rows][on].long()
        loss[r + on] = -logp[on, y]
        if op == "loss":
            continue
        g = logp.exp_()
        g[on, y] -= 1.0
        scale = torch.zeros(g.shape[0], dtype=torch.float64, device="cuda")
        scale[on] = st["dloss"][rows][on].double()
        g *= scale[:, None]
        dh[rows] = g @ w
        dw += g.t() @ h[rows]
        db += g.sum(0)
    if op == "loss":
        return loss
    return (loss, dh, dw) + ((db,) if case["bias"] else ())
