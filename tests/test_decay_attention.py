"""Linear attention with a decay for each head (dgc_decay_attention_*) against plain recurrences in 64 bits.

Tolerances.  Errors are counted against `size`: the same formulas with every input's absolute value, which is
what a rounding error of a term or of a partial sum is relative to.
 * 32 bits.  A result passes at most 128 terms of a product over a head, 128 of one over a chunk and one
   operation a chunk, each with 2^-24, and weights decay^n = 2^(n log2 decay), whose exponent is off by 2^-23 of
   itself (weights below 2^-30 add nothing that counts) and which is off by 2 ulp more: in all under
   (256 + chunks + 30 + 4) 2^-24 < 2.5e-5 for up to 100 chunks.
 * 16-bit calls round decay^n q.k and the state to the type where they enter a product: half a unit of the
   sum over the chunk and half a unit of the state's part, together half a unit of `size`; and the result
   by half a unit of itself.  States are sums of exact products in 32 bits, times weights that may be kept
   as two parts of the type: 2^-17 (7.6e-6) of `size` more."""
import ctypes
import struct

import pytest
import torch

from test_operator_calls import Stream, Tensor, machine  # noqa: F401  (stand-ins for tensors and devices)

DT = [torch.float32, torch.bfloat16, torch.float16]
UNIT = {torch.float32: 0.0, **{d: torch.finfo(d).eps / 2 for d in (torch.bfloat16, torch.float16)}}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
F32 = 2.5e-5
PARTS = 7.7e-6


def _bind():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    from paper_1712_01887_b200 import binding as B
    return B


# ----------------------------------------------------------------- plain recurrences, 64 bits

def plain(q, k, v, decay, scale, s0, lens):
    """(out, s_last), one token after the other."""
    out, last, t = torch.zeros_like(v), s0.clone(), 0
    for s, n in enumerate(lens):
        S = s0[s].clone()
        for t in range(t, t + n):
            S = decay[:, None, None] * S + k[t, :, :, None] * v[t, :, None, :]
            out[t] = scale * (q[t, :, :, None] * S).sum(1)
        t += n > 0
        last[s] = S
    return out, last


def plain_backward(q, k, v, do, decay, scale, s0, ds_last, lens):
    """(dq, dk, dv, ds0)."""
    dq, dk, dv, ds0 = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), ds_last.clone()
    first = 0
    for s, n in enumerate(lens):
        S = s0[s].clone()
        for t in range(first, first + n):
            S = decay[:, None, None] * S + k[t, :, :, None] * v[t, :, None, :]
            dq[t] = scale * (S * do[t, :, None, :]).sum(2)
        E = ds_last[s].clone()
        for t in range(first + n - 1, first - 1, -1):
            D = E + scale * q[t, :, :, None] * do[t, :, None, :]
            dk[t], dv[t] = (D * v[t, :, None, :]).sum(2), (D * k[t, :, :, None]).sum(1)
            E = decay[:, None, None] * D
        ds0[s] = E
        first += n
    return dq, dk, dv, ds0


def test_plain_backward_agrees_with_differences():
    gen = torch.Generator().manual_seed(3)
    N, H, dk, dv, lens, c = 12, 2, 3, 4, [5, 0, 1, 6], 0.7
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    x = [r(N, H, dk), r(N, H, dk), r(N, H, dv), r(4, H, dk, dv)]
    way = [r(*t.shape) for t in x]
    decay, do, dl = torch.tensor([0.9, 0.4], dtype=torch.float64), r(N, H, dv), r(4, H, dk, dv)

    def value(e):
        q, k, v, s0 = (t + e * w for t, w in zip(x, way))
        out, last = plain(q, k, v, decay, c, s0, lens)
        return (out * do).sum() + (last * dl).sum()
    grads = plain_backward(x[0], x[1], x[2], do, decay, c, x[3], dl, lens)
    want = sum((g * w).sum() for g, w in zip(grads, way))
    assert torch.allclose((value(1e-6) - value(-1e-6)) / 2e-6, want, rtol=1e-7)


# ----------------------------------------------------------------- against the library

def _inputs(lens, H, dk, dv, dt, seed=1, lay="joint"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, S = sum(lens), len(lens)

    def three(fill):
        if lay == "joint":       # slices of one wider product's output
            whole = torch.full((N, H * (2 * dk + dv) + 3), 7.0, device="cuda").to(dt)
            parts = whole[:, 1:-2].split([H * dk, H * dk, H * dv], 1)
            parts = [p.unflatten(1, (H, d)) for p, d in zip(parts, (dk, dk, dv))]
        elif lay == "heads":     # heads outermost
            parts = [torch.full((H, N, d), 7.0, device="cuda").to(dt).transpose(0, 1) for d in (dk, dk, dv)]
        else:
            parts = [torch.full((N, H, d), 7.0, device="cuda").to(dt) for d in (dk, dk, dv)]
        if fill:
            for p in parts:
                p.copy_(torch.randn(*p.shape, generator=gen, device="cuda"))
        return parts
    st = dict(q_k_v=three(True), grads=three(False))
    st["out"] = three(False)[2]
    st["dout"] = torch.randn(N, H, dv, generator=gen, device="cuda").to(dt)
    st["decay"] = torch.tensor([[0.97, 1.0, 0.5, 0.0, 0.999][h % 5] for h in range(H)], device="cuda")
    st["s0"], st["ds_last"] = (torch.randn(S, H, dk, dv, generator=gen, device="cuda") for _ in range(2))
    st["starts"] = torch.tensor([sum(lens[:i]) for i in range(S + 1)], dtype=torch.int32, device="cuda")
    return st


def _near(got, want, size, dt, state=False):
    unit = UNIT[dt]
    tol = (F32 + (PARTS if state and unit else 0.0)) * size
    if not state:
        tol = tol + unit * size + unit * want.abs() + TINY[dt] * 2
    bad = ((got.double() - want).abs() > tol + 1e-30) | got.isnan()
    assert not bool(bad.any()), (float((got.double() - want).abs().max()), int(bad.sum()), torch.nonzero(bad)[:4].tolist())


def _check(lens, H, dk, dv, dt, lay="joint", states=True, even=False, seed=1):
    B = _bind()
    st = _inputs(lens, H, dk, dv, dt, seed, lay)
    q, k, v = st["q_k_v"]
    scale = 0.37
    how = dict(seq_start=None if even else st["starts"], num_seqs=len(lens), scale=scale)
    s_last, ds0 = torch.full_like(st["s0"], 7.0), torch.full_like(st["s0"], 7.0)
    B.decay_attention_forward(q, k, v, st["out"], st["decay"], s0=st["s0"] if states else None,
                              s_last=s_last if states else None, **how)
    dq, dkey, dv_ = st["grads"]
    B.decay_attention_backward(q, k, v, st["dout"], dq, dkey, dv_, st["decay"], s0=st["s0"] if states else None,
                               ds_last=st["ds_last"] if states else None, ds0=ds0 if states else None, **how)
    x = [t.double() for t in (q, k, v)]
    do, g, on = st["dout"].double(), st["decay"].double(), 1.0 if states else 0.0
    s0, dl = on * st["s0"].double(), on * st["ds_last"].double()
    c = float(torch.tensor(scale))      # as 32 bits hold it
    want = plain(*x, g, c, s0, lens) + plain_backward(*x, do, g, c, s0, dl, lens)
    x = [t.abs() for t in x]
    size = plain(*x, g, c, s0.abs(), lens) + plain_backward(*x, do.abs(), g, c, s0.abs(), dl.abs(), lens)
    for got, w, z, is_state in zip((st["out"], s_last, dq, dkey, dv_, ds0), want, size, (0, 1, 0, 0, 0, 1)):
        if states or not is_state:
            _near(got, w, z, dt, bool(is_state))


LENS = [[1], [0, 5, 0], [31, 32, 33], [64, 127, 128, 1, 129], [300]]
DIMS = [(1, 1, 1), (2, 16, 16), (3, 37, 53), (2, 64, 64), (1, 128, 128), (5, 64, 128), (2, 128, 72), (2, 8, 120)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths(lens, dt):
    for H, dk, dv in ((2, 64, 64), (1, 128, 128), (2, 24, 40)):
        _check(lens, H, dk, dv, dt, lay="plain")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("H,dk,dv", DIMS)
def test_head_sizes_and_layouts(H, dk, dv, dt):
    for lay in ("joint", "heads", "plain"):
        _check([70, 3, 140], H, dk, dv, dt, lay=lay)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_without_states_and_of_equal_lengths(dt):
    _check([50] * 4, 2, 64, 64, dt, states=False, even=True, lay="plain")
    _check([130] * 3, 2, 32, 48, dt, even=True, lay="heads")
    _check([0, 0], 2, 8, 8, dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_long_sequences_in_parts(dt):
    """A few long sequences are cut into parts (a workspace is taken)."""
    B = _bind()
    for lens, H, dk, dv in (([2500], 2, 64, 64), ([1, 3300, 0, 1700], 1, 128, 96), ([2049], 1, 21, 10)):
        args = B.ATTENTION.pack(B.DTYPES[dt], len(lens), H, dk, dv, 1.0, sum(lens), 4096, *([0] * 31))
        assert B._lib.dgc_decay_attention_workspace_bytes(args, 0) > 0
        assert B._lib.dgc_decay_attention_workspace_bytes(args, 1) > 0
        _check(lens, H, dk, dv, dt, lay="plain")


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 128, 33])
def test_nothing_crosses_from_one_sequence_into_another(dt, dim):
    B = _bind()
    lens, H = [70, 130, 200, 10], 2
    st = _inputs(lens, H, dim, dim, dt, lay="plain")
    q, k, v = st["q_k_v"]
    dq, dk, dv = st["grads"]
    how = dict(seq_start=st["starts"], num_seqs=4)

    def all_of():
        for t in (st["out"], dq, dk, dv):
            t.fill_(7.0)
        B.decay_attention_forward(q, k, v, st["out"], st["decay"], **how)
        B.decay_attention_backward(q, k, v, st["dout"], dq, dk, dv, st["decay"], **how)
        return [t.clone() for t in (st["out"], dq, dk, dv)]
    before = all_of()
    for t in (q, k, v, st["dout"]):
        t[70:200] = float("nan")
        t[390, 0] = float("inf")
    after = all_of()
    for a, b in zip(before, after):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[400:], b[400:])
        assert torch.equal(a[200:400, 1], b[200:400, 1])      # (the other head's)
        assert bool(b[70:200].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_rows_outside_the_sequences_stay(dt):
    B = _bind()
    st = _inputs([300], 2, 64, 64, dt, lay="plain")
    q, k, v = st["q_k_v"]
    dq, dk, dv = st["grads"]
    starts = torch.tensor([20, 150, 270], dtype=torch.int32, device="cuda")
    B.decay_attention_forward(q, k, v, st["out"], st["decay"], seq_start=starts, num_seqs=2)
    B.decay_attention_backward(q, k, v, st["dout"], dq, dk, dv, st["decay"], seq_start=starts, num_seqs=2)
    for t in (st["out"], dq, dk, dv):
        assert bool((t[:20] == 7).all()) and bool((t[270:] == 7).all()) and not bool((t[20:270] == 7).all(2).any())


@pytest.mark.gpu
def test_a_damaged_table_leads_nowhere_else():
    """Offsets outside the tensors are clamped, whatever their order."""
    B = _bind()
    N, H, d = 200, 2, 64
    for dt in (torch.bfloat16, torch.float32):
        room = [torch.full((N + 80, H, d), 3.0, device="cuda").to(dt) for _ in range(4)]
        q, k, v, out = (t[40:-40] for t in room)
        for table in ([-50, 90, 10 ** 9], [150, 20, 400], [2 ** 31 - 1, -2 ** 31, 77]):
            B.decay_attention_forward(q, k, v, out, torch.ones(H, device="cuda"),
                                      seq_start=torch.tensor(table, dtype=torch.int64).to(torch.int32).cuda(), num_seqs=2)
            torch.cuda.synchronize()
            assert bool((room[3][:40] == 3).all()) and bool((room[3][-40:] == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_heads_that_share_keys(dt):
    """Inputs whose heads are one (stride 0): each head's gradient is its own."""
    B = _bind()
    st = _inputs([150, 33], 3, 64, 64, dt, lay="plain")
    q, k, v = st["q_k_v"]
    k1 = k[:, :1].expand(-1, 3, -1)
    dq, dk, dv = st["grads"]
    how = dict(seq_start=st["starts"], num_seqs=2)
    B.decay_attention_forward(q, k1, v, st["out"], st["decay"], **how)
    B.decay_attention_backward(q, k1, v, st["dout"], dq, dk, dv, st["decay"], **how)
    got = [t.clone() for t in (st["out"], dq, dk, dv)]
    whole = k1.contiguous()
    B.decay_attention_forward(q, whole, v, st["out"], st["decay"], **how)
    B.decay_attention_backward(q, whole, v, st["dout"], dq, dk, dv, st["decay"], **how)
    for a, b in zip(got, (st["out"], dq, dk, dv)):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("R,H,dk,dv", [(1, 1, 1, 1), (5, 3, 37, 53), (64, 2, 128, 128), (3, 8, 64, 96), (2, 2, 128, 6)])
def test_step(R, H, dk, dv, dt):
    B = _bind()
    gen = torch.Generator(device="cuda").manual_seed(R)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k, v = r(R, H, dk).to(dt), r(R, H, dk).to(dt), r(H, R, dv).to(dt).transpose(0, 1)
    slots = R + 2
    state, out = r(slots, H, dk, dv), torch.full((R, H, dv), 7.0, device="cuda").to(dt)
    at = torch.randperm(slots, generator=gen, device="cuda")[:R].to(torch.int32)
    if R > 2:
        at[1], at[2] = -1, slots
    decay = torch.linspace(0, 1, H, device="cuda")
    before = state.double()
    B.decay_attention_step(q, k, v, state, out, decay, slots=at, scale=0.5)
    want = before.clone()
    for row, s in enumerate(at.tolist()):
        if not 0 <= s < slots:
            assert bool((out[row] == 0).all())
            continue
        new = decay.double()[:, None, None] * before[s] + k[row].double()[:, :, None] * v[row].double()[:, None, :]
        want[s] = new
        size = 0.5 * (q[row].double().abs()[:, :, None] * (before[s].abs() + (k[row].double()[:, :, None] * v[row].double()[:, None, :]).abs())).sum(1)
        w = 0.5 * (q[row].double()[:, :, None] * new).sum(1)
        assert bool(((out[row].double() - w).abs() <= 130 * 2.0 ** -24 * size + UNIT[dt] * w.abs() + TINY[dt]).all())
    assert bool(((state.double() - want).abs() <= 2.0 ** -22 * (before.abs() + want.abs() + 8)).all())
    untouched = torch.ones(slots, dtype=torch.bool, device="cuda")
    untouched[at[(at >= 0) & (at < slots)].long()] = False
    assert torch.equal(state[untouched].double(), before[untouched])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_steps_continue_a_prompt(dt):
    """A prompt's state, then single tokens, against the whole at once."""
    B = _bind()
    H, d, n, m = 4, 64, 140, 9
    st = _inputs([n + m] * 2, H, d, d, dt, lay="plain")
    q, k, v = (t.view(2, n + m, H, d) for t in st["q_k_v"])
    whole, last = torch.empty_like(v), torch.empty(2, H, d, d, device="cuda")
    B.decay_attention_forward(*st["q_k_v"], whole.view(-1, H, d), st["decay"], num_seqs=2, s_last=last)
    cache = torch.zeros(5, H, d, d, device="cuda")
    state = torch.empty(2, H, d, d, device="cuda")
    head = [t[:, :n].reshape(-1, H, d) for t in (q, k, v)]
    out = torch.empty_like(head[2])
    B.decay_attention_forward(*head, out, st["decay"], num_seqs=2, s_last=state)
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    cache[slots.long()] = state
    one = torch.empty(2, H, d, dtype=dt, device="cuda")
    bound = 8 * d                                       # |q . S| of standard normal numbers, far out
    for t in range(n, n + m):
        B.decay_attention_step(q[:, t], k[:, t], v[:, t], cache, one, st["decay"], slots=slots)
        assert float((one.double() - whole[:, t].double()).abs().max()) <= (4 * UNIT[dt] + 1e-4) * bound * 4
    assert float((cache[slots.long()] - last).abs().max()) <= 2 * (F32 + PARTS) * 20 * 20


@pytest.mark.gpu
def test_a_captured_call_follows_its_inputs():
    B = _bind()
    st = _inputs([2000], 2, 64, 64, torch.bfloat16, lay="plain")     # with a workspace
    q, k, v = st["q_k_v"]
    dq, dk, dv = st["grads"]

    def both():
        B.decay_attention_forward(q, k, v, st["out"], st["decay"])
        B.decay_attention_backward(q, k, v, st["dout"], dq, dk, dv, st["decay"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            both()
    v.copy_(torch.randn_like(v.float()))
    both()
    want = [t.clone() for t in (st["out"], dq, dk, dv)]
    for g in graphs:
        for t in (st["out"], dq, dk, dv):
            t.fill_(7.0)
        g.replay()
        for a, b in zip(want, (st["out"], dq, dk, dv)):
            assert torch.equal(a, b)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """A cache of states and rows that lie further than 2^31 elements on."""
    B = _bind()
    H, d = 32, 128
    slots = 2 ** 31 // (H * d * d) + 3
    cache = torch.empty(slots, H, d, d, device="cuda")
    q, k, v = (torch.randn(2, H, d, device="cuda") for _ in range(3))
    at, out, g = torch.tensor([slots - 1, 1], dtype=torch.int32, device="cuda"), torch.empty(2, H, d, device="cuda"), torch.ones(H, device="cuda")
    few = torch.randn(2, H, d, d, device="cuda")
    cache[at.long()] = few
    B.decay_attention_step(q, k, v, cache, out, g, slots=at)
    same, ref = few.clone(), torch.empty_like(out)
    B.decay_attention_step(q, k, v, same, ref, g)
    assert torch.equal(out, ref) and torch.equal(cache[at.long()], same)
    del cache
    N, ld = 70000, 32768                                   # 2^31 elements are passed at token 65536
    for dt, dim in ((torch.bfloat16, 64), (torch.bfloat16, 63), (torch.float32, 32)):
        wide = torch.empty(N, ld, dtype=dt, device="cuda")
        parts = [wide[:, i * 64:i * 64 + dim].unflatten(1, (1, dim)) for i in range(4)]
        small = [torch.randn(N, 1, dim, device="cuda").to(dt) for _ in range(3)]
        for p, s in zip(parts, small):
            p.copy_(s)
        decay, ref = torch.full((1,), 0.9, device="cuda"), torch.empty_like(small[2])
        starts = torch.tensor([0, 65000, N], dtype=torch.int32, device="cuda")
        B.decay_attention_forward(*parts, decay, seq_start=starts, num_seqs=2)
        B.decay_attention_forward(*small, ref, decay, seq_start=starts, num_seqs=2)
        assert torch.equal(parts[3].reshape(ref.shape), ref)
        del wide, parts


# ----------------------------------------------------------------- refusals, device and stream

def _packed(B, **change):
    at = 4096
    a = dict(dtype=1, num_seqs=2, heads=3, dk=16, dv=24, scale=1.0, tokens=10, seq_start=at, decay=at,
             q=(at, 48, 16), k=(at, 48, 16), v=(at, 72, 24), out=(at, 72, 24), s0=at, s_last=at,
             dout=(at, 72, 24), dq=(at, 48, 16), dk_=(at, 48, 16), dv_=(at, 72, 24), ds_last=at, ds0=at, work=0, bytes=0)
    a.update(change)
    flat = []
    for v in a.values():
        flat += list(v) if isinstance(v, tuple) else [v]
    return B.ATTENTION.pack(*flat)


def test_refusals():
    """Found on the host: nothing is enqueued, so that this runs without a GPU."""
    from paper_1712_01887_b200 import binding as B
    both = (B._lib.dgc_decay_attention_forward, B._lib.dgc_decay_attention_backward)
    at = 4096
    for change in (dict(dtype=3), dict(dtype=-1), dict(num_seqs=0), dict(heads=0), dict(heads=65536), dict(dk=0), dict(dk=129),
                   dict(dv=0), dict(dv=129), dict(scale=float("nan")), dict(scale=float("inf")), dict(tokens=-1),
                   dict(tokens=2 ** 31), dict(seq_start=0, tokens=11), dict(seq_start=at + 2), dict(decay=0),
                   dict(q=(0, 48, 16)), dict(q=(at + 1, 48, 16)), dict(k=(at, -1, 16)), dict(v=(at, 72, -24)), dict(s0=at + 1),
                   dict(work=at + 8, bytes=64)):
        for call in both:
            assert call(_packed(B, **change), None) == B.EINVAL, change
    for change in (dict(out=(at, 71, 24)), dict(out=(at, 72, 23)), dict(out=(at, 0, 24)), dict(s_last=at + 2)):
        assert both[0](_packed(B, **change), None) == B.EINVAL, change
    for change in (dict(dout=(0, 72, 24)), dict(dq=(at, 47, 16)), dict(dk_=(at, 16, 159)), dict(dv_=(at, 72, 0)),
                   dict(ds_last=at + 1), dict(ds0=at + 2)):
        assert both[1](_packed(B, **change), None) == B.EINVAL, change
    assert both[0](None, None) == B.EINVAL and both[1](None, None) == B.EINVAL
    assert B._lib.dgc_decay_attention_workspace_bytes(_packed(B, dk=129), 0) == B.EINVAL
    long = dict(num_seqs=1, tokens=60000, work=at)
    need = B._lib.dgc_decay_attention_workspace_bytes(_packed(B, **long), 1)
    assert need > 0 and both[1](_packed(B, bytes=need - 1, **long), None) == B.ECAPACITY
    step = B._lib.dgc_decay_attention_step
    good = [1, 4, 3, 16, 24, 5, 1.0, 0, at, at, 48, 16, at, 48, 16, at, 72, 24, at, 72, 24, at, at]
    for place, value in ((0, 5), (1, -1), (2, 0), (3, 129), (4, 0), (5, -1), (6, float("nan")), (8, 0), (9, 0), (10, -1), (12, at + 1),
                         (19, 71), (21, 0), (21, at + 2), (22, at + 1)):
        bad = list(good)
        bad[place] = value
        assert step(B.ATTENTION_ONE.pack(*bad), None) == B.EINVAL, (place, value)
    bad = list(good)
    bad[5], bad[22] = 3, 0                      # fewer slots than rows, and no table
    assert step(B.ATTENTION_ONE.pack(*bad), None) == B.EINVAL and step(None, None) == B.EINVAL


def _calls(B, device, **how):
    h = lambda d=16: Tensor((10, 3, d), device=device)  # noqa: E731
    g = Tensor((3,), device=device)
    yield lambda: B.decay_attention_forward(h(), h(), h(24), h(24), g, **how)
    yield lambda: B.decay_attention_backward(h(), h(), h(24), h(24), h(), h(), h(24), g, **how)
    yield lambda: B.decay_attention_step(h(), h(), h(24), Tensor((10, 3, 16, 24), device=device), h(24), g, **how)


def test_device_and_stream(machine, monkeypatch):  # noqa: F811
    from paper_1712_01887_b200 import binding as B

    def called(args, stream):
        machine.calls.append((machine.current, stream))
        return 0
    for name in ("dgc_decay_attention_forward", "dgc_decay_attention_backward", "dgc_decay_attention_step"):
        monkeypatch.setattr(B._lib, name, called)
    for call in _calls(B, 1):
        call()
    for call in _calls(B, 1, stream=Stream(77, 1)):
        call()
    assert machine.calls == [(1, 101)] * 3 + [(1, 77)] * 3 and machine.current == 0
    for call in _calls(B, 1, stream=Stream(0, 0)):
        with pytest.raises(ValueError):
            call()
    wrong = Tensor((10, 3, 16), torch.float16, 1)
    for call in (lambda: B.decay_attention_forward(wrong, *[Tensor((10, 3, 16))] * 3, Tensor((3,))),
                 lambda: B.decay_attention_forward(*[Tensor((10, 3, 16))] * 3, Tensor((10, 3, 17)), Tensor((3,))),
                 lambda: B.decay_attention_forward(*[Tensor((10, 3, 16))] * 4, Tensor((4,))),
                 lambda: B.decay_attention_forward(*[Tensor((10, 48))] * 4, Tensor((3,)))):
        with pytest.raises(ValueError):
            call()
    assert len(machine.calls) == 6


def test_struct_sizes():
    from paper_1712_01887_b200 import binding as B
    heads = struct.calcsize("@P2q")
    assert heads == 24 and B.ATTENTION.size == 32 + 16 + 8 * heads + 6 * 8 and B.ATTENTION_ONE.size == 32 + 8 + 4 * heads + 16
    assert ctypes.sizeof(ctypes.c_void_p) == 8
