"""Linear attention (dgc_decay_attention_*) over the ranges of its types, in parts of many chunks, in packs of many sequences.

The reference works in chunks, in 64 bits, and is held against the recurrence itself.  Tolerances, beside those of
test_decay_attention.py (F32, UNIT, PARTS there; the errors' `size` is the formula with absolute values):
 * `small`: what is told apart by its 2-norm.  A 16-bit call rounds the weights decay^n q.k, the state and the result by at
   most half a unit each.  For independent inputs of mean zero, the terms' 2-norm is the result's, so that the three come to at
   most 3 UNIT of it, beside 2^-25 for each element of a float16 result (half the step below its range).
 * Factors that are powers of two and the scale's remainder add less than 2 ulp of 32 bits to a term, within F32.
 * float16 states are sums of terms held to 2^-25 of one key (of the scale for the gradient's, half a unit more where that is no
   power of two): 2^-24 of the sum of the other factor's absolute values."""
import pytest
import torch

from test_decay_attention import DT, F32, PARTS, TINY, UNIT, _bind, plain, plain_backward

C = 64


def chunked(q, k, v, decay, scale, s0):
    """(out, s_last) of one sequence."""
    n, S, out = q.shape[0], s0.clone(), torch.empty_like(v)
    g = decay[:, None, None]
    for t in range(0, n, C):
        m = min(C, n - t)
        i = torch.arange(m, device=q.device)
        away = i[:, None] - i
        D = torch.where(away >= 0, g ** away.clamp(min=0), 0.0)
        x, y, z = (a[t:t + m].transpose(0, 1) for a in (q, k, v))
        o = ((x @ y.transpose(1, 2)) * D) @ z + g ** (i + 1)[:, None] * (x @ S)
        out[t:t + m] = scale * o.transpose(0, 1)
        S = g ** m * S + (y * g ** (m - 1 - i)[:, None]).transpose(1, 2) @ z
    return out, S


def chunked_backward(q, k, v, do, decay, scale, s0, ds_last):
    """(dq, dk, dv, ds0) of one sequence: the gradients' walks are forward walks with other roles, the late ones from the
    last token on.  (E reaches a token undecayed, the walk decays its state first: what is put in is E / decay.)"""
    dq = chunked(do, v, k, decay, scale, s0.transpose(1, 2))[0]
    back = [a.flip(0) for a in (q, k, v, do)]
    one = torch.ones_like(decay)
    gap = torch.where(decay > 0, decay, one)[:, None, None]      # (a decay of 0 is tested elsewhere)
    dv, last = chunked(back[1], scale * back[0], back[3], decay, 1.0, ds_last / gap)
    dk = chunked(back[2], scale * back[3], back[0], decay, 1.0, ds_last.transpose(1, 2) / gap)[0]
    return dq, dk.flip(0), dv.flip(0), last * gap


def reference(q, k, v, do, decay, scale, s0, dl, lens):
    """(out, s_last, dq, dk, dv, ds0) of a pack."""
    parts, at = [], 0
    for s, n in enumerate(lens):
        cut = [a[at:at + n] for a in (q, k, v)]
        d = do[at:at + n]
        if n:
            parts.append(chunked(*cut, decay, scale, s0[s]) + chunked_backward(*cut, d, decay, scale, s0[s], dl[s]))
        else:
            parts.append((cut[2], s0[s], cut[0], cut[1], cut[2], dl[s]))
        at += n
    return [torch.cat([p[i] for p in parts]) if i in (0, 2, 3, 4) else torch.stack([p[i] for p in parts]) for i in range(6)]


def test_reference_agrees_with_the_recurrence():
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    N, H, dk, dv, lens = 210, 2, 3, 5, [130, 0, 1, 79]
    x = (r(N, H, dk), r(N, H, dk), r(N, H, dv), r(N, H, dv))
    decay, s0, dl = torch.tensor([0.9, 1.0], dtype=torch.float64), r(4, H, dk, dv), r(4, H, dk, dv)
    got = reference(*x, decay, 0.3, s0, dl, lens)
    want = plain(*x[:3], decay, 0.3, s0, lens) + plain_backward(*x, decay, 0.3, s0, dl, lens)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-10, atol=1e-11)


def _data(lens, H, dk, dv, dt, seed=1, size=(1.0, 1.0, 1.0, 1.0), states=(1.0, 1.0), decays=(0.97, 1.0, 0.5, 0.999)):
    """q, k, v, dout of normal numbers times `size`; s0, ds_last times `states`."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    N, S = sum(lens), len(lens)
    x = [(torch.randn(N, H, d, generator=gen, device="cuda") * a).to(dt) for d, a in zip((dk, dk, dv, dv), size)]
    s = [torch.randn(S, H, dk, dv, generator=gen, device="cuda") * a for a in states]
    decay = torch.tensor([decays[h % len(decays)] for h in range(H)], device="cuda")
    return x, s, decay


def _run(lens, x, s, decay, scale):
    B = _bind()
    q, k, v, do = x
    starts = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    how = dict(seq_start=starts, num_seqs=len(lens), scale=scale)
    out, dq, dk, dv = (torch.full_like(t, 7.0) for t in (v, q, k, v))
    last, ds0 = torch.full_like(s[0], 7.0), torch.full_like(s[0], 7.0)
    B.decay_attention_forward(q, k, v, out, decay, s0=s[0], s_last=last, **how)
    B.decay_attention_backward(q, k, v, do, dq, dk, dv, decay, s0=s[0], ds_last=s[1], ds0=ds0, **how)
    B.tensor_check()
    return [out, last, dq, dk, dv, ds0]


NAMES = ("out", "s_last", "dq", "dk", "dv", "ds0")


def _verify(got, x, s, decay, scale, lens, only=range(6)):
    """By element against `size` and, for rows, by 2-norm as `small` says."""
    dt, c = x[0].dtype, float(torch.tensor(scale))
    x, s, g = [t.double() for t in x], [t.double() for t in s], decay.double()
    want = reference(*x, g, c, *s, lens)
    size = reference(*[t.abs() for t in x], g, abs(c), *[t.abs() for t in s], lens)
    floor = [0.0] * 6
    if dt == torch.float16:
        y = [torch.stack([p.abs().sum(0) for p in t.split(lens)])[:, :, None, :] for t in (x[2], x[3])]     # [seqs, heads, 1, dv]
        floor[1], floor[5] = 2.0 ** -24 * y[0], 2.0 ** -24 * abs(c) * y[1]
    for name, a, w, z, low in [r for i, r in enumerate(zip(NAMES, got, want, size, floor)) if i in only]:
        assert bool(a.isfinite().all()), name
        err, is_state = (a.double() - w).abs(), name in ("s_last", "ds0")
        unit = 0.0 if is_state else UNIT[dt]
        tol = (F32 + (PARTS if is_state and UNIT[dt] else 0.0)) * z + unit * (z + w.abs()) + (low if is_state else TINY[dt])
        assert bool((err <= tol + 1e-30).all()), (name, float(err.max()), float((err / (tol + 1e-30)).max()))
        if unit:
            bound = 3 * unit * w.norm() + TINY[dt] * w.numel() ** 0.5 + F32 * z.norm()
            assert float(err.norm()) <= float(bound), (name, float(err.norm() / w.norm()), float(bound / w.norm()))


# ----------------------------------------------------------------- the types' ranges

@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale,size,states", [
    (1e-8, (1.0, 1.0, 1.0, 1e4), (1.0, 1e-4)),          # (results of some 1e-3)
    (1e-6, (1.0, 1.0, 1.0, 3e3), (1.0, 1e-2)),
    (-3e-4, (1.0, 1.0, 1.0, 30.0), (1.0, 1e-2)),
    (1e5, (0.01, 0.01, 0.01, 1e-3), (1e-3, 1.0)),
    (1e6, (0.01, 0.003, 0.003, 1e-3), (1e-4, 1.0)),
    (0.0, (1.0, 1.0, 1.0, 1.0), (1.0, 1.0)),
], ids=lambda p: str(p) if isinstance(p, float) else "")
def test_scales_of_any_size(scale, size, states, dim, dt):
    """The scale is any finite number: what counts is that the results are in range."""
    lens = [300, 0, 129]
    x, s, decay = _data(lens, 2, dim, dim, dt, size=size, states=states)
    _verify(_run(lens, x, s, decay, scale), x, s, decay, scale, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("small", [1e-3, 1e-4, 1e-5])
def test_small_gradients(small, dim, dt):
    """A mean loss over a few thousand tokens: dout far below 1."""
    lens = [1000, 24]
    x, s, decay = _data(lens, 2, dim, dim, dt, size=(1.0, 1.0, 1.0, small), states=(1.0, small), decays=(0.99, 0.9))
    _verify(_run(lens, x, s, decay, dim ** -0.5), x, s, decay, dim ** -0.5, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 128])
def test_gradients_of_very_different_tokens(dim, dt):
    """dout 2^-12 of its usual size in some chunks, none in others, and a whole sequence far below the rest: each is held against
    its own sequence's reference."""
    lens = [700, 260]
    x, s, decay = _data(lens, 2, dim, dim, dt, states=(1.0, 0.0), decays=(0.99, 0.9))
    x[3][128:256] = 0
    x[3][256:300] *= 2.0 ** -12
    x[3][700:] *= 2.0 ** -12
    got = _run(lens, x, s, decay, dim ** -0.5)
    _verify(got, x, s, decay, dim ** -0.5, lens)
    behind = lambda t: t[1:] if t.dim() == 4 else t[700:]  # noqa: E731
    _verify([behind(t) for t in got], [t[700:] for t in x], [t[1:] for t in s], decay, dim ** -0.5, [260])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("dim", [64, 128])
def test_states_of_the_gradient_above_the_types_range(dim, dt):
    """The state's gradient is of some 1e6, where float16 ends at 65504."""
    lens = [900, 200]
    x, s, decay = _data(lens, 2, dim, dim, dt, size=(1.0, 1e-3, 1e-3, 1.0), states=(1.0, 1e6), decays=(1.0, 0.999))
    _verify(_run(lens, x, s, decay, 0.01), x, s, decay, 0.01, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("g", [2e-5, 1e-20, 1e-37, 1e-44])
def test_decays_near_0(g, dt):
    """A token's own weight is decay^0, one, whatever the decay."""
    lens = [200]
    x, s, decay = _data(lens, 2, 64, 64, dt, states=(0.0, 0.0), decays=(g, g * 1.37))
    _verify(_run(lens, x, s, decay, 0.3), x, s, decay, 0.3, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_captured_calls_and_two_streams(dt):
    """A captured backward call follows its inputs (dout a thousand times smaller than at the capture), and calls on two streams at
    once give what they give alone."""
    B = _bind()
    lens = [400, 0, 90]
    x, s, decay = _data(lens, 3, 64, 64, dt)
    scale = 0.125
    q, k, v, do = x
    starts = torch.tensor([0, 400, 400, 490], dtype=torch.int32, device="cuda")
    sets = [[torch.empty_like(t) for t in (q, k, v)] + [torch.empty_like(s[0])] for _ in range(3)]

    def call(to, stream=None):
        B.decay_attention_backward(q, k, v, do, *to[:3], decay, seq_start=starts, num_seqs=3, s0=s[0], ds_last=s[1], ds0=to[3], scale=scale,
                                   stream=stream)
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    side[0].wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side[0]):
        call(sets[0])
    torch.cuda.current_stream().wait_stream(side[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(sets[0])
    do.mul_(1e-3)
    s[1].mul_(1e-3)
    graph.replay()
    call(sets[1])
    for a, b in zip(sets[0], sets[1]):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, to in zip(side, (sets[0], sets[2])):
            call(to, stream)
    torch.cuda.synchronize()
    for to in (sets[0], sets[2]):
        for a, b in zip(to, sets[1]):
            assert torch.equal(a, b)
    _verify([torch.zeros_like(v), s[0]] + sets[1], x, s, decay, scale, lens, only=(2, 3, 4, 5))
