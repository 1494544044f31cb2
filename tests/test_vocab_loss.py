"""Softmax cross entropy from hidden rows and output matrix (dgc_vocab_loss_*) against the definition in 64 bits.

Tolerances.  A logit is a sum of `hidden` products in 32 bits: off by at most A = (hidden + 2) 2^-23 of the sum of
their absolute values (2^-23: a tensor core's additions may cut off instead of rounding), at most L for
a row.  The loss is off by 2 L and a few ulp of its parts (the exponents of the sum: 2^-23 of their size,
under 64, each).  A probability is off by d = 2 L + 2^-16 of itself, so G by d |dloss| (p + [label]) and, in a 16-bit call,
by half a unit of itself, in f16 also by the step below its range, 2^-25 of the scaled G's unit (2^-10 |dloss|).  The
gradients sum these over their terms in 32 bits (2^-23 a term at worst, which for the longest sum here is
70000 * 2^-23 and in practice its root; the bound taken is 2^-15 of the sum of absolute values) and are rounded once."""
import pytest
import torch

from test_operator_calls import Stream, Tensor, machine  # noqa: F401  (stand-ins for tensors and devices)

DT = [torch.float32, torch.bfloat16, torch.float16]
UNIT = {torch.float32: 0.0, **{d: torch.finfo(d).eps / 2 for d in (torch.bfloat16, torch.float16)}}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
INF = float("inf")


def _bind():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    from paper_1712_01887_b200 import binding as B
    return B


def plain(h, w, b, labels, dloss):
    """(loss, G, L) in 64 bits: G [rows, vocab], L the bound of a row's logits' errors."""
    there = (labels >= 0) & (labels < w.shape[0])
    h = torch.where(there[:, None], h.double(), 0.0)
    logits = h @ w.double().t()
    size = (h.abs() @ w.double().abs().t())
    if b is not None:
        logits = logits + b.double()
        size = size + torch.where(b <= -1e4, 0.0, b.double().abs())       # (masked words: no part of the sum)
    y = torch.where(there, labels, 0).long()[:, None]
    m = logits.amax(1, keepdim=True).clamp(min=-1e300)
    e = torch.exp(logits - m)
    total = e.sum(1, keepdim=True)
    loss = torch.where(there, (torch.log(total) + m - logits.gather(1, y))[:, 0], 0.0)
    p = torch.where(total > 0, e / total, 0.0)
    hot = torch.zeros_like(p).scatter_(1, y, 1.0)
    weight = torch.where(there, dloss.double(), 0.0)[:, None]
    L = (h.shape[1] + 2) * 2.0 ** -23 * size.amax(1)
    return loss, weight * (p - hot), weight.abs() * (p + hot), L


def test_plain_gradient_agrees_with_differences():
    gen = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    h, w, b, d = r(4, 5), r(7, 5), r(7), r(4)
    y = torch.tensor([3, 0, -1, 6], dtype=torch.int32)
    vh, vw, vb = r(4, 5), r(7, 5), r(7)
    value = lambda e: (plain(h + e * vh, w + e * vw, b + e * vb, y, d)[0] * d).sum()  # noqa: E731
    _, G, _, _ = plain(h, w, b, y, d)
    h = torch.where((y >= 0)[:, None], h, 0.0)
    want = ((G @ w) * vh).sum() + ((G.t() @ h) * vw).sum() + (G.sum(0) * vb).sum()
    assert torch.allclose((value(1e-6) - value(-1e-6)) / 2e-6, want, rtol=1e-7)


def _inputs(R, V, D, dt, bias, seed=1, spread=2.0, pad=(0, 0)):
    gen = torch.Generator(device="cuda").manual_seed(seed + V)
    n = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    lead, more = pad
    h = (n(R, lead + D + more)).to(dt)[:, lead:lead + D]
    w = (n(V, lead + D + more) * spread * D ** -0.5).to(dt)[:, lead:lead + D]
    b = n(V).to(dt) if bias else None
    y = torch.randint(0, V, (R,), generator=gen, device="cuda", dtype=torch.int32)
    if R >= 3:
        y[R // 2] = -1
    if R >= 5:
        y[1] = V
    return h, w, b, y, torch.rand(R, generator=gen, device="cuda") + 0.5


def _near(got, want, size, noise, dt):
    """size: sum of absolute values of the terms; noise: of their errors."""
    tol = noise + 2.0 ** -15 * size + UNIT[dt] * want.abs() + 2 * TINY[dt]
    bad = ((got.double() - want).abs() > tol + 1e-30) | got.isnan()
    assert not bool(bad.any()), (float((got.double() - want).abs().max()), int(bad.sum()), torch.nonzero(bad)[:4].tolist())


def _verify(h, w, b, y, d, dt, loss, dh, dw, db):
    want, G, size, L = plain(h, w, b, y, d)
    there = (y >= 0) & (y < w.shape[0])
    fine = torch.isfinite(want)
    assert torch.equal(loss[~fine].double(), want[~fine])
    assert bool(((loss.double() - want).abs() <= 2 * L + 2.0 ** -22 * (64 + want.abs()))[fine].all()), float((loss.double() - want)[fine].abs().max())
    assert bool((loss[~there] == 0).all())
    noise = size * (2 * L + 2.0 ** -16)[:, None] + UNIT[dt] * G.abs()
    if dt == torch.float16:
        noise = noise + torch.where(there, d.abs().max() * 2.0 ** -35, 0.0)[:, None]
    W, H = w.double().abs(), torch.where(there[:, None], h.double(), 0.0)
    _near(dh, G @ w.double(), size @ W, noise @ W, dt)
    _near(dw, G.t() @ H, size.t() @ H.abs(), noise.t() @ H.abs(), dt)
    if db is not None:
        _near(db, G.sum(0), size.sum(0), noise.sum(0), dt)
    assert bool((dh[~there] == 0).all())


def _run(B, h, w, b, y, d, dt):
    """All calls; the one-call form has to give what the two give."""
    R, V = h.shape[0], w.shape[0]
    out = []
    for joint in (False, True):
        loss, stats = torch.full((R,), 7.0, device="cuda"), torch.full((R, 2), 7.0, device="cuda")
        dh, dw = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
        db = None if b is None else torch.full((V,), 7.0, device="cuda").to(dt)
        if joint:
            B.vocab_loss_grad(h, w, y, d, loss, dh, dw, bias=b, dbias=db)
        else:
            B.vocab_loss_forward(h, w, y, loss, stats, bias=b)
            B.vocab_loss_backward(h, w, y, stats, d, dh, dw, bias=b, dbias=db)
        out.append((loss, dh, dw, db))
    return out


def _check(R, V, D, dt, bias, **how):
    h, w, b, y, d = _inputs(R, V, D, dt, bias, **how)
    for got in _run(_bind(), h, w, b, y, d, dt):
        _verify(h, w, b, y, d, dt, *got)


SIZES = [(1, 1, 1), (1, 7, 64), (3, 300, 8), (5, 257, 33), (40, 1000, 129), (129, 513, 64), (257, 2049, 200), (300, 4099, 72), (2, 20011, 520)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("R,V,D", SIZES)
def test_sizes(R, V, D, dt):
    _check(R, V, D, dt, bias=R % 2 == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("pad", [(1, 0), (8, 8), (0, 3), (16, 5)])
def test_strides_and_alignments(dt, pad):
    _check(130, 700, 96, dt, bias=True, pad=pad)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_many_pieces_of_a_large_vocabulary(dt):
    _check(1500, 70001, 64, dt, bias=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_large_logits_and_masked_words(dt):
    h, w, b, y, d = _inputs(70, 600, 64, dt, True, spread=60.0)
    b[::3] = -INF
    b[301] = torch.finfo(dt).min
    y[7], y[8], y[9] = 300, 299, 301       # a masked word, one that is not, one of the type's lowest value
    for loss, dh, dw, db in _run(_bind(), h, w, b, y, d, dt):
        want, _, _, L = plain(h, w, b, y, d)
        assert float(want[7]) == INF and torch.equal(loss == INF, want == INF)
        if dt != torch.float16:
            assert float(loss[9]) > 1e37
        else:
            assert 6e4 < float(loss[9]) < 7e4
        keep = torch.isfinite(want)
        keep[9] = False
        assert bool(((loss.double() - want).abs() <= 2 * L + 2.0 ** -22 * (64 + want.abs()))[keep].all())
        assert not bool(dh.isnan().any() | dw.isnan().any() | db.isnan().any())
        listed = torch.zeros(600, dtype=torch.bool, device="cuda")
        listed[y[(y >= 0) & (y < 600)].long()] = True
        assert not bool(db[::3][~listed[::3]].any())           # a masked word's p is 0


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_padding_rows_may_hold_anything(dt):
    B = _bind()
    h, w, b, y, d = _inputs(140, 500, 64, dt, True)
    y[10:20] = -1
    first = _run(B, h, w, b, y, d, dt)
    h[10:15], d[10:20] = float("nan"), float("nan")
    h[15:20] = INF
    for a, c in zip(first, _run(B, h, w, b, y, d, dt)):
        for s, t in zip(a, c):
            assert torch.equal(s, t)
    y[:] = -1
    for loss, dh, dw, db in _run(B, h, w, b, y, d, dt):
        assert not bool(loss.any() | dh.any()) and not bool(dw.any() | db.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_small_weights_of_rows(dt):
    """A mean over many tokens: G is far below what 16 bits of a narrow range hold."""
    h, w, b, y, d = _inputs(200, 3000, 64, dt, False)
    for scale in (1e-5, 1e3) if dt == torch.float16 else (1e-9, 1e6):
        dd = d * scale
        up = 1.0 if dt != torch.float16 else 2.0 ** 12 if scale < 1 else 1.0
        for loss, dh, dw, _ in _run(_bind(), h, (w * up).to(dt) if up != 1.0 else w, None, y, dd, dt)[:1]:
            ww = (w * up).to(dt) if up != 1.0 else w
            if up == 1.0:
                _verify(h, ww, None, y, dd, dt, loss, dh, dw, None)
            else:
                _, G, size, L = plain(h, ww, None, y, dd)
                noise = size * (2 * L + 2.0 ** -16)[:, None] + UNIT[dt] * G.abs() + dd.abs().max() * 2.0 ** -35
                _near(dh, G @ ww.double(), size @ ww.double().abs(), noise @ ww.double().abs(), dt)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_offsets_beyond_32_bits(dt):
    """An output matrix and its gradient whose rows lie further than 2^31 elements on."""
    B = _bind()
    V, D, ld = 70000, 64, 32768
    h, w, b, y, d = _inputs(20, V, D, dt, True)
    wide = torch.empty(V, ld, dtype=dt, device="cuda")
    far, dfar = wide[:, :D], wide[:, 1024:1024 + D]
    far.copy_(w)
    ref = _run(B, h, w, b, y, d, dt)[1]
    loss, dh, db = torch.empty(20, device="cuda"), torch.empty_like(h), torch.empty_like(b)
    B.vocab_loss_grad(h, far, y, d, loss, dh, dfar, bias=b, dbias=db)
    for got, want in zip((loss, dh, dfar, db), ref):
        assert torch.equal(got, want)


@pytest.mark.gpu
def test_waits_do_not_run_out():
    _bind().tensor_check()


@pytest.mark.gpu
def test_no_rows():
    B = _bind()
    for dt in DT:
        h, w, y = torch.empty(0, 16, device="cuda", dtype=dt), torch.randn(50, 16, device="cuda").to(dt), torch.empty(0, dtype=torch.int32, device="cuda")
        dw, db, e = torch.full_like(w, 7.0), torch.full((50,), 7.0, device="cuda").to(dt), torch.empty(0, device="cuda")
        B.vocab_loss_forward(h, w, y, e)
        B.vocab_loss_grad(h, w, y, e, e, torch.empty_like(h), dw, bias=db.clone(), dbias=db)
        assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_a_captured_call_follows_its_inputs(dt):
    B = _bind()
    h, w, b, y, d = _inputs(200, 1500, 64, dt, True)
    loss, dh, dw, db = torch.empty(200, device="cuda"), torch.empty_like(h), torch.empty_like(w), torch.empty_like(b)
    call = lambda: B.vocab_loss_grad(h, w, y, d, loss, dh, dw, bias=b, dbias=db)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for g in graphs:
        with torch.cuda.graph(g):
            call()
    h.copy_(torch.randn_like(h.float()))
    call()
    want = [t.clone() for t in (loss, dh, dw, db)]
    for g in graphs:
        for t in (loss, dh, dw, db):
            t.fill_(7.0)
        g.replay()
        for a, c in zip(want, (loss, dh, dw, db)):
            assert torch.equal(a, c)


# ----------------------------------------------------------------- refusals, device and stream

def _packed(B, **change):
    at = 4096
    a = dict(dtype=1, vocab=100, hidden=16, reserved=0, rows=10, h=at, h_ld=16, w=at, w_ld=16, bias=at, labels=at, loss=at,
             stats=at, dloss=at, dh=at, dh_ld=16, dw=at, dw_ld=16, dbias=at, work=at, bytes=1 << 40)
    a.update(change)
    return B.VOCAB_LOSS.pack(*a.values())


def test_refusals():
    """Found on the host: nothing is enqueued, so that this runs without a GPU."""
    from paper_1712_01887_b200 import binding as B
    at, lib = 4096, B._lib
    calls = dict(f=lib.dgc_vocab_loss_forward, b=lib.dgc_vocab_loss_backward, g=lib.dgc_vocab_loss_grad)
    for change in (dict(dtype=3), dict(vocab=0), dict(vocab=2 ** 31 - 1), dict(hidden=0), dict(hidden=65537), dict(rows=-1),
                   dict(rows=2 ** 31), dict(h=0), dict(h=at + 1), dict(h_ld=15), dict(w=0), dict(w_ld=15), dict(bias=at + 1),
                   dict(labels=0), dict(labels=at + 2), dict(work=at + 128), dict(bytes=-1)):
        for call in calls.values():
            assert call(_packed(B, **change), None) == B.EINVAL, change
    for which, change in (("f", dict(loss=0)), ("g", dict(loss=0)), ("f", dict(loss=at + 1)), ("f", dict(stats=at + 2)), ("b", dict(stats=0)),
                          ("b", dict(dloss=0)), ("g", dict(dloss=0)), ("b", dict(dh=0)), ("b", dict(dh_ld=15)), ("g", dict(dw=0)),
                          ("g", dict(dw_ld=3)), ("g", dict(dbias=at + 1))):
        assert calls[which](_packed(B, **change), None) == B.EINVAL, (which, change)
    for which, call in calls.items():
        need = lib.dgc_vocab_loss_workspace_bytes(_packed(B), which != "f")
        assert need > 0 and call(_packed(B, bytes=need - 1), None) == B.ECAPACITY and call(_packed(B, work=0), None) == B.ECAPACITY
        assert call(None, None) == B.EINVAL
    assert lib.dgc_vocab_loss_workspace_bytes(_packed(B, hidden=0), 0) == B.EINVAL
    # the workspace does not grow with rows x vocab
    big = lib.dgc_vocab_loss_workspace_bytes(_packed(B, rows=16384, vocab=262144, hidden=1024, h_ld=1024, w_ld=1024), 1)
    assert 0 < big < 16384 * 262144 * 2 // 8


def test_device_and_stream(machine, monkeypatch):  # noqa: F811
    from paper_1712_01887_b200 import binding as B
    asked = []

    def called(args, stream):
        machine.calls.append((machine.current, stream))
        return 0
    for name in ("dgc_vocab_loss_forward", "dgc_vocab_loss_backward", "dgc_vocab_loss_grad"):
        monkeypatch.setattr(B._lib, name, called)
    monkeypatch.setattr(B, "_work", lambda need, stream, device: asked.append((need > 0, stream, device)) or Tensor((need,), torch.uint8, device))

    def all_calls(device, **how):
        m, v = lambda n=6: Tensor((n, 40), device=device), lambda *s: Tensor(s, device=device)  # noqa: E731
        y = Tensor((6,), torch.int32, device)
        yield lambda: B.vocab_loss_forward(m(), m(90), y, v(6), **how)
        yield lambda: B.vocab_loss_backward(m(), m(90), y, v(6, 2), v(6), m(), m(90), **how)
        yield lambda: B.vocab_loss_grad(m(), m(90), y, v(6), v(6), m(), m(90), **how)
    for call in all_calls(1):
        call()
    stream = Stream(77, 1)
    for call in all_calls(1, stream=stream):
        call()
    assert machine.calls == [(1, 101)] * 3 + [(1, 77)] * 3 and machine.current == 0
    assert asked == [(True, None, 1)] * 3 + [(True, stream, 1)] * 3
    for call in all_calls(1, stream=Stream(0, 0)):
        with pytest.raises(ValueError):
            call()
    y = Tensor((6,), torch.int32, 1)
    for call in (lambda: B.vocab_loss_forward(Tensor((6, 40)), Tensor((90, 41)), y, Tensor((6,))),
                 lambda: B.vocab_loss_forward(Tensor((6, 40)), Tensor((90, 40)), Tensor((7,), torch.int32), Tensor((6,))),
                 lambda: B.vocab_loss_forward(Tensor((6, 40)), Tensor((90, 40), torch.float16), y, Tensor((6,)))):
        with pytest.raises(ValueError):
            call()
