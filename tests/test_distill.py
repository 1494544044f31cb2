"""The teacher's lists (dgc_top_logits) and the distillation loss over them (dgc_distill_*)
against plain definitions in 64 bits.

Tolerances.  The lists hold copies of the logits: no tolerance.  In the loss a logarithm of a
probability is (s - m) / T - log(sum): with |s - m| / T < 64 the products and differences are off by
at most 4 * 2^-24 * 64 = 1.6e-5, the sum by the same (the exponents of its terms) plus a few ulp: in
all under 4e-5 of a unit, times the weights.  A probability is off by 4e-5 of itself, hence
a gradient by 4e-5 of w_soft T (p + q) + w_hard (p1 + [label]), plus half an ulp of a 16-bit type."""
import math

import numpy as np
import pytest
import torch

DT = [torch.float32, torch.bfloat16, torch.float16]
HALF_ULP = {torch.float32: 0.0, **{d: torch.finfo(d).eps / 2 for d in (torch.bfloat16, torch.float16)}}
TINY = {torch.float32: 1e-38, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}
TOL = 4e-5
INF = math.inf


def _bind():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    from paper_1712_01887_b200 import binding as B
    return B


# ----------------------------------------------------------------- plain definitions, 64 bits

def plain_top(row, k):
    """The list of one row (a float32 numpy array)."""
    order = sorted((i for i in range(row.size) if not row[i] == -INF),
                   key=lambda i: (0 if np.isnan(row[i]) else 1, 0 if np.isnan(row[i]) else -float(row[i]), i))[:k]
    idx, val = np.full(k, -1, np.int32), np.full(k, -INF, np.float32)
    idx[:len(order)], val[:len(order)] = order, row[order]
    return idx, val


def _softmax(x):
    m = x.max() if x.numel() else -INF
    if m == -INF:
        return torch.zeros_like(x)
    e = torch.exp(x - m)
    return e / e.sum()


def _log_softmax(x):
    m = x.max()
    return torch.full_like(x, -INF) if m == -INF else x - m - torch.log(torch.exp(x - m).sum())


def plain_distill(logits, idx, val, labels, T, soft, hard, w=None):
    """(loss, gradient, the size against which its error counts) in float64."""
    R, V = logits.shape
    loss, grad, size = torch.zeros(R, dtype=torch.float64), torch.zeros(R, V, dtype=torch.float64), torch.zeros(R, V, dtype=torch.float64)
    for r in range(R):
        s = logits[r].double()
        on = [j for j in range(idx.shape[1]) if 0 <= int(idx[r, j]) < V and float(val[r, j]) > -INF]
        wr = 1.0 if w is None else float(w[r])
        if on:
            at, q = idx[r, on].long(), _softmax(val[r, on].double() / T)
            logp, p = _log_softmax(s / T)[at], _softmax(s / T)
            terms = torch.where(q > 0, q * (torch.log(q) - logp), 0.0)
            loss[r] += soft * T * T * terms.sum()
            taught = torch.zeros(V, dtype=torch.float64).index_add_(0, at, q)
            grad[r] += wr * soft * T * (p - taught)
            size[r] += abs(wr) * soft * T * (p + taught)
        y = -1 if labels is None else int(labels[r])
        if 0 <= y < V and hard != 0:
            p1 = _softmax(s)
            loss[r] -= hard * _log_softmax(s)[y]
            hot = torch.zeros(V, dtype=torch.float64)
            hot[y] = 1.0
            grad[r] += wr * hard * (p1 - hot)
            size[r] += abs(wr) * hard * (p1 + hot)
    return loss, grad, size


def test_plain_gradient_agrees_with_differences():
    gen = torch.Generator().manual_seed(1)
    s = torch.randn(3, 11, generator=gen, dtype=torch.float64)
    idx, val = torch.tensor([[3, 0, 7], [5, 5, -1], [-1, -1, -1]], dtype=torch.int32), torch.randn(3, 3, generator=gen)
    lab = torch.tensor([3, -1, 2], dtype=torch.int32)
    d = torch.randn(3, 11, generator=gen, dtype=torch.float64)
    _, g, _ = plain_distill(s, idx, val, lab, 2.0, 0.7, 0.3)
    eps = 1e-6
    up, dn = (plain_distill(s + e * d, idx, val, lab, 2.0, 0.7, 0.3)[0] for e in (eps, -eps))
    assert torch.allclose((up - dn) / (2 * eps), (g * d).sum(1), atol=1e-8)


# ----------------------------------------------------------------- lists

def _lists(B, logits, k):
    R = logits.shape[0]
    idx = torch.full((R, k), -7, dtype=torch.int32, device="cuda")
    val = torch.full((R, k), 7.0, device="cuda")
    B.top_logits(logits, idx, val)
    return idx.cpu().numpy(), val.cpu().numpy()


def _check_lists(B, logits, k, rows=None):
    idx, val = _lists(B, logits, k)
    host = logits.float().cpu().numpy()
    for r in rows if rows is not None else range(host.shape[0]):
        ri, rv = plain_top(host[r], k)
        assert np.array_equal(idx[r], ri), (r, idx[r][:8], ri[:8])
        assert np.array_equal(val[r], rv, equal_nan=True), r


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("R,V,k", [(1, 1, 1), (2, 1, 5), (3, 7, 7), (5, 29, 4), (4, 1000, 256), (9, 4099, 64), (3, 10000, 16),
                                   (2, 50021, 255), (40, 20011, 33), (1, 131075, 128), (3, 70001, 1)])
def test_top_logits(R, V, k, dt):
    gen = torch.Generator(device="cuda").manual_seed(V + k)
    whole = torch.randn(R, V + 3, generator=gen, device="cuda").mul_(2.5).to(dt)
    _check_lists(_bind(), whole[:, :V].contiguous(), k)
    _check_lists(_bind(), whole[:, 1:V + 1], k)         # rows at other addresses


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_top_logits_of_rows_that_are_not_ordinary(dt):
    B = _bind()
    V, k = 6001, 40
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(14, V, generator=gen, device="cuda").to(dt)
    x[0] = 1.5                                                   # all equal: the lowest indices
    x[1] = -INF                                                  # nothing left
    x[2, 5:] = -INF                                              # fewer than k left
    x[3, ::7] = float("nan")
    x[4] = torch.arange(V, device="cuda").to(dt)                 # ascending
    x[5] = -torch.arange(V, device="cuda").to(dt)
    x[6] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0).to(dt)
    x[7] = torch.finfo(dt).min
    x[8] = torch.finfo(dt).min
    x[8, 17] = torch.finfo(dt).max
    x[9, 100] = INF
    x[10] = (torch.randint(0, 3, (V,), generator=gen, device="cuda")).to(dt)     # few distinct values
    x[11] = float("nan")
    x[12] = torch.where(torch.arange(V, device="cuda") < V // 2, 2.0, 3.0).to(dt)
    x[13] = -INF
    x[13, V - 1] = torch.finfo(dt).min
    _check_lists(B, x, k)
    _check_lists(B, x, 1)
    _check_lists(B, x[:, 1:], 256)


@pytest.mark.gpu
def test_top_logits_of_orders_that_defeat_the_bound():
    """All large values dealt to a few threads, and rows of equal values too long for the list."""
    B = _bind()
    V = 1_200_011
    x = torch.randn(3, V, device="cuda")
    at = torch.arange(V, device="cuda")
    x[0] = torch.where((at // 4) % 512 < 3, x[0] + 50, x[0])
    x[1] = 0.25
    x[1, 700_000:700_030] = 0.5
    x[2, :] = torch.where(at % 5 == 0, 9.0, x[2].clamp(max=5))
    idx, val = _lists(B, x, 64)
    for r in range(3):
        v, i = torch.sort(x[r], descending=True, stable=True)
        assert np.array_equal(idx[r], i[:64].cpu().numpy()) and np.array_equal(val[r], v[:64].cpu().numpy())
    y = torch.zeros(300, 20001, device="cuda", dtype=torch.bfloat16)
    idx, val = _lists(B, y, 50)
    assert (idx == np.arange(50)).all() and (val == 0).all()


# ----------------------------------------------------------------- loss and gradient

def _problem(R, V, K, dt, seed, labels, std=2.5):
    gen = torch.Generator().manual_seed(seed)
    s = (torch.randn(R, V, generator=gen) * std).to(dt)
    idx = torch.stack([torch.randperm(V, generator=gen)[:K] if V >= K else torch.arange(K) for _ in range(R)]).to(torch.int32)
    val = torch.randn(R, K, generator=gen) * 2
    w = torch.rand(R, generator=gen) + 0.25
    lab = torch.randint(0, V, (R,), generator=gen).to(torch.int32) if labels else None
    return s, idx, val, lab, w


def _check_distill(B, s, idx, val, lab, w, T=1.0, soft=1.0, hard=0.0, place="same", finite=True):
    dt = s.dtype
    R, V = s.shape
    want, grad, size = plain_distill(s, idx, val, lab, T, soft, hard, w)
    dev = lambda t: None if t is None else t.cuda()
    how = dict(temperature=T, soft_weight=soft, hard_weight=hard, labels=dev(lab))

    def logits():
        if place == "odd":
            wide = torch.zeros(R, V + 5, dtype=dt, device="cuda")
            wide[:, 3:3 + V] = s.cuda()
            return wide[:, 3:3 + V]
        return s.cuda()

    def near_loss(x):
        x = x.double().cpu()
        assert torch.equal(torch.isinf(x), torch.isinf(want)) and not torch.isnan(x).any()
        f = torch.isfinite(want)
        assert ((x - want).abs()[f] <= TOL * (soft * T * T + hard + want.abs()[f])).all(), (x - want)[f].abs().max()

    def near_grad(x):
        x = x.double().cpu()
        tol = TOL * size + HALF_ULP[dt] * grad.abs() + TINY[dt]
        bad = (x - grad).abs() > tol
        assert not bad.any() and torch.isfinite(x).all(), (int(bad.sum()), float(((x - grad).abs() / tol).max()))
    ld = logits()
    loss, stats = torch.full((R,), -9.0, device="cuda"), torch.empty(R, 2, device="cuda")
    B.distill_forward(ld, dev(idx), dev(val), loss, stats, **how)
    near_loss(loss)
    whole = torch.full((R, V + 4), -5.0, dtype=dt, device="cuda")
    out = whole[:, 1:V + 1] if place == "odd" else torch.full((R, V), -5.0, dtype=dt, device="cuda")
    B.distill_backward(ld, dev(idx), dev(val), stats, dev(w), out, **how)
    near_grad(out)
    loss2 = torch.full((R,), -9.0, device="cuda")
    out2 = torch.full((R, V), -5.0, dtype=dt, device="cuda")
    B.distill_loss_grad(ld, dev(idx), dev(val), dev(w), loss2, out2, **how)
    near_loss(loss2)
    near_grad(out2)
    if place == "odd":
        assert (whole[:, 0] == -5).all() and (whole[:, V + 1:] == -5).all()
    # over the logits themselves
    over = logits()
    B.distill_loss_grad(over, dev(idx), dev(val), dev(w), loss2, over, **how)
    assert torch.equal(over, out2)
    near_loss(loss2)
    over = logits()
    B.distill_backward(over, dev(idx), dev(val), stats, dev(w), over, **how)
    assert torch.equal(over, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("R,V,K,T,labels,place", [
    (1, 1, 1, 1.0, True, "same"), (3, 5, 5, 2.0, True, "odd"), (7, 29, 4, 1.0, False, "odd"), (4, 1000, 256, 3.5, True, "same"),
    (5, 4099, 64, 1.0, True, "odd"), (3, 10000, 16, 2.0, True, "same"), (2, 50021, 100, 1.0, True, "same"), (2, 50021, 33, 0.5, False, "odd"),
    (200, 9001, 20, 2.0, True, "same"), (1, 131075, 128, 2.0, True, "odd"), (300, 515, 7, 1.0, True, "same")])
def test_distill(R, V, K, T, labels, place, dt):
    s, idx, val, lab, w = _problem(R, V, K, dt, R * V + K, labels)
    if R >= 3:
        idx[1, K // 2:] = -1                 # a shorter list
        val[2, 0] = -INF                     # an absent entry
        if lab is not None:
            lab[0] = idx[0, 0]               # the label is listed
            lab[1] = -1                      # a padding token
    if dt == torch.float16:
        w = w * 64                           # a loss scale
    _check_distill(_bind(), s, idx, val, lab, w, T, 0.75 if labels else 1.0, 0.25 if labels else 0.0, place)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_distill_rows_that_are_not_ordinary(dt, T):
    B = _bind()
    R, V, K = 12, 9001, 12
    s, idx, val, lab, w = _problem(R, V, K, dt, 77, True, std=1.0)
    idx[0], lab[0] = -1, -1                                  # nothing to learn from: zeros
    idx[1] = V                                               # outside the vocabulary: absent
    idx[2], lab[2] = 5, 5                                    # one word listed K times, and the label
    w[3] = 0.0
    s[4, 100:] = -INF                                        # a masked vocabulary
    idx[4], lab[4] = torch.arange(K).to(torch.int32), 3
    s[5] = torch.finfo(dt).min                               # a mask of the lowest value in every place: uniform
    s[6, 4000:] = torch.finfo(dt).min
    idx[6], lab[6] = torch.arange(K).to(torch.int32) * 2, 7
    s[7] = s[7] + (1000.0 if dt != torch.float16 else 500.0)  # a large logarithm of the sum
    val[8] = val[8] + 3.0e4
    lab[9] = V + 5
    idx[10] = torch.flip(idx[10], [0])
    s[11] = 0.0
    _check_distill(B, s, idx, val, lab, w, T, 0.5, 0.5)


@pytest.mark.gpu
def test_distill_where_the_student_cannot_say_the_word():
    """A listed word or a label with p = 0: the loss is +infinity, the gradient still the formula's;
    a row whose mask leaves nothing has p = 0 everywhere."""
    B = _bind()
    s, idx, val, lab, w = _problem(3, 700, 4, torch.float32, 2, True)
    s[0, int(idx[0, 1])] = -INF
    s[1, int(lab[1])] = -INF
    s[2] = -INF
    loss, stats, out = torch.empty(3, device="cuda"), torch.empty(3, 2, device="cuda"), torch.empty(3, 700, device="cuda")
    how = dict(temperature=2.0, soft_weight=1.0, hard_weight=0.5, labels=lab.cuda())
    _, grad, size = plain_distill(s, idx, val, lab, 2.0, 1.0, 0.5, w)
    B.distill_loss_grad(s.cuda(), idx.cuda(), val.cuda(), w.cuda(), loss, out, **how)
    assert torch.equal(loss.cpu(), torch.full((3,), INF))
    assert ((out.double().cpu() - grad).abs() <= TOL * size + 1e-38).all()
    B.distill_forward(s.cuda(), idx.cuda(), val.cuda(), loss, stats, **how)
    assert torch.equal(loss.cpu(), torch.full((3,), INF)) and (stats[2] == 0).all()
    B.distill_backward(s.cuda(), idx.cuda(), val.cuda(), stats, w.cuda(), out, **how)
    assert ((out.double().cpu() - grad).abs() <= TOL * size + 1e-38).all()


@pytest.mark.gpu
def test_not_a_number_stays_in_its_row_and_runs_repeat():
    B = _bind()
    s, idx, val, lab, w = _problem(4, 30011, 8, torch.bfloat16, 3, True)
    bad = s.clone()
    bad[1, 7], bad[2, 9] = float("nan"), INF
    outs = []
    for x in (s, bad, s):
        loss, out = torch.empty(4, device="cuda"), torch.empty(4, 30011, dtype=torch.bfloat16, device="cuda")
        B.distill_loss_grad(x.cuda(), idx.cuda(), val.cuda(), w.cuda(), loss, out, labels=lab.cuda(), hard_weight=0.5)
        outs.append((loss, out))
    assert torch.equal(outs[0][0], outs[2][0]) and torch.equal(outs[0][1], outs[2][1])
    keep = torch.tensor([0, 3], device="cuda")
    assert torch.equal(outs[0][0][keep], outs[1][0][keep]) and torch.equal(outs[0][1][keep], outs[1][1][keep])
    assert torch.isnan(outs[1][0][1:3]).all() and torch.isnan(outs[1][1][1]).all()


@pytest.mark.gpu
def test_a_teachers_lists_feed_the_loss_on_another_stream():
    """Lists of the student's own logits with k = vocab: the divergence is zero, so is the gradient."""
    B = _bind()
    s = torch.randn(6, 200, device="cuda")
    idx, val = torch.empty(6, 200, dtype=torch.int32, device="cuda"), torch.empty(6, 200, device="cuda")
    loss, out, w = torch.empty(6, device="cuda"), torch.empty(6, 200, device="cuda"), torch.ones(6, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.top_logits(s, idx, val, stream=side)
    B.distill_loss_grad(s, idx, val, w, loss, out, stream=side)
    side.synchronize()
    assert float(loss.abs().max()) <= TOL and float(out.abs().max()) <= 2 * TOL


@pytest.mark.gpu
def test_matrices_whose_offsets_pass_32_bits():
    B = _bind()
    R, V = 5, 1000
    big = torch.zeros(R, 1 << 29, dtype=torch.bfloat16, device="cuda")     # 5 GB: the last row starts past 2^31 elements
    s, idx, val, lab, w = _problem(R, V, 8, torch.bfloat16, 5, True)
    big[:, 7:7 + V] = s.cuda()
    view = big[:, 7:7 + V]
    _check_lists(B, view, 8)
    loss, out = torch.empty(R, device="cuda"), torch.empty(R, V, dtype=torch.bfloat16, device="cuda")
    B.distill_loss_grad(view, idx.cuda(), val.cuda(), w.cuda(), loss, out, labels=lab.cuda(), hard_weight=0.5)
    ref, ro = torch.empty_like(loss), torch.empty_like(out)
    B.distill_loss_grad(s.cuda(), idx.cuda(), val.cuda(), w.cuda(), ref, ro, labels=lab.cuda(), hard_weight=0.5)
    # the rows start at another distance from a 16-byte boundary: other threads hold other elements
    assert float((loss - ref).abs().max()) <= TOL * float(1 + ref.abs().max())
    assert ((out.float() - ro.float()).abs() <= 2 * (HALF_ULP[torch.bfloat16] + TOL) * (ro.float().abs() + 1e-6)).all()


def test_refusals_of_the_c_calls():
    from paper_1712_01887_b200 import binding as B
    lib, p, off = B._lib, 4096, 4097

    def top(dtype=0, rows=2, v=8, k=4, x=p, ld=8, i=p, o=p):
        return lib.dgc_top_logits(B.TOP.pack(dtype, v, k, 0, rows, x, ld, i, o), None)
    for bad in (dict(dtype=3), dict(rows=-1), dict(v=0), dict(k=0), dict(k=257), dict(ld=7), dict(x=0), dict(i=0), dict(o=0),
                dict(x=off), dict(i=off), dict(o=off), dict(rows=1 << 31)):
        assert top(**bad) == B.EINVAL, bad
    assert top(rows=0) == B.OK and lib.dgc_top_logits(None, None) == B.EINVAL

    def call(which, dtype=1, rows=2, v=8, k=4, x=p, ld=8, i=p, t=p, T=1.0, ws=1.0, wh=0.0, stats=p, dl=p, loss=p, g=p, ldg=8, lab=0):
        return getattr(lib, "dgc_distill_" + which)(B.DISTILL.pack(dtype, v, k, 0, rows, x, ld, i, t, lab, T, ws, wh, 0.0, loss, stats,
                                                                   dl, g, ldg), None)
    every = [dict(dtype=-1), dict(dtype=3), dict(rows=-2), dict(v=0), dict(k=0), dict(k=300), dict(x=0), dict(ld=7), dict(i=0),
             dict(t=0), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=INF), dict(ws=INF), dict(wh=float("nan")), dict(x=off),
             dict(i=off), dict(lab=off)]
    only = {"forward": [dict(loss=0), dict(loss=off), dict(stats=off)],
            "backward": [dict(stats=0), dict(dl=0), dict(g=0), dict(ldg=7), dict(g=off)],
            "loss_grad": [dict(dl=0), dict(loss=0), dict(g=0), dict(ldg=0)]}
    for which, more in only.items():
        for bad in every + more:
            assert call(which, **bad) == B.EINVAL, (which, bad)
        assert call(which, rows=0) == B.OK
        assert getattr(lib, "dgc_distill_" + which)(None, None) == B.EINVAL


@pytest.mark.gpu
def test_refusals_of_the_binding():
    B = _bind()
    s, i, v = torch.zeros(3, 50, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, device="cuda")
    loss = torch.zeros(3, device="cuda")
    for bad in ((s.double(), i, v), (s, i.long(), v), (s, i, v.half()), (s, i[:2], v), (s.t(), i, v), (s.cpu(), i, v)):
        with pytest.raises(ValueError):
            B.top_logits(*bad)
        with pytest.raises(ValueError):
            B.distill_forward(*bad, loss)
    with pytest.raises(ValueError):
        B.distill_loss_grad(s, i, v, loss, loss.clone(), s.half())
    with pytest.raises(ValueError):
        B.distill_forward(s, i, v, loss, labels=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(B.DgcError):
        B.distill_forward(s, i, v, loss, temperature=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0, 3.5, 0.25])
def test_distill_rows_of_large_logits(dt, T):
    """Rows whose maximum is so large that its product with log2(e) / T is off by whole numbers: masks of
    -1e9 to -1e20 in every place, a few words far above the rest, and both sides of 2^24 / log2(e) = 1.16e7
    and T times that.  (Tolerance as above; there (s - m) / T < 64 for every word that has a share, and a
    word without one is off by 2^-22 of its own logarithm, which the term in |loss| covers.)"""
    B = _bind()
    V, K = 9001, 12
    full = [-1e9, -1e10, -1e20, -1e29, -1e31, 1e10, 1e20, 1e29]
    limit = 2.0 ** 24 / 1.4426950408889634
    near = [sign * by * limit * t for t in (1.0, T) for by in (0.96, 1.04) for sign in (1, -1)]
    R = len(full) + 3 + len(near)
    s, idx, val, lab, w = _problem(R, V, K, dt, 91, True, std=1.0)
    for r, v in enumerate(full):
        s[r] = v
    r = len(full)
    s[r], s[r + 1], s[r + 2] = s[r].clamp(-4, 4), s[r + 1].clamp(-4, 4), -1e10
    s[r, 77] = 1e10                                          # one word far above the rest
    s[r + 1, [5, 6000, 9000]] = 1e11                         # three of them
    s[r + 2, 4000:] = -1e20
    idx[r, 0], lab[r] = 77, 77
    idx[r + 1, :2], lab[r + 1] = torch.tensor([5, 6000]).to(torch.int32), 9000
    idx[r + 2], lab[r + 2] = torch.arange(K).to(torch.int32), 9
    steps = torch.randint(-8, 1, (V,), generator=torch.Generator().manual_seed(92)).float()
    for q, v in enumerate(near):                             # (f32: whole numbers, exact at this size)
        s[r + 3 + q] = (round(v) + steps).to(dt)
    _check_distill(B, s, idx, val, lab, w, T, 0.5, 0.5)
    _check_distill(B, s, idx, val, None, w, T, 1.0, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_no_soft_term_where_its_weight_is_zero(dt, T):
    """Labels alone: a list that names words masked in the student, or holds infinities, says nothing."""
    B = _bind()
    R, V, K = 4, 5003, 6
    s, idx, val, lab, w = _problem(R, V, K, dt, 17, True)
    s[0, int(idx[0, 1])] = -INF
    s[1, idx[1].long()] = -INF
    lab[1] = (int(idx[1].max()) + 1) % V
    while int(lab[1]) in idx[1].tolist():
        lab[1] = (int(lab[1]) + 1) % V
    lab[0] = lab[1]
    s[:2, int(lab[1])] = 0.5
    val[2, 3] = INF
    lab[3] = -1
    absent = torch.full_like(idx, -1)
    want, grad, size = plain_distill(s, absent, val, lab, T, 0.0, 0.75, w)
    assert torch.isfinite(want).all() and float(want[3]) == 0
    dev = [t.cuda() for t in (s, idx, val)]
    how = dict(temperature=T, soft_weight=0.0, hard_weight=0.75, labels=lab.cuda())
    loss, stats = torch.empty(R, device="cuda"), torch.empty(R, 2, device="cuda")
    out, out2 = (torch.empty(R, V, dtype=dt, device="cuda") for _ in range(2))
    B.distill_forward(*dev, loss, stats, **how)
    B.distill_backward(*dev, stats, w.cuda(), out, **how)
    loss2 = torch.empty_like(loss)
    B.distill_loss_grad(*dev, w.cuda(), loss2, out2, **how)
    for x in (loss, loss2):
        assert ((x.double().cpu() - want).abs() <= TOL * (0.75 + want.abs())).all()
    for x in (out, out2):
        assert ((x.double().cpu() - grad).abs() <= TOL * size + HALF_ULP[dt] * grad.abs() + TINY[dt]).all()
    B.distill_loss_grad(*dev, w.cuda(), loss2, out2, temperature=T, soft_weight=0.0)     # neither term
    assert (loss2 == 0).all() and (out2 == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_an_infinite_teacher_is_not_passed_over(dt, T):
    """A listed value of +infinity leaves q undefined: the row's loss and its gradient at the listed places
    are NaN, as by the definition; the other places and rows have the formula's values."""
    B = _bind()
    R, V, K = 4, 3001, 6
    s, idx, val, lab, w = _problem(R, V, K, dt, 23, True)
    val[1, 2] = INF
    val[2, 0], val[2, 5] = INF, INF
    idx[2, 5] = -1                                           # (an absent entry's value does not count)
    want, grad, size = plain_distill(s, idx, val, lab, T, 0.5, 0.5, w)
    want[1:3] = float("nan")                                 # q log q of them
    dev = [t.cuda() for t in (s, idx, val)]
    how = dict(temperature=T, soft_weight=0.5, hard_weight=0.5, labels=lab.cuda())
    loss, stats = torch.empty(R, device="cuda"), torch.empty(R, 2, device="cuda")
    out, out2 = (torch.empty(R, V, dtype=dt, device="cuda") for _ in range(2))
    B.distill_forward(*dev, loss, stats, **how)
    B.distill_backward(*dev, stats, w.cuda(), out, **how)
    loss2 = torch.empty_like(loss)
    B.distill_loss_grad(*dev, w.cuda(), loss2, out2, **how)
    fine, rows = ~torch.isnan(grad), ~torch.isnan(want)
    assert int((~fine).sum()) == K + K - 1
    for x in (loss, loss2):
        x = x.double().cpu()
        assert torch.equal(torch.isnan(x), torch.isnan(want))
        assert ((x - want).abs()[rows] <= TOL * (0.5 * T * T + 0.5 + want.abs()[rows])).all()
    for x in (out, out2):
        x = x.double().cpu()
        assert torch.equal(torch.isnan(x), ~fine)
        assert ((x - grad).abs()[fine] <= (TOL * size + HALF_ULP[dt] * grad.abs() + TINY[dt])[fine]).all()


def test_temperatures_out_of_range_are_refused():
    """T^2 or 1 / T would not be a normal 32-bit number (the loss 0 x infinity)."""
    from paper_1712_01887_b200 import binding as B
    for which in ("forward", "backward", "loss_grad"):
        for T in (1e-45, 1e-39, 1e-30, 0.99 * 2.0 ** -60, 1.01 * 2.0 ** 60, 1e30, 3e38):
            args = B.DISTILL.pack(0, 8, 4, 0, 2, 4096, 8, 4096, 4096, 0, T, 1.0, 0.0, 0.0, 4096, 4096, 4096, 4096, 8)
            assert getattr(B._lib, "dgc_distill_" + which)(args, None) == B.EINVAL, (which, T)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
def test_temperatures_at_the_ends_of_the_range(T):
    for dt in (torch.float32, torch.bfloat16):
        s, idx, val, _, w = _problem(5, 3001, 7, dt, 41, False)
        idx[1, 4:] = -1
        _check_distill(_bind(), s, idx, val, None, w, T, 1.0, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("T", [1.0, 2.0, 3.5])
def test_listed_words_masked_with_the_lowest_value(dt, T):
    """Their log p is finite, -3.4e38 / T in f32 and bf16, and so is the loss (weights that keep it below 3.4e38)."""
    R, V, K = 5, 4001, 8
    s, idx, val, lab, w = _problem(R, V, K, dt, 61, True)
    low = torch.finfo(dt).min
    s[0, int(idx[0, 3])] = low
    s[1, idx[1].long()] = low
    s[2, int(lab[2])] = low
    s[3, 100:] = low
    s[4], s[4, 7] = low, torch.finfo(dt).max / 8                # a row that is taken with care
    _check_distill(_bind(), s, idx, val, lab, w, T, 1 / 32, 1 / 16)
