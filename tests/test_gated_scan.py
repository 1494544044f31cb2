"""The gated linear recurrence (dgc_gated_scan_*) against a plain recurrence in 64 bits.

Tolerances.  f and 1 - f come from one exponential and one division in 32 bits: at most 4 ulp,
2.4e-7.  A relative error d of every f moves a state by at most d / (1 - f_max); with the gates'
logits inside [-6, 6] that is d * 404 < 1e-4 of the largest state, and the same holds for the
gradients (their recurrence has the same coefficients).  Rounding to a 16-bit type adds half a
unit in the last place: at most eps / 2 = 2^-8 (bf16) or 2^-11 (f16) of the value; where the backward pass starts a
run from a stored state, that state's rounding enters dgate once more, times f (1 - f) |g|."""
import numpy as np
import pytest
import torch

UNIT = {torch.float32: 0.0, **{d: torch.finfo(d).eps / 2 for d in (torch.bfloat16, torch.float16)}}   # half an ulp
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}   # f16 subnormals
DT = [torch.float32, torch.bfloat16, torch.float16]
F32_TOL = 1e-4


def plain(z, x, h0, starts, reverse):
    """float64, one step after the other."""
    h, before = torch.zeros_like(x), torch.zeros_like(x)
    last = h0.clone()
    f = torch.sigmoid(z)
    for s in range(len(starts) - 1):
        order = list(range(starts[s], starts[s + 1]))
        cur = h0[s]
        for t in (order[::-1] if reverse else order):
            before[t] = cur
            cur = f[t] * cur + torch.sigmoid(-z[t]) * x[t]
            h[t] = cur
        last[s] = cur
    return h, last, before


def plain_backward(z, x, h0, starts, reverse, dh, dlast):
    _, _, before = plain(z, x, h0, starts, reverse)
    f, omf = torch.sigmoid(z), torch.sigmoid(-z)
    g, dh0 = torch.zeros_like(x), dlast.clone()
    for s in range(len(starts) - 1):
        order = list(range(starts[s], starts[s + 1]))
        e = dlast[s]
        for t in (order if reverse else order[::-1]):
            g[t] = dh[t] + e
            e = f[t] * g[t]
        dh0[s] = e
    return f * omf * g * (before - x), omf * g, dh0, g


def test_plain_backward_agrees_with_differences():
    """The formulas the kernels are tested against, against the forward recurrence itself."""
    gen = torch.Generator().manual_seed(5)
    starts, C = [0, 7, 7, 8, 20], 3
    z, x, dh = (torch.randn(20, C, generator=gen, dtype=torch.float64) for _ in range(3))
    h0, dl = (torch.randn(4, C, generator=gen, dtype=torch.float64) for _ in range(2))
    for reverse in (False, True):
        gz, gx, g0, _ = plain_backward(z, x, h0, starts, reverse, dh, dl)
        vz, vx = torch.randn(20, C, generator=gen, dtype=torch.float64), torch.randn(20, C, generator=gen, dtype=torch.float64)
        v0 = torch.randn(4, C, generator=gen, dtype=torch.float64)

        def value(e):
            h, last, _ = plain(z + e * vz, x + e * vx, h0 + e * v0, starts, reverse)
            return (h * dh).sum() + (last * dl).sum()
        eps = 1e-5
        num = (value(eps) - value(-eps)) / (2 * eps)
        ana = (gz * vz).sum() + (gx * vx).sum() + (g0 * v0).sum()
        assert abs(num - ana) <= 1e-8 * (1 + abs(ana))


def _bind():
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device: the gpu tests need a B200")
    from paper_1712_01887_b200 import binding as B
    return B


def _near(got, want, dt, what, extra=0.0):
    got = got.double().cpu()
    tol = UNIT[dt] * want.abs() + TINY[dt] + F32_TOL * max(1e-30, float(want.abs().max()) if want.numel() else 0) + extra
    bad = (got - want).abs() > tol
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / tol).max()))
    assert torch.isfinite(got).all(), what


def _case(lens, C, dt, joint, seed, gate_mean=1.5):
    gen = torch.Generator().manual_seed(seed)
    N, S = sum(lens), len(lens)
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(int).tolist()
    z = (torch.randn(N, C, generator=gen) * 2 + gate_mean).clamp(-6, 6).to(dt)
    x = torch.randn(N, C, generator=gen).to(dt)
    dh = torch.randn(N, C, generator=gen).to(dt)
    h0, dl = torch.randn(S, C, generator=gen), torch.randn(S, C, generator=gen)

    def dev(t):
        if not joint:
            return t.cuda()
        wide = torch.full((N, 2 * C + joint), 7.0, dtype=dt, device="cuda")   # joint: extra columns of the row
        wide[:, joint:joint + C] = t.cuda()
        return wide[:, joint:joint + C]
    return starts, z, x, dh, h0, dl, dev


def _check(B, lens, C, dt, joint=0, reverse=False, packed=True, seed=0, with_h0=True, gate_mean=1.5):
    starts, z, x, dh, h0, dl, dev = _case(lens, C, dt, joint, seed, gate_mean)
    N, S = sum(lens), len(lens)
    how = dict(num_seqs=S, reverse=reverse, h0=h0.cuda() if with_h0 else None,
               seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda") if packed else None)
    zd, xd, gd = dev(z), dev(x), dev(dh)
    whole = torch.full((N + 2, C + 3), -5.0, dtype=dt, device="cuda")
    h = whole[1:N + 1, 1:C + 1] if joint else torch.empty(N, C, dtype=dt, device="cuda")
    last = torch.full((S, C), float("nan"), device="cuda")
    B.gated_scan_forward(zd, xd, h, h_last=last, **how)
    start = h0.double() if with_h0 else torch.zeros(S, C, dtype=torch.float64)
    rh, rl, _ = plain(z.double(), x.double(), start, starts, reverse)
    _near(h, rh, dt, "h")
    _near(last, rl, torch.float32, "h_last")
    if joint:   # nothing outside the matrix was written
        assert (whole[0] == -5).all() and (whole[-1] == -5).all()
        assert (whole[:, 0] == -5).all() and (whole[:, C + 1:] == -5).all()
    pair = torch.full((N, 2 * C + 1), -5.0, dtype=dt, device="cuda")
    dgate, dx = (pair[:, :C], pair[:, C + 1:]) if joint else (torch.empty(N, C, dtype=dt, device="cuda") for _ in range(2))
    dh0 = torch.full((S, C), float("nan"), device="cuda")
    B.gated_scan_backward(zd, xd, h, gd, dgate, dx, dh_last=dl.cuda(), dh0=dh0, **how)
    rz, rx, r0, g = plain_backward(z.double(), x.double(), start, starts, reverse, dh.double(), dl.double())
    f = torch.sigmoid(z.double())
    hmax = float(rh.abs().max()) if N else 0.0
    _near(dgate, rz, dt, "dgate", UNIT[dt] * hmax * (f * (1 - f) * g).abs())
    _near(dx, rx, dt, "dx")
    _near(dh0, r0, torch.float32, "dh0")
    if joint:
        assert (pair[:, C] == -5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("lens,C,joint", [
    ([1], 1, 0), ([1], 64, 0), ([2, 0, 1], 65, 1), ([0, 0, 5, 0], 66, 2), ([15, 16, 17], 128, 0), ([127, 128, 129], 33, 0),
    ([255, 1, 513], 70, 2), ([1025], 64, 0), ([3001], 10, 1), ([40, 0, 2500, 3], 96, 4), ([7] * 50, 130, 0)])
def test_scan_and_gradients(lens, C, joint, reverse, dt):
    _check(_bind(), lens, C, dt, joint, reverse, seed=len(lens) * 100 + C)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_scan_of_equal_lengths_without_a_table(dt):
    _check(_bind(), [35] * 20, 150, dt, packed=False)
    _check(_bind(), [300] * 3, 1500, dt, packed=False, with_h0=False, reverse=True)


@pytest.mark.gpu
@pytest.mark.parametrize("mean", [-4.0, 5.0])
def test_scan_with_gates_that_forget_or_keep(mean):
    _check(_bind(), [2000, 90], 64, torch.float32, gate_mean=mean)
    _check(_bind(), [2000, 90], 64, torch.bfloat16, gate_mean=mean)


@pytest.mark.gpu
def test_scan_of_many_sequences_and_long_ones():
    _check(_bind(), [i % 5 for i in range(700)], 40, torch.bfloat16)
    _check(_bind(), [9000], 32, torch.float32, reverse=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("lens,C,joint,packed", [
    ([8192], 64, 0, False), ([16385], 33, 0, True), ([8447], 1, 1, True), ([0, 20000, 64, 1, 32764], 10, 2, True),
    ([24000, 63, 1025], 130, 0, True), ([8192, 8192], 100, 4, False), ([4096], 512, 0, True)])
@pytest.mark.parametrize("reverse", [False, True])
def test_long_and_narrow_sequences_go_by_runs(lens, C, joint, packed, reverse, dt):
    """The sizes that take a workspace: runs that end inside a stage, empty sequences, one step."""
    B = _bind()
    assert B._lib.dgc_gated_scan_workspace_bytes(B.SCAN.pack(B.DTYPES[dt], len(lens), C, 0, sum(lens), *[0] * 19)) > 0
    _check(B, lens, C, dt, joint, reverse, packed=packed, seed=C)
    _check(B, lens, C, dt, joint, reverse, packed=packed, seed=C + 1, with_h0=False)


@pytest.mark.gpu
def test_long_sequences_on_two_streams_at_once():
    """Calls on a given stream beside calls on the current one: each has a workspace of its own."""
    B = _bind()
    g = torch.Generator(device="cuda").manual_seed(5)
    z, x = (torch.randn(40000, 96, device="cuda", generator=g) for _ in range(2))
    want = [torch.empty_like(z) for _ in range(2)]
    B.gated_scan_forward(z, x, want[0])
    B.gated_scan_forward(x, z, want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [[torch.empty_like(z) for _ in range(2)] for _ in range(6)]
    torch.cuda.synchronize()
    for a, b in got:
        B.gated_scan_forward(z, x, a)
        B.gated_scan_forward(x, z, b, stream=side)
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.gpu
def test_extreme_gates_and_neighbours_that_are_not_finite():
    """Gates of +-inf and of the type's lowest value are exactly 1 and 0; a sequence full of NaN
    and infinities leaves its neighbours in the pack untouched, bit for bit."""
    B = _bind()
    for dt in DT:
        lens, C = [70, 200, 33], 64
        starts, z, x, dh, h0, dl, _ = _case(lens, C, dt, 0, 3)
        z[5], z[6], z[7] = float("inf"), -float("inf"), torch.finfo(dt).min
        clean = None
        for poison in (False, True):
            zz, xx, gg = z.clone(), x.clone(), dh.clone()
            if poison:
                zz[80:90], xx[100:150], gg[70:270] = float("nan"), float("inf"), float("nan")
            tab = torch.tensor(starts, dtype=torch.int32, device="cuda")
            zd, xd, gd = zz.cuda(), xx.cuda(), gg.cuda()
            h, gz, gx = (torch.empty(303, C, dtype=dt, device="cuda") for _ in range(3))
            last, d0 = (torch.empty(3, C, device="cuda") for _ in range(2))
            how = dict(seq_start=tab, num_seqs=3, h0=h0.cuda())
            B.gated_scan_forward(zd, xd, h, h_last=last, **how)
            B.gated_scan_backward(zd, xd, h, gd, gz, gx, dh_last=dl.cuda(), dh0=d0, **how)
            keep = [t[i].clone() for t in (h, gz, gx) for i in (slice(0, 70), slice(270, 303))] + [last[::2].clone(), d0[::2].clone()]
            assert all(torch.isfinite(k).all() for k in keep)
            if clean is None:
                clean = keep
            else:
                assert all(torch.equal(a, b) for a, b in zip(clean, keep))
        # gate = 1: the state passes unchanged; gate = 0: the state is the input
        assert torch.equal(h[5], h[4]) and torch.equal(h[6], x[6].cuda()) and torch.equal(h[7], x[7].cuda())


@pytest.mark.gpu
def test_scan_is_the_same_from_run_to_run_and_on_another_stream():
    B = _bind()
    starts, z, x, *_ = _case([5000, 3], 64, torch.bfloat16, 0, 9)
    zd, xd = z.cuda(), x.cuda()
    tab = torch.tensor(starts, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(xd), torch.empty_like(xd)
    B.gated_scan_forward(zd, xd, a, seq_start=tab, num_seqs=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.gated_scan_forward(zd, xd, b, seq_start=tab, num_seqs=2, stream=side)
    side.synchronize()
    assert torch.equal(a, b)


@pytest.mark.gpu
def test_damaged_offsets_stay_inside():
    """Offsets beyond the pack and descending ones are clamped; guard rows keep their bits."""
    B = _bind()
    N, C = 100, 32
    z, x = torch.randn(N, C, device="cuda"), torch.randn(N, C, device="cuda")
    whole = torch.full((N + 64, C), -5.0, device="cuda")
    tab = torch.tensor([-30, 40, 20, 130], dtype=torch.int32, device="cuda")
    B.gated_scan_forward(z, x, whole[32:32 + N], seq_start=tab, num_seqs=3)
    torch.cuda.synchronize()
    assert (whole[:32] == -5).all() and (whole[32 + N:] == -5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("S,C,slots", [(1, 1, 1), (3, 7, 5), (64, 1500, 96), (130, 66, 130)])
def test_step(S, C, slots, dt):
    B = _bind()
    gen = torch.Generator().manual_seed(S)
    z, x = (torch.randn(S, C, generator=gen) * 2).to(dt), torch.randn(S, C, generator=gen).to(dt)
    state = torch.randn(slots, C, generator=gen)
    at = torch.randperm(slots, generator=gen)[:S].to(torch.int32)
    if S > 2:
        at[1], at[2] = -1, slots          # idle rows
    sd, out = state.cuda(), torch.full((S, C), -5.0, dtype=dt, device="cuda")
    B.gated_scan_step(z.cuda(), x.cuda(), sd, out, slots=at.cuda())
    want, ro = state.double(), torch.zeros(S, C, dtype=torch.float64)
    for r in range(S):
        i = int(at[r])
        if 0 <= i < slots:
            want[i] = torch.sigmoid(z[r].double()) * want[i] + torch.sigmoid(-z[r].double()) * x[r].double()
            ro[r] = want[i]
    _near(sd, want, torch.float32, "state")
    _near(out, ro, dt, "out")


@pytest.mark.gpu
def test_steps_continue_a_scan():
    """The prompt by the scan, the next tokens one by one: the same states as one scan of all."""
    B = _bind()
    S, L, C = 4, 50, 96
    z, x = torch.randn(S, L, C, device="cuda"), torch.randn(S, L, C, device="cuda")
    h, last = torch.empty(S * L, C, device="cuda"), torch.empty(S, C, device="cuda")
    B.gated_scan_forward(z.view(-1, C), x.view(-1, C), h, num_seqs=S, h_last=last)
    h1, st = torch.empty(S * 40, C, device="cuda"), torch.empty(S, C, device="cuda")
    B.gated_scan_forward(z[:, :40].reshape(-1, C), x[:, :40].reshape(-1, C), h1, num_seqs=S, h_last=st)
    out = torch.empty(S, C, device="cuda")
    for t in range(40, L):
        B.gated_scan_step(z[:, t], x[:, t], st, out)
        assert float((out - h.view(S, L, C)[:, t]).abs().max()) <= F32_TOL * float(h.abs().max())
    assert float((st - last).abs().max()) <= F32_TOL * float(last.abs().max())


@pytest.mark.gpu
def test_scan_in_a_graph():
    B = _bind()
    starts, z, x, *_ = _case([300, 20], 64, torch.float16, 0, 2)
    zd, xd = z.cuda(), x.cuda()
    tab = torch.tensor(starts, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(xd), torch.empty_like(xd)
    B.gated_scan_forward(zd, xd, a, seq_start=tab, num_seqs=2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.gated_scan_forward(zd, xd, b, seq_start=tab, num_seqs=2)
    b.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, b)


def test_refusals_of_the_c_calls():
    """Bad arguments come back as DGC_EINVAL before anything is enqueued (no GPU needed)."""
    from paper_1712_01887_b200 import binding as B
    p = 4096

    def scan(call, dtype=0, tokens=8, seqs=2, ch=4, table=0, z=p, ldz=4, x=p, ldx=4, h=p, ldh=4, h0=0, last=0, dh=p, lddh=4, dz=p,
             lddz=4, dx=p, lddx=4, dlast=0, dh0=0, work=0, size=0):
        return call(B.SCAN.pack(dtype, seqs, ch, 0, tokens, table, z, ldz, x, ldx, h, ldh, h0, last, dh, lddh, dz, lddz, dx, lddx,
                                dlast, dh0, work, size), None)
    both = [dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(tokens=7), dict(tokens=1 << 31), dict(seqs=0), dict(seqs=-1), dict(ch=0),
            dict(ch=-4), dict(ldz=3), dict(ldx=0), dict(ldh=-4), dict(z=0), dict(x=0), dict(h=0), dict(x=p + 2), dict(dtype=1, h=p + 1),
            dict(table=p + 2), dict(h0=p + 1), dict(work=p + 4, size=64), dict(work=p, size=-1)]
    for bad in both + [dict(last=p + 2)]:
        assert scan(B._lib.dgc_gated_scan_forward, **bad) == B.EINVAL, bad
    for bad in both + [dict(dh=0), dict(dz=0), dict(dx=0), dict(lddh=3), dict(lddz=3), dict(lddx=3), dict(dh=p + 1), dict(dlast=p + 1),
                       dict(dh0=p + 2)]:
        assert scan(B._lib.dgc_gated_scan_backward, **bad) == B.EINVAL, bad

    for call in (B._lib.dgc_gated_scan_forward, B._lib.dgc_gated_scan_backward):   # a workspace that is too small
        assert scan(call, tokens=8192, seqs=1, work=p, size=100) == B.ECAPACITY
    size = B._lib.dgc_gated_scan_workspace_bytes
    pack = lambda dtype, seqs, ch, tokens: B.SCAN.pack(dtype, seqs, ch, 0, tokens, *[0] * 19)  # noqa: E731
    assert size(pack(1, 1, 100, 8192)) == (8192 // 64 + 1) * 100 * 8
    assert size(pack(1, 1, 100, 100)) == 0 and size(pack(1, 8, 4096, 65536)) == 0
    assert size(pack(7, 1, 1, 1)) == B.EINVAL and size(None) == B.EINVAL

    def step(dtype=0, rows=2, ch=4, n=2, z=p, ldz=4, x=p, ldx=4, out=p, ldo=4, state=p, slots=0):
        return B._lib.dgc_gated_scan_step(B.SCAN_ONE.pack(dtype, rows, ch, n, z, ldz, x, ldx, out, ldo, state, slots), None)
    for bad in (dict(dtype=5), dict(rows=-1), dict(ch=0), dict(ldz=1), dict(ldx=3), dict(ldo=2), dict(z=0), dict(x=p + 2), dict(out=0),
                dict(state=0), dict(state=p + 2), dict(n=1), dict(n=-1), dict(slots=p + 1)):
        assert step(**bad) == B.EINVAL, bad
    assert step(rows=0) == B.OK and scan(B._lib.dgc_gated_scan_forward, tokens=0) == B.OK
    assert scan(B._lib.dgc_gated_scan_backward, tokens=0) == B.OK
    for call in (B._lib.dgc_gated_scan_forward, B._lib.dgc_gated_scan_backward, B._lib.dgc_gated_scan_step):
        assert call(None, None) == B.EINVAL


@pytest.mark.gpu
def test_refusals_of_the_binding():
    B = _bind()
    z = torch.zeros(8, 4, device="cuda")
    for gate, x, h in ((z.double(), z, z), (z, z[:, :3], z), (z, z.half(), z), (z, z, z.t().contiguous().t()), (z, z.cpu(), z), (z[0], z, z)):
        with pytest.raises(ValueError):
            B.gated_scan_forward(gate, x, h)
    with pytest.raises(ValueError):
        B.gated_scan_forward(z, z.clone(), z.clone(), seq_start=torch.zeros(3, dtype=torch.int64, device="cuda"), num_seqs=2)
    with pytest.raises(ValueError):
        B.gated_scan_forward(z, z.clone(), z.clone(), h0=torch.zeros(3, 4, device="cuda"))
    with pytest.raises(B.DgcError):
        B.gated_scan_forward(z, z.clone(), z.clone(), num_seqs=3)


def test_channels_up_to_the_last_tile_of_32_bit_indices():
    """A tile of channels that ends past 2^31 is refused; nothing is enqueued."""
    from paper_1712_01887_b200 import binding as B
    p, lib = 4096, B._lib
    for ch in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 1024):
        scan = B.SCAN.pack(0, 1, ch, 0, 1, 0, *[p, ch] * 3, 0, 0, *[p, ch] * 3, 0, 0, 0, 0)
        assert lib.dgc_gated_scan_forward(scan, None) == B.EINVAL
        assert lib.dgc_gated_scan_backward(scan, None) == B.EINVAL
        assert lib.dgc_gated_scan_workspace_bytes(scan) == B.EINVAL
        assert lib.dgc_gated_scan_step(B.SCAN_ONE.pack(0, 1, ch, 1, *[p, ch] * 3, p, 0), None) == B.EINVAL
    for ch in (1, 2 ** 31 - 1025):
        assert lib.dgc_gated_scan_workspace_bytes(B.SCAN.pack(0, 1, ch, 0, 1, *[0] * 19)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("lens,C", [([400, 3, 150], 40), ([2600, 90], 64), ([9000], 32)])
@pytest.mark.parametrize("reverse", [False, True])
def test_infinite_states_and_gradients_stay_infinite(lens, C, reverse, dt):
    """A gate that forgets, f > 0, leaves an infinite state infinite, however many such steps follow: the
    product of a run's f must not become 0 (0 x infinity).  All other values keep their tolerance: every f
    may be taken too large by 2e-38 and no result here is larger than 1e3."""
    B, INF = _bind(), float("inf")
    starts, z, x, dh, h0, dl, _ = _case(lens, C, dt, 0, 31)
    z = (z * 0.3 - 9).to(dt)                                   # f about e^-9: sixteen of them are below 2^-126
    N, S = sum(lens), len(lens)
    tab = torch.tensor(starts, dtype=torch.int32, device="cuda")
    how = dict(seq_start=tab, num_seqs=S, reverse=reverse)
    xi, hi = x.clone(), h0.clone()
    hi[0, 1], hi[S - 1, 2] = INF, -INF
    xi[starts[1] // 2, 3], xi[starts[1] // 2, 4] = INF, -INF
    h, last = torch.empty(N, C, dtype=dt, device="cuda"), torch.empty(S, C, device="cuda")
    B.gated_scan_forward(z.cuda(), xi.cuda(), h, h_last=last, h0=hi.cuda(), **how)
    rh, rl, _ = plain(z.double(), xi.double(), hi.double(), starts, reverse)
    assert int(torch.isinf(rh).sum()) > N // 4 and not torch.isnan(rh).any()

    def same(got, want, unit, what, scale):
        got = got.double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, int(torch.isnan(got).sum()))
        odd = torch.isinf(want)
        assert torch.equal(got[odd], want[odd]) and not torch.isinf(got[~odd]).any(), what
        fine = torch.isfinite(want)
        assert ((got - want).abs()[fine] <= unit * want.abs()[fine] + TINY[dt] + F32_TOL * scale).all(), what
    same(h, rh, UNIT[dt], "h", 5.0)
    same(last, rl, 0.0, "h_last", 5.0)

    # backward: infinite gradients of the states, of finite states
    B.gated_scan_forward(z.cuda(), x.cuda(), h, h0=h0.cuda(), **how)
    gi, li = dh.clone(), dl.clone()
    gi[starts[1] // 2, 5], li[0, 6], li[S - 1, 7] = INF, -INF, INF
    dz, dx = (torch.empty(N, C, dtype=dt, device="cuda") for _ in range(2))
    d0 = torch.empty(S, C, device="cuda")
    B.gated_scan_backward(z.cuda(), x.cuda(), h, gi.cuda(), dz, dx, h0=h0.cuda(), dh_last=li.cuda(), dh0=d0, **how)
    rz, rx, r0, g = plain_backward(z.double(), x.double(), h0.double(), starts, reverse, gi.double(), li.double())
    assert int(torch.isinf(rx).sum()) > N // 8
    same(dx, rx, UNIT[dt], "dx", 5.0)
    same(d0, r0, 0.0, "dh0", 5.0)
    # (where the stored state before a step is the step's input, dgate is 0 x infinity and may be NaN)
    _, _, before = plain(z.double(), x.double(), h0.double(), starts, reverse)
    some = before.to(dt) != x
    same(dz.cpu()[some], rz[some], 2 * UNIT[dt], "dgate", 5.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
@pytest.mark.parametrize("lens,C,joint,packed", [
    ([16385], 33, 0, True),                # 16 blocks of a cluster, 9 rounds forward and 17 backward
    ([30011, 0, 777], 40, 1, True),        # 8 (f32) or 16, rows at any address; a short one and an empty one
    ([8192, 8192], 100, 4, False)])        # 8 (f32) or 16, without a table
@pytest.mark.parametrize("reverse", [False, True])
def test_long_sequences_by_clusters_without_a_workspace(lens, C, joint, packed, reverse, dt, monkeypatch):
    """A C call without a workspace: the clusters' barriers are used over many rounds and phases."""
    B = _bind()
    monkeypatch.setattr(B, "_scan", lambda call, name, args, tokens, num_seqs, stream, device: B._enqueue(call, name, args, stream, device))
    _check(B, lens, C, dt, joint, reverse, packed=packed, seed=C + 7)
    B.gated_scan_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_long_and_wide_sequences_by_clusters(dt):
    """More tiles of channels than go by runs (18 of 32 words): twenty rounds and more of eight blocks a
    cluster, then of four."""
    B = _bind()
    C = 18 * 128 // torch.tensor([], dtype=dt).element_size()
    assert B._lib.dgc_gated_scan_workspace_bytes(B.SCAN.pack(B.DTYPES[dt], 1, C, 0, 21000, *[0] * 19)) == 0
    _check(B, [21000], C, dt, packed=False, seed=3)
    _check(B, [300, 20500], C, dt, reverse=True, seed=4)
    B.gated_scan_check()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=str)
def test_both_weights_of_a_gate_over_its_whole_range(dt):
    """A step from state 1 with input 0 is f, from state 0 with input 1 it is 1 - f.  The logit's product with
    log2(e) is rounded: 2^-24 |z| of the exponential, and 1.4e-8 |z| for the constant's own rounding; the
    exponential, the sum, the reciprocal and the product add at most 2^-22 + 2^-24 + 2^-23 + 2^-24."""
    B = _bind()
    z = torch.cat([torch.linspace(-86, 86, 40001), torch.linspace(-8, 8, 40001)]).to(dt)[None]
    n = z.shape[1]
    one, none = torch.ones(1, n), torch.zeros(1, n)
    f64 = z.double()
    tol = f64.abs() * (2.0 ** -24 + 1.4e-8) + 2.0 ** -22 + 2.0 ** -23 + 2.0 ** -23
    for state, x, want in ((one, none, torch.sigmoid(f64)), (none, one, torch.sigmoid(-f64))):
        sd, out = state.cuda(), torch.empty(1, n, dtype=dt, device="cuda")
        B.gated_scan_step(z.cuda(), x.to(dt).cuda(), sd, out)
        off = (sd.double().cpu() - want).abs() / want
        assert (off <= tol).all(), (float((off / tol).max()), float(f64[0, (off / tol).argmax()]))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", DT, ids=str)
def test_scan_with_finite_gates_of_any_size(dt):
    """Logits far beyond [-6, 6].  f and 1 - f come from the same exponential, so its error moves h by
    f (1 - f) of itself: with the roundings above less than 4e-7 of the largest value a step and 1e-6 with both
    products, and at most as many steps as the sequence has: 3e-4 for 300."""
    B = _bind()
    lens, C = [300, 7, 250], 96
    starts, _, x, dh, h0, dl, _ = _case(lens, C, dt, 0, 12)
    z = (torch.randn(sum(lens), C, generator=torch.Generator().manual_seed(13)) * 20).clamp(-80, 80).to(dt)
    how = dict(seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), num_seqs=3, h0=h0.cuda())
    h, dz, dx = (torch.empty(sum(lens), C, dtype=dt, device="cuda") for _ in range(3))
    d0 = torch.empty(3, C, device="cuda")
    B.gated_scan_forward(z.cuda(), x.cuda(), h, **how)
    B.gated_scan_backward(z.cuda(), x.cuda(), h, dh.cuda(), dz, dx, dh_last=dl.cuda(), dh0=d0, **how)
    zz, xx, hh = z.double(), x.double(), h0.double()
    rh, _, _ = plain(zz, xx, hh, starts, False)
    rz, rx, r0, g = plain_backward(zz, xx, hh, starts, False, dh.double(), dl.double())
    f = torch.sigmoid(zz)
    stored = UNIT[dt] * float(rh.abs().max()) * (f * (1 - f) * g).abs()     # the stored state's rounding
    for got, want, unit, more in ((h, rh, UNIT[dt], 0.0), (dx, rx, UNIT[dt], 0.0), (d0, r0, 0.0, 0.0), (dz, rz, UNIT[dt], stored)):
        off = (got.double().cpu() - want).abs()
        assert (off <= unit * want.abs() + TINY[dt] + 3e-4 * float(want.abs().max()) + more).all()


@pytest.mark.gpu
@pytest.mark.parametrize("workspace", [True, False])
def test_scan_of_matrices_whose_offsets_pass_32_bits(workspace, monkeypatch):
    """Slices of a [8192, 2^19] product (its last rows start past 2^32 elements): the bits of packed copies."""
    B = _bind()
    if not workspace:
        monkeypatch.setattr(B, "_scan", lambda call, name, args, tokens, num_seqs, stream, device: B._enqueue(call, name, args, stream, device))
    N, C, dt = 8192, 64, torch.bfloat16
    starts, z, x, dh, h0, dl, _ = _case([N - 3, 3], C, dt, 0, 6)
    big = torch.empty(N, 1 << 19, dtype=dt, device="cuda")
    wide = [big[:, (1 << 19) - (6 - i) * C:][:, :C] for i in range(6)]
    flat = [torch.empty(N, C, dtype=dt, device="cuda") for _ in range(6)]
    how = dict(seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), num_seqs=2, h0=h0.cuda(), reverse=True)
    for m in (wide, flat):
        for to, t in zip(m, (z, x, dh)):
            to.copy_(t)
        B.gated_scan_forward(m[0], m[1], m[3], **how)
        B.gated_scan_backward(m[0], m[1], m[3], m[2], m[4], m[5], dh_last=dl.cuda(), **how)
    for a, b in zip(wide, flat):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_step_in_a_cache_whose_offsets_pass_32_bits():
    B = _bind()
    slots, C = (1 << 21) + 3, 1024                             # 8.6 GB of states
    state = torch.empty(slots, C, device="cuda")
    at = torch.tensor([slots - 1, 0, (1 << 21) - 1, slots], dtype=torch.int32, device="cuda")
    z, x = torch.randn(4, C, device="cuda"), torch.randn(4, C, device="cuda")
    before = torch.randn(3, C, device="cuda")
    state[at[:3].long()] = before
    out = torch.empty(4, C, device="cuda")
    B.gated_scan_step(z, x, state, out, slots=at)
    want, got = before.clone(), torch.empty(3, C, device="cuda")
    B.gated_scan_step(z[:3], x[:3], want, got)                 # the same rows in a small cache
    assert torch.equal(out[:3], got) and torch.equal(state[at[:3].long()], want) and (out[3] == 0).all()
