"""The gated leaky integrator (lif_gated_scan, lif_gated_scan_backward,
lif_gated_step) against the float64 reference on identical inputs.

Tolerances.  With u = 2^-24, a gate sigmoid(f) or its complement has a
relative error of at most d = (6 + 2 |f|) u (an exponential whose argument
is rounded to |f| u, a sum, a quotient, a product).  A state is a sum of
inputs decayed by products of gates, whatever the order in which the maps are
composed, so with M_t = a M_{t-1} + |input| (M_{-1} = |h_first|) its error is
at most E_t = a E_{t-1} + (2 d + 4 u) M_t.  The adjoints obey the same
recursion backwards with |dL/dh| as the input, and the gradients' products add
the errors of their factors.  A result in a narrower type is rounded once."""
import numpy as np
import pytest

from oracle import sequence as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUND = {"f32": (U, 0.0), "bf16": (2.0 ** -8, 1e-37), "f16": (2.0 ** -11, 2.0 ** -25)}
SHAPES = [(1, 1, 1), (2, 1, 5), (1, 2, 3), (3, 63, 7), (2, 64, 64), (2, 65, 130), (1, 200, 257), (4, 129, 20),
          (1, 3001, 33), (2, 1025, 512), (5, 17, 1024), (1, 5000, 4), (96, 70, 700)]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


def _dt(torch, dtype):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _scan_bound(a, f, mag0, inp):
    """(M, E) of the recursion M_t = a_t M_{t-1} + inp_t, in time order."""
    M, E = np.zeros_like(a), np.zeros_like(a)
    m, e = mag0.copy(), np.zeros_like(mag0)
    for t in range(a.shape[1]):
        d = (6 + 2 * np.minimum(np.abs(f[:, t]), 200)) * U
        m = a[:, t] * m + inp[:, t]
        e = a[:, t] * e + (2 * d + 4 * U) * m
        M[:, t], E[:, t] = m, e
    return M, E


def _check(got, want, tol, dtype, label):
    rel, ab = ROUND[dtype]
    err = np.abs(got - want)
    lim = tol + rel * (np.abs(want) + tol) + ab
    assert np.isfinite(got).all(), f"{label}: not finite"
    bad = np.argwhere(err > lim)
    assert len(bad) == 0, f"{label}: {len(bad)} off, first {tuple(bad[0])}: {got[tuple(bad[0])]!r} for " \
                          f"{want[tuple(bad[0])]!r}, bound {lim[tuple(bad[0])]:.3g}"


def _valid(n, B, T):
    return np.ones((B, T, 1), bool) if n is None else (np.arange(T)[None, :] < np.clip(n, 0, T)[:, None])[:, :, None]


def run(env, x, f, dtype, n=None, h0=None, coupled=True, gh=None, gl=None, label=""):
    """Forward and backward on device tensors x, f against the reference."""
    torch, lif = env
    B, T, D = x.shape
    print(f"[case] gated {label} B={B} T={T} D={D} {dtype} coupled={coupled} strides={x.stride()} {f.stride()}",
          flush=True)
    dn = None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda:0")
    o = lif.gated_scan(x, f, length=dn, h_first=h0, coupled=coupled, marks=True)
    gx, gf, g0 = lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl, length=dn, coupled=coupled)
    torch.cuda.synchronize()
    X, F, H0, GH, GL = (_np(v) for v in (x, f, h0, gh, gl))
    h, last, before = S.gated_scan(X, F, n, H0, coupled)
    valid = _valid(n, B, T)
    X, F = np.where(valid, X, 0.0), np.where(valid, F, 0.0)      # what lies past the length plays no part
    a, na = S._gate(F)
    a1, na1 = np.where(valid, a, 1.0), np.where(valid, na, 0.0)
    inp = np.abs(X) * (na1 if coupled else valid)
    M, E = _scan_bound(a1, F * valid, np.zeros((B, D)) if H0 is None else np.abs(H0), inp)
    _check(_np(o.h), h, E * valid, dtype, label + " h")
    _check(_np(o.h_last), last, E[:, -1], "f32", label + " h_last")
    Mb = np.concatenate([np.zeros((B, 1, D)) if H0 is None else np.abs(H0)[:, None], M[:, :-1]], 1)
    Eb = np.concatenate([np.zeros((B, 1, D)), E[:, :-1]], 1)
    _check(_np(o.marks), before[:, ::64], Eb[:, ::64], "f32", label + " marks")
    wx, wf, w0 = S.gated_scan_grad(X, F, GH, GL, n, H0, coupled)
    g = np.zeros((B, T, D)) if GH is None else np.where(valid, np.abs(GH), 0.0)
    if GL is not None:
        g[:, -1] += np.abs(GL)
    after = np.concatenate([a1[:, 1:], np.ones((B, 1, D))], 1)
    Fa = np.concatenate([(F * valid)[:, 1:], np.zeros((B, 1, D))], 1)
    L, EL = (v[:, ::-1] for v in _scan_bound(after[:, ::-1], Fa[:, ::-1], np.zeros((B, D)), g[:, ::-1]))
    d = (6 + 2 * np.minimum(np.abs(F), 200)) * U
    na_x = na1 if coupled else valid
    _check(_np(gx), wx, na_x * (EL + (d + 4 * U) * L), dtype, label + " grad_x")
    mag = Mb + (np.abs(X) if coupled else 0)
    _check(_np(gf), wf, a1 * na1 * (EL * (mag + Eb) + L * (Eb + (4 * d + 8 * U) * mag)), dtype, label + " grad_f")
    _check(_np(g0), w0, a1[:, 0] * EL[:, 0] + (2 * d[:, 0] + 4 * U) * a1[:, 0] * L[:, 0], "f32", label + " grad_h_first")
    return o, (gx, gf, g0)


def _inputs(env, B, T, D, dtype, seed, shift=2.0, spread=2.0):
    torch, _ = env
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T, D, generator=g).to(_dt(torch, dtype)).cuda()
    f = (torch.randn(B, T, D, generator=g) * spread + shift).to(_dt(torch, dtype)).cuda()
    gh = torch.randn(B, T, D, generator=g).to(_dt(torch, dtype)).cuda()
    h0, gl = torch.randn(B, D, generator=g).cuda(), torch.randn(B, D, generator=g).cuda()
    return x, f, gh, h0, gl


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,D", SHAPES)
def test_scan_shapes(env, B, T, D, dtype):
    x, f, gh, h0, gl = _inputs(env, B, T, D, dtype, B * 1000 + T + D)
    run(env, x, f, dtype, h0=h0, gh=gh, gl=gl, label="shape")


@pytest.mark.parametrize("coupled", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ragged_lengths_and_padding(env, dtype, coupled):
    """Lengths 0, 1, at the edges of blocks, T and outside [0, T]; what lies
    past a length is NaN and infinite and has no effect."""
    torch, _ = env
    n = np.array([0, 1, 63, 64, 65, 200, 300, 10 ** 6, -5, 127, 128, 129])
    x, f, gh, h0, gl = _inputs(env, len(n), 300, 66, dtype, 7)
    for b, k in enumerate(n):
        k = min(max(k, 0), 300)
        x[b, k:], f[b, k:], gh[b, k:] = float("nan"), float("inf"), float("nan")
        f[b, k + 1:] = float("nan")
    o, (gx, gf, g0) = run(env, x, f, dtype, n=n, h0=h0, gh=gh, gl=gl, coupled=coupled, label="ragged")
    assert torch.equal(o.h_last[0], h0[0]) and torch.equal(g0[0], gl[0]) and not o.h[0].any() and not gx[8].any()
    assert torch.equal(o.marks[0, 3], h0[0])             # the last state stays past the length


@pytest.mark.parametrize("split", [(1, 20000, 24), (2, 6000, 48), (1, 9999, 501)])
def test_long_sequences_of_few_channels(env, split):
    """Shapes whose time axis is shared out over workgroups, with slow leaks
    that carry a state over thousands of steps."""
    B, T, D = split
    x, f, gh, h0, gl = _inputs(env, B, T, D, "f32", 5, shift=7.0, spread=1.0)
    n = np.array([T - 17] + [T // 3] * (B - 1))
    run(env, x, f, "f32", n=n, h0=h0, gh=gh, gl=gl, label="long")
    run(env, x, f, "f32", gh=gh, coupled=False, label="long, no first state")
    run(env, x, f, "f32", gl=gl, label="long, a gradient of the last state only")


def test_strides_offsets_and_expanded_inputs(env):
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 3, 150, 72, "bf16", 11)
    want = run(env, x, f, "bf16", h0=h0, gh=gh, gl=gl, label="contiguous")
    tm = lambda v: v.transpose(0, 1).contiguous().transpose(0, 1)                 # noqa: E731
    wide = torch.zeros(3, 160, 91, dtype=torch.bfloat16, device="cuda:0")
    wide[:, 4:154, 13:85] = x
    odd = torch.empty(x.numel() + 3, dtype=torch.bfloat16, device="cuda:0")[3:].view(x.shape).copy_(f)
    for xs, fs, gs in ((tm(x), f, tm(gh)), (wide[:, 4:154, 13:85], odd, gh), (x, tm(f), wide[:, 4:154, 13:85] * 0 + gh),
                       (x.transpose(1, 2).contiguous().transpose(1, 2), f, gh)):
        got = run(env, xs, fs, "bf16", h0=h0, gh=gs, gl=gl, label="strided")
        for p, q in zip((want[0].h, want[0].h_last, *want[1]), (got[0].h, got[0].h_last, *got[1])):
            assert torch.equal(p, q)
    for fs in (f[:, :1].expand(-1, 150, -1), f[:1].expand(3, -1, -1), f[:1, :1].expand(3, 150, -1)):
        run(env, x, fs, "bf16", h0=h0, gh=gh, gl=gl, label="one gate for several steps or samples")
    run(env, x, f, "bf16", h0=h0, gh=gh[:, :1].expand(-1, 150, -1), label="expanded upstream gradient")


def test_offsets_past_32_bits(env):
    """Time and batch strides whose element offsets pass 2^31."""
    torch, lif = env
    base = torch.zeros(2_400_000_000, dtype=torch.bfloat16, device="cuda:0")
    x, f, gh, h0, gl = _inputs(env, 2, 3, 40, "bf16", 3)
    far = torch.as_strided(base, (2, 3, 40), (600_000_000, 850_000_000, 1))
    far.copy_(x)
    want = run(env, x, f, "bf16", h0=h0, gh=gh, gl=gl, label="near")
    got = run(env, far, f, "bf16", h0=h0, gh=gh, gl=gl, label="far")
    assert torch.equal(want[0].h, got[0].h) and torch.equal(want[1][1], got[1][1])
    del base, far


def test_extreme_gates(env):
    """f of +-infinity holds and replaces the state; large |f| keeps the small
    one of a and 1 - a to its relative precision."""
    torch, lif = env
    B, T, D = 1, 130, 8
    x, f, gh, h0, gl = _inputs(env, B, T, D, "f32", 2)
    f[..., 1], f[..., 2], f[..., 3], f[..., 4] = 30.0, -30.0, 88.0, -88.0
    f[0, ::2, 5], f[0, 1::2, 5] = 25.0, -25.0
    run(env, x, f, "f32", h0=h0, gh=gh, gl=gl, label="large |f|")
    run(env, x, f, "f32", h0=h0, gh=gh, gl=gl, coupled=False, label="large |f|")
    f[..., 6], f[..., 7] = float("inf"), float("-inf")
    o = lif.gated_scan(x, f, h_first=h0)
    assert torch.equal(o.h[0, :, 6], h0[0, 6].expand(T)) and torch.equal(o.h[0, :, 7], x[0, :, 7])


def test_a_nan_stays_in_its_channel(env):
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 2, 4000, 48, "f32", 9)
    clean = lif.gated_scan(x, f, h_first=h0, marks=True)
    cg = lif.gated_scan_backward(x, f, clean.marks, gh, grad_last=gl)
    x[1, 1000, 17] = float("nan")
    o = lif.gated_scan(x, f, h_first=h0, marks=True)
    g = lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl)
    torch.cuda.synchronize()
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[1, 1000:, 17] = True
    assert torch.isnan(o.h[hit]).all() and torch.equal(o.h[~hit], clean.h[~hit])
    assert torch.isnan(o.h_last[1, 17]) and torch.equal(g[0], cg[0])
    other = torch.arange(48, device="cuda:0") != 17
    assert torch.equal(g[1][..., other], cg[1][..., other]) and torch.equal(g[2], cg[2])


def test_absent_inputs_and_outputs(env):
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 3, 100, 40, "f32", 4)
    full = lif.gated_scan(x, f, h_first=h0)
    only = lif.gated_scan(x, f, h_first=h0, states=False)
    assert only.h is None and only.marks is None and torch.equal(full.h_last, only.h_last)
    run(env, x, f, "f32", gl=gl, label="no grad_h")
    run(env, x, f, "f32", gh=gh, label="no grad_last")
    o, (gx, gf, g0) = run(env, x, f, "f32", label="no gradient")
    assert not gx.any() and not gf.any() and not g0.any()
    # no steps, no samples
    e = lif.gated_scan(x[:, :0], f[:, :0], h_first=h0, marks=True)
    assert torch.equal(e.h_last, h0) and e.h.shape == (3, 0, 40) and e.marks.shape == (3, 0, 40)
    assert torch.equal(lif.gated_scan_backward(x[:, :0], f[:, :0], e.marks, grad_last=gl)[2], gl)
    assert not lif.gated_scan(x[:, :0], f[:, :0]).h_last.any()
    assert lif.gated_scan(x[:0], f[:0]).h.shape == (0, 100, 40)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,D,slots", [(1, 1, 1), (1, 512, 64), (7, 33, 20), (64, 700, 64), (5, 1030, 9)])
def test_step(env, B, D, slots, dtype):
    torch, lif = env
    g = torch.Generator().manual_seed(B + D)
    x = torch.randn(B, D, generator=g).to(_dt(torch, dtype)).cuda()
    f = (torch.randn(B, D, generator=g) * 3).to(_dt(torch, dtype)).cuda()
    pool = torch.randn(slots, D, generator=g).cuda()
    slot = torch.randperm(slots, generator=g)[:B].to(torch.int32)
    if B > 4:
        slot[1], slot[3] = -1, slots                     # streams that are left out
    print(f"[case] step B={B} D={D} slots={slots} {dtype}", flush=True)
    for coupled in (True, False):
        for sl in (slot, None):
            state = pool.clone()
            h = lif.gated_step(x, f, state, slot=None if sl is None else sl.cuda(), coupled=coupled)
            torch.cuda.synchronize()
            wh, ws = S.gated_step(_np(x), _np(f), _np(pool), None if sl is None else sl.numpy(), coupled)
            a, na = S._gate(_np(f))
            inp = np.abs(_np(x)) * (na if coupled else 1)
            at = np.arange(B) if sl is None else np.clip(sl.numpy(), 0, slots - 1)
            tol = ((6 + 2 * np.abs(_np(f))) * U * 2 + 4 * U) * (a * np.abs(_np(pool))[at] + inp)
            _check(_np(h), wh, tol, dtype, "h")
            lim = np.zeros((slots, D))
            lim[at] = np.maximum(lim[at], tol)
            _check(_np(state), ws, lim, "f32", "state")
            rest = np.setdiff1d(np.arange(slots), at if sl is None else sl.numpy())
            assert torch.equal(state[rest], pool[rest])


def test_steps_follow_a_scan(env):
    """A sequence's last state goes on step by step as the longer sequence."""
    torch, lif = env
    x, f, _, h0, _ = _inputs(env, 4, 90, 130, "f32", 21)
    whole = lif.gated_scan(x, f, h_first=h0)
    state = lif.gated_scan(x[:, :70], f[:, :70], h_first=h0).h_last
    for t in range(70, 90):
        h = lif.gated_step(x[:, t], f[:, t], state)
    torch.cuda.synchronize()
    # 20 further roundings of a state below 8 in magnitude, in another order
    assert (h - whole.h[:, -1]).abs().max() <= 8 * 90 * 16 * U
    assert torch.equal(h, state)


def test_reproducible_and_on_another_stream(env):
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 2, 7000, 100, "bf16", 31)

    def go(stream=None):
        o = lif.gated_scan(x, f, h_first=h0, marks=True, stream=stream)
        return (o.h, o.h_last, o.marks, *lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl, stream=stream))
    want = go()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = go(side)
    torch.cuda.current_stream().wait_stream(side)
    for p, q, r in zip(want, got, go()):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_copies_run_on_the_given_stream(env):
    """With a stream of its own, a call copies what it has to copy (inputs in
    another order) on that stream: it does not wait for the current one, which
    is busy here."""
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 2, 300, 64, "f32", 51)
    turned = lambda v: v.transpose(-1, -2).contiguous().transpose(-1, -2)         # noqa: E731
    z, tok = x[0], torch.zeros(300, dtype=torch.int32, device="cuda:0")
    lp, idx = lif.token_logprobs(z, k=4).top_logp, lif.token_logprobs(z, k=4).top_idx
    args = [turned(v) for v in (x, f, gh, h0, gl, z, lp, idx)]

    def go(x, f, gh, h0, gl, z, lp, idx, stream=None):
        o = lif.gated_scan(x, f, h_first=h0, marks=True, stream=stream)
        return (o.h, *lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl, stream=stream),
                lif.token_logprobs(z, tok, stream=stream).logp, *lif.distill_top(z, lp, idx, stream=stream))
    want = go(x, f, gh, h0, gl, z, lp, idx)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    got = go(*args, stream=side)
    side.synchronize()
    for p, q in zip(want, got):
        assert torch.equal(p, q.to(p.device))
    torch.cuda.synchronize()


def test_graph_replays(env):
    """Scan, backward and step captured once and replayed on new inputs."""
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 1, 5000, 40, "f32", 41)
    state = h0.clone()

    def go():
        o = lif.gated_scan(x, f, h_first=h0, marks=True)
        return (o.h, o.h_last, *lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl),
                lif.gated_step(x[:, 0], f[:, 0], state))
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go()
    for i in range(3):
        x.normal_()
        gh.normal_()
        state.copy_(h0)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        state.copy_(h0)
        for p, q in zip(got, go()):
            assert torch.equal(p, q)
        torch.cuda.synchronize()


def test_refusals(env):
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, 2, 10, 8, "f32", 1)
    o = lif.gated_scan(x, f, marks=True)
    bad = [lambda: lif.gated_scan(x.double(), f), lambda: lif.gated_scan(x, f.half()),
           lambda: lif.gated_scan(x, f[:, :9]), lambda: lif.gated_scan(x[0], f[0]), lambda: lif.gated_scan(x.cpu(), f),
           lambda: lif.gated_scan(x, f, length=torch.zeros(2, device="cuda:0")),
           lambda: lif.gated_scan(x, f, h_first=h0[:1]), lambda: lif.gated_scan_backward(x, f, None, gh),
           lambda: lif.gated_scan_backward(x, f, o.marks[:, :0], gh),
           lambda: lif.gated_scan_backward(x, f, o.marks, gh.half()),
           lambda: lif.gated_step(x[:, 0], f[:, 0], h0[:, :4]), lambda: lif.gated_step(x[:, 0], f[:, 0], h0.half()),
           lambda: lif.gated_step(x[:, 0], f[:, 0], h0, slot=torch.zeros(3, dtype=torch.int32, device="cuda:0"))]
    for fn in bad:
        with pytest.raises(ValueError):
            fn()
    with pytest.raises(lif.LifError):
        lif.gated_step(x[:, 0], f[:, 0], h0[:1])          # fewer states than streams and no slots
