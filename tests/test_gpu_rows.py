"""Token log probabilities, entropies, alternatives (lif_token_logprobs) and
distillation from a teacher's list (lif_distill_top) against the float64
reference on identical inputs.

Tolerances.  With u = 2^-24 and d_j = (x_j - m) / T the distance to the row's
largest logit, a term e^{d_j} has a relative error of at most
eta_j = (4 |d_j| + 4) u (the rounded difference, the rounded product with
log2(e) / T, the exponential), and a sum S of positive terms adds at most
160 u (at most 128 terms in a row in one lane, then trees), so its relative
error is etaS = sum p_j eta_j + 160 u.  From these follow, term by term, the
errors of log S, of log p = d - log S, of the entropy and of the gradients'
products.  |m| / T enters once more where the exponent's offset is rounded.
A term below 2^-126 may count as 0.
A gradient is rounded once to its type.  Indices have to be equal."""
import numpy as np
import pytest

from oracle import sequence as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -126
ROUND = {"f32": (U, 1e-44), "bf16": (2.0 ** -8, 1e-37), "f16": (2.0 ** -11, 2.0 ** -25)}
WIDTHS = [1, 2, 3, 7, 8, 20, 33, 63, 64, 65, 100, 255, 511, 513, 1000, 1025, 2049, 4097, 8193, 16383, 16385, 32767,
          32769, 50021, 65537, 131071, 131073, 200003]


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


def _check(got, want, tol, rel, ab, label):
    got, want, tol = (np.asarray(v, np.float64) for v in (got, want, tol))
    with np.errstate(over="ignore"):
        want = np.where(np.isinf(want.astype(np.float32)), np.copysign(np.inf, want), want)    # past float32's range
    fin = np.isfinite(want)
    assert np.array_equal(fin, np.isfinite(got)) and np.array_equal(np.isnan(want), np.isnan(got)), \
        f"{label}: infinities or NaN in other places"
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), label
    g, w, t = got[fin], want[fin], np.broadcast_to(tol, want.shape)[fin]
    lim = t + rel * (np.abs(w) + t) + ab
    bad = np.nonzero(np.abs(g - w) > lim)[0]
    assert len(bad) == 0, f"{label}: {len(bad)} off, first {g[bad[0]]!r} for {w[bad[0]]!r}, bound {lim[bad[0]]:.3g}"


def _terms(x, T):
    """d, p, eta, etaS, log S and the offset's rounding, per row; rows that are
    not finite get zeros (their results are compared for what they are)."""
    z = x / T
    m = np.max(np.where(np.isnan(z), -np.inf, z), axis=1, keepdims=True)
    odd = ~np.isfinite(m) | np.isnan(z).any(1, keepdims=True)
    d = np.where(odd, 0.0, z - np.where(odd, 0.0, m))
    d = np.maximum(d, -1e4)                      # e^d is 0 there, in both
    e = np.exp(d)
    s = e.sum(1, keepdims=True)
    p = e / s
    eta = (4 * np.abs(d) + 4) * U
    etaS = (p * eta).sum(1, keepdims=True) + 160 * U
    return d, p, eta, etaS, np.log(s), 2 * U * np.where(odd, 0.0, np.abs(m)), odd


def run_logprobs(env, x, dtype, tokens=None, k=0, T=1.0, gl=None, ge=None, label=""):
    torch, lif = env
    R, V = x.shape
    print(f"[case] logprobs {label} R={R} V={V} k={k} T={T} {dtype} stride={x.stride(0)}", flush=True)
    dev = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device="cuda:0")       # noqa: E731
    o = lif.token_logprobs(x, dev(tokens, torch.int32), k=k, temperature=T, grad_logp=dev(gl, torch.float32),
                           grad_entropy=dev(ge, torch.float32))
    torch.cuda.synchronize()
    X = _np(x)
    gl, ge = (None if g is None else np.asarray(g, np.float32).astype(np.float64) for g in (gl, ge))
    with np.errstate(over="ignore", invalid="ignore"):
        w = S.token_logprobs(X, tokens, k, T, gl, ge)
        d, p, eta, etaS, ls, off, odd = _terms(X, T)
    ls, off, es = ls[:, 0], off[:, 0], etaS[:, 0]
    t_ls = es + 2 * U * np.abs(ls) + off
    tok = np.zeros(R, int) if tokens is None else np.clip(np.asarray(tokens), 0, V - 1)
    d_tok = np.abs(d[np.arange(R), tok])
    _check(_np(o.lse), w["lse"], t_ls, 2 * U, 0, label + " lse")
    _check(_np(o.logp), w["logp"], t_ls + 4 * U * (d_tok + np.abs(ls)), 2 * U, 0, label + " logp")
    bar = (p * np.abs(d)).sum(1)
    t_H = t_ls + (p * np.abs(d) * (eta + 160 * U)).sum(1) + bar * es + 4 * U * (bar + np.abs(ls))
    _check(_np(o.entropy), w["entropy"], t_H, 2 * U, 0, label + " entropy")
    if k:
        assert np.array_equal(o.top_idx.cpu().numpy(), w["top_idx"]), label + " top_idx"
        dt = np.abs(np.take_along_axis(d, w["top_idx"], 1))
        _check(_np(o.top_logp), w["top_logp"], t_ls[:, None] + 4 * U * (dt + np.abs(ls)[:, None]), 2 * U, 0,
               label + " top_logp")
    if o.grad is not None:
        G = np.zeros(R) if gl is None else np.abs(gl)
        Ge = np.zeros(R) if ge is None else np.abs(ge)
        lpH = np.abs(d) + np.abs(ls)[:, None] + np.abs(np.where(odd[:, 0], 0, w["entropy"]))[:, None]
        tol = p * (G[:, None] + Ge[:, None] * lpH) * (eta + etaS + 6 * U) + p * Ge[:, None] * (
            2 * t_ls + t_H + 4 * U * d_tok)[:, None]
        tol += TINY * (G[:, None] + Ge[:, None] * lpH)
        if tokens is not None:
            tol[np.arange(R), tok] += 4 * U * G
        _check(_np(o.grad), w["grad"], tol / T, *ROUND[dtype], label + " grad")
    return o


def run_distill(env, x, lp, idx, dtype, T=1.0, tail=False, weight=None, label=""):
    torch, lif = env
    R, V = x.shape
    print(f"[case] distill {label} R={R} V={V} k={idx.shape[1]} T={T} tail={tail} {dtype} stride={x.stride(0)}",
          flush=True)
    lp = np.asarray(lp, np.float32)
    dev = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device="cuda:0")       # noqa: E731
    loss, grad = lif.distill_top(x, dev(lp, torch.float32), dev(idx, torch.int32), temperature=T, tail=tail,
                                 weight=dev(weight, torch.float32))
    torch.cuda.synchronize()
    X, wt = _np(x), np.ones(R) if weight is None else np.asarray(weight, np.float32).astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        wl, wg = S.distill_top(X, lp, idx, T, tail, wt)
        d, p, eta, etaS, ls, off, odd = _terms(X, T)
    used = (idx >= 0) & (idx < V)
    at = np.clip(idx, 0, V - 1)
    lt = np.where(used, lp, -np.inf).astype(np.float64)
    q = np.exp(lt)
    total = q.sum(1, keepdims=True)
    eta_q = np.where(q > 0, (2 * np.abs(np.where(q > 0, lt, 0)) + 6) * U, 0)
    scale = np.where(total > 0, total, 1.0) if not tail else 1.0
    qn = q / scale
    dl = np.abs(np.take_along_axis(d, at, 1))
    t_lp = (etaS + off[:, :1]) + 4 * U * (dl + np.abs(ls))
    t_loss = (qn * (t_lp + (eta_q + 8 * U) * (np.abs(np.where(q > 0, lt, 0)) + dl + np.abs(ls) + 2))).sum(1)
    listed = np.zeros((R, V), bool)
    for r in range(R):
        listed[r, at[r][used[r]]] = True
    q_rest, p_rest = np.zeros((R, 1)), (p * ~listed).sum(1, keepdims=True)
    t_rest = np.zeros((R, 1))
    if tail:
        q_rest = np.where((1 - total >= S.TAIL_MIN) & ~listed.all(1, keepdims=True), 1 - total, 0.0)
        dq = (q * eta_q).sum(1, keepdims=True)
        t_rest = np.where(q_rest > 0, dq / np.where(q_rest > 0, q_rest, 1), 0) + 8 * U + etaS + (
            p * ~listed * eta).sum(1, keepdims=True) / np.maximum(p_rest, 1e-300) + 160 * U
        ratio = np.abs(np.log(np.maximum(q_rest, 1e-30) / np.maximum(p_rest, 1e-300)))
        t_loss = t_loss + (q_rest * t_rest + dq * (ratio + 1))[:, 0]
    _check(_np(loss), wl, t_loss, 2 * U, 0, label + " loss")
    tol = TINY * 4 + p * (eta + etaS + 8 * U + (q * eta_q).sum(1, keepdims=True))
    np.add.at(tol, (np.arange(R)[:, None], at), qn * (eta_q + 8 * U))
    tol = tol + np.where(listed, 0, p * (q_rest / np.maximum(p_rest, 1e-300)) * (t_rest + eta))
    _check(_np(grad), wg, tol * np.abs(wt)[:, None] / T, *ROUND[dtype], label + " grad")
    return loss, grad


def _logits(env, R, V, dtype, seed, spread=2.5):
    torch, _ = env
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(R, V, generator=g) * spread).to(_dt(torch, dtype)).cuda()


def _teacher(R, V, k, seed, T=1.0, spread=2.5):
    r = np.random.default_rng(seed)
    t = r.standard_normal((R, V)) * spread / T
    t = t - np.log(np.exp(t).sum(1, keepdims=True))
    idx = np.argsort(-t, axis=1)[:, :k]
    return np.take_along_axis(t, idx, 1).astype(np.float32), idx.astype(np.int32)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", WIDTHS)
def test_logprobs_widths(env, V, dtype):
    R = 5 if V < 60000 else 2
    r = np.random.default_rng(V)
    x = _logits(env, R, V, dtype, V)
    tok = r.integers(0, V, R)
    tok[-1] = -1 if V % 2 else V
    k = min(V, (5, 20, 64, 128)[V % 4])
    run_logprobs(env, x, dtype, tok, k, 0.7 if V % 3 else 1.0, label="alternatives")
    run_logprobs(env, x, dtype, tok, 0, 1.3, r.standard_normal(R), r.standard_normal(R), label="gradient")
    run_logprobs(env, x, dtype, tok, min(V, 3), 1.0, r.standard_normal(R), None, label="both")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", WIDTHS)
def test_distill_widths(env, V, dtype):
    R = 5 if V < 60000 else 2
    k = min(V, (1, 5, 64, 128)[V % 4])
    x = _logits(env, R, V, dtype, V + 1)
    lp, idx = _teacher(R, V, k, V)
    idx[R - 1, k // 2:] = -1                       # a shorter list (none at all for k = 1)
    w = np.random.default_rng(V).random(R) + 0.5
    for tail in (False, True):
        run_distill(env, x, lp, idx, dtype, 1.0, tail, w, label="widths")
    run_distill(env, x, lp, idx, dtype, 2.5, True, None, label="temperature")


@pytest.mark.parametrize("R,V", [(1000, 20), (3001, 64), (700, 65), (513, 300), (300, 2000)])
def test_many_narrow_rows(env, R, V):
    r = np.random.default_rng(R)
    for dtype in ("f32", "bf16"):
        x = _logits(env, R, V, dtype, R)
        tok = r.integers(-1, V + 1, R)
        run_logprobs(env, x, dtype, tok, min(V, 7), 1.0, r.standard_normal(R), r.standard_normal(R), label="narrow")
        lp, idx = _teacher(R, V, 6, R)
        run_distill(env, x, lp, idx, dtype, 1.0, True, r.random(R), label="narrow")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [20, 64, 300, 3000, 20011, 70001])
def test_masks_ties_and_rows_that_are_not_finite(env, V, dtype):
    """Rows masked by -infinity or by the type's lowest value down to nothing,
    one or a few logits, constant rows, many ties, signed zeros, NaN and
    infinities."""
    torch, _ = env
    x = _logits(env, 14, V, dtype, 5)
    low = torch.finfo(x.dtype).min
    inf = float("inf")
    x[0] = -inf                                     # nothing left
    x[1, :V - 1] = -inf                             # one left, the last
    x[2, 4:] = -inf                                 # fewer left than alternatives asked for
    x[3] = low                                      # all at the lowest value
    x[4, 3:] = low
    x[5] = 1.5                                      # constant
    x[6] = torch.round(x[6])                        # few distinct values
    x[7] = 0.0
    x[7, 1::2] = -0.0                               # signed zeros are equal
    x[8, V // 2] = float("nan")
    x[9, V // 3] = inf
    x[10] = torch.finfo(x.dtype).max / 4            # large offsets: only differences matter
    x[10, 5] = torch.finfo(x.dtype).max / 2
    x[11, ::2] = -inf
    x[12] = -torch.arange(V, device=x.device).to(x.dtype)     # decreasing: the first ones are the likeliest
    x[13] = torch.arange(V, device=x.device).to(x.dtype)      # increasing, with ties from rounding
    r = np.random.default_rng(6)
    tok = np.array([0, V - 1, 6, 1, 0, V - 1, 3, 2, 1, 1, 5, 0, 0, V - 1])
    for T in (1.0, 0.5, 3.0):
        run_logprobs(env, x, dtype, tok, min(V, 20), T, label="special")
        run_logprobs(env, x, dtype, tok, 0, T, r.standard_normal(14), r.standard_normal(14), label="special gradient")
    lp, idx = _teacher(14, V, min(V, 16), 6)
    with np.errstate(all="ignore"):
        for tail in (False, True):
            loss, grad = run_distill(env, x, lp, idx, dtype, 1.0, tail, label="special")
            assert torch.isposinf(loss[0]) and not grad[0].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_over_many_segments(env, dtype):
    """Constant rows, few distinct values and alternatives that all lie in one
    segment, in rows that are cut into many."""
    torch, _ = env
    V = 300000
    for v in (torch.zeros(1, V), torch.randn(1, V).round(), torch.arange(V).flip(0)[None] / 8.0,
              torch.where(torch.arange(V) % 2999 == 7, 1.0, -float("inf"))[None]):
        x = v.to(_dt(torch, dtype)).cuda()
        for k in (128, 20, 1):
            run_logprobs(env, x, dtype, np.array([5]), k, label="many segments")


@pytest.mark.parametrize("V", [20, 64, 1000, 40009, 140001])
def test_teacher_lists(env, V):
    """Unused entries, empty lists, entries of probability 0, repeated classes,
    a list with all mass, every class listed, a masked vocabulary."""
    torch, _ = env
    k = min(V, 20)
    x = _logits(env, 8, V, "f32", 9)
    lp, idx = _teacher(8, V, k, 10)
    idx[0] = -1
    idx[1, ::2] = V + 5
    lp[2, 3:] = -np.inf
    lp[3] = -np.inf
    idx[4, 1] = idx[4, 0]
    lp[5] = np.log(1.0 / k)                        # no mass left for the tail
    lp[6, 1:], lp[6, 0] = -np.inf, 0.0             # a certain teacher
    keep = idx[7, :k // 2]
    x[7] = -float("inf")
    x[7, keep.tolist()] = torch.randn(len(keep), device="cuda:0")
    q = np.exp(lp[7, :k // 2].astype(np.float64))
    lp[7, :k // 2], lp[7, k // 2:] = np.log(q / q.sum()), -np.inf     # teacher and student masked alike
    w = np.array([1.0, 0.5, 0.0, 2.0, -1.0, 1.0, 1.0, 1.0])
    for tail in (False, True):
        loss, grad = run_distill(env, x, lp, idx, "f32", 1.0, tail, w, label="lists")
        assert loss[0] == 0 and not grad[0].any() and loss[3] == 0 and not grad[3].any() and not grad[2].any()
        assert torch.isfinite(loss).all() and torch.isfinite(grad).all()


def test_a_teachers_alternatives_train_its_own_copy_to_nothing(env):
    torch, lif = env
    x = _logits(env, 6, 5000, "f32", 12)
    o = lif.token_logprobs(x, k=64, temperature=2.0)
    loss, grad = run_distill(env, x, o.top_logp.cpu().numpy(), o.top_idx.cpu().numpy(), "f32", 2.0, True, label="own")
    # the bounds of the logarithms above, at p <= 1 and |log p| <= 20
    assert loss.abs().max() < 400 * U and grad.abs().max() < 400 * U


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 1003, 9001, 40009])
def test_strides_and_alignment(env, V, dtype):
    """Padded rows, rows off the vector grid, a view that starts off it, rows
    in other orders: the same bits."""
    torch, lif = env
    R, k = 6, 16
    x = _logits(env, R, V, dtype, 14)
    r = np.random.default_rng(15)
    tok = torch.tensor(r.integers(0, V, R), dtype=torch.int32, device="cuda:0")
    g = torch.randn(R, device="cuda:0")
    lp, idx = _teacher(R, V, k, 16)
    lp, idx = torch.tensor(lp, device="cuda:0"), torch.tensor(idx, device="cuda:0")

    def go(v):
        o = lif.token_logprobs(v, tok, k=k, grad_logp=g, grad_entropy=g)
        return (o.logp, o.entropy, o.lse, o.top_logp, o.top_idx, o.grad, *lif.distill_top(v, lp, idx, tail=True))
    want = go(x)
    for pad, lead in ((0, 1), (3, 0), (5, 7), (8, 8)):
        wide = torch.full((R, lead + V + pad), float("nan"), dtype=x.dtype, device="cuda:0")
        view = wide[:, lead:lead + V]
        view.copy_(x)
        for p, q in zip(want, go(view)):
            assert torch.equal(p, q), (pad, lead)
    for view in (x.t().contiguous().t(), x[:1].expand(R, V)):          # copied by the binding
        for p, q in zip(go(view.contiguous()), go(view)):
            assert torch.equal(p, q)


def test_row_offsets_past_32_bits(env):
    torch, lif = env
    base = torch.zeros(2_500_000_000, dtype=torch.bfloat16, device="cuda:0")
    for V in (50, 3000, 40009):
        x = _logits(env, 3, V, "bf16", 17)
        far = torch.as_strided(base, (3, V), (1_200_000_000, 1))
        far.copy_(x)
        tok = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda:0")
        a, b = (lif.token_logprobs(v, tok, k=9, grad_logp=torch.ones(3, device="cuda:0")) for v in (x, far))
        torch.cuda.synchronize()
        assert torch.equal(a.logp, b.logp) and torch.equal(a.top_idx, b.top_idx) and torch.equal(a.grad, b.grad)
    del base, far


def test_reproducible_streams_and_graphs(env):
    torch, lif = env
    for R, V, k in ((1, 131072, 20), (700, 20, 5), (4, 50021, 64), (9, 600, 30)):
        x = _logits(env, R, V, "bf16", 19)
        lp, idx = _teacher(R, V, k, 20)
        lp, idx = torch.tensor(lp, device="cuda:0"), torch.tensor(idx, device="cuda:0")
        tok, g = torch.zeros(R, dtype=torch.int32, device="cuda:0"), torch.ones(R, device="cuda:0")

        def go(stream=None):
            o = lif.token_logprobs(x, tok, k=k, grad_logp=g, stream=stream)
            return (o.logp, o.entropy, o.lse, o.top_logp, o.top_idx, o.grad,
                    *lif.distill_top(x, lp, idx, tail=True, stream=stream))
        want = go()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = go(side)
        torch.cuda.current_stream().wait_stream(side)
        for p, q in zip(want, got):
            assert torch.equal(p, q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = go()
        for _ in range(3):
            x.normal_()
            graph.replay()
            torch.cuda.synchronize()
            for p, q in zip([v.clone() for v in out], go()):
                assert torch.equal(p, q)
            torch.cuda.synchronize()


def test_gradients_against_differences(env):
    """The float32 gradients against central differences of the float32
    losses: step 2^-6, truncation h^2 / 6 max |f'''| < 2e-4 (third derivatives
    of a log-softmax are below 2 / T^3), rounding 2 * 300 u * 8 / (2 h) < 1e-2
    relative to losses below 8."""
    torch, lif = env
    h = 2.0 ** -6
    x = _logits(env, 1, 23, "f32", 21)
    lp, idx = (torch.tensor(v, device="cuda:0") for v in _teacher(1, 23, 5, 22))
    tok, one, e = torch.tensor([4], dtype=torch.int32, device="cuda:0"), torch.ones(1, device="cuda:0"), 0.5
    steps = torch.eye(23, device="cuda:0") * h
    up, down = x + steps, x - steps
    toks = tok.expand(23).contiguous()
    many = lambda v: lif.token_logprobs(v, toks)                                   # noqa: E731
    a, b = many(up), many(down)
    want = ((a.logp + e * a.entropy) - (b.logp + e * b.entropy)) / (2 * h)
    got = lif.token_logprobs(x, tok, grad_logp=one, grad_entropy=one * e).grad[0]
    tol = 2e-4 * (1 + 8 * e) + 300 * U * 16 / (2 * h)
    assert (got - want).abs().max() < tol
    for tail in (False, True):
        a, b = (lif.distill_top(v, lp.expand(23, -1).contiguous(), idx.expand(23, -1).contiguous(), tail=tail,
                                want_grad=False)[0] for v in (up, down))
        got = lif.distill_top(x, lp, idx, tail=tail)[1][0]
        assert (got - (a - b) / (2 * h)).abs().max() < tol


def test_empty_calls_and_refusals(env):
    torch, lif = env
    x = _logits(env, 4, 30, "f32", 1)
    o = lif.token_logprobs(x[:0], k=3)
    assert o.logp.shape == (0,) and o.top_idx.shape == (0, 3)
    assert lif.distill_top(x[:0], torch.zeros(0, 3, device="cuda:0"),
                           torch.zeros(0, 3, dtype=torch.int32, device="cuda:0"))[1].shape == (0, 30)
    o = lif.token_logprobs(x)
    assert not o.logp.any() and o.top_idx is None and o.grad is None
    lp, idx = torch.zeros(4, 0, device="cuda:0"), torch.zeros(4, 0, dtype=torch.int32, device="cuda:0")
    loss, grad = lif.distill_top(x, lp, idx)          # a list of nothing teaches nothing
    assert not loss.any() and not grad.any()
    z32 = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    lp, idx = torch.zeros(4, 2, device="cuda:0"), torch.zeros(4, 2, dtype=torch.int32, device="cuda:0")
    for fn in (lambda: lif.token_logprobs(x.double()), lambda: lif.token_logprobs(x[0]),
               lambda: lif.token_logprobs(x.cpu()), lambda: lif.token_logprobs(x, z32.long()),
               lambda: lif.token_logprobs(x, z32[:3]), lambda: lif.token_logprobs(x, z32, grad_logp=z32),
               lambda: lif.distill_top(x, lp.double(), idx), lambda: lif.distill_top(x, lp, idx.long()),
               lambda: lif.distill_top(x, lp[:3], idx), lambda: lif.distill_top(x, lp, idx[0]),
               lambda: lif.distill_top(x, lp, idx, weight=z32)):
        with pytest.raises(ValueError):
            fn()
    for fn in (lambda: lif.token_logprobs(x, k=31), lambda: lif.token_logprobs(x, k=-1),
               lambda: lif.token_logprobs(x, temperature=0.0), lambda: lif.token_logprobs(x, temperature=float("nan")),
               lambda: lif.token_logprobs(torch.zeros(1, 500, device="cuda:0"), k=129),
               lambda: lif.distill_top(x, lp, idx, temperature=-1.0)):
        with pytest.raises(lif.LifError):
            fn()
