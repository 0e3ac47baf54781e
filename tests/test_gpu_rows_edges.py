"""Rows of logits (lif_token_logprobs, lif_distill_top) where float32 would
run out of range, lose an offset or depend on an order, against the float64
reference.  Every case runs on the three ways a row can take: staged in LDS (V <= 256), held by
one workgroup (many rows), and cut into segments (few rows).

Tolerances are those of test_gpu_rows unless a test says otherwise."""
import numpy as np
import pytest

import test_gpu_rows as rows
from oracle import sequence as S
from test_gpu_rows import ROUND, _dt, _logits, _np, env, run_distill, run_logprobs       # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# rows, logits: LDS with 2, 4 and 16 lanes a row; one workgroup of 512, 512 and
# 1024 threads and segments (float32), of 256 to 1024 (16 bits); segments
PLACES = [(5, 20), (6, 64), (4, 200), (256, 4100), (256, 20011), (256, 40009), (256, 70001), (3, 20011), (3, 300000)]


def _repeat(torch, x, R):
    """x's rows over and over, R in all."""
    return x[torch.arange(R, device=x.device) % x.shape[0]].contiguous()


def run_repeated(env, x, lp, idx, dtype, R, T=1.0, tail=False, weight=None, label=""):
    """run_distill on a few rows for the reference's values, then the call of
    R rows that holds them over and over: every one has to be the few's."""
    torch, lif = env
    n = x.shape[0]
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device="cuda:0")[np.arange(R) % n].contiguous()  # noqa: E731
    big = _repeat(torch, x, R)
    print(f"[case] {label} R={R} V={x.shape[1]} k={idx.shape[1]} T={T} tail={tail} {dtype}", flush=True)
    loss, grad = lif.distill_top(big, dev(lp, torch.float32), dev(idx, torch.int32), temperature=T, tail=tail,
                                 weight=None if weight is None else dev(weight, torch.float32))
    torch.cuda.synchronize()
    for r in range(n, R):
        assert torch.equal(grad[r], grad[r % n]) or torch.isnan(grad[r % n]).any(), f"{label}: row {r}"
    assert torch.equal(loss[n:].nan_to_num(7.0), loss[torch.arange(n, R) % n].nan_to_num(7.0)), label

    class First:                                  # run_distill's checks on the rows of the large call
        LifError = lif.LifError

        @staticmethod
        def distill_top(*a, **k):
            return loss[:n], grad[:n]
    return run_distill((torch, First), x, lp, idx, dtype, T, tail, weight, label)


@pytest.mark.parametrize("R,V", PLACES)
def test_lists_of_unlikely_classes(env, R, V):
    """Classes whose probabilities lie below float32's range: made to sum to 1
    they teach as any others do, and as a part of all mass they leave it to
    the tail."""
    torch, _ = env
    n, k = min(R, 3), 6
    x = _logits(env, n, V, "f32", V)
    r = np.random.default_rng(V)
    idx = np.stack([r.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    # subnormal in float32, 0 in float32, 0 in float64
    lp = np.stack([-r.uniform(a, b, k) for a, b in ((90.0, 104.0), (110.0, 130.0), (800.0, 820.0))])
    lp = lp[:n].astype(np.float32)
    for tail in (False, True):
        loss, grad = run_repeated(env, x, lp, idx, "f32", R, 1.0, tail, label="unlikely classes")
        assert (loss > 0).all() and grad.any(1).all()


@pytest.mark.parametrize("R,V", PLACES)
@pytest.mark.parametrize("offset,T", [(5000.0, 1.0), (-1e6, 1.0), (1e8, 8.0)])
def test_rows_far_from_zero(env, monkeypatch, R, V, offset, T):
    """A common offset of a row's logits cancels in everything but lse: the
    bounds of test_gpu_rows without the term of the offset's rounding."""
    torch, _ = env
    terms = rows._terms
    monkeypatch.setattr(rows, "_terms", lambda x, T: [0.0 * v if i == 5 else v for i, v in enumerate(terms(x, T))])
    n = min(R, 3)
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(n, V, generator=g, dtype=torch.float64) * 2.5 * T + offset).float().cuda()
    big = _repeat(torch, x, R)
    r = np.random.default_rng(V)
    tok = np.resize(r.integers(0, V, n), R)
    gl, ge = np.resize(r.standard_normal(n), R), np.resize(r.standard_normal(n), R)
    first = lambda v: None if v is None else v[:n]                                # noqa: E731

    class First:                                  # the first rows of the call with all of them
        @staticmethod
        def token_logprobs(_, tokens, **k):
            dev = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device="cuda:0")   # noqa: E731
            if k["grad_logp"] is not None:
                k["grad_logp"], k["grad_entropy"] = dev(gl, torch.float32), dev(ge, torch.float32)
            o = env[1].token_logprobs(big, dev(tok, torch.int32), **k)
            return type(o)(*(first(v) for v in (o.logp, o.entropy, o.lse, o.top_logp, o.top_idx, o.grad)))
    run_logprobs((torch, First), x, "f32", tok[:n], min(V, 5), T, label="far")
    run_logprobs((torch, First), x, "f32", tok[:n], 0, T, gl[:n], ge[:n], label="far")
    idx = np.stack([r.permutation(V)[:6] for _ in range(n)]).astype(np.int32)
    lp = np.log(r.random((n, 6)) / 6).astype(np.float32)
    for tail in (False, True):
        run_repeated(env, x, lp, idx, "f32", R, T, tail, label="far")


def _far_bounds(x, lp, idx, T, w):
    """Bounds on the error of loss and gradient for a list with a tail whose
    distance to the rest is anything: the terms of test_gpu_rows, those of the
    rest by its own largest logit."""
    R, V = x.shape
    z = x / T
    listed = np.zeros((R, V), bool)
    np.put_along_axis(listed, idx.astype(np.int64), True, 1)
    q = np.exp(lp.astype(np.float64))
    eta_q = (2 * np.abs(lp.astype(np.float64)) + 6) * U
    dq, q_rest = (q * eta_q).sum(1, keepdims=True), 1 - q.sum(1, keepdims=True)

    def terms(z):
        m = z.max(1, keepdims=True)
        d = np.where(np.isinf(z), 0.0, z - m)
        e = np.exp(z - m)
        p = e / e.sum(1, keepdims=True)
        eta = (4 * np.abs(d) + 4) * U
        return d, p, eta, (p * eta).sum(1, keepdims=True) + 160 * U, m + np.log(e.sum(1, keepdims=True))
    with np.errstate(over="ignore"):
        d, p, eta, etaS, lse = terms(z)
        _, share, eta_r, etaS_r, lse_r = terms(np.where(listed, -np.inf, z))
        lp_rest, dl = np.abs(lse_r - lse), np.abs(np.take_along_axis(d, idx.astype(np.int64), 1))
    off = 2 * U * np.abs(z.max(1, keepdims=True))
    t_lp = etaS + off + 4 * U * (dl + 12)                                 # log S < 12
    t_loss = (q * (t_lp + (eta_q + 8 * U) * (np.abs(lp) + dl + 14))).sum(1)
    t_loss += (q_rest * (etaS + etaS_r + 2 * off + 8 * U * (24 + np.abs(np.log(q_rest))) + dq / q_rest)
               + dq * (np.abs(np.log(q_rest)) + lp_rest + 1))[:, 0]
    tol = 2.0 ** -126 * 4 + p * (eta + etaS + 8 * U + dq)
    tol += share * q_rest * (eta_r + etaS_r + 8 * U + dq / q_rest)
    np.add.at(tol, (np.arange(R)[:, None], idx), q * (eta_q + 8 * U))
    return t_loss, tol * np.abs(w)[:, None] / T


GAPS = [0.0, 20.0, 60.0, 84.0, 87.5, 90.0, 104.0, 150.0, 400.0, 700.0, 5000.0, None]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,V", PLACES)
def test_the_tail_far_below_the_list(env, R, V, dtype):
    """Unlisted logits far below the listed ones, up to the type's lowest value
    (None): the loss is q_rest times the distance, the unlisted classes share
    -q_rest, and the gradient of a row sums to 0.  Weights as a loss scale sets
    them, temperatures that stretch a small distance."""
    torch, lif = env
    n, k = 3, 6
    r = np.random.default_rng(V)
    idx = np.stack([r.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    q = r.random((n, k)) + 0.05
    lp = np.log(q / q.sum(1, keepdims=True) * np.array([[0.9], [0.5], [0.99]])).astype(np.float32)
    base = r.standard_normal((n, V))
    for T in (1.0, 0.1):
        for gap in GAPS:
            x = torch.tensor(base, dtype=_dt(torch, dtype))
            for i in range(n):
                rest = np.setdiff1d(np.arange(V), idx[i])
                x[i, rest] = torch.finfo(x.dtype).min if gap is None else (x[i, rest].double() - gap * T).to(x.dtype)
            x[0, np.setdiff1d(np.arange(V), idx[0])[::3]] = -float("inf")
            w = np.array([1.0, 0.25, 65536.0 if dtype != "f16" else 16.0])
            at = np.arange(R) % n
            dev = lambda a, t: torch.tensor(a[at], dtype=t, device="cuda:0")      # noqa: E731
            print(f"[case] far tail R={R} V={V} {dtype} T={T} gap={gap}", flush=True)
            loss, grad = lif.distill_top(x.cuda()[torch.tensor(at, device="cuda:0")], dev(lp, torch.float32),
                                         dev(idx, torch.int32), temperature=T, tail=True,
                                         weight=dev(w, torch.float32))
            torch.cuda.synchronize()
            for i in range(n, R):
                assert torch.equal(grad[i], grad[i % n]) and loss[i] == loss[i % n]
            X = x.double().numpy()
            wl, wg = S.distill_top(X, lp, idx, T, True, w)
            t_loss, t_grad = _far_bounds(X, lp, idx, T, w)
            rows._check(loss[:n].cpu().numpy(), wl, t_loss, 2 * U, 0, f"gap {gap} loss")
            rows._check(_np(grad[:n]), wg, t_grad, *ROUND[dtype], f"gap {gap} grad")


@pytest.mark.parametrize("R,V", [(256, 300), (256, 4100), (1024, 20011), (512, 40009), (256, 70001), (3, 20011)])
def test_a_class_listed_twice_counts_at_its_first_entry(env, R, V):
    """Entries of probability 0 that repeat earlier ones' classes, in another
    wave's part of the list or in the same, change nothing: not a bit, and not
    from call to call."""
    torch, lif = env
    k = 128
    x = _logits(env, R, V, "f32", V)
    g = torch.Generator().manual_seed(1)
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(R)]).to(torch.int32)
    lp = torch.log(torch.rand(R, k, generator=g) / k)
    lp[:, 90:], idx[:, 90:] = -float("inf"), -1
    print(f"[case] repeated classes R={R} V={V}", flush=True)
    lp = lp.cuda()
    want = lif.distill_top(x, lp, idx.cuda(), tail=True)
    for where in (slice(0, 38), slice(52, 90)):
        twice = idx.clone()
        twice[:, 90:] = idx[:, where]
        for _ in range(3):
            got = lif.distill_top(x, lp, twice.cuda(), tail=True)
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("R,V", PLACES)
def test_an_unlikely_class_that_the_student_rules_out(env, R, V):
    """However small its q, a listed class of the student's probability 0 makes
    the loss infinite; one of q = 0 does not."""
    torch, _ = env
    n, k = min(R, 3), 4
    x = _logits(env, n, V, "f32", V)
    r = np.random.default_rng(V)
    idx = np.stack([r.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    lp = np.log(np.array([[0.5, 0.2, 0.1, 0.1]] * n)).astype(np.float32)
    for i, v in enumerate((-90.0, -200.0, -np.inf)):
        lp[i, 2] = v
        x[i, int(idx[i, 2])] = -float("inf")
    for tail in (False, True):
        loss, _ = run_repeated(env, x, lp, idx, "f32", R, 1.0, tail, label="ruled out")
        assert torch.isposinf(loss[:2]).all() and torch.isfinite(loss[2])


@pytest.mark.parametrize("R,V", PLACES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_row_that_is_not_finite_next_to_unlikely_classes(env, R, V, value):
    """A NaN or +infinity is in every result of its row, however small the q of
    the listed classes."""
    torch, _ = env
    n, k = min(R, 3), min(V, 128)
    x = _logits(env, n, V, "f32", V)
    r = np.random.default_rng(V)
    idx = np.stack([r.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    lp = np.full((n, k), -200.0, np.float32)
    for i in range(n):
        x[i, int(idx[i, k - 1] if i else r.integers(0, V))] = value
    for tail in (False, True):
        loss, grad = run_repeated(env, x, lp, idx, "f32", R, 1.0, tail, label="not finite")
        assert torch.isnan(loss).all() and torch.isnan(grad).all()
