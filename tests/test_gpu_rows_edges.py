"""Rows of logits (lif_token_logprobs, lif_distill_top) where float32 would
run out of range, lose an offset or depend on an order, against the float64
reference.  Every case runs on the three ways a row can take: staged in LDS (V <= 256), held by
one workgroup (many rows), and cut into segments (few rows).

Tolerances are those of test_gpu_rows unless a test says otherwise."""
import numpy as np
import pytest

import test_gpu_rows as rows
from test_gpu_rows import _logits, env, run_distill, run_logprobs       # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
#         rows, logits: LDS with 2, 4 and 16 lanes a row; one workgroup of 256, 512, 512 and 1024 threads; segments
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
