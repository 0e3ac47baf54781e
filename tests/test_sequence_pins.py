"""The float64 reference of the sequence and answer operators against closed
forms and central differences (no GPU)."""
import numpy as np
import pytest

from oracle import sequence as S

EPS = 1e-6
# central differences of a smooth float64 function at step 1e-6: truncation
# ~ h^2 f''' ~ 1e-12 and rounding ~ 2^-53 |f| / h ~ 1e-10 |f|; losses here stay
# below 100
DIFF_TOL = 5e-8


def _diff(fn, v):
    g = np.zeros_like(v)
    it = np.nditer(v, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        keep = v[i]
        v[i] = keep + EPS
        up = fn()
        v[i] = keep - EPS
        down = fn()
        v[i] = keep
        g[i] = (up - down) / (2 * EPS)
    return g


def test_constant_gate_is_the_leaky_integrator():
    """With a constant input and gate, h_t = x + a^{t+1} (h_first - x): the
    exact decay of tau dh/dt = -h + x over t + 1 bins."""
    a, x0, h0 = 0.95, 0.7, -0.3
    f = np.full((1, 50, 1), np.log(a / (1 - a)))
    h, last, _ = S.gated_scan(np.full((1, 50, 1), x0), f, h_first=np.array([[h0]]))
    want = x0 + a ** np.arange(1, 51) * (h0 - x0)
    assert np.allclose(h[0, :, 0], want, rtol=0, atol=1e-14)
    assert last[0, 0] == h[0, -1, 0]


@pytest.mark.parametrize("coupled", [True, False])
def test_scan_gradient_against_differences(coupled):
    r = np.random.default_rng(1)
    B, T, D = 3, 7, 2
    x, f, h0 = r.standard_normal((B, T, D)), r.standard_normal((B, T, D)), r.standard_normal((B, D))
    gh, gl, n = r.standard_normal((B, T, D)), r.standard_normal((B, D)), np.array([7, 0, 4])

    def loss():
        h, last, _ = S.gated_scan(x, f, n, h0, coupled)
        return float((gh * h).sum() + (gl * last).sum())
    gx, gf, g0 = S.gated_scan_grad(x, f, gh, gl, n, h0, coupled)
    for got, v in ((gx, x), (gf, f), (g0, h0)):
        assert np.abs(got - _diff(loss, v)).max() < DIFF_TOL
    assert not gx[1].any() and not gf[2, 4:].any() and np.array_equal(g0[1], gl[1])


def test_step_is_one_step_of_the_scan():
    r = np.random.default_rng(2)
    x, f, pool = r.standard_normal((3, 1, 4)), r.standard_normal((3, 1, 4)), r.standard_normal((6, 4))
    slot = np.array([4, -1, 0])
    h, after = S.gated_step(x[:, 0], f[:, 0], pool, slot)
    want, _, _ = S.gated_scan(x[[0, 2]], f[[0, 2]], h_first=pool[[4, 0]])
    assert np.array_equal(h[[0, 2]], want[:, 0]) and not h[1].any()
    assert np.array_equal(after[[1, 2, 3, 5]], pool[[1, 2, 3, 5]])
    assert np.array_equal(after[[4, 0]], h[[0, 2]])


def test_logprobs_gradient_against_differences():
    r = np.random.default_rng(3)
    x, tok, T = r.standard_normal((4, 6)) * 2, np.array([0, -1, 5, 6]), 0.7
    gl, ge = r.standard_normal(4), r.standard_normal(4)
    x[2, 1] = -np.inf

    def loss():
        o = S.token_logprobs(x, tok, temperature=T)
        return float((gl * o["logp"]).sum() + (ge * o["entropy"]).sum())
    g = S.token_logprobs(x, tok, temperature=T, grad_logp=gl, grad_entropy=ge)["grad"]
    fin = np.isfinite(x)
    with np.errstate(invalid="ignore"):
        want = _diff(loss, x)
    assert np.abs(g - want)[fin].max() < DIFF_TOL and g[2, 1] == 0


def test_logprobs_of_uniform_masked_and_empty_rows():
    x = np.zeros((3, 8))
    x[1, 3:] = -np.inf
    x[2] = -np.inf
    o = S.token_logprobs(x, np.array([2, 5, 0]), k=4)
    assert np.allclose(o["entropy"], [np.log(8), np.log(3), 0.0]) and np.allclose(o["lse"][:2], [np.log(8), np.log(3)])
    assert np.isneginf(o["lse"][2]) and np.isneginf(o["logp"][1:]).all()
    assert np.array_equal(o["top_idx"], np.tile(np.arange(4), (3, 1)))
    low = S.token_logprobs(np.full((1, 8), -3e38), np.array([2]))         # masked by a huge finite value: uniform
    assert np.allclose(low["logp"], -np.log(8)) and np.allclose(low["entropy"], np.log(8))


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(tail):
    r = np.random.default_rng(4)
    R, V, k, T = 5, 7, 3, 1.7
    x = r.standard_normal((R, V)) * 2
    t = r.standard_normal((R, V))
    t = t - np.log(np.exp(t).sum(1, keepdims=True))
    idx = np.argsort(-t, axis=1)[:, :k]
    lp = np.take_along_axis(t, idx, 1)
    idx[1, 2], idx[2] = -1, V                        # a shorter list and an empty one
    idx[3, 1] = idx[3, 0]                            # a class listed twice
    w = r.random(R)

    def loss():
        return float((w * S.distill_top(x, lp, idx, T, tail)[0]).sum())
    l, g = S.distill_top(x, lp, idx, T, tail, w)
    assert l[2] == 0 and not g[2].any()
    assert np.abs(g - _diff(loss, x)).max() < DIFF_TOL


def test_distill_is_zero_for_the_teacher_itself():
    r = np.random.default_rng(5)
    x = r.standard_normal((3, 9))
    o = S.token_logprobs(x, k=4, temperature=2.0)
    for tail, k in ((True, 4), (False, 9)):
        o = S.token_logprobs(x, k=k, temperature=2.0)
        l, g = S.distill_top(x, o["top_logp"], o["top_idx"], 2.0, tail)
        assert np.abs(l).max() < 1e-15 and np.abs(g).max() < 1e-15
