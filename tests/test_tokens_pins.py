"""Pins of the float64 reference of the operators over tokens: its gradients
against central differences of its values, and small cases by hand."""
import numpy as np
import pytest

from oracle import tokens as O


def differences(value, v, step=1e-6):
    """d value / dv by central differences; error about step^2 third
    derivatives + 2^-53 / step, 1e-9 for values and derivatives around 1."""
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        keep = v[i]
        v[i] = keep + step
        up = value()
        v[i] = keep - step
        down = value()
        v[i] = keep
        g[i] = (up - down) / (2 * step)
    return g


def test_embed_by_hand():
    W = np.array([[1.0, 2.0], [3.0, 4.0]])
    tokens = np.array([[1, -1, 2, 0], [0, 0, 0, 0]])
    out = O.embed(tokens, W, 2.0, [4, 1])
    assert (out[0] == [[6, 8], [0, 0], [0, 0], [2, 4]]).all() and (out[1] == [[2, 4], [0, 0], [0, 0], [0, 0]]).all()
    g, mag = O.embed_grad(tokens, np.ones((2, 4, 2)), 2, 2.0, [4, 1])
    assert (g == [[4, 4], [2, 2]]).all() and (mag == g).all()


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("K,length", [(2, None), (4, [5, 2, 0]), (3, [1, 5, 9])])
def test_conv_gradients(K, length, silu):
    r = np.random.default_rng(K)
    B, T, D = 3, 5, 2
    v = {"x": r.normal(size=(B, T, D)), "w": r.normal(size=(D, K)), "bias": r.normal(size=D),
         "x_first": r.normal(size=(B, K - 1, D))}
    gy, gl = r.normal(size=(B, T, D)), r.normal(size=(B, K - 1, D))

    def value():
        y, last = O.causal_conv(v["x"], v["w"], v["bias"], length, v["x_first"], silu)
        return (gy * y).sum() + (gl * last).sum()
    got = O.causal_conv_grad(v["x"], v["w"], gy, v["bias"], length, v["x_first"], gl, silu)
    for name, g in zip(("x", "w", "bias", "x_first"), got):
        assert np.abs(g - differences(value, v[name])).max() < 1e-7, name


@pytest.mark.parametrize("gated,soft", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("length", [None, [4, 0]])
def test_select_gradients(length, gated, soft):
    r = np.random.default_rng(5)
    nb, T, W, N, G = 2, 4, 4, 3, 2
    v = {"x": r.normal(size=(nb, T, W)), "dt": r.normal(size=(nb, T, W)), "A": -np.exp(r.normal(size=(W, N))),
         "B": r.normal(size=(nb, T, G, N)), "C": r.normal(size=(nb, T, G, N)), "D": r.normal(size=W),
         "z": r.normal(size=(nb, T, W)), "dt_bias": r.normal(size=W), "h_first": r.normal(size=(nb, W, N))}
    if not soft:
        v["dt"], v["dt_bias"] = np.abs(v["dt"]) * 0.3, np.abs(v["dt_bias"]) * 0.3
    gy, gl = r.normal(size=(nb, T, W)), r.normal(size=(nb, W, N))
    z = lambda: v["z"] if gated else None                                       # noqa: E731

    def value():
        y, last, _ = O.selective_scan(v["x"], v["dt"], v["A"], v["B"], v["C"], v["D"], z(), v["dt_bias"], length,
                                      v["h_first"], soft)
        return (gy * y).sum() + (gl * last).sum()
    got = O.selective_scan_grad(v["x"], v["dt"], v["A"], v["B"], v["C"], gy, v["D"], z(), v["dt_bias"], length,
                                v["h_first"], gl, soft)
    for name in v:
        if name != "z" or gated:
            assert np.abs(got[name] - differences(value, v[name])).max() < 1e-7, name


def test_select_is_a_leaky_integrator():
    """One state, B = C = 1, A = -1 and a step length without softplus: h decays
    by e^{-delta} and takes in delta x."""
    x, dt = np.array([[[1.0], [0.0], [2.0]]]), np.array([[[0.5], [1.0], [0.25]]])
    one = np.ones((1, 3, 1, 1))
    y, last, _ = O.selective_scan(x, dt, np.array([[-1.0]]), one, one, softplus_=False)
    h = [0.5, 0.5 * np.exp(-1.0)]
    h.append(h[1] * np.exp(-0.25) + 0.5)
    assert np.abs(y[0, :, 0] - h).max() < 1e-15 and abs(last[0, 0, 0] - h[2]) < 1e-15
