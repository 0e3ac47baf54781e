"""What the GPU tests of the convolution and the scan compare with: the values
of their error analyses are those of oracle/tokens.py, whose gradients are
pinned to differences.  Both are float64 from the same formulas: 1e-12."""
import numpy as np
import pytest

import test_gpu_conv as conv
import test_gpu_select as select
from oracle import tokens as O


def same(got, want, label):
    assert got.shape == want.shape, label
    assert np.abs(got - want).max(initial=0.0) <= 1e-12 * max(1.0, np.abs(want).max(initial=0.0)), label


@pytest.mark.parametrize("act", [True, False])
@pytest.mark.parametrize("missing", [None, "bias", "x_first", "grad_last", "grad_y"])
@pytest.mark.parametrize("K,length", [(2, [6, 6, 6]), (4, [5, 2, 0]), (8, [1, 6, 3])])
def test_conv(K, length, missing, act):
    r = np.random.default_rng(K)
    nb, T, W = 3, 6, 5
    v = {"x": r.normal(size=(nb, T, W)), "w": r.normal(size=(W, K)), "bias": r.normal(size=W),
         "x_first": r.normal(size=(nb, K - 1, W)), "grad_y": r.normal(size=(nb, T, W)),
         "grad_last": r.normal(size=(nb, K - 1, W))}
    if missing:
        v[missing] = None
    got = conv.reference(v, np.asarray(length), act)
    y, last = O.causal_conv(v["x"], v["w"], v["bias"], length, v["x_first"], act)
    gy = np.zeros((nb, T, W)) if v["grad_y"] is None else v["grad_y"]
    gx, gw, gb, g0 = O.causal_conv_grad(v["x"], v["w"], gy, v["bias"], length, v["x_first"], v["grad_last"], act)
    for k, w in {"y": y, "grad_x": gx, "grad_w": gw, "grad_bias": gb, "grad_x_first": g0}.items():
        same(got[k].v, w, k)
    same(got["x_last"], last, "x_last")


@pytest.mark.parametrize("soft", [True, False])
@pytest.mark.parametrize("missing", [(), ("D",), ("z",), ("dt_bias",), ("h_first",), ("grad_last",),
                                     ("D", "z", "dt_bias", "h_first", "grad_last")])
@pytest.mark.parametrize("G,length", [(1, [7, 7]), (2, [7, 3]), (3, [0, 5])])
def test_select(G, length, missing, soft):
    r = np.random.default_rng(G)
    nb, T, W, N = 2, 7, 6, 3
    rn = lambda *s: r.normal(size=s)                                                      # noqa: E731
    v = {"x": rn(nb, T, W), "dt": np.abs(rn(nb, T, W)) * 0.3, "A": -np.exp(rn(W, N)), "B": rn(nb, T, G, N),
         "C": rn(nb, T, G, N), "D": rn(W), "z": rn(nb, T, W), "dt_bias": np.abs(rn(W)) * 0.3, "h_first": rn(nb, W, N),
         "grad_y": rn(nb, T, W), "grad_last": rn(nb, W, N)}
    for k in missing:
        v[k] = None
    got = select.reference(v, np.asarray(length), soft)
    inputs = [v[k] for k in ("x", "dt", "A", "B", "C")]
    y, last, _ = O.selective_scan(*inputs, v["D"], v["z"], v["dt_bias"], length, v["h_first"], soft)
    same(got["y"].v, y, "y")
    same(got["h_last"].v, last, "h_last")
    want = O.selective_scan_grad(*inputs, v["grad_y"], v["D"], v["z"], v["dt_bias"], length, v["h_first"],
                                 v["grad_last"], soft)
    for k, w in want.items():
        if k != "z" or v["z"] is not None:
            same(got["grad_" + k].v, w, "grad_" + k)
