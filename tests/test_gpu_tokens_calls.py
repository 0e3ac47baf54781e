"""Calls of the operators over tokens that the other tests do not make: steps of
convolutions whose width is no multiple of a vector's, masked steps, the widest
and longest calls, growing states; tolerances by running error analysis
(tests/rounding.py)."""
import numpy as np
import pytest

import test_gpu_conv as conv
import test_gpu_select as select
from rounding import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nb,W,K", [(300, 33, 8), (512, 33, 4), (1, 257, 4), (64, 257, 2), (8, 1001, 4), (512, 1001, 3),
                                    (1, 2049, 4), (130, 2049, 8), (5, 2050, 4), (300, 7, 2), (300, 6, 5)])
def test_step_widths(env, nb, W, K, dtype):
    """Streams whose last channels lie in another wave or workgroup than those
    before them: outputs and states by the formula, repeated steps too."""
    torch, lif = env
    print(f"[case] conv step {nb} x {W} K={K} {dtype}", flush=True)
    v = conv.make(torch, (nb, 6, W, K), dtype, seed=W)
    state = v["x_first"].clone()
    ys = [lif.causal_conv_step(v["x"][:, t], v["w"], state, bias=v["bias"]) for t in range(6)]
    want = conv.reference({k: conv.arr(t) for k, t in v.items()}, np.full(nb, 6))
    check(conv.arr(torch.stack(ys, 1)), want["y"], dtype, "y")
    assert np.array_equal(conv.arr(state), want["x_last"])


def scan(env, v, length=None, soft=True):
    """Forward and backward on v: results by the names of select.reference."""
    torch, lif = env
    n = None if length is None else torch.tensor(length, dtype=torch.int32, device="cuda:0")
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], dt_bias=v["dt_bias"], length=n, softplus=soft)
    o = lif.selective_scan(*args, h_first=v["h_first"], marks=True, **kw)
    g = lif.selective_scan_backward(*args, o.marks, v["grad_y"], grad_last=v["grad_last"], **kw)
    torch.cuda.synchronize()
    return {"y": o.y, "h_last": o.h_last, **{"grad_" + k: getattr(g, k) for k in
                                             ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h_first")}}


def compare(env, got, v, dtype, label, length=None, soft=True):
    nb, T = v["x"].shape[:2]
    want = select.reference({k: select.arr(t) for k, t in v.items()}, select.steps_of(length, nb, T), soft,
                            select.segment_of(env[1], v))
    for k, w in want.items():
        if got[k] is not None:
            check(select.arr(got[k]), w, "f32" if k in select.FLOAT32 else dtype, f"{label} {k}")


def masked(torch, v, part):
    """Which steps of which channels have a step length of 0: single ones, a
    channel's whole sequence, a whole sample."""
    g = torch.Generator().manual_seed(5)
    off = torch.rand(v["dt"].shape, generator=g) < 0.2
    if part == "sample":
        off[0] = True
    off[..., 1] = True
    return off.to("cuda:0")


# few columns share out the time axis in the last two
MASKED = [(2, 40, 33, 9, 1), (2, 37, 70, 6, 2), (1, 20, 5, 64, 1), (2, 1200, 40, 16, 1), (1, 1100, 20, 33, 1)]


@pytest.mark.parametrize("part", ["steps", "sample"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", MASKED)
def test_masked_steps(env, shape, dtype, part):
    """dt = -infinity is a step length of 0: the step leaves the state alone,
    and no gradient goes through dt.  The reference takes -200 there, whose step
    length is 10^-87."""
    torch, lif = env
    print(f"[case] masked {shape} {dtype} {part}", flush=True)
    v = select.make(torch, shape, dtype, seed=3)
    off = masked(torch, v, part)
    v["dt"][off] = float("-inf")
    got = scan(env, v)
    assert not got["grad_dt"][off].any() and not got["grad_dt_bias"][1]
    if part == "sample":
        assert torch.equal(got["h_last"][0], v["h_first"][0])
    v["dt"][off] = -200.0
    compare(env, got, v, dtype, "masked")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masked_streams(env, dtype):
    """The same for single steps: such a stream's state keeps its bits."""
    torch, lif = env
    v = select.make(torch, (5, 1, 66, 16, 2), dtype, seed=4, step=True)
    off = masked(torch, v, "sample")
    v["dt"][off] = float("-inf")
    state, kept = v["h_first"].clone(), v["h_first"]
    y = lif.selective_step(*[v[k] for k in ("x", "dt", "A", "B", "C")], state, D=v["D"], z=v["z"],
                           dt_bias=v["dt_bias"])
    assert torch.equal(state[off], kept[off])
    v["dt"][off] = -200.0
    ref = {k: select.arr(t)[:, None] if k in ("x", "dt", "B", "C", "z", "grad_y") else select.arr(t)
           for k, t in v.items()}
    want = select.reference(ref, np.full(5, 1))
    check(select.arr(y), want["y"][:, 0], dtype, "y")
    check(select.arr(state), want["h_last"], "f32", "state")


def test_longest_steps(env):
    """Step lengths near the largest float32: the state is forgotten, an input
    of 0 comes in as 0."""
    torch, lif = env
    v = select.make(torch, (2, 40, 33, 9, 1), "f32", seed=6)
    v["dt"][:, 20], v["x"][:, 20], v["dt_bias"] = 3e38, 0.0, None
    args = [v[k] for k in ("dt", "A", "B", "C")]
    o = lif.selective_scan(v["x"][:, :21], *[t if k == 1 else t[:, :21] for k, t in enumerate(args)],
                           h_first=v["h_first"])
    assert not o.h_last.any() and torch.isfinite(o.y).all()
    state = v["h_first"].clone()
    lif.selective_step(v["x"][:, 20], *[t if k == 1 else t[:, 20, 0] if k > 1 else t[:, 20]
                                        for k, t in enumerate(args)], state)
    assert not state.any()


@pytest.mark.parametrize("shape", MASKED)
def test_infinite_rates(env, shape):
    """A = -infinity: a state that keeps nothing over a step of positive length,
    and stays over one of length 0.  The reference takes -10^30."""
    torch, lif = env
    v = select.make(torch, shape, "f32", seed=7)
    off = masked(torch, v, "steps")
    v["dt"][off] = float("-inf")
    v["A"][::3, 0] = float("-inf")
    v["A"][2, :] = float("-inf")
    got = scan(env, v)
    v["dt"][off] = -200.0
    v["A"][torch.isinf(v["A"])] = -1e30
    compare(env, got, v, "f32", "infinite rates")


def test_infinite_rates_of_streams(env):
    torch, lif = env
    v = select.make(torch, (5, 1, 66, 17, 2), "f32", seed=8, step=True)
    off = masked(torch, v, "steps")
    v["dt"][off] = float("-inf")
    v["A"][::3, 0], v["A"][2, :] = float("-inf"), float("-inf")
    state, kept = v["h_first"].clone(), v["h_first"]
    y = lif.selective_step(*[v[k] for k in ("x", "dt", "A", "B", "C")], state, D=v["D"], z=v["z"],
                           dt_bias=v["dt_bias"])
    assert torch.equal(state[off], kept[off])
    v["dt"][off] = -200.0
    v["A"][torch.isinf(v["A"])] = -1e30
    ref = {k: select.arr(t)[:, None] if k in ("x", "dt", "B", "C", "z", "grad_y") else select.arr(t)
           for k, t in v.items()}
    want = select.reference(ref, np.full(5, 1))
    check(select.arr(y), want["y"][:, 0], "f32", "y")
    check(select.arr(state), want["h_last"], "f32", "state")


@pytest.mark.parametrize("N", [4, 20])
def test_growing_states(env, N):
    """A > 0 where a shared-out time axis has no state yet: the decay over a
    segment lies past the largest float32, the state is 0.  Inputs come in the
    last 40 steps, gradients in the first 40."""
    torch, lif = env
    nb, T, W = 1, 2048, 6
    v = select.make(torch, (nb, T, W, N, 1), "f32", seed=9)
    p = lif.lif_select_params(nb, T, W, N, 1, 0, 0, 0, *([0] * 12))
    assert lif.lif_selective_scan_workspace_size(p) > 0, "the time axis is not shared out"
    v["A"] = torch.full_like(v["A"], 1.5)
    v["dt"], v["dt_bias"], v["h_first"], v["grad_last"] = torch.ones_like(v["dt"]), None, None, None
    v["x"][:, :-40] = 0.0
    v["grad_y"][:, 40:] = 0.0
    got = scan(env, v, soft=False)
    # the last 48 steps alone give the outputs, the first 48 the gradients
    ref = {k: select.arr(t) for k, t in v.items()}
    part = lambda sl: {k: t[:, sl] if k in ("x", "dt", "B", "C", "z", "grad_y") else t for k, t in ref.items()}  # noqa: E731
    tail, head = (select.reference(part(sl), np.full(nb, 48), False, 48) for sl in (slice(T - 48, T), slice(0, 48)))
    assert np.isfinite(tail["h_last"].e).all() and np.isfinite(head["grad_h_first"].e).all()
    check(select.arr(got["y"][:, -48:]), tail["y"], "f32", "growing y")
    check(select.arr(got["h_last"]), tail["h_last"], "f32", "growing h_last")
    for k in ("x", "B", "C", "dt", "z"):
        check(select.arr(got["grad_" + k][:, :48]), head["grad_" + k], "f32", "growing grad_" + k)
        assert not got["grad_" + k][:, 48:].any(), k
    check(select.arr(got["grad_h_first"]), head["grad_h_first"], "f32", "growing grad_h_first")
    assert not got["y"][:, :-48].any() and not got["grad_A"].any()


def test_long_steps_in_segments(env):
    """Rates of 0 and steps whose sum passes the largest float32: the state
    stays."""
    torch, lif = env
    nb, T, W, N = 1, 2048, 6, 4
    v = select.make(torch, (nb, T, W, N, 1), "f32", seed=10)
    v["A"], v["x"] = torch.zeros_like(v["A"]), torch.zeros_like(v["x"])
    v["dt"] = torch.full_like(v["dt"], 2e38)
    o = lif.selective_scan(*[v[k] for k in ("x", "dt", "A", "B", "C")], h_first=v["h_first"])
    assert torch.equal(o.h_last, v["h_first"]) and torch.isfinite(o.y).all()


def test_most_places(env):
    """As many places as 32 bits count: the last of them lie in pieces whose end
    is the largest whole number.  Counts below 2^24 are exact; the sum of 2^31 - 8
    ones takes at most one rounding a piece and one a sum of two."""
    torch, lif = env
    R = (1 << 31) - 1
    print(f"[case] embed {R} places", flush=True)
    tokens = torch.zeros((1, R), dtype=torch.int32, device="cuda:0")
    tokens[0, :3], tokens[0, -4:] = 1, 1
    grad = torch.ones((1, 1, 1), device="cuda:0").expand(1, R, 1)
    g = lif.embed_backward(tokens, grad, 3)
    assert g[1, 0] == 7 and g[2, 0] == 0
    assert abs(float(g[0, 0]) - (R - 7)) <= (R - 7) * 8192 * 2.0 ** -24
    W = torch.tensor([[2.0], [3.0], [5.0]], device="cuda:0")
    out = lif.embed(tokens, W, dtype=torch.bfloat16)
    assert (out[0, :3] == 3).all() and (out[0, -4:] == 3).all()
    assert all(bool((part == 2).all()) for part in out[0, 3:-4, 0].split(1 << 28))


def test_most_states(env):
    """The gradient of as many states as the checks accept at one step: its sums
    are more than a launch has threads.  Channels from every part are compared."""
    torch, lif = env
    D, N = 1 << 24, 64
    print(f"[case] select {D} x {N}", flush=True)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    rn = lambda *s: torch.randn(*s, device="cuda:0", generator=g)                         # noqa: E731
    v = {"x": rn(1, 1, D), "dt": rn(1, 1, D), "A": -torch.rand(D, N, device="cuda:0", generator=g),
         "B": rn(1, 1, 1, N), "C": rn(1, 1, 1, N), "D": rn(D), "z": None, "dt_bias": rn(D), "h_first": rn(1, D, N),
         "grad_y": rn(1, 1, D), "grad_last": None}
    got = scan(env, v)
    at = torch.cat([torch.arange(i, i + 70) for i in (0, 70000, D // 2 - 35, D - 70)]).to("cuda:0")
    take = lambda t, axis: t.index_select(axis, at)                                       # noqa: E731
    axis = {"x": 2, "dt": 2, "A": 0, "D": 0, "dt_bias": 0, "h_first": 1, "grad_y": 2}
    want = select.reference({k: select.arr(t if k not in axis else take(t, axis[k])) for k, t in v.items()}, np.ones(1))
    for k, i in {"y": 2, "h_last": 1, "grad_x": 2, "grad_dt": 2, "grad_A": 0, "grad_D": 0, "grad_dt_bias": 0,
                 "grad_h_first": 1}.items():
        check(select.arr(take(got[k], i)), want[k], "f32", k)


def test_most_taps(env):
    """The gradient of so many taps that their sums are more than a launch has
    threads; channels from every part are compared."""
    torch, lif = env
    T, D, K = 3, 30_000_001, 8
    print(f"[case] conv {D} x {K}", flush=True)
    g = torch.Generator(device="cuda:0").manual_seed(4)
    rn = lambda *s: torch.randn(*s, device="cuda:0", generator=g)                         # noqa: E731
    v = {"x": rn(1, T, D), "w": rn(D, K) / K ** 0.5, "bias": rn(D), "x_first": None, "grad_y": rn(1, T, D),
         "grad_last": None}
    o = lif.causal_conv(v["x"], v["w"], v["bias"])
    grads = lif.causal_conv_backward(v["x"], v["w"], v["grad_y"], v["bias"])
    got = {"y": o.y, "grad_x": grads.x, "grad_w": grads.w, "grad_bias": grads.bias}
    at = torch.cat([torch.arange(i, i + 70) for i in (0, 70000, D // 2 - 35, D - 70)]).to("cuda:0")
    axis = {"x": 2, "w": 0, "bias": 0, "grad_y": 2, "y": 2, "grad_x": 2, "grad_w": 0, "grad_bias": 0}
    take = lambda k, t: t if t is None else conv.arr(t.index_select(axis[k], at))         # noqa: E731
    want = conv.reference({k: take(k, t) for k, t in v.items()}, np.full(1, T))
    for k, t in got.items():
        check(take(k, t), want[k], "f32", k)


def test_gradients_of_many_steps(env):
    """Equal terms, whose roundings all go one way, over 51200 strips of 64
    steps: a term passes 64 roundings of its strip, 32 and 100 of its wave's
    strips, 16 of the waves and its product's and last one's."""
    torch, lif = env
    nb, T, W, gy, x = 50, 65536, 20, 0.123, 0.456
    one = torch.ones((nb, T, W), device="cuda:0")
    g = lif.causal_conv_backward(x * one, torch.ones((W, 2), device="cuda:0"), gy * one,
                                 torch.zeros(W, device="cuda:0"), silu=False)
    gy, x = float(np.float32(gy)), float(np.float32(x))
    for got, want in ((g.w[:, 1], nb * T * gy * x), (g.w[:, 0], nb * (T - 1) * gy * x), (g.bias, nb * T * gy)):
        assert np.abs(conv.arr(got) / want - 1.0).max() <= (64 + 32 + 100 + 16 + 2) * 2.0 ** -24


@pytest.mark.parametrize("shape", [(1, 3000, 6, 4, 1), (2, 1111, 130, 16, 2), (1, 2005, 40, 33, 1), (3, 2000, 300, 8, 1)])
def test_errors_of_long_sums(env, shape):
    """The bounds of the error analysis add up all roundings; those of a long
    chain have random signs.  3000 steps of four roundings are off by about
    sqrt(12000) 2^-24 = 6.5e-6 relative to the whole: 1e-5."""
    torch, lif = env
    v = select.make(torch, shape, "f32", seed=12)
    got = scan(env, v)
    want = select.reference({k: select.arr(t) for k, t in v.items()}, np.full(shape[0], shape[1]))
    for k, w in want.items():
        err = np.linalg.norm(select.arr(got[k]) - w.v) / np.linalg.norm(w.v)
        print(f"{k} {err:.1e}", flush=True)
        assert err <= 1e-5, k
