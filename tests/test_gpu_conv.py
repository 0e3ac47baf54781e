"""The short causal convolution (lif_causal_conv), its gradient and its single
step against the float64 formulas on identical inputs; tolerances by running
error analysis (tests/rounding.py)."""
import numpy as np
import pytest

from rounding import Num, check, silu

pytestmark = pytest.mark.gpu

TYPES = ("f32", "bf16", "f16")
# (samples, steps, channels, taps)
SHAPES = [(1, 1, 1, 2), (2, 1, 3, 8), (1, 2, 4, 4), (3, 7, 5, 3), (2, 63, 9, 4), (2, 64, 64, 5), (1, 65, 130, 6),
          (2, 200, 33, 7), (3, 129, 20, 8), (1, 1000, 7, 4), (70, 9, 20, 2)]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


def dt_of(torch, dtype):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]


def arr(t):
    return None if t is None else t.detach().double().cpu().numpy()


def make(torch, shape, dtype, seed=0):
    nb, T, W, K = shape
    g = torch.Generator().manual_seed(seed * 1000 + T)
    rn = lambda *s: torch.randn(*s, generator=g)                                          # noqa: E731
    v = {"x": rn(nb, T, W), "w": rn(W, K) / K ** 0.5, "bias": rn(W) * 0.3, "x_first": rn(nb, K - 1, W),
         "grad_y": rn(nb, T, W), "grad_last": rn(nb, K - 1, W)}
    wide = ("w", "bias", "grad_last")
    return {k: t.to("cuda:0", torch.float32 if k in wide else dt_of(torch, dtype)) for k, t in v.items()}


def reference(v, n, act=True):
    """Values with bounds of what forward and backward give."""
    nb, T, W = v["x"].shape
    K = v["w"].shape[1]
    first = np.zeros((nb, K - 1, W)) if v["x_first"] is None else v["x_first"]
    on = (np.arange(T)[None, :] < n[:, None])[:, :, None]
    seen = np.concatenate([first, np.where(on, v["x"], 0.0)], 1)
    taps = Num(np.stack([seen[:, j:j + T] * 1.0 for j in range(K)], -1)) * Num(v["w"])
    c = taps.sum(-1) + Num(np.zeros(W) if v["bias"] is None else v["bias"])
    y, slope = silu(c) if act else (c, Num(np.ones_like(c.v)))
    nothing = Num(np.zeros((nb, T, W)))
    last = np.stack([seen[b, m:m + K - 1] for b, m in enumerate(n)])
    out = {"y": Num.where(on, y, nothing), "x_last": last}
    gy = np.zeros((nb, T, W)) if v["grad_y"] is None else np.where(on, v["grad_y"], 0.0)
    gc = Num.where(on, Num(gy) * slope, nothing)
    val, err, mag = np.zeros_like(seen), np.zeros_like(seen), np.zeros_like(seen)
    for j in range(K):
        p = gc * Num(v["w"][:, j])
        val[:, j:j + T] += p.v
        err[:, j:j + T] += p.e
        mag[:, j:j + T] += np.abs(p.v) + p.e
    if v["grad_last"] is not None:
        for b, m in enumerate(n):
            val[b, m:m + K - 1] += v["grad_last"][b]
            mag[b, m:m + K - 1] += np.abs(v["grad_last"][b])
    gs = Num(val, err + (K + 1) * 2.0 ** -24 * mag)
    out["grad_x"], out["grad_x_first"] = Num.where(on, gs[:, K - 1:], nothing), gs[:, :K - 1]
    shifted = Num(np.stack([seen[:, j:j + T] for j in range(K)], -1))
    out["grad_w"] = (gc[..., None] * shifted).sum((0, 1))
    out["grad_bias"] = gc.sum((0, 1))
    return out


def steps_of(length, nb, T):
    return np.full(nb, T) if length is None else np.clip(np.asarray(length), 0, T)


def run(env, v, dtype, length=None, act=True, label=""):
    torch, lif = env
    nb, T, W = v["x"].shape
    print(f"[case] conv {label} {tuple(v['x'].shape)} K={v['w'].shape[1]} {dtype} strides={v['x'].stride()}",
          flush=True)
    n = None if length is None else torch.tensor(length, dtype=torch.int32, device="cuda:0")
    kw = dict(bias=v["bias"], length=n, x_first=v["x_first"], silu=act)
    o = lif.causal_conv(v["x"], v["w"], **kw)
    g = lif.causal_conv_backward(v["x"], v["w"], v["grad_y"], grad_last=v["grad_last"], **kw)
    torch.cuda.synchronize()
    want = reference({k: arr(t) for k, t in v.items()}, steps_of(length, nb, T), act)
    assert np.array_equal(arr(o.x_last), want.pop("x_last")), f"{label} x_last"
    got = {"y": o.y, "grad_x": g.x, "grad_w": g.w, "grad_bias": g.bias, "grad_x_first": g.x_first}
    for k, w in want.items():
        if got[k] is not None:
            check(arr(got[k]), w, dtype if k in ("y", "grad_x") else "f32", f"{label} {k}")
    return {**got, "x_last": o.x_last}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(env, shape, dtype):
    run(env, make(env[0], shape, dtype), dtype, act=shape[1] % 2 == 1, label="shapes")


@pytest.mark.parametrize("length", [[0, 0, 0], [1, 2, 3], [70, -3, 99], [64, 66, 63]])
def test_lengths(env, length):
    """What lies past a sample's length has no effect, whatever it holds."""
    v = make(env[0], (3, 70, 37, 4), "bf16")
    for b, n in enumerate(steps_of(length, 3, 70)):
        for k in ("x", "grad_y"):
            v[k][b, n:] = float("nan") if b != 1 else float("inf")
    run(env, v, "bf16", length, label="lengths")


@pytest.mark.parametrize("missing", ["bias", "x_first", "grad_last", "grad_y"])
def test_without_an_input(env, missing):
    v = make(env[0], (2, 40, 33, 4), "f32")
    v[missing] = None
    got = run(env, v, "f32", label="without " + missing)
    assert (got["grad_bias"] is None) == (missing == "bias")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views(env, dtype):
    torch, _ = env
    v = make(torch, (3, 37, 41, 4), dtype, seed=3)
    wide = torch.zeros((3, 37, 2 * 41 + 1), dtype=v["x"].dtype, device="cuda:0")
    wide[:, :, 1:42] = v["x"]
    v["x"] = wide[:, :, 1:42]
    v["grad_y"] = v["grad_y"].transpose(0, 1).contiguous().transpose(0, 1)
    run(env, v, dtype, label="slices")
    v["x"], v["grad_y"] = v["x"][:1].expand(3, -1, -1), v["grad_y"][:, :1].expand(-1, 37, -1)
    run(env, v, dtype, [37, 20, 5], label="repeated")


def test_pieces(env):
    """Two pieces, the last inputs and their gradient handed on, give the same
    bits as the whole; pieces shorter than the taps too."""
    torch, lif = env
    v = make(torch, (2, 50, 20, 5), "bf16", seed=4)
    whole = run(env, v, "bf16", label="whole")
    for cut in (20, 1, 2, 49):
        x, gy = v["x"], v["grad_y"]
        a = lif.causal_conv(x[:, :cut], v["w"], v["bias"], x_first=v["x_first"])
        b = lif.causal_conv(x[:, cut:], v["w"], v["bias"], x_first=a.x_last)
        gb = lif.causal_conv_backward(x[:, cut:], v["w"], gy[:, cut:], v["bias"], x_first=a.x_last,
                                      grad_last=v["grad_last"])
        ga = lif.causal_conv_backward(x[:, :cut], v["w"], gy[:, :cut], v["bias"], x_first=v["x_first"],
                                      grad_last=gb.x_first)
        assert torch.equal(torch.cat([a.y, b.y], 1), whole["y"]) and torch.equal(b.x_last, whole["x_last"])
        want = reference({k: arr(t) for k, t in v.items()}, np.full(2, 50))
        check(arr(torch.cat([ga.x, gb.x], 1)), want["grad_x"], "bf16", "pieces grad_x")
        check(arr(ga.x_first), want["grad_x_first"], "f32", "pieces grad_x_first")


def test_nan_stays_in_its_channel(env):
    torch, lif = env
    v = make(torch, (2, 40, 10, 4), "f32")
    clean = lif.causal_conv(v["x"], v["w"]).y
    v["x"][0, 20, 3] = float("nan")
    y = lif.causal_conv(v["x"], v["w"]).y
    same = torch.ones_like(y, dtype=torch.bool)
    same[0, 20:24, 3] = False
    assert torch.equal(y[same], clean[same]) and torch.isnan(y[0, 20:24, 3]).all()


def test_empty(env):
    torch, lif = env
    v = make(torch, (2, 3, 5, 4), "f32")
    o = lif.causal_conv(v["x"][:, :0], v["w"], x_first=v["x_first"])
    g = lif.causal_conv_backward(v["x"][:, :0], v["w"], v["grad_y"][:, :0], v["bias"], x_first=v["x_first"],
                                 grad_last=v["grad_last"])
    assert torch.equal(o.x_last, v["x_first"]) and torch.equal(g.x_first, v["grad_last"])
    assert not g.w.any() and not g.bias.any()
    g = lif.causal_conv_backward(v["x"][:0], v["w"], v["grad_y"][:0], v["bias"])
    assert not g.w.any() and not g.bias.any() and lif.causal_conv(v["x"][:0], v["w"]).y.numel() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1, 2), (3, 1, 5, 3), (4, 1, 64, 4), (300, 1, 33, 8)])
def test_step(env, shape, dtype):
    torch, lif = env
    nb, _, W, K = shape
    v = make(torch, shape, dtype)
    slots = nb + 3
    g = torch.Generator().manual_seed(1)
    state = torch.randn((slots, K - 1, W), generator=g).to("cuda:0", dt_of(torch, dtype))
    slot = torch.randperm(slots, generator=g)[:nb].to("cuda:0", torch.int32)
    rows = list(range(nb))
    if nb > 2:
        slot[1], slot[2] = -1, slots
        rows = [0] + rows[3:]
    kept, at = state.clone(), slot.long()[rows]
    y = lif.causal_conv_step(v["x"][:, 0], v["w"], state, slot=slot, bias=v["bias"])
    ref = {k: arr(t)[rows] if k in ("x", "grad_y", "grad_last") else arr(t) for k, t in v.items()}
    ref["x_first"] = arr(kept[at])
    want = reference(ref, np.full(len(rows), 1))
    check(arr(y)[rows], want["y"][:, 0], dtype, "step y")
    assert np.array_equal(arr(state[at]), want["x_last"])
    others = torch.ones(slots, dtype=torch.bool, device="cuda:0")
    others[at] = False
    assert torch.equal(state[others], kept[others])
    if nb > 2:
        assert not y[1].any() and not y[2].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_steps_follow_the_sequence(env, dtype):
    """A stream run step by step gives the sequence's bits."""
    torch, lif = env
    v = make(torch, (3, 20, 33, 4), dtype, seed=7)
    state = v["x_first"].clone()
    ys = [lif.causal_conv_step(v["x"][:, t], v["w"], state, bias=v["bias"]) for t in range(20)]
    o = lif.causal_conv(v["x"], v["w"], v["bias"], x_first=v["x_first"])
    assert torch.equal(torch.stack(ys, 1), o.y) and torch.equal(state, o.x_last)


def test_same_bits_and_graphs(env):
    torch, lif = env
    v = make(torch, (3, 300, 65, 4), "bf16", seed=9)
    length = torch.full((3,), 300, dtype=torch.int32, device="cuda:0")

    def both(**more):
        kw = dict(bias=v["bias"], length=length, x_first=v["x_first"], **more)
        o = lif.causal_conv(v["x"], v["w"], **kw)
        g = lif.causal_conv_backward(v["x"], v["w"], v["grad_y"], grad_last=v["grad_last"], **kw)
        return [o.y, o.x_last, g.x, g.w, g.bias, g.x_first]
    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        v["x"].copy_(torch.randn_like(v["x"]))
        length.fill_(300 - 7 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, both())), i
