"""The selective state space scan (lif_selective_scan), its gradient and its
single step against the float64 formulas on identical inputs; tolerances by
running error analysis (tests/rounding.py).  Where a call shares out the time
axis, the decay over a segment is e^{A sum of delta}, whose sum has as many
roundings as the segment has steps: a relative error of delta of that many U."""
import numpy as np
import pytest

from rounding import U, Num, check, exp_of, silu, softplus

pytestmark = pytest.mark.gpu

TYPES = ("f32", "bf16", "f16")
# (samples, steps, channels, states, groups)
SHAPES = [(1, 1, 1, 1, 1), (2, 1, 5, 3, 1), (1, 2, 64, 4, 1), (3, 15, 7, 5, 1), (2, 16, 65, 8, 1), (2, 17, 130, 16, 2),
          (1, 33, 63, 17, 3), (2, 48, 40, 32, 2), (1, 50, 20, 33, 1), (2, 35, 66, 64, 3), (1, 700, 24, 16, 1),
          (40, 20, 20, 16, 1), (1, 3000, 6, 4, 1), (2, 1111, 130, 16, 2), (1, 2005, 40, 33, 1)]


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


def make(torch, shape, dtype, seed=0, step=False):
    """Inputs of a call; time constants of 1 to 1000 steps."""
    nb, T, W, N, G = shape
    g = torch.Generator().manual_seed(seed * 1000 + T)
    lead = (nb,) if step else (nb, T)
    rn = lambda *s: torch.randn(*s, generator=g)                                          # noqa: E731
    delta = torch.exp(torch.rand(W, generator=g) * np.log(100.0) + np.log(0.001))
    v = {"x": rn(*lead, W), "dt": 0.5 * rn(*lead, W), "A": -torch.arange(1, N + 1) * torch.exp(0.1 * rn(W, N)),
         "B": rn(*lead, G, N), "C": rn(*lead, G, N) / N ** 0.5, "D": rn(W), "z": rn(*lead, W),
         "dt_bias": torch.log(torch.expm1(delta)), "h_first": rn(nb, W, N), "grad_y": rn(*lead, W),
         "grad_last": rn(nb, W, N)}
    wide = ("A", "D", "dt_bias", "h_first", "grad_last")
    return {k: t.to("cuda:0", torch.float32 if k in wide else dt_of(torch, dtype)) for k, t in v.items()}


def steps_of(length, nb, T):
    return np.full(nb, T) if length is None else np.clip(np.asarray(length), 0, T)


def reference(v, n, soft=True, segment=0):
    """Values with bounds of everything that forward and backward give, for
    inputs v (arrays; z, D, dt_bias, h_first, grad_last may be None)."""
    nb, T, W = v["x"].shape
    G, N = v["B"].shape[2:]
    of = np.arange(W) // (W // G)
    zero = lambda *s: np.zeros(s)                                                         # noqa: E731
    on = (np.arange(T)[None, :] < n[:, None])[:, :, None]
    clean = lambda a: np.where(on if a.ndim == 3 else on[..., None], a, 0.0)              # noqa: E731
    x, raw, B, C, gy = (clean(v[k]) for k in ("x", "dt", "B", "C", "grad_y"))
    r = Num(raw) + Num(zero(W) if v["dt_bias"] is None else v["dt_bias"])
    delta, slope = softplus(r) if soft else (r, Num(np.ones_like(raw)))
    D = zero(W) if v["D"] is None else v["D"]
    A = v["A"]
    u = delta * Num(x)
    Bf, Cf = B[:, :, of], C[:, :, of]                                   # [nb, T, W, N]
    a = exp_of(delta[..., None], A, segment * U)
    into = u[..., None] * Num(Bf)
    h = Num(zero(nb, W, N) if v["h_first"] is None else v["h_first"])
    before, hs = [], []
    for t in range(T):
        before.append(h)
        h = Num.where(on[:, t][..., None], a[:, t] * h + into[:, t], h)
        hs.append(h)
    stack = lambda l: Num(np.stack([i.v for i in l], 1), np.stack([i.e for i in l], 1))   # noqa: E731
    last, before, hs = h, stack(before), stack(hs)
    y0 = (Num(Cf) * hs).sum(-1, slack=2) + Num(D) * Num(x)
    if v["z"] is None:
        gate, gslope = Num(np.ones_like(x)), None
    else:
        gate, gslope = silu(Num(clean(v["z"])))
    out = {"y": Num.where(on, y0 * gate, Num(zero(nb, T, W))), "h_last": last}
    g = Num(gy) * gate
    mu = Num(zero(nb, W, N) if v["grad_last"] is None else v["grad_last"])
    lam = [None] * T
    out_of = g[..., None] * Num(Cf)
    for t in reversed(range(T)):
        lam[t] = mu + out_of[:, t]
        mu = Num.where(on[:, t][..., None], a[:, t] * lam[t], mu)
    out["grad_h_first"] = mu
    nothing = Num(zero(nb, T, W))
    lam = Num.where(on[..., None], stack(lam), Num(zero(nb, T, W, N)))
    q = lam * a * before
    group = lambda p: Num(p.v.reshape(nb, T, G, W // G, N), p.e.reshape(nb, T, G, W // G, N)).sum(3)   # noqa: E731
    out["grad_B"] = group(Num.where(on[..., None], lam * u[..., None], Num(zero(nb, T, W, N))))
    out["grad_C"] = group(Num.where(on[..., None], g[..., None] * hs, Num(zero(nb, T, W, N))))
    Q = (lam * Num(Bf)).sum(-1)
    P = (Num(A) * q).sum(-1)
    gdt = Num.where(on, (P + Num(x) * Q) * slope, nothing)
    out["grad_dt"] = gdt
    out["grad_dt_bias"] = gdt.sum((0, 1))
    out["grad_x"] = Num.where(on, delta * Q + Num(D) * g, nothing)
    out["grad_D"] = Num.where(on, g * Num(x), nothing).sum((0, 1))
    out["grad_A"] = Num.where(on[..., None], delta[..., None] * q, Num(zero(nb, T, W, N))).sum((0, 1))
    if gslope is not None:
        out["grad_z"] = Num.where(on, Num(gy) * y0 * gslope, nothing)
    return out


FLOAT32 = ("h_last", "grad_A", "grad_D", "grad_dt_bias", "grad_h_first")


def segment_of(lif, v, length=None):
    """Steps of a segment, 0 where the time axis is not shared out: all steps
    are an upper bound."""
    nb, T, W = v["x"].shape
    G = v["B"].shape[2] if v["B"].dim() == 4 else 1
    return T if lif._select_ws(nb, T, W, v["A"].shape[1], G, lif._dtype_code("x", v["x"]), False) else 0


def run(env, v, dtype, length=None, soft=True, label=""):
    torch, lif = env
    nb, T, W = v["x"].shape
    print(f"[case] select {label} {tuple(v['x'].shape)} N={v['A'].shape[1]} B={tuple(v['B'].shape)} {dtype}",
          flush=True)
    n = None if length is None else torch.tensor(length, dtype=torch.int32, device="cuda:0")
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], dt_bias=v["dt_bias"], length=n, softplus=soft)
    o = lif.selective_scan(*args, h_first=v["h_first"], marks=True, **kw)
    g = lif.selective_scan_backward(*args, o.marks, v["grad_y"], grad_last=v["grad_last"], **kw)
    torch.cuda.synchronize()
    got = {"y": o.y, "h_last": o.h_last, **{"grad_" + k: getattr(g, k) for k in
                                            ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h_first")}}
    ref = {k: arr(t) for k, t in v.items()}
    for k in ("B", "C"):
        ref[k] = ref[k].reshape(nb, T, -1, ref[k].shape[-1])
    if ref["grad_y"] is None:
        ref["grad_y"] = np.zeros((nb, T, W))
    want = reference(ref, steps_of(length, nb, T), soft, segment_of(lif, v))
    for k, w in want.items():
        if got[k] is not None:
            check(arr(got[k]).reshape(w.v.shape), w, "f32" if k in FLOAT32 else dtype, f"{label} {k}")
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(env, shape, dtype):
    v = make(env[0], shape, dtype)
    if dtype == "f16" and shape[4] == 1:                      # one group without its axis
        v["B"], v["C"] = v["B"][:, :, 0], v["C"][:, :, 0]
    run(env, v, dtype, label="shapes")


@pytest.mark.parametrize("length", [[0, 0, 0], [1, 16, 37], [17, -3, 99], [32, 33, 31]])
def test_lengths(env, length):
    """What lies past a sample's length has no effect, whatever it holds."""
    torch, _ = env
    v = make(torch, (3, 37, 70, 6, 2), "bf16")
    for b, n in enumerate(steps_of(length, 3, 37)):
        for k in ("x", "dt", "B", "C", "z", "grad_y"):
            v[k][b, n:] = float("nan") if b != 1 else float("inf")
    run(env, v, "bf16", length, label="lengths")


@pytest.mark.parametrize("missing", ["D", "z", "dt_bias", "h_first", "grad_last", "grad_y", "all"])
def test_without_an_input(env, missing):
    v = make(env[0], (2, 40, 33, 9, 1), "f32")
    for k in ("D", "z", "dt_bias", "h_first", "grad_last") if missing == "all" else (missing,):
        v[k] = None
    got = run(env, v, "f32", label="without " + missing)
    assert (got["grad_D"] is None) == (v["D"] is None) and (got["grad_z"] is None) == (v["z"] is None)


def test_without_softplus(env):
    v = make(env[0], (2, 40, 33, 9, 1), "f32")
    v["dt"], v["dt_bias"] = v["dt"].abs() * 0.1, v["dt_bias"].abs() * 0.01
    run(env, v, "f32", [40, 21], soft=False, label="no softplus")


def test_extreme_values(env):
    """Steps near 0 and very long ones, gates far out, rates of 0, slow growth
    and states that decay at once."""
    torch, _ = env
    v = make(torch, (2, 40, 16, 8, 1), "f32")
    v["dt"][:, ::3] = -60.0
    v["dt"][:, 1::5] = 40.0
    v["z"][:, ::4] = 80.0
    v["z"][:, 1::4] = -80.0
    v["A"][:4] = 0.0
    v["A"][4:6] = 0.001
    v["A"][6:8] = -1e4
    run(env, v, "f32", label="extreme")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views(env, dtype):
    """Inputs that are slices of one projection, at odd offsets, or one row for
    all samples or steps."""
    torch, _ = env
    nb, T, W, N = 2, 37, 67, 5
    v = make(torch, (nb, T, W, N, 1), dtype, seed=3)
    wide = torch.zeros((nb, T, 3 * W + 2 * N + 1), dtype=v["x"].dtype, device="cuda:0")
    at = 1
    for k in ("x", "dt", "z"):
        wide[:, :, at:at + W] = v[k]
        v[k] = wide[:, :, at:at + W]
        at += W
    for k in ("B", "C"):
        wide[:, :, at:at + N] = v[k][:, :, 0]
        v[k] = wide[:, :, at:at + N]
        at += N
    run(env, v, dtype, label="slices")
    for k in ("x", "dt", "z", "grad_y"):
        v[k] = v[k].transpose(0, 1).contiguous().transpose(0, 1)       # time before samples
    v["B"] = v["B"][:1].expand(nb, -1, -1)
    v["C"] = v["C"][:, :1].expand(-1, T, -1)
    run(env, v, dtype, [37, 20], label="repeated")
    v["x"] = v["x"].transpose(1, 2).contiguous().transpose(1, 2)       # channels apart: copied
    run(env, v, dtype, label="channels apart")


def test_pieces(env):
    """A sequence in two pieces, the state and its gradient handed on, gives
    what the whole gives; a boundary at a mark gives the same bits."""
    torch, lif = env
    nb, T, W, N = 2, 64, 40, 7
    v = make(torch, (nb, T, W, N, 1), "f32", seed=4)
    seq = ("x", "dt", "B", "C", "z", "grad_y")
    whole = run(env, v, "f32", label="whole")
    for cut in (32, 21):
        a = {k: (t[:, :cut] if k in seq else t) for k, t in v.items()}
        b = {k: (t[:, cut:] if k in seq else t) for k, t in v.items()}
        args = lambda p: [p[k] for k in ("x", "dt", "A", "B", "C")]                       # noqa: E731
        kw = lambda p: dict(D=p["D"], z=p["z"], dt_bias=p["dt_bias"])                     # noqa: E731
        oa = lif.selective_scan(*args(a), h_first=v["h_first"], marks=True, **kw(a))
        ob = lif.selective_scan(*args(b), h_first=oa.h_last, marks=True, **kw(b))
        gb = lif.selective_scan_backward(*args(b), ob.marks, b["grad_y"], grad_last=v["grad_last"], **kw(b))
        ga = lif.selective_scan_backward(*args(a), oa.marks, a["grad_y"], grad_last=gb.h_first, **kw(a))
        if cut % 16 == 0:
            assert torch.equal(torch.cat([oa.y, ob.y], 1), whole["y"]) and torch.equal(ob.h_last, whole["h_last"])
            assert torch.equal(torch.cat([ga.x, gb.x], 1), whole["grad_x"])
            assert torch.equal(torch.cat([ga.B, gb.B], 1), whole["grad_B"])
            assert torch.equal(ga.h_first, whole["grad_h_first"])
        v2 = {k: arr(t) for k, t in v.items()}
        want = reference(v2, np.full(nb, T))
        check(arr(torch.cat([oa.y, ob.y], 1)), want["y"], "f32", "pieces y")
        check(arr(torch.cat([ga.dt, gb.dt], 1)), want["grad_dt"], "f32", "pieces grad_dt")
        check(arr(ga.h_first), want["grad_h_first"], "f32", "pieces grad_h_first")
        check(arr(ga.A + gb.A), want["grad_A"], "f32", "pieces grad_A")


def test_nan_stays_in_its_channel(env):
    torch, lif = env
    v = make(torch, (2, 40, 70, 6, 1), "f32")
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], dt_bias=v["dt_bias"], h_first=v["h_first"])
    clean = lif.selective_scan(*args, **kw)
    v["x"][0, 20, 3] = float("nan")
    o = lif.selective_scan(*args, **kw)
    same = torch.ones((2, 40, 70), dtype=torch.bool, device="cuda:0")
    same[0, 20:, 3] = False
    assert torch.equal(o.y[same], clean.y[same]) and torch.isnan(o.y[0, 20:, 3]).all()


def test_no_outputs(env):
    torch, lif = env
    v = make(torch, (2, 40, 33, 9, 1), "bf16")
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    full = lif.selective_scan(*args, z=v["z"], h_first=v["h_first"])
    o = lif.selective_scan(*args, z=v["z"], h_first=v["h_first"], outputs=False)
    assert o.y is None and torch.equal(o.h_last, full.h_last)


def test_empty(env):
    torch, lif = env
    v = make(torch, (2, 3, 5, 4, 1), "f32")
    for sl in ((slice(0, 0), slice(None)), (slice(None), slice(0, 0))):
        p = {k: (t[sl] if k in ("x", "dt", "B", "C", "z", "grad_y") else t) for k, t in v.items()}
        h0, gl = v["h_first"][sl[0]], v["grad_last"][sl[0]]
        args = [p[k] for k in ("x", "dt", "A", "B", "C")]
        o = lif.selective_scan(*args, D=v["D"], z=p["z"], h_first=h0, marks=True)
        g = lif.selective_scan_backward(*args, o.marks, p["grad_y"], D=v["D"], z=p["z"], grad_last=gl)
        assert torch.equal(o.h_last, h0) and torch.equal(g.h_first, gl)
        assert not g.A.any() and not g.D.any() and g.x.numel() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1), (3, 1, 5, 3, 1), (2, 1, 66, 16, 2), (7, 1, 33, 64, 3),
                                   (5, 1, 130, 17, 1), (300, 1, 40, 4, 1)])
def test_step(env, shape, dtype):
    torch, lif = env
    nb, _, W, N, G = shape
    v = make(torch, shape, dtype, step=True)
    slots = nb + 3
    state = torch.randn((slots, W, N), generator=torch.Generator().manual_seed(1)).to("cuda:0")
    slot = torch.randperm(slots, generator=torch.Generator().manual_seed(2))[:nb].to("cuda:0", torch.int32)
    left_out = nb > 2
    if left_out:
        slot[1], slot[2] = -1, slots
    kept = state.clone()
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], dt_bias=v["dt_bias"])
    y = lif.selective_step(*args, state, slot=slot, **kw)
    rows = [i for i in range(nb) if not (left_out and i in (1, 2))]
    at = slot.long()[rows]
    ref = {k: arr(t)[:, None] if k in ("x", "dt", "B", "C", "z", "grad_y") else arr(t) for k, t in v.items()}
    for k in ("x", "dt", "B", "C", "z", "grad_y", "grad_last"):
        ref[k] = ref[k][rows]
    ref["h_first"] = arr(kept[at])
    want = reference(ref, np.full(len(rows), 1))
    check(arr(y)[rows], want["y"][:, 0], dtype, "step y")
    check(arr(state[at]), want["h_last"], "f32", "step state")
    others = torch.ones(slots, dtype=torch.bool, device="cuda:0")
    others[at] = False
    assert torch.equal(state[others], kept[others])
    if left_out:
        assert not y[1].any() and not y[2].any()
    # without slots: the first rows
    first = kept.clone()
    y2 = lif.selective_step(*args, first, **kw)
    ref = {**{k: arr(t)[:, None] if k in ("x", "dt", "B", "C", "z", "grad_y") else arr(t) for k, t in v.items()},
           "h_first": arr(kept[:nb])}
    check(arr(y2), reference(ref, np.full(nb, 1))["y"][:, 0], dtype, "step y without slots")
    assert torch.equal(first[nb:], kept[nb:])


def test_steps_follow_the_scan(env):
    """A stream run step by step gives what the scan gives."""
    torch, lif = env
    nb, T, W, N = 3, 20, 33, 6
    v = make(torch, (nb, T, W, N, 1), "f32", seed=7)
    state = v["h_first"].clone()
    kw = dict(D=v["D"], dt_bias=v["dt_bias"])
    ys = [lif.selective_step(*[v[k][:, t] if k != "A" else v[k] for k in ("x", "dt", "A", "B", "C")], state,
                             z=v["z"][:, t], **kw) for t in range(T)]
    want = reference({k: arr(t) for k, t in v.items()}, np.full(nb, T))
    check(arr(torch.stack(ys, 1)), want["y"], "f32", "steps y")
    check(arr(state), want["h_last"], "f32", "steps state")


@pytest.mark.parametrize("shape", [(2, 300, 100, 16, 1), (1, 2500, 64, 16, 1)])
def test_same_bits_and_graphs(env, shape):
    """Calls repeat bit for bit, on another stream too; captured calls give
    what eager ones give on every replay, with eager work in between."""
    torch, lif = env
    v = make(torch, shape, "bf16", seed=9)
    length = torch.full((shape[0],), shape[1], dtype=torch.int32, device="cuda:0")
    args = [v[k] for k in ("x", "dt", "A", "B", "C")]
    kw = dict(D=v["D"], z=v["z"], dt_bias=v["dt_bias"], length=length)
    keys = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h_first")

    def both(**more):
        o = lif.selective_scan(*args, h_first=v["h_first"], marks=True, **kw, **more)
        g = lif.selective_scan_backward(*args, o.marks, v["grad_y"], grad_last=v["grad_last"], **kw, **more)
        return [o.y, o.h_last] + [getattr(g, k) for k in keys]
    first = [t.clone() for t in both()]
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
        length.fill_(shape[1] - 7 * i)
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i
