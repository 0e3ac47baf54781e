"""The operators over tokens where calls go wrong: arrays past 2^31 elements,
more streams than a grid has rows, samples that end inside a shared-out time
axis, calls on two streams at once, workspaces that come from the caller."""
import numpy as np
import pytest

from rounding import check
from test_gpu_select import arr, make, reference, run, steps_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


def test_lookup_past_32_bits(env):
    torch, lif = env
    R, D, V = (1 << 21) + 70, 1030, 3                         # 2^31 elements and more
    tokens = torch.zeros((1, R), dtype=torch.int32, device="cuda:0")
    tokens[0, -5:] = torch.tensor([1, 2, -1, 1, 0], dtype=torch.int32, device="cuda:0")
    W = torch.randn((V, D), device="cuda:0", dtype=torch.bfloat16)
    out = lif.embed(tokens, W)
    assert torch.equal(out[0, -5], W[1]) and torch.equal(out[0, -4], W[2]) and not out[0, -3].any()
    assert torch.equal(out[0, -2], W[1]) and torch.equal(out[0, -1], W[0]) and torch.equal(out[0, 12345], W[0])
    out.fill_(1.0)
    out[0, -5:] = 2.0
    g = lif.embed_backward(tokens, out, V)
    # whole numbers below 2^24: exact
    assert (g[0] == R - 5 + 2).all() and (g[1] == 4).all() and (g[2] == 2).all()


def test_sequences_past_32_bits(env):
    """The last steps of a long sequence, whole or as a piece of their own."""
    torch, lif = env
    T, D, cut = (1 << 21) + 77, 1030, 1 << 21
    x = torch.randn((1, T, D), device="cuda:0", dtype=torch.bfloat16)
    w = torch.randn((D, 4), device="cuda:0")
    y = lif.causal_conv(x, w).y
    tail = lif.causal_conv(x[:, cut:], w, x_first=x[:, cut - 3:cut].contiguous())
    assert torch.equal(y[:, cut:], tail.y)
    g = lif.causal_conv_backward(x, w, y)
    gt = lif.causal_conv_backward(x[:, cut:], w, y[:, cut:], x_first=x[:, cut - 3:cut].contiguous())
    assert torch.equal(g.x[:, cut:], gt.x)
    del y, g, gt, tail
    A = -torch.rand((D, 1), device="cuda:0") - 0.5
    B, C = (torch.randn((1, T, 1), device="cuda:0", dtype=torch.bfloat16) for _ in range(2))
    o = lif.selective_scan(x, x, A, B, C, marks=True)
    h = lif.selective_scan(x[:, :cut], x[:, :cut], A, B[:, :cut], C[:, :cut], outputs=False).h_last
    args = (x[:, cut:], x[:, cut:], A, B[:, cut:], C[:, cut:])
    t = lif.selective_scan(*args, h_first=h, marks=True)
    # float32 states that are put together in another order, each result rounded
    # to bf16: half a step of the largest on either side
    scale = t.y.float().abs().max()
    assert (o.y[:, cut:].float() - t.y.float()).abs().max() <= scale * 2.0 ** -7
    g = lif.selective_scan_backward(x, x, A, B, C, o.marks, x)
    gt = lif.selective_scan_backward(*args, t.marks, x[:, cut:])
    scale = gt.x.float().abs().max()
    assert (g.x[:, cut:].float() - gt.x.float()).abs().max() <= scale * 2.0 ** -7
    scale = gt.B.float().abs().max()
    assert (g.B[:, cut:].float() - gt.B.float()).abs().max() <= scale * 2.0 ** -7


@pytest.mark.parametrize("shape,length", [((3, 1200, 40, 16, 1), [1200, 700, 0]), ((2, 1500, 24, 5, 2), [1, 961]),
                                          ((1, 2000, 70, 33, 1), [1999]), ((2, 1200, 40, 24, 1), [1200, 333]),
                                          ((1, 1500, 66, 64, 2), [1490])])
def test_lengths_in_segments(env, shape, length):
    """Samples that end inside a segment of a time axis that is shared out,
    before the others, or have no step at all."""
    torch, lif = env
    v = make(torch, shape, "f32", seed=11)
    p = lif.lif_select_params(*shape, 0, 0, 0, *([0] * 12))
    assert lif.lif_selective_scan_workspace_size(p) > 0, "the time axis is not shared out"
    for b, n in enumerate(steps_of(length, shape[0], shape[1])):
        for k in ("x", "dt", "B", "C", "z", "grad_y"):
            v[k][b, n:] = float("nan")
    run(env, v, "f32", length, label="segments")


def test_many_streams(env):
    """More streams than a grid has rows, and more than one to a workgroup."""
    torch, lif = env
    nb, D, N = 70001, 3, 5
    v = make(torch, (nb, 1, D, N, 1), "f32", step=True)
    state = v["h_first"].clone()
    y = lif.selective_step(*[v[k] for k in ("x", "dt", "A", "B", "C")], state, D=v["D"], z=v["z"], dt_bias=v["dt_bias"])
    ref = {k: arr(t)[:, None] if k in ("x", "dt", "B", "C", "z", "grad_y") else arr(t) for k, t in v.items()}
    want = reference(ref, np.full(nb, 1))
    check(arr(y), want["y"][:, 0], "f32", "y")
    check(arr(state), want["h_last"], "f32", "state")
    conv = torch.randn((nb, 2, D), device="cuda:0")
    w, kept = torch.randn((D, 3), device="cuda:0"), conv.clone()
    y = lif.causal_conv_step(v["x"], w, conv, silu=False)
    whole = lif.causal_conv(v["x"][:, None], w, x_first=kept, silu=False)
    assert torch.equal(y, whole.y[:, 0]) and torch.equal(conv, whole.x_last)


def test_more_samples_than_are_ordered(env):
    """600 samples of different lengths (up to 512 are put in order)."""
    torch, lif = env
    length = np.random.default_rng(3).integers(0, 20, 600)
    run(env, make(torch, (600, 19, 5, 3, 1), "bf16", seed=5), "bf16", list(length), label="600 samples")
    run(env, make(torch, (512, 19, 5, 3, 1), "bf16", seed=6), "bf16", list(length[:512]), label="512 samples")


def test_two_streams_at_once(env):
    """Calls on two streams at the same time do not touch each other."""
    torch, lif = env
    cases = []
    for i in range(2):
        v = make(torch, (2, 600, 64, 16, 1), "bf16", seed=20 + i)
        tokens = torch.randint(0, 50, (2, 600), dtype=torch.int32, device="cuda:0")
        cases.append((v, tokens, torch.cuda.Stream()))

    def all_of(v, tokens, stream):
        a = [v[k] for k in ("x", "dt", "A", "B", "C")]
        o = lif.selective_scan(*a, z=v["z"], h_first=v["h_first"], marks=True, stream=stream)
        g = lif.selective_scan_backward(*a, o.marks, v["grad_y"], z=v["z"], stream=stream)
        e = lif.embed_backward(tokens, v["x"], 50, stream=stream)
        w = v["A"][:, :4].contiguous()
        c = lif.causal_conv_backward(v["x"], w, v["grad_y"], stream=stream)
        return [o.y, o.h_last, g.x, g.dt, g.A, g.B, g.C, g.z, e, c.x, c.w]
    want = [all_of(v, t, None) for v, t, _ in cases]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(3):
        for i, (v, t, s) in enumerate(cases):
            got[i] = all_of(v, t, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(got[i], want[i]))


def test_given_workspaces(env):
    """A workspace that held something else gives the same; too small a one is
    replaced; the bytes behind it stay."""
    torch, lif = env
    v = make(torch, (1, 1200, 40, 16, 1), "f32", seed=8)
    a = [v[k] for k in ("x", "dt", "A", "B", "C")]
    tokens = torch.randint(0, 300, (1, 6000), dtype=torch.int32, device="cuda:0")
    grad = torch.randn((1, 6000, 20), device="cuda:0")
    w = torch.randn((40, 4), device="cuda:0")
    f = lambda ws: lif.selective_scan(*a, marks=True, ws=ws)                              # noqa: E731
    o = f(None)
    calls = [(lambda ws: f(ws).y, lif._select_ws(1, 1200, 40, 16, 1, 0, False)),
             (lambda ws: lif.selective_scan_backward(*a, o.marks, v["grad_y"], ws=ws).A,
              lif._select_ws(1, 1200, 40, 16, 1, 0, True)),
             (lambda ws: lif.embed_backward(tokens, grad, 300, ws=ws), lif._embed_ws(1, 6000, 300, 20)),
             (lambda ws: lif.causal_conv_backward(v["x"], w, v["grad_y"], ws=ws).w, lif._conv_ws(1, 1200, 40, 4, 0))]
    for call, need in calls:
        want = call(None)
        for fill in (0xff, 0x00, 0x3f):
            ws = torch.full((need + 4096,), fill, dtype=torch.uint8, device="cuda:0")
            assert torch.equal(call(ws[:need]), want)
            assert (ws[need:] == fill).all(), "bytes behind the workspace"
        assert torch.equal(call(torch.empty(16, dtype=torch.uint8, device="cuda:0")), want)


def test_outputs_are_written_whole(env):
    """Outputs in memory that held NaN have none left."""
    torch, lif = env
    for shape in ((2, 37, 67, 5, 1), (3, 100, 70, 16, 2)):
        v = make(torch, shape, "bf16", seed=9)
        junk = [torch.full((1 << 20,), float("nan"), device="cuda:0") for _ in range(8)]
        del junk
        got = run(env, v, "bf16", [shape[1], 5, 0][:shape[0]], label="after junk")
        for k, t in got.items():
            assert t is None or torch.isfinite(t.float()).all(), k
