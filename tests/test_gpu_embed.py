"""Rows of a table by token (lif_embed) and the table's gradient
(lif_embed_backward) against the float64 sums.  A looked-up row has one product
and one rounding to its type; a sum of m terms in any order has at most m
roundings a term and one for the scale."""
import numpy as np
import pytest

from oracle import tokens as O
from rounding import HALF, TINY, U

pytestmark = pytest.mark.gpu

TYPES = ("f32", "bf16", "f16")
# (samples, places, rows, width)
SHAPES = [(1, 1, 1, 1), (2, 3, 2, 3), (3, 70, 5, 4), (1, 65, 700, 20), (4, 333, 50, 33), (2, 1500, 1023, 7),
          (2, 900, 1024, 130), (1, 4000, 5000, 9), (5, 200, 300, 257), (1, 20000, 2, 5), (1, 300, 1 << 21, 1),
          (1, 64, 9, 4), (1, 4096, 70000, 6), (2, 2048, 3, 8), (1, 4097, 255, 3)]


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
    return t.detach().double().cpu().numpy()


def tokens_of(torch, B, T, V, seed=0):
    """Some rows often, and padding on both sides of the table."""
    g = torch.Generator().manual_seed(seed)
    t = ((V + 1.0) ** torch.rand((B, T), generator=g, dtype=torch.float64) - 1.0).long().clamp(0, V - 1)
    t[torch.rand((B, T), generator=g) < 0.05] = -1
    t[torch.rand((B, T), generator=g) < 0.05] = V
    return t.to(torch.int32)


def check_lookup(env, tokens, W, out, scale, length, dtype):
    want = O.embed(arr(tokens).astype(np.int64), arr(W), scale, length)
    lim = (U + HALF[dtype]) * (1 + U) * np.abs(want) + TINY[dtype]
    assert (np.abs(arr(out) - want) <= lim).all()


def check_grad(tokens, grad, got, scale, length):
    want, mag = O.embed_grad(arr(tokens).astype(np.int64), arr(grad), got.shape[0], scale, length)
    named = tokens.cpu().numpy()
    most = np.bincount(named[(named >= 0) & (named < got.shape[0])], minlength=1).max() if (named >= 0).any() else 0
    lim = (most + 2) * U * 1.01 * mag
    err = np.abs(arr(got) - want)
    assert np.isfinite(arr(got)).all() and (err <= lim).all(), f"{(err > lim).sum()} off, largest {err.max()}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(env, shape, dtype):
    torch, lif = env
    B, T, V, D = shape
    print(f"[case] embed {shape} {dtype}", flush=True)
    tokens = tokens_of(torch, B, T, V).to("cuda:0")
    g = torch.Generator().manual_seed(1)
    W = torch.randn((V, D), generator=g).to("cuda:0", dt_of(torch, dtype))
    for out_type in {"f32", dtype}:
        out = lif.embed(tokens, W, 1.7, dtype=dt_of(torch, out_type))
        check_lookup(env, tokens, W, out, float(np.float32(1.7)), None, out_type)
    grad = torch.randn((B, T, D), generator=g).to("cuda:0", dt_of(torch, dtype))
    check_grad(tokens, grad, lif.embed_backward(tokens, grad, V, 1.7), float(np.float32(1.7)), None)


@pytest.mark.parametrize("length", [[0, 0, 0], [1, 64, 99], [100, -5, 999]])
def test_lengths(env, length):
    torch, lif = env
    tokens = tokens_of(torch, 3, 100, 40).to("cuda:0")
    W, grad = torch.randn((40, 12), device="cuda:0"), torch.randn((3, 100, 12), device="cuda:0")
    n = torch.tensor(length, dtype=torch.int32, device="cuda:0")
    check_lookup(env, tokens, W, lif.embed(tokens, W, length=n), 1.0, length, "f32")
    for b, m in enumerate(np.clip(length, 0, 100)):
        grad[b, m:] = float("nan")
    got = lif.embed_backward(tokens, grad, 40, length=n)
    grad = torch.nan_to_num(grad)
    check_grad(tokens, grad, got, 1.0, length)


def test_views(env):
    """Rows of the table apart, gradients in any order of axes or repeated, and
    single places of a batch."""
    torch, lif = env
    tokens = tokens_of(torch, 4, 50, 30).to("cuda:0")
    wide = torch.randn((30, 41), device="cuda:0", dtype=torch.bfloat16)
    W = wide[:, 3:24]
    check_lookup(env, tokens, W, lif.embed(tokens, W), 1.0, None, "bf16")
    grad = torch.randn((50, 4, 21), device="cuda:0").transpose(0, 1)
    check_grad(tokens, grad, lif.embed_backward(tokens, grad, 30), 1.0, None)
    one = grad[:, :1].expand(4, 50, 21)
    check_grad(tokens, one, lif.embed_backward(tokens, one, 30), 1.0, None)
    flat = tokens[:, 0]
    out = lif.embed(flat, W, 3.0)
    assert out.shape == (4, 21) and torch.equal(out, lif.embed(tokens[:, :1].contiguous(), W, 3.0)[:, 0])
    got = lif.embed_backward(flat, grad[:, 0], 30)
    check_grad(tokens[:, :1], grad[:, :1], got, 1.0, None)


def test_nan_stays_in_its_row(env):
    torch, lif = env
    tokens = tokens_of(torch, 2, 500, 9).to("cuda:0")
    grad = torch.randn((2, 500, 12), device="cuda:0")
    tokens[1, 250] = 4
    grad[1, 250, 5] = float("nan")
    g = lif.embed_backward(tokens, grad, 9)
    bad = torch.isnan(g)
    assert bad[4, 5] and bad.sum() == 1


def test_nothing_named(env):
    """No place names a row: the gradient is 0 everywhere; no places at all."""
    torch, lif = env
    grad = torch.randn((2, 300, 12), device="cuda:0")
    assert not lif.embed_backward(torch.full((2, 300), -1, dtype=torch.int32, device="cuda:0"), grad, 1000).any()
    none = torch.empty((2, 0), dtype=torch.int32, device="cuda:0")
    assert not lif.embed_backward(none, grad[:, :0], 1000).any()
    assert lif.embed(none, torch.randn((5, 3), device="cuda:0")).shape == (2, 0, 3)


def test_same_bits_and_graphs(env):
    torch, lif = env
    tokens = tokens_of(torch, 8, 3000, 400).to("cuda:0")
    grad = torch.randn((8, 3000, 70), device="cuda:0", dtype=torch.bfloat16)
    W = torch.randn((400, 70), device="cuda:0")
    both = lambda **k: (lif.embed(tokens, W, 2.0, **k), lif.embed_backward(tokens, grad, 400, 2.0, **k))   # noqa: E731
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
        tokens.copy_(tokens_of(torch, 8, 3000, 400, seed=i + 1))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, both())), i
