"""A training step of the model over tokens against the same step in float64 on
the CPU (torch's cross-entropy and gradients), an event queue as its tokens, and
lookups between types; tolerances as in test_gpu_token_model.py and
test_gpu_embed.py."""
import numpy as np
import pytest

from test_gpu_embed import check_lookup, dt_of, tokens_of
from test_gpu_token_model import close, make, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    from paper_2603_13283_amd.tokens import TokenModel
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif, TokenModel


@pytest.mark.parametrize("ragged", [True, False])
def test_training_step(env, ragged):
    """Loss and gradients of the targets that count: those in [0, K) before
    their sample's length; then one update against Adam's formula."""
    torch = env[0]
    model, tokens, length, x0, h0, g = make(env, seed=4)
    B, T = tokens.shape
    targets = torch.randint(-3, 14, (B, T), generator=g, dtype=torch.int32)               # K is 10
    n = length if ragged else torch.full((B,), T, dtype=torch.int32)
    before = {k: v.double().cpu() for k, v in model.params.items()}
    dev = [v.to("cuda:0") for v in (tokens, targets, length)]
    loss, grads = model.train_step(dev[0], dev[1], dev[2] if ragged else None, update=False)
    leaves = {k: v.clone().requires_grad_() for k, v in before.items()}
    zeros = torch.zeros(x0.shape, dtype=torch.float64), torch.zeros(h0.shape, dtype=torch.float64)
    logits, _, _ = reference(torch, model, leaves, tokens, n, *zeros)
    on = (targets >= 0) & (targets < 10) & (torch.arange(T)[None, :] < n[:, None])
    assert 0 < int(on.sum()) < B * T
    want = torch.nn.functional.cross_entropy(logits[on.view(-1)], targets[on].long())
    want.backward()
    close(torch, loss, want, "loss")
    for k, v in leaves.items():
        close(torch, grads[k], v.grad, "gradient of " + k)
    assert all(torch.equal(model.params[k].double().cpu(), v) for k, v in before.items()), "update=False updates"
    _, grads = model.train_step(dev[0], dev[1], dev[2] if ragged else None)
    a = model.adam
    for k, v in before.items():
        gr = grads[k].double().cpu()
        # the first step: both moments over 1 - beta are the gradient and its square
        want = v - a.lr * gr / (gr.abs() + a.eps)
        err = (model.params[k].double().cpu() - want).abs()
        # the parameter is rounded once, the step is off by a few of its roundings
        assert (err <= 2.0 ** -24 * want.abs() + 1e-5 * a.lr).all(), k


def test_without_targets(env):
    """No target counts: no loss, no gradients."""
    torch = env[0]
    model, tokens, length, _, _, _ = make(env, seed=5)
    loss, grads = model.train_step(tokens.to("cuda:0"), torch.full(tokens.shape, -1, dtype=torch.int32, device="cuda:0"),
                                   length.to("cuda:0"), update=False)
    assert float(loss) == 0.0 and not any(v.any() for v in grads.values())


def test_event_queue(env):
    """The source channels of an event queue in the order of its events are
    tokens, its counts are lengths."""
    torch, lif, TokenModel = env
    import workloads
    ev = workloads.random_small(7, B=4, C=50, N=8, n_events=40, T=0.3, gain=1.0).events
    model = TokenModel.random(50, 24, 36, 6, 10, seed=6)
    src, n = torch.from_numpy(np.ascontiguousarray(ev.ev_src)), torch.from_numpy(np.ascontiguousarray(ev.ev_n))
    assert len(set(n.tolist())) > 1
    out = model.forward(src.to("cuda:0"), n.to("cuda:0"))
    zeros = [torch.zeros((4, *s), dtype=torch.float64) for s in ((model.taps - 1, model.D), (model.D, model.N))]
    params = {k: v.double().cpu() for k, v in model.params.items()}
    logits, last, state = reference(torch, model, params, src, n, *zeros)
    close(torch, out.logits, logits, "logits")
    close(torch, out.x_last, last, "x_last")
    close(torch, out.h_last, state, "h_last")


@pytest.mark.parametrize("table", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(2, 3, 2, 3), (3, 70, 50, 33), (2, 500, 300, 130)])
def test_lookup_types(env, shape, dtype, table):
    """Tables of one type looked up into another."""
    torch, lif, _ = env
    B, T, V, D = shape
    tokens = tokens_of(torch, B, T, V).to("cuda:0")
    W = torch.randn((V, D), generator=torch.Generator().manual_seed(2)).to("cuda:0", dt_of(torch, table))
    check_lookup(env[:2], tokens, W, lif.embed(tokens, W, 1.7, dtype=dt_of(torch, dtype)), float(np.float32(1.7)), None,
                 dtype)
