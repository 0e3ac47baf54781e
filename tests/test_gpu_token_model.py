"""The model over tokens: the operators run together as a user runs them.  The
reference is the same model in float64 on the CPU from elementary operations,
differentiated by torch; both sides take the same float32 parameters.  The
tolerance is that of float32 dense products and sums over up to 96 terms in a
chain of about 20 operations: 2^-24 x 96 x 20 = 1.2e-4 of the largest magnitude
of each result."""
import pytest

pytestmark = pytest.mark.gpu
TOL = 1.2e-4


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    from paper_2603_13283_amd.tokens import TokenModel
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif, TokenModel


def reference(torch, model, params, tokens, length, x_first, h_first):
    """Logits, last inputs and last states in float64."""
    F = torch.nn.functional
    p, D, N, R, K = params, model.D, model.N, model.R, model.taps
    B, T = tokens.shape
    on = (torch.arange(T)[None, :] < length[:, None])
    named = on & (tokens >= 0) & (tokens < model.V)
    e = torch.where(named[..., None], p["E"][tokens.clamp(0, model.V - 1).long()] * model.scale, 0.0)
    xz = e @ p["Win"]
    x, z = xz[..., :D], xz[..., D:]
    outs, lasts, states = [], [], []
    for b in range(B):
        seen, h, ys = list(x_first[b]), h_first[b], []
        for t in range(int(length[b])):
            seen.append(x[b, t])
            c = F.silu(p["b"] + sum(p["w"][:, j] * seen[len(seen) - K + j] for j in range(K)))
            pr = c @ p["Wp"]
            delta = F.softplus(pr[:R] @ p["Wdt"] + p["dt_bias"])
            h = torch.exp(delta[:, None] * -p["A_log"].exp()) * h + (delta * c)[:, None] * pr[R:R + N]
            ys.append(((h * pr[R + N:]).sum(1) + p["skip"] * c) * F.silu(z[b, t]))
        ys += [torch.zeros(D, dtype=torch.float64)] * (T - int(length[b]))
        outs.append(torch.stack(ys))
        lasts.append(torch.stack(seen[len(seen) - K + 1:]))
        states.append(h)
    m = e + torch.stack(outs) @ p["Wout"]
    return (m @ p["Wo"]).view(B * T, -1), torch.stack(lasts), torch.stack(states)


def close(torch, got, want, label):
    got, want = got.detach().double().cpu(), want.detach()
    err = (got - want).abs().max().item()
    assert err <= TOL * want.abs().max().item() + 1e-12, f"{label}: {err} of {want.abs().max().item()}"


def make(env, B=3, T=40, V=50, seed=1):
    torch, _, TokenModel = env
    model = TokenModel.random(V, 24, 36, 6, 10, seed=seed)
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(-1, V + 1, (B, T), generator=g, dtype=torch.int32)
    length = torch.tensor([T, 17, 0][:B], dtype=torch.int32)
    x0 = torch.randn((B, model.taps - 1, model.D), generator=g)
    h0 = torch.randn((B, model.D, model.N), generator=g)
    return model, tokens, length, x0, h0, g


def test_gradients(env):
    torch = env[0]
    model, tokens, length, x0, h0, g = make(env)
    B, T = tokens.shape
    gl = torch.randn((B * T, 10), generator=g)
    gx, gh = torch.randn(x0.shape, generator=g), torch.randn(h0.shape, generator=g)
    dev = [v.to("cuda:0") for v in (tokens, length, x0, h0, gl, gx, gh)]
    out = model.forward(dev[0], dev[1], dev[2], dev[3], train=True)
    grads = model.backward(dev[0], out, dev[4], dev[1], grad_x_last=dev[5], grad_h_last=dev[6])
    leaves = {k: v.double().cpu().requires_grad_() for k, v in model.params.items()}
    first = {"x_first": x0.double().requires_grad_(), "h_first": h0.double().requires_grad_()}
    logits, last, state = reference(torch, model, leaves, tokens, length, first["x_first"], first["h_first"])
    close(torch, out.logits, logits, "logits")
    close(torch, out.x_last, last, "x_last")
    close(torch, out.h_last, state, "h_last")
    ((logits * gl.double()).sum() + (last * gx.double()).sum() + (state * gh.double()).sum()).backward()
    for k, v in {**leaves, **first}.items():
        close(torch, grads[k], v.grad, "gradient of " + k)


def test_streams_follow_the_sequence(env):
    torch, lif, _ = env
    model, tokens, _, _, _, g = make(env, B=2, T=12)
    tokens = tokens.to("cuda:0")
    out = model.forward(tokens)
    state = model.stream_state(5)
    slot = torch.tensor([4, 1], dtype=torch.int32, device="cuda:0")
    for t in range(12):
        last = model.stream_step(tokens[:, t], state, slot, k=3)
        rows = out.logits.view(2, 12, -1)[:, t]
        want = torch.log_softmax(rows.double().cpu(), dim=1).topk(3, dim=1).values
        close(torch, last.top_logp, want, f"step {t}")
    assert not state.h[[0, 2, 3]].any() and not state.x[[0, 2, 3]].any()
    close(torch, state.h[slot.long()], out.h_last.double().cpu(), "states")
    close(torch, state.x[slot.long()], out.x_last.double().cpu(), "inputs")


def test_pieces_and_training(env):
    """Two pieces give the whole's logits; steps on the next token change the
    parameters by finite amounts, events of a queue are tokens."""
    torch, lif, _ = env
    model, tokens, _, _, _, g = make(env, B=2, T=40)
    tokens = tokens.to("cuda:0")
    whole = model.forward(tokens)
    a = model.forward(tokens[:, :23].contiguous())
    b = model.forward(tokens[:, 23:].contiguous(), x_first=a.x_last, h_first=a.h_last)
    both = torch.cat([a.logits.view(2, 23, -1), b.logits.view(2, 17, -1)], 1)
    close(torch, both, whole.logits.view(2, 40, -1).double().cpu(), "pieces")
    length = torch.tensor([40, 11], dtype=torch.int32, device="cuda:0")
    targets = torch.where(tokens < 10, tokens, -1).roll(-1, dims=1).contiguous()
    for _ in range(3):
        loss, grads = model.train_step(tokens, targets, length)
        assert torch.isfinite(loss) and all(torch.isfinite(v).all() for v in grads.values())
    assert all(torch.isfinite(v).all() for v in model.params.values())


def test_captured_training_step(env):
    """Forward and backward in a graph give what eager calls give on every
    replay, with eager work in between."""
    torch = env[0]
    model, tokens, length, _, _, g = make(env)
    tokens, length = tokens.to("cuda:0"), length.to("cuda:0")
    targets = torch.randint(0, 10, tokens.shape, generator=g, dtype=torch.int32).to("cuda:0")
    run = lambda: model.train_step(tokens, targets, length, update=False)[1]              # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for i in range(3):
        tokens.copy_(torch.randint(-1, 51, tokens.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for k, v in run().items():
            close(torch, held[k], v.double().cpu(), f"replay {i}: {k}")
