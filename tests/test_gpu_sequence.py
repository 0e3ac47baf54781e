"""The sequence head (gated leaky integrator, logits, label and distillation
losses) as it is used: gradients against a float64 autograd graph of the same
formulas, streams against whole sequences, and the example that distils one
head into another."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GRAD_RTOL = 1e-4          # the gradient tolerance of the parity bar, relative in norm


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


def _reference(torch, head, counts, length, loss_of):
    """Gradients of loss_of(log probabilities [B * T, K]) in float64 on the
    CPU, step by step."""
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in head.params.items()}
    c = counts.double().cpu()
    B, T, _ = c.shape
    n = torch.full((B,), T) if length is None else length.cpu().long()
    h, rows = torch.zeros(B, p["bf"].shape[0], dtype=torch.float64), []
    for t in range(T):
        a = torch.sigmoid(c[:, t] @ p["Wf"] + p["bf"])
        on = (t < n)[:, None]
        h = torch.where(on, a * h + (1 - a) * (c[:, t] @ p["Wx"]), h)
        rows.append(torch.where(on, h, 0.0))
    logits = torch.stack(rows, 1).reshape(B * T, -1) @ p["Wo"]
    loss = loss_of(logits)
    loss.backward()
    return float(loss.detach()), {k: v.grad.numpy() for k, v in p.items()}


def _close(got, want):
    for k, w in want.items():
        g = got[k].double().cpu().numpy()
        assert np.linalg.norm(g - w) <= GRAD_RTOL * np.linalg.norm(w), k


@pytest.mark.parametrize("ragged", [False, True])
def test_head_gradients(env, ragged):
    torch, lif = env
    from paper_2603_13283_amd.sequence import SequenceHead
    B, T, N, D, K, k, temp = 3, 70, 11, 12, 7, 3, 1.5
    g = torch.Generator().manual_seed(3)
    counts = torch.poisson(torch.full((B, T, N), 0.4), generator=g).cuda()
    labels = torch.tensor([0, 6, 3], dtype=torch.int32, device="cuda:0")
    length = torch.tensor([T, 0, 41], dtype=torch.int32, device="cuda:0") if ragged else None
    head, teacher = SequenceHead.random(N, D, K, seed=4), SequenceHead.random(N, 20, K, seed=5)
    w = head._bins(counts, length).double().cpu()
    rows = torch.arange(B * T)

    def ce(logits):
        return -(w * torch.log_softmax(logits, 1)[rows, labels.cpu().long().repeat_interleave(T)]).sum()
    loss, grads = head.train_step(counts, labels, length, update=False)
    want, ref = _reference(torch, head, counts, length, ce)
    assert abs(float(loss) - want) <= 1e-5 * abs(want)
    _close(grads, ref)

    lists = teacher.alternatives(counts, k, temp, length)
    q, idx = lists.top_logp.double().cpu().exp(), lists.top_idx.cpu().long()

    def divergence(logits):
        p = torch.softmax(logits / temp, 1)
        pq, rest = p.gather(1, idx), 1 - p.gather(1, idx).sum(1)
        q_rest = 1 - q.sum(1)
        return (w * ((q * (q / pq).log()).sum(1) + q_rest * (q_rest / rest).log())).sum()
    loss, grads = head.distill_step(counts, lists, temp, length=length, update=False)
    want, ref = _reference(torch, head, counts, length, divergence)
    assert abs(float(loss) - want) <= 1e-5 * abs(want)
    _close(grads, ref)


def test_example_distils_and_streams(env):
    """The example runs: the teacher learns the labels, the student the
    teacher, and the student's streams end in the states of its whole
    sequences."""
    torch, lif = env
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import distill_sequence as E
    finally:
        sys.path.pop(0)
    res = E.main(steps=40, verbose=False)
    assert res["teacher"][-1] < 0.5 * res["teacher"][0]
    assert res["student"][-1] < 0.5 * res["student"][0]
    assert res["streams"]["accuracy"] > 0.5
    diff = (res["streams"]["state"] - res["whole"].h_last).abs().max()
    # 100 further roundings, in another order, of states below 8 and of products summed in another order
    assert float(diff) < 1e-4
    assert torch.isfinite(res["streams"]["logp"]).all() and (res["streams"]["entropy"] >= 0).all()


def test_bins_count_every_spike(env):
    torch, lif = env
    from paper_2603_13283_amd.sequence import bin_spikes
    t = torch.tensor([[[0.0, 0.0049, 0.005, float("inf")], [0.0149, 0.015, 0.5, 0.6]]], device="cuda:0")
    n = torch.tensor([[3, 3]], dtype=torch.int32, device="cuda:0")
    c = bin_spikes(lif.ForwardOut(t, n, None, None), 3, 0.005)
    assert c.shape == (1, 3, 2) and c[0].tolist() == [[2.0, 0.0], [1.0, 0.0], [0.0, 1.0]]
