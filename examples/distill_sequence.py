"""A small sequence classifier learns from a larger one.

Input events pass an event-driven LIF layer; its spikes, counted in bins,
drive two heads with a gated leaky integrator.  The wide one is trained on the
labels.  The narrow one never sees a label: it is trained on the wide one's
likeliest classes at every bin.  Last, the narrow head runs on the samples as
streams, one bin at a time.

    python examples/distill_sequence.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2603_13283_amd as lif                                               # noqa: E402
import workloads as W                                                            # noqa: E402
from paper_2603_13283_amd.sequence import SequenceHead, bin_spikes               # noqa: E402
from paper_2603_13283_amd.train import AdamParams                                # noqa: E402

BINS, DT, CLASSES, LIST, TEMPERATURE = 100, 0.005, 20, 5, 2.0


def data(B: int = 64, C: int = 100, N: int = 128, seed: int = 0):
    """Spike counts [B, BINS, N] of a LIF layer on random events, and labels:
    the samples of a class share their events up to a tenth."""
    dev = "cuda:0"
    g = torch.Generator().manual_seed(seed)
    cfg = W.random_small(seed, B=CLASSES, C=C, N=N, n_events=1500, T=BINS * DT, gain=14.0, ragged=False)
    labels = torch.randint(0, CLASSES, (B,), generator=g)
    ev = cfg.events
    src = torch.from_numpy(ev.ev_src)[labels]
    noise = torch.rand(src.shape, generator=g) < 0.1
    src = torch.where(noise, torch.randint(0, C, src.shape, generator=g), src.long()).to(torch.int32)
    t, n = torch.from_numpy(ev.ev_t)[labels], torch.from_numpy(ev.ev_n)[labels]
    WT = torch.from_numpy(cfg.layers[0].WT)
    out = lif.forward(t.to(dev).contiguous(), src.to(dev), n.to(dev).contiguous(), WT.to(dev), lif.Params(s_max=64))
    return bin_spikes(out, BINS, DT), labels.to(dev, torch.int32)


def main(steps: int = 60, verbose: bool = True) -> dict:
    say = print if verbose else lambda *a, **k: None
    counts, labels = data()
    N = counts.shape[2]
    adam = AdamParams(lr=3e-3)
    teacher = SequenceHead.random(N, 256, CLASSES, seed=1, adam=adam)
    student = SequenceHead.random(N, 48, CLASSES, seed=2, adam=AdamParams(lr=1e-2))
    res = {"teacher": [], "student": []}
    for i in range(steps):
        loss, _ = teacher.train_step(counts, labels)
        res["teacher"].append(float(loss))
    say(f"teacher: cross-entropy {res['teacher'][0]:.3f} -> {res['teacher'][-1]:.3f}")
    lists = teacher.alternatives(counts, LIST, TEMPERATURE)
    for i in range(steps):
        loss, _ = student.distill_step(counts, lists, TEMPERATURE)
        res["student"].append(float(loss))
    say(f"student: divergence from the teacher {res['student'][0]:.3f} -> {res['student'][-1]:.3f}")
    # the student on streams: one bin of all samples at a time, their states in a pool
    B = counts.shape[0]
    state = torch.zeros((2 * B, student.params["bf"].shape[0]), device=counts.device)
    slot = torch.randperm(2 * B, device=counts.device)[:B].to(torch.int32)
    for t in range(BINS):
        last = student.stream_step(counts[:, t], state, slot, labels, k=3)
    hits = (last.top_idx[:, 0] == labels).float().mean()
    res["streams"] = {"accuracy": float(hits), "logp": last.logp, "entropy": last.entropy, "state": state[slot.long()]}
    res["whole"] = student.forward(counts)
    say(f"student on streams: {100 * float(hits):.0f} % of the labels at the last bin, entropy "
        f"{float(last.entropy.mean()):.2f}")
    return res


if __name__ == "__main__":
    main()
