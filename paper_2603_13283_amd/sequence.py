"""A classifier head over binned spikes: a hidden layer's spikes counted in
time bins drive a gated leaky integrator (lif_gated_scan), whose states give
one row of logits per bin.  It is trained on labels (lif_token_logprobs) or on
a teacher's likeliest classes (lif_distill_top), with the gradients through
lif_gated_scan_backward and lif_adam_step, and it runs on streams one bin at a
time (lif_gated_step).  The dense products are torch matrix products."""
from __future__ import annotations

from dataclasses import dataclass

from . import (ForwardOut, LogprobOut, adam_step, distill_top, gated_scan, gated_scan_backward, gated_step,
               token_logprobs, _torch)
from .train import AdamParams


def bin_spikes(fwd: ForwardOut, bins: int, dt: float, dtype=None):
    """Spike counts [B, bins, N] of a layer's output in bins of dt seconds
    from t = 0; earlier and later spikes are left out."""
    torch = _torch()
    B, N, S = fwd.out_t.shape
    at = fwd.out_t / dt
    there = (torch.arange(S, device=at.device) < fwd.out_n[:, :, None]) & (at >= 0) & (at < bins)
    at = torch.where(there, at, float(bins)).long()
    counts = torch.zeros((B, N, bins + 1), dtype=torch.float32, device=fwd.out_t.device)
    counts.scatter_add_(2, at, there.float())
    return counts[:, :, :bins].transpose(1, 2).contiguous().to(dtype or torch.float32)


@dataclass
class HeadOut:
    h: "object"              # [B, T, D] states
    logits: "object"         # [B * T, K]
    h_last: "object"         # float32 [B, D]: where a stream goes on
    x: "object" = None       # [B, T, D] the integrator's inputs, and the states that its gradient starts from
    f: "object" = None
    marks: "object" = None


class SequenceHead:
    """x = counts Wx, f = counts Wf + bf, h the gated leaky integrator of x
    and f, logits = h Wo.  Parameters are float32 device tensors: Wx, Wf
    [N, D], bf [D], Wo [D, K]."""

    def __init__(self, Wx, Wf, bf, Wo, adam: AdamParams = AdamParams(), coupled: bool = True):
        torch = _torch()
        self.params = {"Wx": Wx, "Wf": Wf, "bf": bf, "Wo": Wo}
        self.m1 = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.m2 = {k: torch.zeros_like(v) for k, v in self.params.items()}
        self.adam, self.coupled, self.t = adam, coupled, 0

    @classmethod
    def random(cls, N: int, D: int, K: int, seed: int = 0, device="cuda:0", leak_bins: float = 20.0, **kw):
        """Random weights; the gate's bias gives a leak over leak_bins bins."""
        torch = _torch()
        g = torch.Generator().manual_seed(seed)
        w = lambda a, b: (torch.randn(a, b, generator=g) / a ** 0.5).to(device)      # noqa: E731
        a = 1.0 - 1.0 / leak_bins
        return cls(w(N, D), 0.1 * w(N, D), torch.full((D,), float(torch.logit(torch.tensor(a))), device=device),
                   w(D, K), **kw)

    def _gates(self, counts):
        p = self.params
        flat = counts.reshape(-1, counts.shape[-1]).to(p["Wx"].dtype)
        return flat @ p["Wx"], flat @ p["Wf"] + p["bf"]

    def forward(self, counts, length=None, h_first=None, train: bool = False) -> HeadOut:
        """counts [B, T, N] of any type, length int32 [B]: logits of every bin
        (those of bins past a sample's length come from h = 0)."""
        B, T, _ = counts.shape
        x, f = (v.view(B, T, v.shape[1]) for v in self._gates(counts))
        o = gated_scan(x, f, length=length, h_first=h_first, coupled=self.coupled, marks=train)
        return HeadOut(o.h, o.h.view(B * T, o.h.shape[2]) @ self.params["Wo"], o.h_last, x, f, o.marks)

    def backward(self, counts, out: HeadOut, grad_logits, length=None, h_first=None, *, grad_last=None) -> dict:
        """Gradients of the parameters for dL/dlogits [B * T, K] of a forward
        with train=True, and dL/dh_last = grad_last (float32 [B, D]).  With
        the forward's h_first, its gradient is there too: what a sequence that
        goes on in pieces hands to the piece before as grad_last."""
        B, T, N = counts.shape
        flat = counts.reshape(B * T, N).to(self.params["Wx"].dtype)
        D = out.x.shape[2]
        gh = (grad_logits @ self.params["Wo"].t()).view(B, T, D)
        gx, gf, g0 = gated_scan_backward(out.x, out.f, out.marks, gh, grad_last=grad_last, length=length,
                                         coupled=self.coupled)
        gx, gf = gx.view(B * T, D), gf.view(B * T, D)
        grads = {"Wx": flat.t() @ gx, "Wf": flat.t() @ gf, "bf": gf.sum(0),
                 "Wo": out.h.view(B * T, D).t() @ grad_logits}
        return grads if h_first is None else {**grads, "h_first": g0}

    def update(self, grads: dict) -> None:
        self.t += 1
        a = self.adam
        for k, w in self.params.items():
            adam_step(w, grads[k].contiguous(), self.m1[k], self.m2[k], self.t, a.lr, a.beta1, a.beta2, a.eps)

    def _bins(self, counts, length):
        """1 / (number of bins) for the bins of each sample, 0 past its
        length: float32 [B * T]."""
        torch = _torch()
        B, T, _ = counts.shape
        if length is None:
            return torch.full((B * T,), 1.0 / max(B * T, 1), device=counts.device)
        on = (torch.arange(T, device=counts.device) < length[:, None]).float()
        return (on / on.sum().clamp(min=1.0)).reshape(-1)

    def train_step(self, counts, labels, length=None, update: bool = True):
        """Cross-entropy of the samples' labels (int32 [B]) at every bin,
        averaged over bins.  Returns (loss, gradients)."""
        w = self._bins(counts, length)
        out = self.forward(counts, length, train=True)
        tokens = labels[:, None].expand(-1, counts.shape[1]).reshape(-1).contiguous()
        lp = token_logprobs(out.logits, tokens, grad_logp=-w)
        grads = self.backward(counts, out, lp.grad, length)
        if update:
            self.update(grads)
        return -(lp.logp * w).sum(), grads

    def alternatives(self, counts, k: int, temperature: float = 1.0, length=None) -> LogprobOut:
        """The k likeliest classes of every bin: what a student learns from."""
        return token_logprobs(self.forward(counts, length).logits, k=k, temperature=temperature)

    def distill_step(self, counts, teacher: LogprobOut, temperature: float = 1.0, tail: bool = True, length=None,
                     update: bool = True):
        """One step towards a teacher's alternatives (at the same
        temperature).  Returns (loss, gradients)."""
        w = self._bins(counts, length)
        out = self.forward(counts, length, train=True)
        loss, grad = distill_top(out.logits, teacher.top_logp, teacher.top_idx, temperature=temperature, tail=tail,
                                 weight=w)
        grads = self.backward(counts, out, grad, length)
        if update:
            self.update(grads)
        return (loss * w).sum(), grads

    def stream_step(self, counts, state, slot=None, tokens=None, k: int = 0) -> LogprobOut:
        """One bin of B running streams: counts [B, N], their states rows
        `slot` of state (float32 [n_slots, D], updated in place)."""
        x, f = self._gates(counts)
        h = gated_step(x, f, state, slot=slot, coupled=self.coupled)
        return token_logprobs(h @ self.params["Wo"], tokens, k=k)
