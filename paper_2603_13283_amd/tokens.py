"""A sequence model over tokens: the source channels of an event queue in the
order of its events, or words.  Each token's row of a table (lif_embed) is
projected to an input and a gate; the input passes a short causal convolution
(lif_causal_conv) and a selective state space (lif_selective_scan) whose steps,
inputs and readouts are projections of the convolution's output; the gated
result is projected back onto the row, and that to one row of logits per token.
It is trained on the labels of the sequences or on the tokens that follow
(lif_token_logprobs), with the gradients through the operators' backward passes
and lif_adam_step, and it runs on streams one token at a time.  The dense
products are torch matrix products."""
from __future__ import annotations

from dataclasses import dataclass

from . import (LogprobOut, adam_step, causal_conv, causal_conv_backward, causal_conv_step, embed, embed_backward,
               selective_scan, selective_scan_backward, selective_step, token_logprobs, _torch)
from .train import AdamParams


@dataclass
class TokenOut:
    logits: "object"             # [B * T, K]
    x_last: "object"             # [B, taps - 1, D]: where the convolution of a stream goes on
    h_last: "object"             # float32 [B, D, N]: its states
    kept: "object" = None        # what the backward pass needs


@dataclass
class StreamState:
    """Pools of running streams: one slot each."""
    x: "object"                  # [n_slots, taps - 1, D] last inputs of the convolution
    h: "object"                  # float32 [n_slots, D, N]


class TokenModel:
    """Parameters are float32 device tensors: E [V, M] the table, Win [M, 2 D],
    w [D, taps] and b [D] the convolution, Wp [D, R + 2 N] (step lengths, B and
    C), Wdt [R, D], dt_bias [D], A_log [D, N] (the rates are -e^A_log), skip
    [D], Wout [D, M], Wo [M, K]."""

    def __init__(self, params: dict, adam: AdamParams = AdamParams()):
        torch = _torch()
        self.params = params
        self.m1 = {k: torch.zeros_like(v) for k, v in params.items()}
        self.m2 = {k: torch.zeros_like(v) for k, v in params.items()}
        self.adam, self.t = adam, 0
        (self.V, self.M), (self.D, self.N) = params["E"].shape, params["A_log"].shape
        self.taps, self.R = params["w"].shape[1], params["Wdt"].shape[0]
        self.scale = self.M ** 0.5

    @classmethod
    def random(cls, V: int, M: int, D: int, N: int, K: int, taps: int = 4, R: int = 0, seed: int = 0,
               device="cuda:0", **kw):
        """Random weights; step lengths around 0.001 to 0.1 and rates -1 to -N
        give states that last 1 to 1000 tokens."""
        torch = _torch()
        g = torch.Generator().manual_seed(seed)
        R = R or max(1, M // 16)
        rn = lambda *s: torch.randn(*s, generator=g)                                      # noqa: E731
        w = lambda a, b: rn(a, b) / a ** 0.5                                              # noqa: E731
        step = torch.exp(torch.rand(D, generator=g) * 4.605170186 - 6.907755279)
        p = {"E": rn(V, M) / M ** 0.5, "Win": w(M, 2 * D), "w": rn(D, taps) / taps ** 0.5, "b": torch.zeros(D),
             "Wp": w(D, R + 2 * N), "Wdt": 0.1 * w(R, D), "dt_bias": torch.log(torch.expm1(step)),
             "A_log": torch.log(torch.arange(1, N + 1).float()).repeat(D, 1), "skip": torch.ones(D),
             "Wout": w(D, M), "Wo": w(M, K)}
        return cls({k: v.to(device).contiguous() for k, v in p.items()}, **kw)

    def stream_state(self, n_slots: int) -> StreamState:
        """Pools for n_slots streams that have seen nothing."""
        torch = _torch()
        dev = self.params["E"].device
        return StreamState(torch.zeros((n_slots, self.taps - 1, self.D), device=dev),
                           torch.zeros((n_slots, self.D, self.N), device=dev))

    def _split(self, pr):
        """Step lengths' part, B and C of a projection, as views."""
        R, N = self.R, self.N
        return pr[..., :R], pr[..., R:R + N], pr[..., R + N:]

    def forward(self, tokens, length=None, x_first=None, h_first=None, train: bool = False) -> TokenOut:
        """tokens int32 [B, T] (an event queue's sources; outside the table:
        padding), length int32 [B] (its counts).  x_first and h_first go on from
        an earlier piece's x_last and h_last."""
        p, D = self.params, self.D
        B, T = tokens.shape
        e = embed(tokens, p["E"], self.scale, length)
        xz = e @ p["Win"]
        x, z = xz[..., :D], xz[..., D:]
        c = causal_conv(x, p["w"], p["b"], length, x_first)
        pr = c.y @ p["Wp"]
        r, Bm, C = self._split(pr)
        dt, A = r @ p["Wdt"], -p["A_log"].exp()
        s = selective_scan(c.y, dt, A, Bm, C, D=p["skip"], z=z, dt_bias=p["dt_bias"], length=length, h_first=h_first,
                           marks=train)
        m = (e + s.y @ p["Wout"]).view(B * T, self.M)
        kept = (e, xz, c.y, pr, dt, A, s, m, x_first) if train else None
        return TokenOut(m @ p["Wo"], c.x_last, s.h_last, kept)

    def backward(self, tokens, out: TokenOut, grad_logits, length=None, *, grad_x_last=None, grad_h_last=None) -> dict:
        """Gradients of the parameters, and of x_first and h_first (what a
        sequence that goes on in pieces hands to the piece before as
        grad_x_last and grad_h_last), for dL/dlogits [B * T, K] of a forward
        with train=True."""
        torch, p, D = _torch(), self.params, self.D
        e, xz, y, pr, dt, A, s, m, x_first = out.kept
        B, T = tokens.shape
        flat = lambda v: v.reshape(B * T, v.shape[-1])                                    # noqa: E731
        x, z = xz[..., :D], xz[..., D:]
        r, Bm, C = self._split(pr)
        gm = grad_logits @ p["Wo"].t()
        g = selective_scan_backward(y, dt, A, Bm, C, s.marks, (gm @ p["Wout"].t()).view(B, T, D), D=p["skip"], z=z,
                                    dt_bias=p["dt_bias"], grad_last=grad_h_last, length=length)
        gpr = torch.cat([g.dt @ p["Wdt"].t(), g.B, g.C], dim=-1)
        gc = causal_conv_backward(x, p["w"], g.x + gpr @ p["Wp"].t(), p["b"], length, x_first, grad_x_last)
        gxz = torch.cat([gc.x, g.z], dim=-1)
        ge = gm.view(B, T, self.M) + gxz @ p["Win"].t()
        return {"E": embed_backward(tokens, ge, self.V, self.scale, length), "Win": flat(e).t() @ flat(gxz), "w": gc.w,
                "b": gc.bias, "Wp": flat(y).t() @ flat(gpr), "Wdt": flat(r).t() @ flat(g.dt), "dt_bias": g.dt_bias,
                "A_log": g.A * A, "skip": g.D, "Wout": flat(s.y).t() @ gm, "Wo": m.t() @ grad_logits,
                "x_first": gc.x_first, "h_first": g.h_first}

    def update(self, grads: dict) -> None:
        self.t += 1
        a = self.adam
        for k, w in self.params.items():
            adam_step(w, grads[k].contiguous(), self.m1[k], self.m2[k], self.t, a.lr, a.beta1, a.beta2, a.eps)

    def train_step(self, tokens, targets, length=None, update: bool = True):
        """Cross-entropy of a target per token (int32 [B, T]: the token that
        follows, or a label repeated along T; outside [0, K): none), averaged
        over those that count.  Returns (loss, gradients)."""
        torch = _torch()
        B, T = tokens.shape
        out = self.forward(tokens, length, train=True)
        K = out.logits.shape[1]
        on = (targets >= 0) & (targets < K)
        if length is not None:
            on &= torch.arange(T, device=tokens.device) < length[:, None]
        w = on.reshape(-1).float()
        w = w / w.sum().clamp(min=1.0)
        lp = token_logprobs(out.logits, targets.reshape(-1).contiguous(), grad_logp=-w)
        grads = self.backward(tokens, out, lp.grad, length)
        if update:
            self.update(grads)
        return -(lp.logp * w).sum(), grads

    def stream_step(self, tokens, state: StreamState, slot=None, targets=None, k: int = 0) -> LogprobOut:
        """One token (int32 [B]) of B running streams, whose states are rows
        `slot` of the pools, updated in place."""
        p, D = self.params, self.D
        e = embed(tokens, p["E"], self.scale)
        xz = e @ p["Win"]
        y = causal_conv_step(xz[:, :D], p["w"], state.x, slot=slot, bias=p["b"])
        r, Bm, C = self._split(y @ p["Wp"])
        s = selective_step(y, r @ p["Wdt"], -p["A_log"].exp(), Bm, C, state.h, slot=slot, D=p["skip"], z=xz[:, D:],
                           dt_bias=p["dt_bias"])
        return token_logprobs((e + s @ p["Wout"]) @ p["Wo"], targets, k=k)
