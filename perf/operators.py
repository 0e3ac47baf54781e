"""The sequence and answer operators whose speed is measured: one pass of a
user's program per case, on seeded inputs made on the GPU.

Kinds of case and what each stands for in use:

  step     one time step of a gated leaky integrator for a batch of running
           streams, their states in a pool of slots (serving)
  scan     the same recurrence over whole sequences of binned input, with the
           last state (inference, prefill of a stream's state)
  train    the recurrence forward and its gradients to inputs, gates and first
           state (a training step's share)
  answers  log probability of a given class or token per row of logits, the
           row's entropy and its most likely alternatives (evaluation, serving,
           a teacher's side of distillation)
  policy   the same log probability and entropy with the gradient to the logits
           for given upstream gradients (policy gradients, cross-entropy)
  distill  the divergence of a student's rows of logits from a teacher's most
           likely alternatives, with its gradient

Formulas (t a time step, j a class; T a temperature, w a row's weight):

  recurrence  a = 1 / (1 + e^-f),  h_t = a_t h_{t-1} + (1 - a_t) x_t, or
              h_t = a_t h_{t-1} + x_t where the input is not coupled; steps at
              or past a sample's length leave the state alone and give h = 0
  answers     z = logits / T, p = softmax(z): log p[token], -sum p log p, and
              the k largest log p (ties: lowest index first)
  policy      dL/dlogits = (g (1[j = token] - p_j) - e p_j (log p_j + H)) / T
              for L with dL/dlogp = g and dL/dH = e
  distill     q = the teacher's listed probabilities, made to sum to 1, or
              (tail) kept, with the rest of the mass in one further class:
              loss = sum q (log q - log p), dL/dlogits of sum_r w_r loss_r
"""
import math

import torch

own = False          # False: plain torch operations; True: the framework's operators

DEV = "cuda:0"
F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TAIL_MIN = 2.0 ** -20        # a teacher's tail below this counts as none

MOST_SCAN = 1 << 26          # elements of one sequence input in a drawn case
MOST_ROWS = 200_000_000      # logits in a drawn case


def listed():
    return [
        # a single stream at the width of the 700x512 layer: latency of one call
        dict(name="step_b1_d512", kind="step", B=1, D=512, slots=64, dtype="bf16", coupled=True),
        # a full serving batch of wide states, drawn from a larger pool
        dict(name="step_b256_d4096", kind="step", B=256, D=4096, slots=512, dtype="f32", coupled=True),
        # inference over 1 s in bins of 1 ms at the two-layer network's batch and width, samples of any length
        dict(name="scan_b128_t1000_d512", kind="scan", B=128, T=1000, D=512, dtype="bf16", ragged=True, coupled=True),
        # one long stream: few channels, the time axis has to be split
        dict(name="scan_b1_t65521_d512", kind="scan", B=1, T=65521, D=512, dtype="bf16", ragged=False, coupled=False),
        # training at the 700x256 layer's batch and width in 32 bits, ragged
        dict(name="train_b32_t1000_d256", kind="train", B=32, T=1000, D=256, dtype="f32", ragged=True, coupled=True),
        # training on few long sequences of an odd width
        dict(name="train_b4_t8192_d1001", kind="train", B=4, T=8192, D=1001, dtype="bf16", ragged=False, coupled=True),
        # serving: a few rows of a large vocabulary, with alternatives
        dict(name="answers_r8_v131072", kind="answers", R=8, V=131072, k=20, dtype="bf16", temp=1.0),
        # evaluation of a 20-class readout at every bin of a batch
        dict(name="answers_r128000_v20", kind="answers", R=128000, V=20, k=5, dtype="f32", temp=1.0),
        # a teacher's pass over a batch of text: an odd vocabulary
        dict(name="answers_r4096_v50021", kind="answers", R=4096, V=50021, k=64, dtype="bf16", temp=2.0),
        # a policy-gradient step with an entropy bonus
        dict(name="policy_r2047_v32768", kind="policy", R=2047, V=32768, k=0, dtype="f16", temp=0.7),
        # distillation of a 20-class readout at every bin of a batch
        dict(name="distill_r128000_v20", kind="distill", R=128000, V=20, k=5, dtype="f32", temp=1.0, tail=True),
        # distillation of a large vocabulary from stored lists of 64: the largest case
        dict(name="distill_r4096_v50021", kind="distill", R=4096, V=50021, k=64, dtype="bf16", temp=2.0, tail=True),
    ]


def draw(rng):
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))     # noqa: E731
    kind = rng.choice(["step", "scan", "train", "answers", "policy", "distill"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "step":
        B = logu(1, 512)
        return dict(kind=kind, B=B, D=logu(20, 8192), slots=B + logu(1, 512), dtype=dtype, coupled=rng.random() < 0.5)
    if kind in ("scan", "train"):
        T, D = logu(1, 65536), logu(20, 4096)
        B = min(logu(1, 256), max(1, MOST_SCAN // (T * D)))
        T = min(T, MOST_SCAN // (B * D))
        return dict(kind=kind, B=B, T=T, D=D, dtype=dtype, ragged=rng.random() < 0.5, coupled=rng.random() < 0.5)
    V = logu(2, 131072)
    R = logu(1, min(262144, MOST_ROWS // V))
    case = dict(kind=kind, R=R, V=V, k=0, dtype=dtype, temp=round(rng.uniform(0.5, 4.0), 2))
    if kind != "policy":
        case["k"] = min(logu(1, 128), V)
    if kind == "distill":
        case["tail"] = rng.random() < 0.5
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)                              # noqa: E731
    rand = lambda *s: torch.rand(*s, device=DEV, generator=g)                                # noqa: E731
    s = dict(case)
    if case["kind"] == "step":
        B, D, n = case["B"], case["D"], case["slots"]
        s["x"] = randn(B, D).to(dt)
        s["f"] = (randn(B, D) + 3.0).to(dt)                 # a leak around 20 bins
        s["state"] = randn(n, D)
        s["slot"] = torch.randperm(n, device=DEV, generator=g)[:B].to(torch.int32)
        return s
    if case["kind"] in ("scan", "train"):
        B, T, D = case["B"], case["T"], case["D"]
        s["x"] = randn(B, T, D).to(dt)
        s["f"] = (randn(B, T, D) + 3.0).to(dt)
        s["h0"] = randn(B, D)
        s["length"] = None
        if case["ragged"]:
            s["length"] = (rand(B) * (T + 1)).to(torch.int32).clamp_(max=T)
            s["length"][0] = T
        if case["kind"] == "train":
            s["grad_h"] = randn(B, T, D).to(dt)
            s["grad_last"] = randn(B, D)
        return s
    R, V, k = case["R"], case["V"], case["k"]
    z = randn(R, V) * 2.5
    s["logits"] = z.to(dt, copy=True)
    if case["kind"] == "distill":
        # the teacher agrees with the student in part, and is surer; some rows list half as many classes
        t = (z * 0.8 + randn(R, V) * 2.0) / case["temp"]
        val, idx = t.topk(k, dim=1)
        val = val - torch.logsumexp(t, dim=1, keepdim=True)
        idx = idx.to(torch.int32)
        if k > 1:
            idx[3::7, k // 2:] = -1
        s["t_logp"], s["t_idx"] = val.contiguous(), idx.contiguous()
        s["weight"] = (rand(R) + 0.5) * (rand(R) > 0.1)     # a tenth of the rows is masked out
        return s
    del z
    # the given tokens: likely and unlikely ones, a few rows without one
    s["token"] = (rand(R) * V).to(torch.int32).clamp_(max=V - 1)
    s["token"][5::11] = -1
    if case["kind"] == "policy":
        s["g_logp"], s["g_ent"] = randn(R), randn(R) * 0.01
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    import paper_2603_13283_amd as lif
    kind = s["kind"]
    if kind == "step":
        h = lif.gated_step(s["x"], s["f"], s["state"], slot=s["slot"], coupled=s["coupled"])
        return {"h": h, "state": s["state"]}
    if kind == "scan":
        o = lif.gated_scan(s["x"], s["f"], length=s["length"], h_first=s["h0"], coupled=s["coupled"])
        return {"h": o.h, "h_last": o.h_last}
    if kind == "train":
        o = lif.gated_scan(s["x"], s["f"], length=s["length"], h_first=s["h0"], coupled=s["coupled"], marks=True)
        gx, gf, g0 = lif.gated_scan_backward(s["x"], s["f"], o.marks, s["grad_h"], grad_last=s["grad_last"],
                                             length=s["length"], coupled=s["coupled"])
        return {"h": o.h, "h_last": o.h_last, "grad_x": gx, "grad_f": gf, "grad_h_first": g0}
    if kind == "answers":
        o = lif.token_logprobs(s["logits"], s["token"], k=s["k"], temperature=s["temp"])
        return {"logp": o.logp, "entropy": o.entropy, "lse": o.lse, "top_logp": o.top_logp, "top_idx": o.top_idx}
    if kind == "policy":
        o = lif.token_logprobs(s["logits"], s["token"], temperature=s["temp"], grad_logp=s["g_logp"],
                               grad_entropy=s["g_ent"])
        return {"logp": o.logp, "entropy": o.entropy, "lse": o.lse, "grad": o.grad}
    loss, grad = lif.distill_top(s["logits"], s["t_logp"], s["t_idx"], temperature=s["temp"], tail=s["tail"],
                                 weight=s["weight"])
    return {"loss": loss, "grad": grad}


def run_plain(s):
    kind = s["kind"]
    if kind == "step":
        at = s["slot"].long()
        a, b = maps(s["x"].float(), s["f"].float(), s["coupled"])
        h = a * s["state"][at] + b
        s["state"][at] = h
        return {"h": h.to(s["x"].dtype), "state": s["state"]}
    if kind in ("scan", "train"):
        return plain_sequence(s)
    x = s["logits"].float() / s["temp"]
    m = x.max(dim=1, keepdim=True).values
    e = torch.exp(x - m)
    total = e.sum(dim=1, keepdim=True)
    lse = m + torch.log(total)
    if kind == "distill":
        return plain_distill(s, x, e, total, lse)
    logp = x - lse
    p = e / total
    entropy = -(p * logp).sum(dim=1)
    tok = s["token"].long()
    there = tok >= 0
    tok = tok.clamp(min=0)
    got = torch.where(there, logp.gather(1, tok[:, None])[:, 0], 0.0)
    out = {"logp": got, "entropy": entropy, "lse": lse[:, 0]}
    if kind == "answers":
        # one whole key per element, so that ties go to the lowest index
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        at = torch.arange(x.shape[1], device=x.device)
        top = ((key << 32) + (0x7FFFFFFF - at)).topk(s["k"], dim=1).values
        idx = 0x7FFFFFFF - (top & 0x7FFFFFFF)
        return {**out, "top_logp": logp.gather(1, idx), "top_idx": idx.to(torch.int32)}
    g = torch.where(there, s["g_logp"], 0.0)[:, None]
    grad = -p * (g + s["g_ent"][:, None] * (logp + entropy[:, None]))
    grad.scatter_add_(1, tok[:, None], g)
    return {**out, "grad": (grad / s["temp"]).to(s["logits"].dtype)}


def maps(x, f, coupled):
    """The step's affine map h -> a h + b."""
    return torch.sigmoid(f), torch.sigmoid(-f) * x if coupled else x


def scan(a, b):
    """All h_t of h_t = a_t h_{t-1} + b_t from h_{-1} = 0, by doubling."""
    d = 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], dim=1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], dim=1)
        d *= 2
    return b


def plain_sequence(s):
    x, f, h0, dt = s["x"].float(), s["f"].float(), s["h0"], s["x"].dtype
    B, T, D = x.shape
    a, b = maps(x, f, s["coupled"])
    valid = None
    if s["length"] is not None:
        valid = (torch.arange(T, device=x.device)[None, :] < s["length"][:, None])[:, :, None]
        a, b = torch.where(valid, a, 1.0), torch.where(valid, b, 0.0)
    first = torch.cat([b[:, :1] + a[:, :1] * h0[:, None], b[:, 1:]], dim=1)
    h = scan(a, first)
    last = h[:, -1]
    shown = h if valid is None else torch.where(valid, h, 0.0)
    out = {"h": shown.to(dt), "h_last": last}
    if s["kind"] == "scan":
        return out
    g = s["grad_h"].float()
    if valid is not None:
        g = torch.where(valid, g, 0.0)
    g = torch.cat([g[:, :-1], g[:, -1:] + s["grad_last"][:, None]], dim=1)
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], dim=1)
    lam = scan(after.flip(1), g.flip(1)).flip(1)         # lam_t = g_t + a_{t+1} lam_{t+1}
    before = torch.cat([h0[:, None], h[:, :-1]], dim=1)
    if s["coupled"]:
        gx, ga = lam * torch.sigmoid(-f), lam * (before - x)
    else:
        gx, ga = lam, lam * before
    gf = ga * torch.sigmoid(f) * torch.sigmoid(-f)
    if valid is not None:
        gx, gf = torch.where(valid, gx, 0.0), torch.where(valid, gf, 0.0)
    return {**out, "grad_x": gx.to(dt), "grad_f": gf.to(dt), "grad_h_first": a[:, 0] * lam[:, 0]}


def plain_distill(s, x, e, total, lse):
    idx = s["t_idx"].long()
    there = idx >= 0
    at = idx.clamp(min=0)
    q = torch.where(there, torch.exp(s["t_logp"]), 0.0)
    sum_q = q.sum(dim=1, keepdim=True)
    if not s["tail"]:
        q = q / sum_q
    logp = x.gather(1, at) - lse
    loss = torch.where(q > 0, q * (torch.log(q) - logp), 0.0).sum(dim=1)
    some = there.any(dim=1, keepdim=True)
    if s["tail"]:
        listed_ = torch.zeros_like(x).scatter_add_(1, at, there.float()) > 0
        left = torch.where(listed_, 0.0, e)
        rest = left.sum(dim=1, keepdim=True)
        q_rest = torch.where((1 - sum_q >= TAIL_MIN) & (there.sum(dim=1, keepdim=True) < x.shape[1]), 1 - sum_q, 0.0)
        log_rest = torch.log(rest) - torch.log(total)
        loss = loss + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - log_rest), 0.0)[:, 0]
        grad = e * ((sum_q + q_rest) / total) - torch.where(q_rest > 0, left * (q_rest / rest), 0.0)
    else:
        grad = e / total
    grad.scatter_add_(1, at, -q)
    grad = torch.where(some, grad * (s["weight"][:, None] / s["temp"]), 0.0)
    return {"loss": torch.where(some[:, 0], loss, 0.0), "grad": grad.to(s["logits"].dtype)}


# ---------------------------------------------------------------------------
# the same in 64 bits, step by step and row by row from the definitions
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "step":
        return exact_step(s)
    if case["kind"] in ("scan", "train"):
        return exact_sequence(s)
    outs = []
    for r in range(0, case["R"], max(1, 20_000_000 // case["V"])):      # rows in blocks that fit
        part = {k: v[r:r + max(1, 20_000_000 // case["V"])] if isinstance(v, torch.Tensor) else v for k, v in s.items()}
        outs.append((exact_distill if case["kind"] == "distill" else exact_answers)(part))
    return {k: None if outs[0][k] is None else torch.cat([o[k] for o in outs]) for k in outs[0]}


def exact_gate(s):
    """(a, input) of every step, in 64 bits."""
    f, x = s["f"].to(F64), s["x"].to(F64)
    a = 1.0 / (1.0 + torch.exp(-f))
    return a, x / (1.0 + torch.exp(f)) if s["coupled"] else x


def exact_step(s):
    state = s["state"].to(F64)
    a, u = exact_gate(s)
    rows = s["slot"].tolist()
    h = torch.stack([a[i] * state[r] + u[i] for i, r in enumerate(rows)])
    for i, r in enumerate(rows):
        state[r] = h[i]
    return {"h": h, "state": state}


def exact_sequence(s):
    B, T, D = s["x"].shape
    n = torch.full((B,), T, device=DEV) if s["length"] is None else s["length"].long()
    on = (torch.arange(T, device=DEV)[:, None] < n)[:, :, None]
    a, u = exact_gate(s)
    h = s["h0"].to(F64)
    before, hs = (torch.zeros(B, T, D, dtype=F64, device=DEV) for _ in range(2))
    for t in range(T):
        before[:, t] = h
        h = torch.where(on[t], a[:, t] * h + u[:, t], h)
        hs[:, t] = h
    valid = on.transpose(0, 1)
    out = {"h": hs * valid, "h_last": h}
    if s["kind"] == "scan":
        return out
    lams, lam, g = torch.zeros_like(hs), s["grad_last"].to(F64), s["grad_h"].to(F64)
    for t in reversed(range(T)):
        lam = torch.where(on[t], lam + g[:, t], lam)
        lams[:, t] = lam
        lam = torch.where(on[t], lam * a[:, t], lam)
    x = s["x"].to(F64)
    gx = lams * (1 - a) if s["coupled"] else lams
    gf = lams * a * (1 - a) * (before - x if s["coupled"] else before)
    return {**out, "grad_x": gx * valid, "grad_f": gf * valid, "grad_h_first": lam}


def exact_answers(s):
    z = s["logits"].to(F64) / s["temp"]
    lse = torch.logsumexp(z, dim=1)
    logp = z - lse[:, None]
    p = torch.exp(logp)
    H = -(p * logp).sum(dim=1)
    tok = s["token"].long()
    hit = torch.zeros_like(p)
    rows = (tok >= 0).nonzero()[:, 0]
    hit[rows, tok[rows]] = 1.0
    out = {"logp": (hit * logp).sum(dim=1), "entropy": H, "lse": lse}
    if s["kind"] == "answers":
        return {**out, "top_logp": logp.topk(s["k"], dim=1).values, "top_idx": None}
    g = s["g_logp"].to(F64) * (tok >= 0)
    grad = g[:, None] * (hit - p) - s["g_ent"].to(F64)[:, None] * p * (logp + H[:, None])
    return {**out, "grad": grad / s["temp"]}


def exact_distill(s):
    z = s["logits"].to(F64) / s["temp"]
    p = torch.softmax(z, dim=1)
    idx = s["t_idx"].long()
    r, c = (idx >= 0).nonzero(as_tuple=True)
    q = torch.zeros_like(p)
    q[r, idx[r, c]] = torch.exp(s["t_logp"].to(F64)[r, c])
    listed_ = torch.zeros_like(p, dtype=torch.bool)
    listed_[r, idx[r, c]] = True
    if s["tail"]:
        # one further class for everything that is not listed
        q_rest = 1.0 - q.sum(dim=1)
        q_rest = torch.where((q_rest >= TAIL_MIN) & ~listed_.all(dim=1), q_rest, 0.0)
        p_rest = torch.where(listed_, 0.0, p).sum(dim=1)
        target = torch.where(listed_, q, p * (q_rest / p_rest)[:, None])
        extra = torch.special.xlogy(q_rest, q_rest / p_rest)
        mass = q.sum(dim=1) + q_rest
    else:
        q = q / q.sum(dim=1, keepdim=True)
        target, extra, mass = q, 0.0, 1.0
    loss = (torch.special.xlogy(q, q) - q * torch.log_softmax(z, dim=1)).sum(dim=1) + extra
    mass = mass[:, None] if isinstance(mass, torch.Tensor) else mass
    target = target if not s["tail"] else torch.where((q_rest > 0)[:, None] | listed_, target, 0.0)
    return {"loss": loss, "grad": (mass * p - target) * (s["weight"].to(F64)[:, None] / s["temp"])}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once, and the operations
    of the formulas (an exponential, a logarithm or a quotient counts as one)."""
    e = SIZE[case["dtype"]]
    if case["kind"] == "step":
        n = case["B"] * case["D"]
        return {"bytes": n * (3 * e + 8) + 4 * case["B"], "flops": 6 * n}
    if case["kind"] == "scan":
        n = case["B"] * case["T"] * case["D"]
        return {"bytes": n * 3 * e + 8 * case["B"] * case["D"], "flops": 6 * n}
    if case["kind"] == "train":
        n = case["B"] * case["T"] * case["D"]
        return {"bytes": n * 6 * e + 16 * case["B"] * case["D"], "flops": 16 * n}
    n, R, k = case["R"] * case["V"], case["R"], case["k"]
    if case["kind"] == "answers":
        return {"bytes": n * e + R * (16 + 8 * k), "flops": 7 * n}
    if case["kind"] == "policy":
        return {"bytes": 2 * n * e + R * 24, "flops": 11 * n}
    return {"bytes": 2 * n * e + R * (8 + 8 * k), "flops": 6 * n}
