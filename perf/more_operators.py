"""Operators of models over tokens whose speed is measured: one pass of a
user's program per case, on seeded inputs made on the GPU.

Kinds of case and what each stands for in use:

  lookup        one learned row per token, scaled: tokens are the source channels
                of event queues (rows of events with a count each) or words
  lookup_grad   the gradient of the table for given gradients of the rows
  conv          a short causal convolution along time with its activation, over
                whole sequences, with the inputs where a stream goes on (prompts)
  conv_train    the same and its gradients (a training step's share)
  conv_step     one time step of it for running streams, their last inputs in a
                pool of slots (serving)
  select        a selective state space scan over whole sequences with the last
                state (inference, prefill of a stream's state)
  select_train  the same and its gradients
  select_step   one time step of it, the states in a pool of slots

Formulas (t a time step, d a channel, n a state, g = d's group):

  lookup   out[t] = scale W[token[t]], 0 for a token outside the table and past a
           sample's length; dL/dW[v] = scale sum_{t: token[t] = v} dL/dout[t]
  conv     c_t = bias + sum_j w[j] x_{t-K+1+j},  y = c / (1 + e^-c)
  select   delta = log(1 + e^{dt + dt_bias}),
           h_t[d,n] = e^{delta A[d,n]} h_{t-1}[d,n] + delta x_t[d] B_t[g,n],
           y_t[d] = (sum_n C_t[g,n] h_t[d,n] + skip[d] x_t[d]) z / (1 + e^-z)

Steps at or past a sample's length leave the state alone and give 0.
"""
import math

import torch

own = False          # False: plain torch operations; True: the framework's operators

DEV = "cuda:0"
F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

MOST_ROWS = 1 << 26          # elements of a sequence input, of a table in a drawn case
MOST_STATES = 1 << 28        # states over all steps of a scan in a drawn case


def listed():
    return [
        # event queues of 700 channels, about 5000 events a sample, into the width of the 700x256 layer
        dict(name="lookup_b32_t5000_v700_d256", kind="lookup", B=32, T=5000, V=700, D=256, dtype="f32", table="f32",
             ragged=True, zipf=False),
        # the gradient of that table: few rows, hundreds of events each
        dict(name="lookup_grad_b32_t5000_v700_d256", kind="lookup_grad", B=32, T=5000, V=700, D=256, dtype="f32",
             table="f32", ragged=True, zipf=False),
        # words of an odd vocabulary: a few rows very often, most never
        dict(name="lookup_grad_b8_t4096_v50021_d1001", kind="lookup_grad", B=8, T=4096, V=50021, D=1001, dtype="bf16",
             table="f32", ragged=False, zipf=True),
        # serving: one step of a batch of streams
        dict(name="conv_step_b64_d2048", kind="conv_step", B=64, D=2048, K=4, slots=128, dtype="bf16"),
        # prompts of different lengths
        dict(name="conv_b8_t2048_d2048", kind="conv", B=8, T=2048, D=2048, K=4, dtype="bf16", ragged=True),
        # training on few long sequences of an odd width
        dict(name="conv_train_b4_t8192_d1001", kind="conv_train", B=4, T=8192, D=1001, K=3, dtype="f16", ragged=False),
        # a single stream at the width of the 700x512 layer: latency of one call
        dict(name="select_step_b1_d512", kind="select_step", B=1, D=512, N=16, G=1, slots=64, dtype="bf16"),
        # a full serving batch of wide states, drawn from a larger pool
        dict(name="select_step_b256_d4096", kind="select_step", B=256, D=4096, N=16, G=1, slots=512, dtype="bf16"),
        # inference over 1 s in bins of 1 ms at the two-layer network's batch and width, samples of any length
        dict(name="select_b128_t1000_d512", kind="select", B=128, T=1000, D=512, N=16, G=1, dtype="bf16", ragged=True),
        # one long stream: few channels, the time axis has to be split
        dict(name="select_b1_t65521_d512", kind="select", B=1, T=65521, D=512, N=16, G=1, dtype="f16", ragged=False),
        # training at the 700x256 layer's batch and width in 32 bits, ragged
        dict(name="select_train_b32_t1000_d256", kind="select_train", B=32, T=1000, D=256, N=8, G=2, dtype="f32",
             ragged=True),
        # training of a wide layer: the largest case
        dict(name="select_train_b8_t2048_d2048", kind="select_train", B=8, T=2048, D=2048, N=16, G=1, dtype="bf16",
             ragged=False),
    ]


def draw(rng):
    logu = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))     # noqa: E731
    kind = rng.choice(["lookup", "lookup_grad", "conv", "conv_train", "conv_step", "select", "select", "select_train",
                       "select_train", "select_step"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("conv_step", "select_step"):
        B = logu(1, 512)
        case = dict(kind=kind, B=B, D=logu(20, 8192), slots=B + logu(1, 512), dtype=dtype)
    else:
        T, D = logu(1, 65536), logu(20, 4096)
        B = min(logu(1, 256), max(1, MOST_ROWS // (T * D)))
        T = min(T, MOST_ROWS // (B * D))
        case = dict(kind=kind, B=B, T=T, D=D, dtype=dtype, ragged=rng.random() < 0.5)
    if kind in ("lookup", "lookup_grad"):
        case["V"] = min(logu(2, 131072), MOST_ROWS // case["D"])
        case["table"], case["zipf"] = rng.choice(["f32", dtype]), rng.random() < 0.5
    elif kind.startswith("conv"):
        case["K"] = rng.randint(2, 8)
    else:
        N, G = logu(1, 64), rng.choice([1, 1, 2, 3])
        D = case["D"]
        if "T" in case:
            D = min(D, max(20, MOST_STATES // (N * case["B"])))
            case["T"] = max(1, min(case["T"], MOST_STATES // (N * case["B"] * D)))
        case.update(N=N, G=G, D=max(G, D - D % G))
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
    kind, B, D = case["kind"], case["B"], case["D"]
    s["length"] = None
    if case.get("ragged"):
        s["length"] = (rand(B) * (case["T"] + 1)).to(torch.int32).clamp_(max=case["T"])
        s["length"][0] = case["T"]
    if "slots" in case:
        s["slot"] = torch.randperm(case["slots"], device=DEV, generator=g)[:B].to(torch.int32)
    steps = (B, case["T"]) if "T" in case else (B,)
    if kind in ("lookup", "lookup_grad"):
        V = case["V"]
        # channels alike, or words by rank (the k-th in proportion to 1 / k) in a random order
        at = ((V + 1.0) ** rand(*steps) - 1.0 if case["zipf"] else rand(*steps) * V).long().clamp_(0, V - 1)
        token = torch.randperm(V, device=DEV, generator=g)[at].to(torch.int32)
        token[rand(*steps) < 0.01] = -1                     # padding inside a sample
        s["token"], s["scale"] = token, D ** 0.5
        if kind == "lookup":
            s["W"] = (randn(V, D) / D ** 0.5).to(TYPES[case["table"]])
        else:
            s["grad"] = randn(*steps, D).to(dt)
        return s
    s["x"] = randn(*steps, D).to(dt)
    train = kind.endswith("train")
    if train:
        s["grad_y"] = randn(*steps, D).to(dt)
    if kind.startswith("conv"):
        K = case["K"]
        s["w"], s["bias"] = randn(D, K) / K ** 0.5, randn(D) * 0.1
        if kind == "conv_step":
            s["state"] = randn(case["slots"], K - 1, D).to(dt)
        else:
            s["x_first"] = randn(B, K - 1, D).to(dt)
            if train:
                s["grad_last"] = randn(B, K - 1, D)
        return s
    N, G = case["N"], case["G"]
    # time constants of 1 to 1000 steps: delta around 0.001 .. 0.1, A around -1 .. -N
    delta = torch.exp(rand(D) * math.log(100.0) + math.log(0.001))
    s["dt_bias"] = torch.log(torch.expm1(delta))
    s["dt"] = (randn(*steps, D) * 0.5).to(dt)
    s["A"] = -torch.arange(1, N + 1, device=DEV) * torch.exp(0.1 * randn(D, N))
    s["Bm"], s["C"] = randn(*steps, G, N).to(dt), (randn(*steps, G, N) / N ** 0.5).to(dt)
    s["skip"], s["z"] = randn(D), randn(*steps, D).to(dt)
    if kind == "select_step":
        s["state"] = randn(case["slots"], D, N) * 0.1
    else:
        s["h_first"] = randn(B, D, N) * 0.1
        if train:
            s["grad_last"] = randn(B, D, N)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    import paper_2603_13283_amd as lif
    kind = s["kind"]
    if kind == "lookup":
        return {"out": lif.embed(s["token"], s["W"], scale=s["scale"], length=s["length"], dtype=TYPES[s["dtype"]])}
    if kind == "lookup_grad":
        return {"grad_W": lif.embed_backward(s["token"], s["grad"], s["V"], scale=s["scale"], length=s["length"])}
    if kind == "conv_step":
        y = lif.causal_conv_step(s["x"], s["w"], s["state"], slot=s["slot"], bias=s["bias"])
        return {"y": y, "state": s["state"]}
    if kind in ("conv", "conv_train"):
        kw = dict(bias=s["bias"], length=s["length"], x_first=s["x_first"])
        o = lif.causal_conv(s["x"], s["w"], **kw)
        out = {"y": o.y, "x_last": o.x_last}
        if kind == "conv_train":
            g = lif.causal_conv_backward(s["x"], s["w"], s["grad_y"], grad_last=s["grad_last"], **kw)
            out.update(grad_x=g.x, grad_w=g.w, grad_bias=g.bias, grad_x_first=g.x_first)
        return out
    args = (s["x"], s["dt"], s["A"], s["Bm"], s["C"])
    kw = dict(D=s["skip"], z=s["z"], dt_bias=s["dt_bias"])
    if kind == "select_step":
        return {"y": lif.selective_step(*args, s["state"], slot=s["slot"], **kw), "state": s["state"]}
    o = lif.selective_scan(*args, length=s["length"], h_first=s["h_first"], marks=kind == "select_train", **kw)
    out = {"y": o.y, "h_last": o.h_last}
    if kind == "select_train":
        g = lif.selective_scan_backward(*args, o.marks, s["grad_y"], grad_last=s["grad_last"], length=s["length"], **kw)
        out.update(grad_x=g.x, grad_dt=g.dt, grad_A=g.A, grad_B=g.B, grad_C=g.C, grad_skip=g.D, grad_z=g.z,
                   grad_dt_bias=g.dt_bias, grad_h_first=g.h_first)
    return out


def run_plain(s):
    kind = s["kind"]
    if kind in ("lookup", "lookup_grad"):
        token = s["token"].long()
        there = (token >= 0) & valid(s) if s["length"] is not None else token >= 0
        if kind == "lookup":
            rows = s["W"].float()[token.clamp(min=0)] * s["scale"]
            return {"out": torch.where(there[..., None], rows, 0.0).to(TYPES[s["dtype"]])}
        rows = torch.where(there[..., None], s["grad"].float(), 0.0).view(-1, s["D"])
        grad = torch.zeros(s["V"], s["D"], device=DEV)
        return {"grad_W": grad.index_add_(0, token.clamp(min=0).view(-1), rows) * s["scale"]}
    if kind.startswith("conv"):
        return plain_conv(s)
    return plain_select(s)


def valid(s):
    """[B, T]: the steps before each sample's length."""
    return torch.arange(s["T"], device=DEV)[None, :] < s["length"][:, None]


def plain_conv(s):
    x, w, bias, K, dt = s["x"].float(), s["w"], s["bias"], s["K"], s["x"].dtype
    if s["kind"] == "conv_step":
        at = s["slot"].long()
        seen = torch.cat([s["state"][at].float(), x[:, None]], dim=1)
        c = bias + (seen * w.t()).sum(dim=1)
        s["state"][at] = seen[:, 1:].to(dt)
        return {"y": (c * torch.sigmoid(c)).to(dt), "state": s["state"]}
    T = s["T"]
    seen = torch.cat([s["x_first"].float(), x], dim=1)              # x_t is at t + K - 1
    c = bias + sum(w[:, j] * seen[:, j:j + T] for j in range(K))
    y = c * torch.sigmoid(c)
    n = torch.full((s["B"],), T, device=DEV) if s["length"] is None else s["length"].long()
    tail = (n[:, None] + torch.arange(K - 1, device=DEV))[:, :, None].expand(-1, -1, s["D"])
    on = None if s["length"] is None else valid(s)[:, :, None]
    if on is not None:
        y = torch.where(on, y, 0.0)
    out = {"y": y.to(dt), "x_last": seen.gather(1, tail).to(dt)}
    if s["kind"] == "conv":
        return out
    sg = torch.sigmoid(c)
    gc = s["grad_y"].float() * sg * (1.0 + c * (1.0 - sg))
    if on is not None:
        gc = torch.where(on, gc, 0.0)
    gs = torch.zeros_like(seen).scatter_(1, tail, s["grad_last"])
    for j in range(K):
        gs[:, j:j + T] += w[:, j] * gc
    gw = torch.stack([(gc * seen[:, j:j + T]).sum(dim=(0, 1)) for j in range(K)], dim=1)
    return {**out, "grad_x": gs[:, K - 1:].to(dt), "grad_w": gw, "grad_bias": gc.sum(dim=(0, 1)),
            "grad_x_first": gs[:, :K - 1]}


def scan(a, u, first):
    """All h_t = a_t h_{t-1} + u_t over axis 1: the same place of all blocks of
    about sqrt(T) steps at once, then the blocks one after the other."""
    B, T = a.shape[:2]
    Q = max(1, math.isqrt(T))
    S = -(-T // Q)
    h, p = torch.zeros_like(u), torch.ones_like(a)                   # from 0, and the decay since the block began
    for i in range(Q):
        n = -(-(T - i) // Q)                                         # blocks that have a place i
        h[:, i::Q] = u[:, i::Q] if i == 0 else a[:, i::Q] * h[:, i - 1::Q][:, :n] + u[:, i::Q]
        p[:, i::Q] = a[:, i::Q] if i == 0 else a[:, i::Q] * p[:, i - 1::Q][:, :n]
    carry = first
    for k in range(S):
        part = slice(k * Q, min((k + 1) * Q, T))
        h[:, part] += p[:, part] * carry[:, None]
        carry = h[:, part.stop - 1]
    return h


def plain_select(s):
    dt, G, D, N = s["x"].dtype, s["G"], s["D"], s["N"]
    x, z, raw = s["x"].float(), s["z"].float(), s["dt"].float() + s["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    Bd, Cd = (s[k].float().repeat_interleave(D // G, dim=-2) for k in ("Bm", "C"))
    gate = z * torch.sigmoid(z)
    if s["kind"] == "select_step":
        at = s["slot"].long()
        h = torch.exp(delta[..., None] * s["A"]) * s["state"][at] + (delta * x)[..., None] * Bd
        s["state"][at] = h
        return {"y": (((Cd * h).sum(dim=-1) + s["skip"] * x) * gate).to(dt), "state": s["state"]}
    on = None if s["length"] is None else valid(s)[:, :, None]
    if on is not None:
        delta = torch.where(on, delta, 0.0)                          # e^0 = 1, no input: the state stays
    a = torch.exp(delta[..., None] * s["A"])
    h = scan(a, (delta * x)[..., None] * Bd, s["h_first"])
    y0 = (Cd * h).sum(dim=-1) + s["skip"] * x
    shown = y0 * gate if on is None else torch.where(on, y0 * gate, 0.0)
    out = {"y": shown.to(dt), "h_last": h[:, -1].clone()}
    if s["kind"] == "select":
        return out
    gy = s["grad_y"].float() if on is None else torch.where(on, s["grad_y"].float(), 0.0)
    sg = torch.sigmoid(z)
    gz = gy * y0 * sg * (1.0 + z * (1.0 - sg))
    g = gy * gate
    u = g[..., None] * Cd
    u[:, -1] += s["grad_last"]
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], dim=1)
    lam = scan(after.flip(1), u.flip(1), torch.zeros_like(s["h_first"])).flip(1)
    del u, after
    B, T = x.shape[:2]
    per_group = lambda v: v.view(B, T, G, D // G, N).sum(dim=3)                              # noqa: E731
    gC = per_group(g[..., None] * h)
    gB = per_group(lam * (delta * x)[..., None])
    q = lam * a * torch.cat([s["h_first"][:, None], h[:, :-1]], dim=1)
    into = (lam * Bd).sum(dim=-1)
    gdelta = (s["A"] * q).sum(dim=-1) + x * into
    graw = gdelta * torch.sigmoid(raw)
    gx = delta * into + s["skip"] * g
    if on is not None:
        graw = torch.where(on, graw, 0.0)
    return {**out, "grad_x": gx.to(dt), "grad_dt": graw.to(dt), "grad_A": (delta[..., None] * q).sum(dim=(0, 1)),
            "grad_B": gB.to(dt), "grad_C": gC.to(dt), "grad_skip": (g * x).sum(dim=(0, 1)), "grad_z": gz.to(dt),
            "grad_dt_bias": graw.sum(dim=(0, 1)), "grad_h_first": a[:, 0] * lam[:, 0]}


# ---------------------------------------------------------------------------
# the same in 64 bits, step by step from the definitions
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("lookup", "lookup_grad"):
        return exact_lookup(s)
    if kind.startswith("conv"):
        return exact_conv(s)
    if kind == "select_train" and case["T"] > 20000:
        return None                                                  # a step of both directions at a time: too long
    return exact_select(s)


def steps_of(s):
    """Each sample's steps, on the host."""
    return [s["T"]] * s["B"] if s["length"] is None else s["length"].tolist()


def exact_lookup(s):
    token = s["token"].long().clone()
    for b, n in enumerate(steps_of(s)):
        token[b, n:] = -1
    picked = (token.view(-1) >= 0).nonzero()[:, 0]
    ids = token.view(-1)[picked]
    if s["kind"] == "lookup":
        out = torch.zeros(token.numel(), s["D"], dtype=F64, device=DEV)
        out[picked] = s["W"].to(F64)[ids] * s["scale"]
        return {"out": out.view(*token.shape, s["D"])}
    grad = torch.zeros(s["V"], s["D"], dtype=F64, device=DEV)
    grad.index_put_((ids,), s["grad"].view(-1, s["D"])[picked].to(F64) * s["scale"], accumulate=True)
    return {"grad_W": grad}


def exact_conv(s):
    w, bias, K, D = s["w"].to(F64), s["bias"].to(F64), s["K"], s["D"]
    if s["kind"] == "conv_step":
        state, ys = s["state"].to(F64), []
        for i, r in enumerate(s["slot"].tolist()):
            seen = torch.cat([state[r], s["x"][i:i + 1].to(F64)])
            c = bias + torch.einsum("kd,dk->d", seen, w)
            ys.append(c / (1.0 + torch.exp(-c)))
            state[r] = seen[1:]
        return {"y": torch.stack(ys), "state": state}
    train = s["kind"] == "conv_train"
    y = torch.zeros(s["B"], s["T"], D, dtype=F64, device=DEV)
    last = torch.zeros(s["B"], K - 1, D, dtype=F64, device=DEV)
    gx, g0 = torch.zeros_like(y), torch.zeros_like(last)
    gw, gb = torch.zeros_like(w), torch.zeros_like(bias)
    for b, n in enumerate(steps_of(s)):
        seen = torch.cat([s["x_first"][b], s["x"][b, :n]]).to(F64)
        last[b] = seen[n:]
        seg = seen.unfold(0, K, 1)[:n] if n else seen.new_zeros(0, D, K)      # [n, D, K]
        c = (seg * w).sum(dim=-1) + bias
        y[b, :n] = c / (1.0 + torch.exp(-c))
        if train:
            e = torch.exp(-c)
            gc = s["grad_y"][b, :n].to(F64) * ((1.0 + e + c * e) / (1.0 + e) ** 2)
            gw += (seg * gc[:, :, None]).sum(dim=0)
            gb += gc.sum(dim=0)
            gs = torch.zeros_like(seen)
            gs[n:] += s["grad_last"][b].to(F64)
            for j in range(K):
                gs[j:j + n] += gc * w[:, j]
            gx[b, :n], g0[b] = gs[K - 1:], gs[:K - 1]
    out = {"y": y, "x_last": last}
    return {**out, "grad_x": gx, "grad_w": gw, "grad_bias": gb, "grad_x_first": g0} if train else out


def exact_select(s):
    B, D, G, N = s["B"], s["D"], s["G"], s["N"]
    A, skip = s["A"].to(F64), s["skip"].to(F64)
    of = torch.arange(D, device=DEV) // (D // G)                     # a channel's group

    x, z, raw = s["x"].to(F64), s["z"].to(F64), s["dt"].to(F64) + s["dt_bias"].to(F64)
    delta = torch.log1p(torch.exp(-raw.abs())) + raw.clamp(min=0)
    Bm, C = s["Bm"].to(F64), s["C"].to(F64)
    ez = torch.exp(-z)
    gate = z / (1.0 + ez)
    if s["kind"] == "select_step":
        state = s["state"].to(F64)
        rows = s["slot"].long()
        h = torch.exp(delta[..., None] * A) * state[rows] + (delta * x)[..., None] * Bm[:, of]
        state[rows] = h
        return {"y": ((h * C[:, of]).sum(dim=-1) + skip * x) * gate, "state": state}
    T, train = s["T"], s["kind"] == "select_train"
    n = torch.tensor(steps_of(s), device=DEV)
    on = (torch.arange(T, device=DEV) < n[:, None])[:, :, None]
    delta, u = delta * on, delta * x * on                            # past the length: a = 1, nothing comes in
    h = s["h_first"].to(F64)
    y0 = torch.zeros(B, T, D, dtype=F64, device=DEV)
    hs = torch.zeros(T + 1, B, D, N, dtype=F64, device=DEV) if train else None
    if train:
        hs[0] = h
    for t in range(T):
        h = torch.exp(delta[:, t, :, None] * A) * h + u[:, t, :, None] * Bm[:, t][:, of]
        y0[:, t] = (h * C[:, t][:, of]).sum(dim=-1)
        if train:
            hs[t + 1] = h
    y0 += skip * x
    out = {"y": y0 * gate * on, "h_last": h}
    if not train:
        return out
    gy = s["grad_y"].to(F64) * on
    gz = gy * y0 * (1.0 + ez + z * ez) / (1.0 + ez) ** 2
    g = gy * gate
    into, fall = (torch.zeros(B, T, D, dtype=F64, device=DEV) for _ in range(2))
    gB, gC = (torch.zeros(B, T, G, N, dtype=F64, device=DEV) for _ in range(2))
    gA, lam = torch.zeros_like(A), s["grad_last"].to(F64)
    for t in reversed(range(T)):
        gt, dt_, Bt = g[:, t, :, None], delta[:, t, :, None], Bm[:, t][:, of]
        lam = lam + gt * C[:, t][:, of]
        gC[:, t].index_add_(1, of, gt * hs[t + 1])
        gB[:, t].index_add_(1, of, lam * u[:, t, :, None])
        into[:, t] = (lam * Bt).sum(dim=-1)
        lam = lam * torch.exp(dt_ * A)
        da = lam * hs[t]
        fall[:, t] = (da * A).sum(dim=-1)
        gA += (da * dt_).sum(dim=0)
    graw = (fall + into * x) / (1.0 + torch.exp(-raw)) * on
    return {**out, "grad_x": into * delta + g * skip, "grad_dt": graw, "grad_A": gA, "grad_B": gB, "grad_C": gC,
            "grad_skip": (g * x).sum(dim=(0, 1)), "grad_z": gz, "grad_dt_bias": graw.sum(dim=(0, 1)),
            "grad_h_first": lam}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once (of a table the rows
    that can be met), and the operations of the formulas (an exponential, a
    logarithm or a quotient counts as one).  Ragged samples count as whole."""
    e, B, D, kind = SIZE[case["dtype"]], case["B"], case["D"], case["kind"]
    rows = B * case.get("T", 1)
    n = rows * D
    if kind == "lookup":
        return {"bytes": n * e + 4 * rows + min(rows, case["V"]) * D * SIZE[case["table"]], "flops": n}
    if kind == "lookup_grad":
        return {"bytes": n * e + 4 * rows + 4 * case["V"] * D, "flops": n}
    if kind.startswith("conv"):
        K = case["K"]
        edge = (K - 1) * B * D
        if kind == "conv_step":
            return {"bytes": n * 2 * e + 2 * edge * e + 4 * (K + 1) * D + 4 * B, "flops": (2 * K + 4) * n}
        if kind == "conv":
            return {"bytes": n * 2 * e + 2 * edge * e + 4 * (K + 1) * D, "flops": (2 * K + 4) * n}
        return {"bytes": n * 5 * e + edge * (3 * e + 8) + 12 * (K + 1) * D, "flops": (8 * K + 12) * n}
    N, G = case["N"], case["G"]
    bc, states, params = rows * G * N * e, B * D * N * 4, 4 * D * (N + 2)
    if kind in ("select", "select_step"):
        return {"bytes": n * 4 * e + 2 * bc + 2 * states + params, "flops": n * (7 * N + 8)}
    return {"bytes": n * 11 * e + 6 * bc + 4 * states + 3 * params, "flops": n * (27 * N + 30)}
