"""The gated leaky integrator at the shapes where a lane takes several
channels: four 16-bit ones, two, two on a time axis that is shared out, widths
that the channels of a lane do not divide, and the four-channel step.  Checks
and tolerances are those of test_gpu_gated."""
import numpy as np
import pytest

import test_gpu_gated as gated
from test_gpu_gated import _inputs, env       # noqa: F401

ELEM = {"f32": 4, "bf16": 2, "f16": 2}


def plan_of(B, T, D, dtype, back=False):
    """(channels a lane, segments of the time axis)."""
    e, blocks = ELEM[dtype], -(-T // 64)
    columns = lambda c: -(-B * -(-D // c) // 64)                                   # noqa: E731
    split = blocks >= 8 and B * D * e < (36 << 10) * min(blocks, 16) // 16
    c = 1 if back else 2 if e == 4 else 4
    while c > 1:
        if D >= c and (c == 2 and columns(2) * (blocks // 2) >= 1024 if split else
                       columns(c) >= (512 if c == 4 else 256 if e == 4 else 150)):
            break
        c //= 2
    S = min(-(-1024 // columns(c)), blocks // 2) if split else 1
    per = -(-blocks // S) if blocks else 1
    return c, -(-blocks // per) if blocks else 1


# samples, steps, channels, type -> channels a lane, whether the time axis is shared out
CASES = [(512, 20, 260, "bf16", 4, False), (512, 20, 263, "bf16", 4, False), (300, 40, 513, "f16", 4, False),
         (70, 130, 1999, "bf16", 4, False),
         (96, 70, 701, "bf16", 2, False), (96, 70, 701, "f32", 2, False), (40, 600, 1025, "f32", 2, False),
         (1, 4200, 4099, "bf16", 2, True), (4, 2200, 2047, "f16", 2, True), (1, 4200, 4097, "f32", 2, True),
         (2, 16600, 512, "bf16", 2, True)]


def test_cases_are_what_they_say():
    import paper_2603_13283_amd as lif
    for B, T, D, dtype, cpl, split in CASES:
        c, S = plan_of(B, T, D, dtype)
        assert (c, S > 1) == (cpl, split), (B, T, D, dtype)
        p = lif.lif_gated_params(B, T, D, {"f32": 0, "bf16": 1, "f16": 2}[dtype], 1, 0, *(6 * [0]))
        S = max(S, plan_of(B, T, D, dtype, True)[1])
        assert lif.lif_gated_scan_workspace_size(p) == (S * B * D * 8 if S > 1 else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,D,dtype,cpl,split", CASES)
def test_scan(env, B, T, D, dtype, cpl, split):                                    # noqa: F811
    """Whole and ragged samples, with slow leaks that carry states (and
    adjoints) over many tiles and segments."""
    torch, _ = env
    x, f, gh, h0, gl = _inputs(env, B, T, D, dtype, B + T + D, shift=6.0 if split else 2.0, spread=1.0)
    gated.run(env, x, f, dtype, h0=h0, gh=gh, gl=gl, label="channels of a lane")
    r = np.random.default_rng(D)
    n = r.integers(0, T + 1, B)
    n[0] = T - 17 if B == 1 else T
    if B > 3:
        n[1], n[2], n[3] = 0, 1, T // 2
    for b in range(B):
        x[b, n[b]:], f[b, n[b]:], gh[b, n[b]:] = float("nan"), float("inf"), float("nan")
    o, _ = gated.run(env, x, f, dtype, n=n, h0=h0, gh=gh, gl=gl, coupled=False, label="ragged")
    for b in range(B):
        assert not o.h[b, n[b]:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,D,dtype", [(512, 20, 263, "bf16"), (96, 70, 701, "f32"), (1, 4200, 4099, "bf16")])
def test_strides_give_the_same_bits(env, B, T, D, dtype):                          # noqa: F811
    torch, lif = env
    x, f, gh, h0, gl = _inputs(env, B, T, D, dtype, 5)

    def go(x, f, gh):
        o = lif.gated_scan(x, f, h_first=h0, marks=True)
        return (o.h, o.h_last, o.marks, *lif.gated_scan_backward(x, f, o.marks, gh, grad_last=gl))
    want = go(x, f, gh)
    turn = lambda v: v.transpose(0, 1).contiguous().transpose(0, 1)                # noqa: E731

    def off(v):                                        # inside a wider tensor, off the grid
        wide = torch.full((B, T + 3, D + 5), float("nan"), dtype=v.dtype, device="cuda:0")
        return wide[:, 2:T + 2, 3:D + 3].copy_(v)
    for args in ((turn(x), f, turn(gh)), (off(x), turn(f), gh), (x, f, off(gh))):
        print(f"[case] strides B={B} T={T} D={D} {dtype}", flush=True)
        for p, q in zip(want, go(*args)):
            assert torch.equal(p, q)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,D,slots", [(256, 1024, 256), (300, 1028, 400), (65, 4096, 70)])
def test_step_of_four_channels(env, B, D, slots, dtype):                           # noqa: F811
    assert D % 4 == 0 and B * D >= 4 * 256 * 256
    torch, lif = env
    gated.test_step(env, B, D, slots, dtype)
    # rows of a wider tensor, off the grid of 16 bytes
    x, f, _, _, _ = _inputs(env, 1, B, D, dtype, 3)
    state = torch.randn(slots, D, device="cuda:0")
    slot = torch.randperm(slots, device="cuda:0")[:B].to(torch.int32)
    a, b = state.clone(), state.clone()
    wide = torch.full((B, D + 7), float("nan"), dtype=x.dtype, device="cuda:0")
    view = wide[:, 3:D + 3]
    h = lif.gated_step(x[0], f[0], a, slot=slot)
    assert torch.equal(h, lif.gated_step(view.copy_(x[0]), f[0], b, slot=slot)) and torch.equal(a, b)
