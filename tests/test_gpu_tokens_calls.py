"""Calls of the operators over tokens that the other tests do not make: steps of
convolutions whose width is no multiple of a vector's, masked steps, the widest
and longest calls, growing states; tolerances by running error analysis
(tests/rounding.py)."""
import numpy as np
import pytest

import test_gpu_conv as conv
from rounding import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2603_13283_amd as lif
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    lif.load()
    return torch, lif


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nb,W,K", [(300, 33, 8), (512, 33, 4), (1, 257, 4), (64, 257, 2), (8, 1001, 4), (512, 1001, 3),
                                    (1, 2049, 4), (130, 2049, 8), (5, 2050, 4), (300, 7, 2), (300, 6, 5)])
def test_step_widths(env, nb, W, K, dtype):
    """Streams whose last channels lie in another wave or workgroup than those
    before them: outputs and states by the formula, repeated steps too."""
    torch, lif = env
    print(f"[case] conv step {nb} x {W} K={K} {dtype}", flush=True)
    v = conv.make(torch, (nb, 6, W, K), dtype, seed=W)
    state = v["x_first"].clone()
    ys = [lif.causal_conv_step(v["x"][:, t], v["w"], state, bias=v["bias"]) for t in range(6)]
    want = conv.reference({k: conv.arr(t) for k, t in v.items()}, np.full(nb, 6))
    check(conv.arr(torch.stack(ys, 1)), want["y"], dtype, "y")
    assert np.array_equal(conv.arr(state), want["x_last"])
