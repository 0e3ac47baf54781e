"""Distillation from a teacher's list (lif_distill_top) where float32 would
run out of range or depend on an order, against the float64 reference.  Every
case runs on the three ways a row can take: staged in LDS (V <= 256), held by
one workgroup (many rows), and cut into segments (few rows).

Tolerances are those of test_gpu_rows.run_distill unless a test says
otherwise."""
import numpy as np
import pytest

from test_gpu_rows import _logits, env, run_distill       # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
#         rows, logits: LDS with 2, 4 and 16 lanes a row; one workgroup of 256, 512, 512 and 1024 threads; segments
PLACES = [(5, 20), (6, 64), (4, 200), (256, 4100), (256, 20011), (256, 40009), (256, 70001), (3, 20011), (3, 300000)]


def _repeat(torch, x, R):
    """x's rows over and over, R in all."""
    return x[torch.arange(R, device=x.device) % x.shape[0]].contiguous()


def run_repeated(env, x, lp, idx, dtype, R, T=1.0, tail=False, weight=None, label=""):
    """run_distill on a few rows for the reference's values, then the call of
    R rows that holds them over and over: every one has to be the few's."""
    torch, lif = env
    n = x.shape[0]
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device="cuda:0")[np.arange(R) % n].contiguous()  # noqa: E731
    big = _repeat(torch, x, R)
    print(f"[case] {label} R={R} V={x.shape[1]} k={idx.shape[1]} T={T} tail={tail} {dtype}", flush=True)
    loss, grad = lif.distill_top(big, dev(lp, torch.float32), dev(idx, torch.int32), temperature=T, tail=tail,
                                 weight=None if weight is None else dev(weight, torch.float32))
    torch.cuda.synchronize()
    for r in range(n, R):
        assert torch.equal(grad[r], grad[r % n]) or torch.isnan(grad[r % n]).any(), f"{label}: row {r}"
    assert torch.equal(loss[n:].nan_to_num(7.0), loss[torch.arange(n, R) % n].nan_to_num(7.0)), label

    class First:                                  # run_distill's checks on the rows of the large call
        LifError = lif.LifError

        @staticmethod
        def distill_top(*a, **k):
            return loss[:n], grad[:n]
    return run_distill((torch, First), x, lp, idx, dtype, T, tail, weight, label)


@pytest.mark.parametrize("R,V", PLACES)
def test_lists_of_unlikely_classes(env, R, V):
    """Classes whose probabilities lie below float32's range: made to sum to 1
    they teach as any others do, and as a part of all mass they leave it to
    the tail."""
    torch, _ = env
    n, k = min(R, 3), 6
    x = _logits(env, n, V, "f32", V)
    r = np.random.default_rng(V)
    idx = np.stack([r.permutation(V)[:k] for _ in range(n)]).astype(np.int32)
    # subnormal in float32, 0 in float32, 0 in float64
    lp = np.stack([-r.uniform(a, b, k) for a, b in ((90.0, 104.0), (110.0, 130.0), (800.0, 820.0))])
    lp = lp[:n].astype(np.float32)
    for tail in (False, True):
        loss, grad = run_repeated(env, x, lp, idx, "f32", R, 1.0, tail, label="unlikely classes")
        assert (loss > 0).all() and grad.any(1).all()
