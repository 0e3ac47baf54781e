"""Many long rows (lif_token_logprobs, lif_distill_top): every workgroup shape
that holds a row whole, and segments of many rows, which calls with few rows
never take.  A few distinct rows are repeated over the call: the first ones go
through the checks of test_gpu_rows, all others have to have the same bits."""
import numpy as np
import pytest

import test_gpu_rows as rows
from test_gpu_rows import _dt, _logits, env       # noqa: F401

SHAPES = [(64, 4), (256, 4), (512, 8), (512, 16), (1024, 16)]        # threads, vectors of 16 bytes a thread
ELEM = {"f32": 4, "bf16": 2, "f16": 2}


def shape_of(R, V, dtype):
    """(threads, vectors, segments) that a row takes; (0, 0, 1) staged in LDS."""
    if V <= 256:
        return 0, 0, 1
    vec = 16 // ELEM[dtype]
    holds = [t * n * vec for t, n in SHAPES]
    seg = V if V <= holds[-1] else holds[2]
    if R <= 64 and seg > 4096 * vec:
        seg = min(seg, max(512 * vec, -(-V // -(-512 // R))))
    n = -(-V // seg)
    seg = -(-V // n)
    seg = -(-seg // vec) * vec
    n = -(-V // seg)
    t, v = next(s for s, h in zip(SHAPES, holds) if h >= seg)
    return t, v, n


# rows of the call, logits, type -> the shape: at, below and above what each shape holds, odd lengths
CASES = [(256, 300, "f32", (64, 4, 1)), (256, 1024, "f32", (64, 4, 1)), (256, 1025, "f32", (256, 4, 1)),
         (256, 4096, "f32", (256, 4, 1)), (256, 4097, "f32", (512, 8, 1)), (257, 16383, "f32", (512, 8, 1)),
         (256, 16385, "f32", (512, 16, 1)), (256, 32768, "f32", (512, 16, 1)), (256, 32769, "f32", (1024, 16, 1)),
         (256, 65533, "f32", (1024, 16, 1)), (256, 65537, "f32", (512, 8, 5)), (64, 60001, "f32", (512, 8, 8)),
         (65, 60001, "f32", (1024, 16, 1)), (10, 16385, "f32", (256, 4, 9)), (10, 16384, "f32", (512, 8, 1)),
         (256, 2049, "bf16", (256, 4, 1)), (256, 8192, "f16", (256, 4, 1)), (256, 8193, "bf16", (512, 8, 1)),
         (300, 32767, "f16", (512, 8, 1)), (256, 32769, "f16", (512, 16, 1)), (256, 50021, "bf16", (512, 16, 1)),
         (256, 65536, "bf16", (512, 16, 1)), (256, 65537, "f16", (1024, 16, 1)), (256, 131071, "bf16", (1024, 16, 1)),
         (256, 131073, "f16", (512, 8, 5)), (64, 100003, "bf16", (512, 8, 8)), (65, 100003, "bf16", (1024, 16, 1)),
         (10, 32769, "f16", (256, 4, 9)), (10, 32768, "f16", (512, 8, 1))]


def test_cases_reach_every_shape():
    """The cases are what they say, by the rule and by the library's own count
    of segments (its workspace); each type class reaches each shape whole."""
    import paper_2603_13283_amd as lif
    for R, V, dtype, want in CASES:
        assert shape_of(R, V, dtype) == want, (R, V, dtype)
        p = lif.lif_rows_params(R, V, 0, {"f32": 0, "bf16": 1, "f16": 2}[dtype], V, V, 1.0, 0, 0)
        assert lif.lif_rows_workspace_size(p) == (16 * R * want[2] if want[2] > 1 else 0)
    for some in (("f32",), ("bf16", "f16")):
        whole = {w[:2] for _, _, d, w in CASES if d in some and w[2] == 1}
        assert whole >= set(SHAPES[1:])


class Repeated:
    """The library with every call's rows repeated to R; returns the first."""

    def __init__(self, torch, lif, R):
        self.torch, self.lif, self.R, self.LifError = torch, lif, R, lif.LifError

    def _all(self, v):
        return None if v is None else v[self.torch.arange(self.R, device=v.device) % v.shape[0]].contiguous()

    def _first(self, v, n):
        if v is None:
            return None
        bits = v.view(self.torch.int16 if v.element_size() == 2 else self.torch.int32)
        whole = bits[:bits.shape[0] // n * n].reshape(-1, n, *bits.shape[1:])
        assert (whole == whole[:1]).all() and self.torch.equal(bits[whole.shape[0] * n:], bits[:bits.shape[0] % n])
        return v[:n]

    def token_logprobs(self, x, tokens=None, k=0, temperature=1.0, grad_logp=None, grad_entropy=None):
        print(f"[case] repeated to R={self.R}", flush=True)
        o = self.lif.token_logprobs(self._all(x), self._all(tokens), k=k, temperature=temperature,
                                    grad_logp=self._all(grad_logp), grad_entropy=self._all(grad_entropy))
        return type(o)(*(self._first(v, x.shape[0]) for v in (o.logp, o.entropy, o.lse, o.top_logp, o.top_idx, o.grad)))

    def distill_top(self, x, lp, idx, temperature=1.0, tail=False, weight=None):
        print(f"[case] repeated to R={self.R}", flush=True)
        loss, grad = self.lif.distill_top(self._all(x), self._all(lp), self._all(idx), temperature=temperature,
                                          tail=tail, weight=self._all(weight))
        return self._first(loss, x.shape[0]), self._first(grad, x.shape[0])


@pytest.fixture()
def many(env):                                                                     # noqa: F811
    return lambda R: (env[0], Repeated(*env, R))


@pytest.mark.gpu
@pytest.mark.parametrize("R,V,dtype,shape", CASES)
def test_logprobs_and_distillation(many, R, V, dtype, shape):
    e = many(R)
    rows.test_logprobs_widths(e, V, dtype)
    rows.test_distill_widths(e, V, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("R,V,dtype", [(266, 3000, "f32"), (266, 5001, "bf16"), (266, 9001, "f32"),
                                       (266, 20011, "bf16"), (266, 30011, "f32"), (266, 50021, "bf16"),
                                       (266, 50021, "f16"), (266, 65533, "f32"), (266, 100003, "bf16"),
                                       (266, 100003, "f16"), (266, 70001, "f32"), (266, 140001, "bf16")])
def test_masks_ties_and_rows_that_are_not_finite(many, R, V, dtype):
    rows.test_masks_ties_and_rows_that_are_not_finite(many(R), V, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1000, 4000, 9001, 20011, 40009, 140001])
def test_teacher_lists(many, V):
    rows.test_teacher_lists(many(256), V)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5003, 9001, 20011, 50021, 65533])
def test_ties_over_whole_rows(many, env, V, dtype):                                # noqa: F811
    """More equal or ordered logits than the list of candidates holds, and rows
    masked to a few spread over all threads: the k-th largest is found by
    halving, equal ones fill up by index."""
    torch, _ = env
    e = many(256)
    x = torch.stack([torch.zeros(V), torch.randn(V, generator=torch.Generator().manual_seed(V)).round(),
                     torch.arange(V).flip(0) / 8.0, torch.arange(V) // 700 * 1.0,
                     torch.where(torch.arange(V) % 499 == 7, 1.0, -float("inf")),
                     torch.where(torch.arange(V) < 600, 2.0, 1.0)]).to(_dt(torch, dtype)).cuda()
    for k in (128, 20, 1):
        rows.run_logprobs(e, x, dtype, np.array([5, 0, V - 1, 7, 7, 600]), k, label="whole rows")


@pytest.mark.gpu
@pytest.mark.parametrize("V,dtype", [(4099, "f32"), (30011, "f32"), (60013, "f32"), (5003, "bf16"), (30011, "f16"),
                                     (50021, "bf16"), (100003, "bf16"), (50022, "bf16"), (140001, "f16")])
def test_strides_and_alignment(env, V, dtype):                                     # noqa: F811
    """Padded rows, rows off the vector grid, a view that starts off it: the
    same bits."""
    torch, lif = env
    R, k = 256, 30
    x = _logits(env, R, V, dtype, 14)
    g = torch.randn(R, device="cuda:0")
    tok = torch.randint(0, V, (R,), device="cuda:0", dtype=torch.int32)
    o = lif.token_logprobs(x, k=k)
    lp, idx = o.top_logp - 0.1, torch.roll(o.top_idx, 1, 0).contiguous()

    def go(v):
        o = lif.token_logprobs(v, tok, k=k, grad_logp=g, grad_entropy=g)
        return (o.logp, o.entropy, o.lse, o.top_logp, o.top_idx, o.grad, *lif.distill_top(v, lp, idx, tail=True))
    want = go(x)
    for pad, lead in ((0, 1), (3, 0), (5, 7), (8, 8)):
        print(f"[case] many rows V={V} {dtype} pad={pad} lead={lead}", flush=True)
        wide = torch.full((R, lead + V + pad), float("nan"), dtype=x.dtype, device="cuda:0")
        view = wide[:, lead:lead + V]
        view.copy_(x)
        for p, q in zip(want, go(view)):
            assert torch.equal(p, q), (pad, lead)
