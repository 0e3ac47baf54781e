"""The sequence head on sequences that go on in pieces, on counts of other
types and on sequences of nothing."""
import pytest

from test_gpu_sequence import GRAD_RTOL, env       # noqa: F401

pytestmark = pytest.mark.gpu


def _head(env, N=9, D=14, K=6, seed=4):                                            # noqa: F811
    from paper_2603_13283_amd.sequence import SequenceHead
    torch, _ = env
    g = torch.Generator().manual_seed(seed)
    counts = torch.poisson(torch.full((3, 150, N), 0.4), generator=g).cuda()
    return SequenceHead.random(N, D, K, seed=seed), counts, torch.randn(3 * 150, K, generator=g).cuda()


def test_pieces_of_a_sequence_have_its_gradients(env):                             # noqa: F811
    """Forward in two pieces, the second from the first's last state; backward
    from the second, whose gradient to its first state enters the first as
    that of its last state: the sums are the whole sequence's gradients."""
    torch, _ = env
    head, counts, gl = _head(env)
    B, T, cut = 3, 150, 70
    length = torch.tensor([150, 40, 101], dtype=torch.int32, device="cuda:0")
    whole = head.forward(counts, length, train=True)
    want = head.backward(counts, whole, gl, length)
    parts = (counts[:, :cut], counts[:, cut:])
    lens = (length.clamp(max=cut), (length - cut).clamp(min=0))
    gls = [v.reshape(-1, gl.shape[1]) for v in gl.view(B, T, -1).split([cut, T - cut], 1)]
    a = head.forward(parts[0], lens[0], train=True)
    b = head.forward(parts[1], lens[1], h_first=a.h_last, train=True)
    gb = head.backward(parts[1], b, gls[1], lens[1], h_first=a.h_last)
    ga = head.backward(parts[0], a, gls[0], lens[0], grad_last=gb["h_first"])
    assert "h_first" not in ga and "h_first" not in want
    for k in want:
        got = ga[k] + gb[k]
        assert (got - want[k]).norm() <= GRAD_RTOL * want[k].norm(), k


def test_counts_of_any_type(env):                                                  # noqa: F811
    """Counts are small whole numbers, the same in any type that bin_spikes
    makes: the same results, bit for bit."""
    torch, _ = env
    head, counts, gl = _head(env)
    labels = torch.tensor([0, 5, 2], dtype=torch.int32, device="cuda:0")
    want, wg = head.train_step(counts, labels, update=False)
    state = torch.zeros(3, 14, device="cuda:0")
    step = head.stream_step(counts[:, 0], state.clone(), k=2)
    for dtype in (torch.bfloat16, torch.float16, torch.int32):
        loss, g = head.train_step(counts.to(dtype), labels, update=False)
        assert torch.equal(loss, want) and all(torch.equal(g[k], wg[k]) for k in wg)
        got = head.stream_step(counts[:, 0].to(dtype), state.clone(), k=2)
        assert torch.equal(got.top_idx, step.top_idx) and torch.equal(got.lse, step.lse)


def test_sequences_of_nothing(env):                                                # noqa: F811
    torch, _ = env
    head, counts, _ = _head(env)
    labels = torch.tensor([0, 5, 2], dtype=torch.int32, device="cuda:0")
    for c, lab in ((counts[:, :0], labels), (counts[:0], labels[:0])):
        loss, g = head.train_step(c, lab, update=False)
        assert float(loss) == 0 and all(not v.any() for v in g.values())
        lists = head.alternatives(c, 2)
        assert lists.top_idx.shape == (0, 2)
        assert float(head.distill_step(c, lists, update=False)[0]) == 0
    h0 = torch.randn(3, 14, device="cuda:0")
    assert torch.equal(head.forward(counts[:, :0], h_first=h0).h_last, h0)
