"""The parts of the sequence head that need no GPU: the counting of spikes into
bins."""
import math

import pytest

import paper_2603_13283_amd as L
from paper_2603_13283_amd.sequence import bin_spikes

torch = pytest.importorskip("torch")


def test_only_spikes_inside_the_bins_are_counted():
    """Bins run from t = 0 to bins * dt: earlier, later and absent spikes (a
    time of infinity or NaN) are in none of them."""
    dt = 0.005
    t = torch.tensor([[[-1.0, -0.006, -0.004, -0.0, 0.001, 0.0149, 0.015, 3e38, math.inf, -math.inf, math.nan, 0.001]]])
    n = torch.tensor([[11]], dtype=torch.int32)                # the last one is past the count
    c = bin_spikes(L.ForwardOut(t, n, None, None), 3, dt)
    assert c.shape == (1, 3, 1) and c[0, :, 0].tolist() == [2.0, 0.0, 1.0]
