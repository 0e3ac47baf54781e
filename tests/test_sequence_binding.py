"""What the sequence and row bindings refuse or replace before anything is
launched (no GPU needed: stand-ins for device tensors where one is asked
for)."""
import pytest

import paper_2603_13283_amd as L

torch = pytest.importorskip("torch")


def test_a_workspace_that_is_not_one_block_is_not_written_to():
    """A view with gaps, or one element repeated, has as many elements as are
    needed but not as many bytes behind its pointer."""
    dev = torch.device("cpu")
    block = torch.empty(4096, dtype=torch.uint8)
    ptr, n, kept = L._workspace(torch, 1024, block, dev)
    assert ptr == block.data_ptr() and n == 4096 and kept is block
    for ws in (block[:1].expand(4096), block[::2], torch.empty(64, 64, dtype=torch.uint8)[:, :32]):
        ptr, n, kept = L._workspace(torch, 1024, ws, dev)
        assert n >= 1024 and kept is not ws and kept.is_contiguous() and ptr == kept.data_ptr()


class Stand:
    """As much of a device tensor as the checks look at."""

    def __init__(self, shape, strides=None, dtype=torch.bfloat16, device="cuda:0"):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, torch.device(device), True
        self.strides = strides or [0] * (len(shape) - 1) + [1]

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return tuple(self.strides) if i is None else self.strides[i]


class Stream:
    def __init__(self, device):
        self.device, self.cuda_stream = torch.device(device), 1


def test_a_stream_of_another_device_is_refused():
    with pytest.raises(ValueError, match="cuda:1"):
        L._on(torch, Stand((2, 3)), Stream("cuda:1"))


def test_sizes_past_32_bits_are_refused():
    """The C structures hold 32-bit sizes: a larger one would be taken modulo
    2^32, and most of the output left unwritten."""
    n = (1 << 32) + 5
    for shape, k in (((n, 2), 1), ((3, n), 1), ((3, 4), n)):
        with pytest.raises(ValueError, match="32 bits"):
            L._row_params(Stand(shape, [shape[1], 1]), k, 1.0, 0)
    for shape in ((n, 1, 1), (1, n, 1), (1, 1, n)):
        with pytest.raises(ValueError, match="32 bits"):
            L._gated_inputs(Stand(shape), Stand(shape), None)
    with pytest.raises(ValueError, match="32 bits"):
        L._int32((1 << 31))
    L._int32((1 << 31) - 1, 0)
