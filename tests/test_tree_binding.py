"""What the binding of the calls for drafted trees refuses before it hands an address on.  CPU only: the device's tensors are stand-ins."""
import numpy as np
import pytest
import torch

from paper_2503_05840_amd import binding


class Fake:
    """A tensor that says it is on the device."""

    def __init__(self, *shape, dtype=torch.float32, cuda=True, contiguous=True):
        self.shape, self.dtype, self.is_cuda, self._contiguous = torch.Size(shape), dtype, cuda, contiguous

    def is_contiguous(self):
        return self._contiguous

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return 4

    def data_ptr(self):
        return 4096


def _decode(**kw):
    i32 = torch.int32
    return binding.slim_tree_decode(Fake(2, 4, 64), Fake(2, 20, 64), Fake(64, 64), Fake(2, 4, dtype=i32), Fake(2, 4, 64), 2, 4, 2, 16, 64, dtype="f32", **kw)


def _commit(**kw):
    i32 = torch.int32
    return binding.slim_tree_commit(Fake(2, 20, 64), Fake(2, 4, dtype=i32), Fake(2, dtype=i32), Fake(2, dtype=i32), 2, 4, 2, 16, 64, dtype="f32", **kw)


@pytest.fixture(autouse=True)
def _null_stream(monkeypatch):
    monkeypatch.setattr(binding, "_current_stream", lambda torch: lambda: 0)


@pytest.mark.parametrize("call", [_decode, _commit])
def test_lengths_for_another_batch(call):
    for lens in ([16], [16, 3, 5], 16, np.zeros((1, 2), dtype=np.int32)):
        with pytest.raises(ValueError):
            call(seq_lens_host=lens)
    for lens in (Fake(3, dtype=torch.int32), Fake(2), Fake(2, dtype=torch.int32, cuda=False), Fake(2, dtype=torch.int32, contiguous=False)):
        with pytest.raises(ValueError):
            call(seq_lens=lens)
    with pytest.raises(binding.SlimError):                # (as many as there are sequences: the library looks at them)
        call(seq_lens_host=[16, 17])


def test_workspaces_that_are_not_the_devices():
    for ws in (Fake(1 << 30, cuda=False), Fake(1 << 30, contiguous=False)):
        with pytest.raises(ValueError):
            _decode(workspace=ws)
    with pytest.raises(binding.SlimError):
        _decode(workspace=Fake(16))
