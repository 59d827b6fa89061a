"""Argument checks and stream order of Potential.descriptors and
forces_from_descriptors, with the library's calls and the GPU's tensors and
streams replaced by stand-ins."""
import types

import pytest
import torch

from paper_2608_16329_amd import Potential, binding


class Tensor:
    """What the checks look at of a tensor on the GPU."""

    def __init__(self, *shape, dtype=torch.float64):
        self.shape, self.dtype, self.is_cuda = torch.Size(shape), dtype, True

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 4096


@pytest.fixture
def potential(monkeypatch):
    """A potential of 5 atoms and 64 values a descriptor, and the calls made."""
    p = object.__new__(Potential)
    p.ctx, p.n, p.width = None, 5, 64
    p.torch = torch
    calls = []
    monkeypatch.setattr(binding, "mlip_descriptors", lambda *a: calls.append("descriptors"))
    monkeypatch.setattr(binding, "mlip_forces_from_descriptors", lambda *a: calls.append("forces"))
    return types.SimpleNamespace(p=p, calls=calls)


def rows(n=5):
    return Tensor(n, 64, dtype=torch.float32)


def test_arrays_that_are_too_short_are_refused(potential):
    p = potential.p
    with pytest.raises(AssertionError, match="positions have 12 values"):
        p.descriptors(Tensor(4, 3), rows())
    with pytest.raises(AssertionError, match="positions have 12 values"):
        p.forces_from_descriptors(Tensor(4, 3), rows(), Tensor(5, 3))
    with pytest.raises(AssertionError, match="forces have 12 values"):
        p.forces_from_descriptors(Tensor(5, 3), rows(), Tensor(4, 3))
    with pytest.raises(AssertionError, match="virials have 15 values"):
        p.forces_from_descriptors(Tensor(5, 3), rows(), Tensor(5, 3), Tensor(5, 3))
    with pytest.raises(AssertionError):
        p.forces_from_descriptors(Tensor(5, 3), rows(), Tensor(5, 3), Tensor(5, 9, dtype=torch.float32))
    assert potential.calls == []
