"""Argument checks and stream order of Potential.descriptors and
forces_from_descriptors, with the library's calls and the GPU's tensors and
streams replaced by stand-ins."""
import types

import pytest
import torch

from paper_2608_16329_amd import Potential, binding


class Stream:
    device = 0

    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(f"{self.name} waits for {other.name}")


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
    calls = []
    p.stream, other = Stream("own", calls), Stream("other", calls)
    now = types.SimpleNamespace(stream=other)
    p.torch = types.SimpleNamespace(float32=torch.float32, float64=torch.float64,
                                    cuda=types.SimpleNamespace(current_stream=lambda device=None: now.stream))
    monkeypatch.setattr(binding, "mlip_descriptors", lambda *a: calls.append("descriptors"))
    monkeypatch.setattr(binding, "mlip_forces_from_descriptors", lambda *a: calls.append("forces"))
    return types.SimpleNamespace(p=p, calls=calls, now=now)


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


def test_calls_are_in_order_with_the_current_stream(potential):
    p = potential.p
    p.descriptors(Tensor(5, 3), rows())
    p.forces_from_descriptors(Tensor(5, 3), rows(), Tensor(5, 3), Tensor(5, 9))
    assert potential.calls == ["own waits for other", "descriptors", "other waits for own",
                               "own waits for other", "forces", "other waits for own"]
    potential.calls.clear()
    potential.now.stream = p.stream
    p.descriptors(Tensor(5, 3), rows())
    p.forces_from_descriptors(Tensor(5, 3), rows(), Tensor(5, 3))
    assert potential.calls == ["descriptors", "forces"]
