"""The binding of the calls on rows of logits, without a GPU: tensors that only
say what they are, and a library that must not be reached."""
import pytest

import paper_2606_00722_gb300 as epic

binding = epic.epic


class Said:
    """What the binding asks a tensor for."""

    def __init__(self, shape, dtype, device=1):
        import torch
        self._meta = torch.empty(shape, dtype=dtype, device='meta')
        self.shape, self.dtype, self.index = self._meta.shape, dtype, device
        self.device = ('cuda', device)

    def stride(self):
        return self._meta.stride()

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


class Reached(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Reached(name)
        return call


def calls(logits_device, others=1):
    import torch
    f32, i32 = torch.float32, torch.int32
    z = Said((2, 3, 50), f32, logits_device)
    ids, vals = Said((2, 3, 4), i32, others), Said((2, 3, 4), f32, others)
    row = Said((2, 3), f32, others)
    grad = Said((2, 3, 50), f32, others)
    return [lambda: epic.propose_topk(z, ids, vals), lambda: epic.sample_tokens(z, vals, ids, vals),
            lambda: epic.distill_forward(z, ids, vals, row, row),
            lambda: epic.distill_backward(z, ids, vals, row, row, grad),
            lambda: epic.distill_step(z, ids, vals, row, grad)]


@pytest.fixture
def device(monkeypatch):
    binding._logits_init()
    monkeypatch.setattr(binding, '_lib', Library())
    monkeypatch.setattr(binding, '_raw_stream', lambda device: 0)
    monkeypatch.setattr(binding, '_current_device', lambda: current[0], raising=False)
    current = [1]
    return current


def test_tensors_of_another_device_than_the_current_one_are_refused(device):
    for call in calls(1):
        with pytest.raises(Reached):  # tensors of the current device get as far as the library
            call()
    device[0] = 0
    for call in calls(1):
        with pytest.raises(ValueError, match='current device'):
            call()


def test_tensors_of_two_devices_are_refused(device):
    for call in calls(1, others=0):
        with pytest.raises(ValueError):
            call()
