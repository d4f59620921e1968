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


def fake_loss(monkeypatch):
    """distill_loss on CPU tensors, with calls that note what they were given."""
    import torch
    seen = []

    def forward(z, ids, vals, loss, lse, tau, weight, valid):
        loss.fill_(tau)
        seen.append(('forward', tau, weight, valid))

    def backward(z, ids, vals, lse, grad_loss, grad, tau, weight, valid):
        grad.copy_(grad_loss[..., None].expand_as(grad) * tau)
        seen.append(('backward', tau, weight, valid))
    monkeypatch.setattr(binding, 'distill_forward', forward)
    monkeypatch.setattr(binding, 'distill_backward', backward)
    z = torch.zeros((2, 3, 5), requires_grad=True)
    return z, torch.zeros((2, 3, 4), dtype=torch.int32), torch.zeros((2, 3, 4)), torch.ones((2, 3)), seen


def test_the_loss_is_one_operation(monkeypatch):
    """Every call is of the same torch operation, each with its own temperature and constants."""
    z, ids, vals, weight, seen = fake_loss(monkeypatch)
    one, two = epic.distill_loss(z, ids, vals, 0.5, weight), epic.distill_loss(z, ids, vals, 3.0)
    assert type(one.grad_fn) is type(two.grad_fn)
    two.sum().backward()
    assert (z.grad == 3.0).all()
    z.grad = None
    one.sum().backward()
    assert (z.grad == 0.5).all()
    assert [(form, tau, w is not None) for form, tau, w, _ in seen] == [
        ('forward', 0.5, True), ('forward', 3.0, False), ('backward', 3.0, False), ('backward', 0.5, True)]


def test_constants_of_the_loss_that_ask_for_a_gradient_are_refused(monkeypatch):
    import torch
    z, ids, vals, weight, seen = fake_loss(monkeypatch)
    for bad in (dict(vals=vals.clone().requires_grad_()), dict(vals=vals, weight=weight.clone().requires_grad_())):
        with pytest.raises(ValueError, match='detach'):
            epic.distill_loss(z, ids, **bad)
        with torch.no_grad():
            epic.distill_loss(z, ids, **bad)
    epic.distill_loss(z, ids, vals.clone().requires_grad_().detach(), weight=weight).sum().backward()
    assert (z.grad == 1.0).all() and len(seen) == 4
