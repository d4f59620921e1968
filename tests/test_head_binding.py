"""The binding of the head's calls, without a GPU: tensors that only say what they are, and a library that must not be
reached with wrong ones."""
import pytest

import paper_2606_00722_gb300 as epic

binding = epic.epic


class Said:
    """What the binding asks a tensor for."""

    def __init__(self, shape, dtype, device=1, strides=None):
        import torch
        self._meta = torch.empty(shape, dtype=dtype, device='meta')
        if strides:
            self._meta = torch.empty_strided(shape, strides, dtype=dtype, device='meta')
        self.shape, self.dtype, self.index = self._meta.shape, dtype, device
        self.device = ('cuda', device)

    def stride(self, *at):
        return self._meta.stride(*at)

    def dim(self):
        return self._meta.dim()

    def numel(self):
        return self._meta.numel()

    def element_size(self):
        return self._meta.element_size()

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return self._meta.is_contiguous()

    def data_ptr(self):
        return 4096


class Reached(Exception):
    pass


class Library:
    """Workspace sizes are 512; anything else is the call itself."""

    def __getattr__(self, name):
        def call(*args):
            if name.endswith('_workspace'):
                args[-1]._obj.value = 512
                return 0
            raise Reached(name)
        call.__name__ = name
        return call


def tensors(dev=1, others=1):
    import torch
    b16, f32, i32, i8 = torch.bfloat16, torch.float32, torch.int32, torch.int8
    return dict(h=Said((2, 3, 16), b16, dev), W=Said((50, 16), b16, others), y=Said((2, 3), i32, others),
                row=Said((2, 3), f32, others), gh=Said((2, 3, 16), b16, dev), gw=Said((50, 16), b16, others),
                q=Said((2, 3, 16), i8, others), Wq=Said((50, 16), i8, others), S=Said((50,), f32, others),
                z=Said((2, 3, 50), b16, dev), work=Said((512,), torch.uint8, others))


def calls(t):
    return [lambda: epic.head_loss_forward(t['h'], t['W'], t['y'], t['row'], t['row'], t['row'], workspace=t['work']),
            lambda: epic.head_loss_backward(t['h'], t['W'], t['y'], t['row'], t['row'], t['gh'], t['gw'],
                                            workspace=t['work']),
            lambda: epic.head_loss_step(t['h'], t['W'], t['y'], t['row'], t['gh'], t['gw'], workspace=t['work']),
            lambda: epic.quantize_rows(t['h'], t['q'], t['row']),
            lambda: epic.int8_logits(t['q'], t['row'], t['Wq'], t['S'], t['z'], workspace=t['work'])]


@pytest.fixture
def device(monkeypatch):
    binding._logits_init()
    monkeypatch.setattr(binding, '_lib', Library())
    monkeypatch.setattr(binding, '_raw_stream', lambda device: 0)
    current = [1]
    monkeypatch.setattr(binding, '_current_device', lambda: current[0], raising=False)
    return current


def test_good_calls_reach_the_library(device):
    for call in calls(tensors()):
        with pytest.raises(Reached):
            call()
    t = tensors()
    with pytest.raises(Reached):
        epic.head_loss_backward(t['h'], t['W'], t['y'], t['row'], t['row'], None, None, workspace=t['work'])


def test_tensors_of_other_devices_are_refused(device):
    for call in calls(tensors(1, 0)):
        with pytest.raises(ValueError):
            call()
    device[0] = 0
    for call in calls(tensors()):
        with pytest.raises(ValueError, match='current device'):
            call()


def test_wrong_shapes_and_types_are_refused(device):
    import torch
    b16, f16, f32, i8 = torch.bfloat16, torch.float16, torch.float32, torch.int8
    wrong = [('h', Said((2, 3, 16), f32), (0, 1, 2)), ('h', Said((6, 16), b16), (0, 1, 2, 3)),
             ('h', Said((2, 3, 16), b16, 1, (96, 32, 2)), (0, 1, 2, 3)),
             ('W', Said((50, 16), f16), (0, 1, 2)), ('W', Said((50, 15), b16), (0, 1, 2)),
             ('W', Said((50, 16), b16, 1, (1, 50)), (0, 1, 2)), ('y', Said((2, 3), torch.int64), (0, 1, 2)),
             ('row', Said((2, 4), f32), (0, 1, 2, 3, 4)), ('row', Said((2, 3), f16), (0, 1, 2, 3, 4)),
             ('gh', Said((2, 3, 15), b16), (1, 2)), ('gh', Said((2, 3, 16), f32), (1, 2)),
             ('gw', Said((49, 16), b16), (1, 2)), ('gw', Said((50, 16), f32), (1, 2)),
             ('q', Said((2, 3, 15), i8), (3,)), ('q', Said((2, 3, 16), torch.uint8), (3, 4)),
             ('q', Said((2, 2, 16), i8), (3, 4)), ('Wq', Said((50, 16), torch.uint8), (4,)),
             ('Wq', Said((49, 16), i8), (4,)), ('S', Said((49,), f32), (4,)), ('z', Said((2, 3, 49), b16), (4,)),
             ('z', Said((2, 4, 50), b16), (4,)), ('z', Said((2, 3, 50), i8), (4,)),
             ('work', Said((512,), torch.uint8, 0), (0, 1, 2, 4)),
             ('work', Said((512,), torch.uint8, 1, (2,)), (0, 1, 2, 4))]
    for name, bad, where in wrong:
        t = tensors()
        t[name] = bad
        for i in where:
            with pytest.raises(ValueError):
                calls(t)[i]()


def test_workspaces_that_are_asked_for(device):
    t = tensors()
    for form in ('forward', 'backward', 'step'):
        assert epic.head_loss_workspace(form, t['h'], t['W']) == 512
    with pytest.raises(ValueError):
        epic.head_loss_workspace('both', t['h'], t['W'])


def test_the_loss_is_one_operation_and_refuses_gradients_of_constants(monkeypatch):
    import torch
    seen = []

    def forward(h, W, target, loss, lse, weight):
        loss.fill_(1.0)
        seen.append('forward')

    def backward(h, W, target, lse, grad_loss, gh, gw, weight):
        for g in (gh, gw):
            if g is not None:
                g.fill_(2.0)
        seen.append((gh is not None, gw is not None))
    monkeypatch.setattr(binding, 'head_loss_forward', forward)
    monkeypatch.setattr(binding, 'head_loss_backward', backward)
    h, W = torch.zeros((2, 3, 4), requires_grad=True), torch.zeros((5, 4), requires_grad=True)
    y, w = torch.zeros((2, 3), dtype=torch.int32), torch.ones((2, 3))
    a, b = epic.head_loss(h, W, y, w), epic.head_loss(h.detach(), W, y)
    assert type(a.grad_fn) is type(b.grad_fn)
    a.sum().backward()
    assert (h.grad == 2).all() and (W.grad == 2).all()
    b.sum().backward()
    epic.head_loss(h, W.detach(), y).sum().backward()
    assert seen == ['forward', 'forward', (True, True), (False, True), 'forward', (True, False)]
    with pytest.raises(ValueError, match='detach'):
        epic.head_loss(h, W, y, w.requires_grad_())
    with torch.no_grad():
        epic.head_loss(h, W, y, w)
