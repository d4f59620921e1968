"""Targets of probability 0, and infinite weights.

A logit of finite weights below what 32 bits hold is -inf: its token has probability 0, its loss is +inf, gradients are those of the
others.  Tolerances as in test_gpu_head_loss.py with 2^-12 for a probability (64 products of numbers around 1: (64 + 4) 2^-24
sum |h| |W| < 2^-13, and 2^-14) and 2^-12 for the chains of sums, so of terms' sizes u + 2^-11 (dh) and 2 u + u^2 + 2^-11 (dW)."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize('form', ['step', 'two'])
@pytest.mark.parametrize('d,V,rows', [(64, 50, 20), (64, 700, 300), (40, 50, 9)])
def test_a_target_whose_logit_is_below_32_bits(cuda, form, d, V, rows):
    import torch
    import paper_2606_00722_gb300 as epic
    g = torch.Generator().manual_seed(d + V)
    h, W = torch.randn((1, rows, d), generator=g), torch.randn((V, d), generator=g) / d ** 0.5
    far = [1, rows - 1]                 # positions whose logit of token 3 is -2^200
    h[..., 0], W[:, 0] = 0.0, 0.0
    h[0, far, 0], W[3, 0] = 2.0 ** 100, -2.0 ** 100
    h, W = h.to(torch.bfloat16).to(cuda), W.to(torch.bfloat16).to(cuda)
    target = torch.randint(0, V, (1, rows), generator=g).to(torch.int32)
    target[0, far] = torch.tensor([3, 5], dtype=torch.int32)  # one of them is its target, the other one's is not
    target = target.to(cuda)
    loss, lse = torch.empty((1, rows), device=cuda), torch.empty((1, rows), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    if form == 'step':
        epic.head_loss_step(h, W, target, loss, gh, gw)
    else:
        epic.head_loss_forward(h, W, target, loss, lse)
        epic.head_loss_backward(h, W, target, lse, torch.ones_like(loss), gh, gw)
        assert lse.isfinite().all()
    assert loss[0, far[0]] == math.inf and loss[0, [r for r in range(rows) if r != far[0]]].isfinite().all()
    x, w, y, at = h[0].double(), W.double(), target[0].long(), torch.arange(rows, device=cuda)
    dz = torch.softmax(x @ w.t(), 1)
    dz[at, y] = 0.0
    dz[at, y] = -dz.sum(1)
    u = 2.0 ** -8
    assert gh.isfinite().all() and gw.isfinite().all()
    want, terms = dz @ w, dz.abs() @ w.abs()
    assert ((gh[0].double() - want).abs() <= u * want.abs() + (u + 2.0 ** -11) * terms).all()
    want, terms = dz.t() @ x, dz.abs().t() @ x.abs()
    assert ((gw.double() - want).abs() <= u * want.abs() + (2 * u + u * u + 2.0 ** -11) * terms).all()


@pytest.mark.parametrize('form', ['step', 'two'])
@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_infinite_weights(cuda, dtype, form):
    """A token's weight of -inf: probability 0 at every position, finite gradients of the head, none of hidden states (0 times
    infinity is NaN)."""
    import torch
    import paper_2606_00722_gb300 as epic
    t = {'f16': torch.float16, 'bf16': torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(2)
    rows, d, V = 7, 24, 60
    h, W = torch.randn((1, rows, d), generator=g), torch.randn((V, d), generator=g) / d ** 0.5
    h[..., 4] = h[..., 4].abs() + 0.1
    W[9, 4] = -math.inf
    h, W = h.to(t).to(cuda), W.to(t).to(cuda)
    target = torch.tensor([[0, 9, 11, -1, 9, 59, 20]], dtype=torch.int32, device=cuda)
    loss, lse = torch.empty((1, rows), device=cuda), torch.empty((1, rows), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    if form == 'step':
        epic.head_loss_step(h, W, target, loss, gh, gw)
    else:
        epic.head_loss_forward(h, W, target, loss, lse)
        epic.head_loss_backward(h, W, target, lse, torch.ones_like(loss), gh, gw)
    assert (loss[0, [1, 4]] == math.inf).all() and loss[0, [0, 2, 3, 5, 6]].isfinite().all()
    counts = target[0] >= 0
    assert gh[0][counts][:, 4].isnan().all() and (gh[0][~counts] == 0).all()
    finite = [c for c in range(d) if c != 4]
    assert gh[0][:, finite].isfinite().all()
    x, y = h[0][counts].double(), target[0][counts].long()
    z = x @ W.double().t()
    assert (z[:, 9] == -math.inf).all()
    dz = torch.softmax(z, 1)
    dz[torch.arange(len(y)), y] = 0.0
    dz[torch.arange(len(y)), y] = -dz.sum(1)
    u = {'f16': 2.0 ** -11, 'bf16': 2.0 ** -8}[dtype]
    want, terms = dz.t() @ x, dz.abs().t() @ x.abs()
    assert ((gw.double() - want).abs() <= u * want.abs() + (2 * u + u * u + 2.0 ** -11) * terms + 2.0 ** -25).all()
