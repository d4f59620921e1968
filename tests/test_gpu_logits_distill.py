"""Distillation from a teacher's top logits against its formulas in 64 bits and
against differences.

Tolerances, from the arithmetic: a loss is a sum of p (log p - lq) with lq off
by |lq| 2^-22 (two roundings of the scaled logit, one of the sum's logarithm)
and the sum of exponentials by at most 300 2^-24: per unit of tau^2 w, 40 2^-22 +
2e-5 < 3.2e-5.  A gradient is w tau (q - p) with q to 5e-5 (60 ln2 2^-22 from the exponent, 2^-22, 300 2^-24), p to 1e-6, and one
rounding to the logits' type: half a unit in the last place, 2^-8 (bf16, 8 bits), 2^-11 or, near 0, 2^-25 (f16)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _dtype(name):
    import torch
    return {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}[name]


def make(B, n, V, K, dtype, kind, seed, pad=0, shift=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, n, V), generator=g) * 2.0
    ids = torch.randint(0, max(V, 1), (B, n, K), generator=g).to(torch.int32)
    vals = torch.randn((B, n, K), generator=g) * 2.0
    valid = (torch.rand((B, n, K), generator=g) < 0.7).to(torch.uint8)
    weight = torch.rand((B, n), generator=g) * 2.0 + 0.1
    if kind == 'edges':
        if K > 2:
            ids[..., 1] = ids[..., 0]           # the same token twice
            ids[..., 2] = -1                    # padding
        vals[torch.rand(vals.shape, generator=g) < 0.2] = -math.inf
        valid[0, 0] = 0                         # nothing of the row counts
        valid[-1, -1] = 2                       # a capacity overflow is no valid bit
        weight[0, -1] = 0.0
        ids[0, n // 2, 0] = V                   # out of range
        z[torch.rand(z.shape, generator=g) < 0.1] = -math.inf
        z.scatter_(2, ids.long().clamp(0, V - 1), 0.5)
        z[torch.rand(z.shape, generator=g) < 0.05] = torch.finfo(_dtype(dtype)).min
        z.scatter_(2, ids.long().clamp(0, V - 1), 0.5)
    full = torch.full((B, n, V + pad), math.nan)
    full[..., :V] = z
    flat = torch.full((shift + full.numel() + 16,), math.inf, dtype=_dtype(dtype), device='cuda')
    flat[shift:shift + full.numel()] = full.reshape(-1).cuda()
    logits = flat[shift:shift + full.numel()].view(B, n, V + pad)[..., :V]
    return logits, ids.cuda(), vals.cuda(), valid.cuda(), weight.cuda()


def distill64(logits, ids, vals, valid, weight, tau, up=None):
    """(loss, gradient of sum(up * loss)) in 64 bits by the formulas."""
    z, a = logits.double().cpu().numpy() / tau, vals.double().cpu().numpy() / tau
    ids, w = ids.cpu().numpy(), weight.double().cpu().numpy()
    ok = np.ones(ids.shape, bool) if valid is None else valid.cpu().numpy() == 1
    up = np.ones(w.shape) if up is None else up.double().cpu().numpy()
    B, n, V = z.shape
    loss, grad = np.zeros((B, n)), np.zeros((B, n, V))
    for b in range(B):
        for i in range(n):
            use = [k for k in range(ids.shape[2]) if ok[b, i, k] and 0 <= ids[b, i, k] < V and a[b, i, k] > -np.inf]
            if not use or w[b, i] == 0:
                continue
            p = np.exp(a[b, i, use] - a[b, i, use].max())
            p /= p.sum()
            m = z[b, i].max()
            q = np.exp(z[b, i] - m)
            lse = m + np.log(q.sum())
            q /= q.sum()
            t = ids[b, i, use]
            loss[b, i] = w[b, i] * tau ** 2 * np.sum(p * (np.log(p) - (z[b, i, t] - lse)))
            np.subtract.at(q, t, p)
            grad[b, i] = w[b, i] * tau * up[b, i] * q
    return loss, grad


def check(loss, grad, want_loss, want_grad, ids, weight, tau, dtype, up=None):
    scale = (weight.double().cpu().numpy() * tau ** 2)
    assert (np.abs(loss.double().cpu().numpy() - want_loss) <= 3.2e-5 * scale + 1e-6 * np.abs(want_loss)).all()
    scale = (weight.double() * tau * (1.0 if up is None else up.double())).cpu().numpy()[..., None]
    rel, tiny = {'f32': (2.0 ** -23, 0.0), 'f16': (2.0 ** -11, 2.0 ** -25), 'bf16': (2.0 ** -8, 0.0)}[dtype]
    got = grad.double().cpu().numpy()
    # q is off by 5e-5 of itself; at the teacher's tokens, where p is taken off, that may be of a whole unit
    target = np.zeros(got.shape, bool)
    np.put_along_axis(target, ids.cpu().numpy().astype(np.int64).clip(0, got.shape[-1] - 1), True, -1)
    off = np.abs(got - want_grad)
    assert (off <= np.abs(want_grad) * (rel + 6e-5) + scale * 6e-5 * target + tiny + 1e-30).all()


CASES = [  # B, n, V, K, dtype, kind, pad, shift
    (1, 1, 1, 1, 'f32', 'normal', 0, 0),
    (2, 2, 2, 3, 'bf16', 'normal', 1, 1),
    (1, 3, 7, 5, 'f16', 'edges', 0, 3),
    (2, 3, 256, 8, 'f32', 'edges', 0, 0),
    (2, 3, 1000, 64, 'bf16', 'edges', 3, 1),
    (2, 3, 4099, 16, 'f16', 'edges', 0, 0),
    (1, 4, 32771, 16, 'f32', 'edges', 0, 1),
    (1, 4, 32768, 1024, 'bf16', 'edges', 0, 0),
    (1, 3, 50021, 33, 'bf16', 'edges', 3, 5),
    (1, 2, 126000, 32, 'bf16', 'edges', 16, 0),
    (1, 2, 126000, 32, 'f32', 'normal', 0, 0),
    (1, 2, 420001, 20, 'f32', 'edges', 0, 1),    # past the cluster's shared memory
    (1, 2, 900001, 20, 'bf16', 'edges', 1, 0),
]


@pytest.mark.parametrize('B,n,V,K,dtype,kind,pad,shift', CASES)
@pytest.mark.parametrize('tau', [1.0, 2.5])
def test_loss_and_gradient(cuda, B, n, V, K, dtype, kind, pad, shift, tau):
    import torch
    import paper_2606_00722_gb300 as epic
    logits, ids, vals, valid, weight = make(B, n, V, K, dtype, kind, V + K, pad, shift)
    g = torch.Generator().manual_seed(1)
    up = (torch.rand((B, n), generator=g) + 0.2).cuda()
    want_loss, want_step = distill64(logits, ids, vals, valid, weight, tau)
    _, want_grad = distill64(logits, ids, vals, valid, weight, tau, up)
    for other in (0, 1):  # the gradient's rows at the logits' alignment, and at another
        store = torch.full((B, n, V + pad + 16), 7.0, dtype=logits.dtype, device='cuda')
        at = (logits.data_ptr() % 16) // logits.element_size()
        grad = store.view(-1)[at + other:at + other + B * n * (V + pad)].view(B, n, V + pad)[..., :V]
        loss = torch.full((B, n), -7.0, device='cuda')
        lse = torch.full((B, n), -7.0, device='cuda')
        epic.distill_step(logits, ids, vals, loss, grad, tau=tau, weight=weight, valid=valid)
        check(loss, grad, want_loss, want_step, ids, weight, tau, dtype)
        if pad:
            assert (store.view(-1)[at + other:at + other + B * n * (V + pad)].view(B, n, V + pad)[..., V:] == 7).all()
        assert (store.view(-1)[:at + other] == 7).all()
        assert (store.view(-1)[at + other + B * n * (V + pad):] == 7).all()
        first = loss.clone()
        grad.fill_(7.0)
        epic.distill_forward(logits, ids, vals, loss, lse, tau=tau, weight=weight, valid=valid)
        assert torch.equal(loss, first)
        epic.distill_backward(logits, ids, vals, lse, up, grad, tau=tau, weight=weight, valid=valid)
        check(loss, grad, want_loss, want_grad, ids, weight, tau, dtype, up)
        assert (store.view(-1)[:at + other] == 7).all()


@pytest.mark.parametrize('V,dtype,pad,shift', [(4099, 'bf16', 3, 1), (8192, 'f32', 0, 0), (16411, 'f16', 0, 5)])
def test_many_rows(cuda, V, dtype, pad, shift):
    """Rows enough for every place on the GPU."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, K, tau = 70, 9, 12, 1.5
    logits, ids, vals, valid, weight = make(B, n, V, K, dtype, 'edges', V, pad, shift)
    weight[::3] = 0.0
    want_loss, want_grad = distill64(logits, ids, vals, valid, weight, tau)
    loss, grad = torch.full((B, n), -7.0, device='cuda'), torch.full((B, n, V), 7.0, dtype=logits.dtype, device='cuda')
    epic.distill_step(logits, ids, vals, loss, grad, tau=tau, weight=weight, valid=valid)
    check(loss, grad, want_loss, want_grad, ids, weight, tau, dtype)


def test_without_weights_or_bits(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    logits, ids, vals, _, _ = make(2, 3, 5000, 12, 'f32', 'normal', 5)
    one = torch.ones((2, 3), device='cuda')
    want_loss, want_grad = distill64(logits, ids, vals, None, one, 1.0)
    loss, grad = torch.empty((2, 3), device='cuda'), torch.empty_like(logits)
    epic.distill_step(logits, ids, vals, loss, grad)
    check(loss, grad, want_loss, want_grad, ids, one, 1.0, 'f32')


def test_gradient_against_differences(cuda):
    """Along random directions d, (loss(z + h d) - loss(z - h d)) / 2h is d . grad up to h^2 max|d|^3 (third derivatives
    of logsumexp are below 1) and 2 eps / 2h of the losses' error (eps = 3.2e-5 w tau^2)."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, V, K, tau, h = 2, 3, 700, 9, 1.5, 0.05
    logits, ids, vals, valid, weight = make(B, n, V, K, 'f32', 'normal', 6)
    loss, lse, grad = torch.empty((B, n), device='cuda'), torch.empty((B, n), device='cuda'), torch.empty_like(logits)
    epic.distill_step(logits, ids, vals, loss, grad, tau=tau, weight=weight, valid=valid)
    for seed in range(4):
        d = torch.randn(logits.shape, generator=torch.Generator().manual_seed(seed)).clamp_(-2, 2).cuda()
        side = []
        for sign in (h, -h):
            epic.distill_forward(logits + sign * d, ids, vals, loss, lse, tau=tau, weight=weight, valid=valid)
            side.append(loss.double().clone())
        slope = (side[0] - side[1]) / (2 * h)
        want = (grad.double() * d.double()).sum(-1)
        w = weight.double()
        assert ((slope - want).abs() <= w * (h * h * 8 / tau + 3.2e-5 * tau ** 2 / h)).all()


def test_infinite_and_nan_logits(cuda):
    """A token the student rules out and the teacher wants: loss +inf, finite gradient.  A row of -inf alone likewise.
    NaN and +inf in a row show up as NaN, but in a row of weight 0 they do not."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, V = 1, 6, 300
    z = torch.randn((B, n, V), generator=torch.Generator().manual_seed(1)).cuda()
    ids = torch.tensor([3, 9], dtype=torch.int32, device='cuda').expand(B, n, 2).contiguous()
    vals = torch.zeros((B, n, 2), device='cuda')
    z[0, 1, 3] = -math.inf
    z[0, 2] = -math.inf
    z[0, 3, 200] = math.nan
    z[0, 4, 200] = math.inf
    z[0, 5] = math.nan
    weight = torch.tensor([[1.0, 1, 1, 1, 1, 0]], device='cuda')
    up = torch.ones((B, n), device='cuda')
    loss, lse = torch.empty((B, n), device='cuda'), torch.empty((B, n), device='cuda')
    for form in ('step', 'train'):
        grad = torch.full_like(z, 7.0)
        if form == 'step':
            epic.distill_step(z, ids, vals, loss, grad, weight=weight)
        else:
            epic.distill_forward(z, ids, vals, loss, lse, weight=weight)
            epic.distill_backward(z, ids, vals, lse, up, grad, weight=weight)
        got = loss[0].tolist()
        assert math.isfinite(got[0]) and got[1] == got[2] == math.inf and math.isnan(got[3]) and math.isnan(got[4])
        assert got[5] == 0
        assert torch.isfinite(grad[0, :3]).all()
        assert grad[0, 1, 3] == -0.5 and (grad[0, 2, [3, 9]] == -0.5).all()
        assert (grad[0, 2].abs().sum() == 1.0).all()
        assert torch.isnan(grad[0, 3, 200]) and torch.isnan(grad[0, 4, 200]) and (grad[0, 5] == 0).all()


def test_refusals(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    logits, ids, vals, valid, weight = make(2, 3, 100, 4, 'f32', 'normal', 1)
    loss, grad = torch.empty((2, 3), device='cuda'), torch.empty_like(logits)
    for tau in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(epic.EpicError) as e:
            epic.distill_step(logits, ids, vals, loss, grad, tau=tau)
        assert e.value.status == 1
    many = torch.zeros((2, 3, 1025), dtype=torch.int32, device='cuda')
    with pytest.raises(epic.EpicError) as e:
        epic.distill_step(logits, many, many.float(), loss, grad)
    assert e.value.status == 6
    for args, kw in [((logits, ids.long(), vals, loss, grad), {}), ((logits, ids, vals[:, :2], loss, grad), {}),
                     ((logits, ids, vals, loss[:1], grad), {}), ((logits, ids, vals, loss, grad.half()), {}),
                     ((logits, ids, vals, loss, grad[..., :50]), {}), ((logits, ids, vals, loss, grad), {'valid': valid.float()}),
                     ((logits, ids, vals, loss, grad), {'weight': weight[:1]})]:
        with pytest.raises(ValueError):
            epic.distill_step(*args, **kw)
    # nothing to do, rows of no tokens, no entries
    none = torch.empty((0, 3, 100), device='cuda')
    epic.distill_step(none, ids[:0], vals[:0], loss[:0], none)
    epic.distill_step(logits[..., :0], ids, vals, loss.fill_(7), grad[..., :0])
    assert (loss == 0).all()
    epic.distill_step(logits, ids[..., :0].contiguous(), vals[..., :0].contiguous(), loss.fill_(7), grad.fill_(7))
    assert (loss == 0).all() and (grad == 0).all()


@pytest.mark.parametrize('tau', [0.5, 1.0, 2.5])
@pytest.mark.parametrize('dtype', ['f32', 'f16', 'bf16'])
@pytest.mark.parametrize('n,V,K', [(4, 1000, 5), (3, 40003, 16), (40, 4099, 3)])
def test_backward_far_from_zero(cuda, n, V, K, dtype, tau):
    """Rows at the type's lowest value (a mask that left nothing), and logits of a size whose logsumexp in 32 bits has little
    or nothing left of the sum's logarithm: forward and backward agree with the formulas as the single call does."""
    import torch
    import paper_2606_00722_gb300 as epic
    logits, ids, vals, valid, weight = make(2, n, V, K, dtype, 'normal', V + n)
    logits[0, 0] = torch.finfo(logits.dtype).min
    logits[0, 1] += 20000.0
    logits[0, 2] -= 130.0 * tau
    logits[1, 0] = -3.0e4
    logits[1, 0, ::5] = -1.0e4
    logits[1, 1] = torch.finfo(logits.dtype).max
    logits[1, 2] += 110.0 * tau
    valid.fill_(1)
    g = torch.Generator().manual_seed(1)
    up = (torch.rand((2, n), generator=g) + 0.2).cuda()
    z = logits.double()
    z -= z.amax(-1, keepdim=True)  # which the formulas do not notice, but 64 bits do at 1e38
    want_loss, want_step = distill64(z, ids, vals, valid, weight, tau)
    _, want_grad = distill64(z, ids, vals, valid, weight, tau, up)
    loss, lse = torch.full((2, n), -7.0, device='cuda'), torch.full((2, n), -7.0, device='cuda')
    grad = torch.full((2, n, V), 7.0, dtype=logits.dtype, device='cuda')
    epic.distill_step(logits, ids, vals, loss, grad, tau=tau, weight=weight, valid=valid)
    check(loss, grad, want_loss, want_step, ids, weight, tau, dtype)
    loss.fill_(-7.0)
    grad.fill_(7.0)
    epic.distill_forward(logits, ids, vals, loss, lse, tau=tau, weight=weight, valid=valid)
    epic.distill_backward(logits, ids, vals, lse, up, grad, tau=tau, weight=weight, valid=valid)
    check(loss, grad, want_loss, want_grad, ids, weight, tau, dtype, up)
