"""Gradients where the target's part is nearly all of them: it is not rounded before the last sum, in a hidden state's gradient
however many positions share the target, in the head's for the first four of one.

The targets' rows of the head hold numbers around 1, all others around 2^-8, so what is rounded to 16 bits before a product (u of
each term, and u of h times a factor) is small, and the output's own rounding, u of the value, stands nearly alone.
Tolerances are those of test_gpu_head_loss.py with the target's term apart: of its size T, and A that of the others,
  dh: u |dh| + (u + e + 2^-16) A + (e + 2^-16) T,   dW: u |dW| + (2 u + u^2 + e + 2^-16) A + (e + 2^-16) T
with e = 2 dz + 2^-14 + |lse| 2^-21, dz = (d + 4) 2^-24 sum |h| |W|, the relative error of a probability; 2^-16 for sums cut to
2^-23 in at most 2^7 steps; fp16: half a unit in the last place of subnormals, 2^-25, and 2^-38 of the largest factor a term.  A
target's term that was rounded would be off by u T more, and u is 16 (bf16) and 2 (fp16) times 2^-12."""
import pytest

pytestmark = pytest.mark.gpu


def make(R, d, V, targets, dtype, seed):
    import torch
    t = {'f16': torch.float16, 'bf16': torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((V, d), generator=g) * 2.0 ** -8
    W[:targets] = (torch.rand((targets, d), generator=g) + 0.5) * torch.randn((targets, d), generator=g).sign()
    h = torch.randn((1, R, d), generator=g) * 0.1
    target = (torch.arange(R) % targets).to(torch.int32)[None]
    weight = torch.rand((1, R), generator=g) + 0.5
    return h.to(t).cuda(), W.to(t).cuda(), target.cuda(), weight.cuda()


def check(h, W, target, g, gh, gw):
    """Each of gh and gw (or None) against the formulas in 64 bits."""
    import torch
    u, f16 = (2.0 ** -11, True) if h.dtype == torch.float16 else (2.0 ** -8, False)
    x, w, y, g = h[0].double(), W.double(), target[0].long(), g[0].double()
    at = torch.arange(len(y), device=h.device)
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    dz = torch.exp(z - lse[:, None])
    dz[at, y] = 0.0
    dz[at, y] = -dz.sum(1)
    dz *= g[:, None]
    size = dz.abs()
    own = size[at, y]
    size[at, y] = 0.0
    err = 2.0 ** -14 + 2.0 ** -16 + lse.abs() * 2.0 ** -21 + 2 * (x.shape[1] + 4) * 2.0 ** -24 * (x.abs() @ w.abs().t()).amax(1)
    err += z.abs().amax(1) * 2.0 ** -21  # a power's argument
    low, top = (2.0 ** -25, 2.0 ** -38 * float(g.abs().max())) if f16 else (1e-30, 0.0)
    if gh is not None:
        want = dz @ w
        tol = u * want.abs() + low + (size * (u + err)[:, None]) @ w.abs() + (own * err)[:, None] * w[y].abs() + top * w.abs().sum(0)
        bad = (gh[0].double() - want).abs() > tol
        assert not bad.any(), (int(bad.sum()), gh[0][bad][:4], want[bad][:4], tol[bad][:4])
    if gw is not None:
        want = dz.t() @ x
        tol = u * want.abs() + low + (size * (2 * u + u * u + err)[:, None]).t() @ x.abs() + top * x.abs().sum(0)
        tol.index_add_(0, y, (own * err)[:, None] * x.abs())
        bad = (gw.double() - want).abs() > tol
        assert not bad.any(), (int(bad.sum()), gw[bad][:4], want[bad][:4], tol[bad][:4])


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('far', [False, True])
@pytest.mark.parametrize('R,d,V', [(300, 64, 700), (700, 256, 700), (40, 97, 600)])
def test_hidden_states_of_shared_targets(cuda, R, d, V, far, dtype):
    """Three targets for all positions.  far: one position whose largest logit is 60 above its target's sends all
    others through the second pass."""
    import torch
    import paper_2606_00722_gb300 as epic
    h, W, target, weight = make(R, d, V, 3, dtype, R + d)
    if far:
        h[0, 5] = W[0] * (64.0 / d)  # its target is 2: z about 64 there and 0 at its own
    loss, lse = torch.empty((1, R), device=cuda), torch.empty((1, R), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    check(h, W, target, weight, gh, None)
    up = torch.rand((1, R), generator=torch.Generator().manual_seed(1)).to(cuda) + 0.5
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    check(h, W, target, weight * up, gh, None)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('R,d,V', [(40, 64, 700), (96, 256, 700), (35, 97, 600)])
def test_the_head_at_targets_of_few_positions(cuda, R, d, V, dtype):
    """A target for four positions or fewer: both gradients."""
    import torch
    import paper_2606_00722_gb300 as epic
    h, W, target, weight = make(R, d, V, (R + 3) // 4, dtype, R + d)
    loss, lse = torch.empty((1, R), device=cuda), torch.empty((1, R), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    check(h, W, target, weight, gh, gw)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    epic.head_loss_backward(h, W, target, lse, torch.ones_like(loss), gh, gw, weight=weight)
    check(h, W, target, weight, gh, gw)
