"""Edges of the row calls' arguments: what each answers there is stated in
include/epic.h."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize('dtype', ['float32', 'bfloat16'])
@pytest.mark.parametrize('V', [7, 300, 40001])
def test_temperature_minus_zero_is_zero(cuda, V, dtype):
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, K = 3, 2, 5
    z = torch.randn((B, n, V), generator=torch.Generator().manual_seed(V)).to(getattr(torch, dtype)).cuda()
    u = torch.rand((B, n, K), generator=torch.Generator().manual_seed(1)).cuda()
    top_p = torch.tensor([1.0, 0.9, 0.5], device='cuda')
    out = []
    for zero in (0.0, -0.0):
        T = torch.full((B,), zero, device='cuda')
        for call in ('propose', 'sample', 'top-p'):
            tok = torch.full((B, n, K), -7, dtype=torch.int32, device='cuda')
            p = torch.full((B, n, K), -7.0, device='cuda')
            if call == 'propose':
                epic.propose_topk(z, tok, p, temperature=T)
            else:
                epic.sample_tokens(z, u, tok, p, temperature=T, top_p=top_p if call == 'top-p' else None)
                assert (tok == z.float().argmax(-1, keepdim=True)).all() and (p == 1).all()
            out.append((tok, p))
    for (tok, p), (tok2, p2) in zip(out[:3], out[3:]):
        assert (tok == tok2).all() and (p == p2).all()


def both_forms(z, ids, vals, tau, weight):
    """(name, loss, gradient) of the single call and of the two calls."""
    import torch
    import paper_2606_00722_gb300 as epic
    loss, lse = torch.full(z.shape[:2], -7.0, device='cuda'), torch.full(z.shape[:2], -7.0, device='cuda')
    grad = torch.full_like(z, 7.0)
    epic.distill_step(z, ids, vals, loss, grad, tau=tau, weight=weight)
    yield 'step', loss.clone(), grad.clone()
    loss.fill_(-7.0)
    grad.fill_(7.0)
    epic.distill_forward(z, ids, vals, loss, lse, tau=tau, weight=weight)
    epic.distill_backward(z, ids, vals, lse, torch.ones_like(loss), grad, tau=tau, weight=weight)
    yield 'two calls', loss, grad


@pytest.mark.parametrize('n,V', [(4, 300), (4, 70001), (400, 300)])
def test_nan_shows_where_the_wanted_token_is_ruled_out(cuda, n, V):
    """NaN or +inf in a row makes its loss NaN also if the one token that the teacher wants is at -inf there."""
    import torch
    z = torch.randn((1, n, V), generator=torch.Generator().manual_seed(1)).cuda()
    ids = torch.full((1, n, 1), 3, dtype=torch.int32, device='cuda')
    vals = torch.zeros((1, n, 1), device='cuda')
    weight = torch.ones((1, n), device='cuda')
    z[..., 3] = -math.inf
    z[0, 1, 200] = math.nan
    z[0, 2, 200] = math.inf
    z[0, 3] = -math.inf
    for form, loss, grad in both_forms(z, ids, vals, 1.0, weight):
        assert loss[0, 0] == loss[0, 3] == math.inf, form
        assert torch.isnan(loss[0, 1:3]).all(), form
        assert torch.isnan(grad[0, 1:3, 200]).all() and torch.isfinite(grad[0, 0]).all(), form
        assert torch.isfinite(grad[0, 3]).all() and (loss[0, 4:] == math.inf).all(), form


def distill_rows64(z, ids, vals, tau, weight):
    """The loss by its definition in 64 bits, without a quotient by tau until differences are taken, and the gradient."""
    z, v, ids = z.double().cpu().numpy(), vals.double().cpu().numpy(), ids.cpu().numpy()
    w = weight.double().cpu().numpy()
    loss, grad = np.zeros(z.shape[:2]), np.zeros(z.shape)
    for b, i in np.ndindex(*z.shape[:2]):
        da, dz = v[b, i] - v[b, i].max(), z[b, i] - z[b, i].max()
        with np.errstate(under='ignore'):
            p, q = np.exp(da / tau), np.exp(dz / tau)
        log_a, log_z = math.log(p.sum()), math.log(q.sum())
        p, q = p / p.sum(), q / q.sum()
        for k, t in enumerate(ids[b, i]):
            if p[k] > 0:
                loss[b, i] += w[b, i] * tau * p[k] * (da[k] - dz[t] + tau * (log_z - log_a))
            q[t] -= p[k]
        grad[b, i] = w[b, i] * tau * q
    return loss, grad


@pytest.mark.parametrize('tau', [0.1, 0.5, 1.0, 1e-3, 1e-30, 1e-39])
@pytest.mark.parametrize('dtype', ['float32', 'float16', 'bfloat16'])
@pytest.mark.parametrize('n,V', [(6, 300), (6, 70001)])
def test_quotients_by_the_temperature_stay_in_range(cuda, n, V, dtype, tau):
    """Values and logits at the lowest and largest of 32 bits, divided by a small temperature, would pass 32 bits: entries
    that all are at the lowest value are alike, and a wanted token at the student's lowest value costs what it costs.
    Tolerances: 3.2e-5 w tau^2 of a loss and 6e-5 w tau of a gradient element, as derived in the distillation tests, 1e-6 of
    a loss, half a unit of the gradient's type, and for results below 2^-126 four units of 2^-149."""
    import torch
    low, most = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    dt = getattr(torch, dtype)
    z = torch.randn((1, n, V), generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    ids = torch.tensor([3, 9, 250], dtype=torch.int32, device='cuda').expand(1, n, 3).contiguous()
    vals = torch.tensor([0.5, -0.3, 0.1], device='cuda').expand(1, n, 3).contiguous()
    vals[0, 0] = low
    vals[0, 1, 1:] = low
    vals[0, 2, 0] = most
    z[0, 3, 3] = torch.finfo(dt).min
    z[0, 4] = torch.finfo(dt).min
    z[0, 4, 9] = 0.0
    weight = torch.tensor([[0.4, 0.3, 0.2, 0.1, 0.1, 1.0]], device='cuda')
    tau32 = float(np.float32(tau))
    want_loss, want_grad = distill_rows64(z, ids, vals, tau32, weight)
    assert np.isfinite(want_loss).all() and (np.abs(want_loss) < 3e38).all()
    w = weight.double().cpu().numpy()
    rel, tiny = {'float32': (2.0 ** -23, 2.0 ** -147), 'float16': (2.0 ** -11, 2.0 ** -25),
                 'bfloat16': (2.0 ** -8, 2.0 ** -132)}[dtype]  # bf16's smallest number is 2^-133
    for form, loss, grad in both_forms(z, ids, vals, tau, weight):
        loss, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
        assert (np.abs(loss - want_loss) <= 3.2e-5 * w * tau32 ** 2 + 1e-6 * np.abs(want_loss) + 2.0 ** -147).all(), form
        assert (np.abs(grad - want_grad) <= np.abs(want_grad) * rel + w[..., None] * tau32 * 6e-5 + tiny).all(), form


@pytest.mark.parametrize('tau,weight', [(0.5, 1.0), (0.999, 0.9), (1.0, 0.9), (10.0, 0.09), (10.0, 0.05), (1e-3, 50.0)])
@pytest.mark.parametrize('K', [1, 3, 40, 1000])
def test_costs_near_the_largest_number_do_not_overflow_on_the_way(cuda, K, tau, weight):
    """All wanted tokens at the lowest value of 32 bits: w tau 3.4e38, where that is a number.  Tolerance: 2.2e-6 of it for
    the probabilities' sum (2^-24 for each of 32 additions in a lane and 5 between lanes) and 1e-6 for what else rounds."""
    import torch
    n, V = 3, 5000
    z = torch.randn((1, n, V), generator=torch.Generator().manual_seed(1)).cuda()
    ids = torch.randperm(V, generator=torch.Generator().manual_seed(2))[:K].to(torch.int32)
    ids = ids.expand(1, n, K).contiguous().cuda()
    vals = torch.randn((1, n, K), generator=torch.Generator().manual_seed(3)).cuda()
    z.scatter_(2, ids.long(), torch.finfo(torch.float32).min)
    w = torch.full((1, n), weight, device='cuda')
    want = weight * tau * torch.finfo(torch.float32).max
    assert want < torch.finfo(torch.float32).max
    for form, loss, grad in both_forms(z, ids, vals, tau, w):
        assert ((loss.double() - want).abs() <= 3.2e-6 * want).all(), form
        assert torch.isfinite(grad).all(), form


@pytest.mark.parametrize('tau', [1e20, 1e30, 3e38])
def test_a_row_that_agrees_costs_nothing_at_any_temperature(cuda, tau):
    """One token, wanted: loss and gradient 0, also where tau^2 passes 32 bits."""
    import torch
    z = torch.tensor([[[2.5]], [[-3.0]]], device='cuda')
    ids = torch.zeros((2, 1, 1), dtype=torch.int32, device='cuda')
    vals = torch.tensor([[[0.0]], [[7.0]]], device='cuda')
    for form, loss, grad in both_forms(z, ids, vals, tau, torch.ones((2, 1), device='cuda')):
        assert (loss == 0).all() and (grad == 0).all(), form


@pytest.mark.parametrize('V,dtype', [(9, 'float32'), (3000, 'bfloat16'), (3000, 'float32'), (70001, 'float32')])
@pytest.mark.parametrize('top_k,top_p', [(0, 1.0), (100, 1.0), (1500, 0.7), (0, 0.4)])
def test_infinite_temperature_of_logits_whose_differences_pass_32_bits(cuda, V, dtype, top_k, top_p):
    """All tokens weigh 1 at T = +inf, also where the largest logit less theirs is no 32-bit number.  The reference takes
    the logits times 2^-40, which changes neither their order nor, at that temperature, their weights."""
    import torch
    import paper_2606_00722_gb300 as epic
    from test_gpu_logits_pick import sample_whole
    B, S, K = 3, 9, 8
    z = (torch.randn((B, 1, V), generator=torch.Generator().manual_seed(V)) * 1.1e38).clamp_(-3.3e38, 3.3e38)
    z = z.to(getattr(torch, dtype)).cuda()
    z[:, 0, 0], z[:, 0, 1] = torch.finfo(z.dtype).min, torch.finfo(z.dtype).max
    z[1, 0, 2::3] = -math.inf
    z[2, 0, 3] = math.nan
    u = torch.rand((B, 1, S), generator=torch.Generator().manual_seed(1)).cuda()
    T = torch.full((B,), math.inf, device='cuda')
    rules = [torch.full((B,), top_k, dtype=torch.int32, device='cuda'), torch.full((B,), top_p, device='cuda'),
             torch.zeros((B,), device='cuda')]
    tok = torch.full((B, 1, S), -7, dtype=torch.int32, device='cuda')
    prob = torch.full((B, 1, S), -7.0, device='cuda')
    epic.sample_tokens(z, u, tok, prob, temperature=T, top_k=rules[0], top_p=rules[1], min_p=rules[2])
    want_tok, want_prob, _ = sample_whole(z.float() * 2.0 ** -40, T, *rules, u)
    assert torch.equal(tok, want_tok)
    np.testing.assert_allclose(prob.cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)
    cand = torch.full((B, 1, K), -7, dtype=torch.int32, device='cuda')
    conf = torch.full((B, 1, K), -7.0, device='cuda')
    epic.propose_topk(z, cand, conf, temperature=T)
    there = (z > -math.inf).sum(-1, keepdim=True)
    want = torch.where(torch.arange(K, device='cuda') < there, 1.0 / there.double(), 0.0)
    assert ((conf.double() - want).abs() <= 2.4e-5 * want).all()
    assert ((cand >= 0) == (want > 0)).all()
