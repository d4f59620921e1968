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
