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
