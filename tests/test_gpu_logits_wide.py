"""Rows of 126,000 tokens that one CTA has alone (more than 152 rows in the call),
and slices of that length in a cluster: draws against the definition in whole
numbers, ranks and distillation against 64 bits.  Tokens are equal; tolerances
are those of the tests of shorter rows, whose derivations hold here too: the two
sums of one of 384 threads have 165 elements of a row each, and 300 are allowed
for."""
import math

import numpy as np
import pytest

import test_gpu_logits_distill as distill
from test_gpu_logits_pick import RTOL, RULES, make_logits, propose64, rows64, run_sample, sample_whole

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan

# A row's values and how many tokens have them; the last one takes the rest.  In each, more than 65,538 elements of one
# slice share a bin of a histogram, and their masses' low 15 bits are above 16,384 on average.
ROWS = {
    'two in one bin': [(10.75, 1), (1.0078125, 120000), (1.0, None)],
    'target in the last': [(10.0, 1), (1.1328125, 120000), (1.125, None)],
    'three in the first bin': [(0.0, 1), (-0.25, 90000), (-0.5, None)],   # at a temperature of 1000
    'NaN in every warp': [(0.0, 1), (-10.5, 125000), (NAN, None)],
    # neighbouring floats that the temperature's factor rounds to one exponent: told apart by digits of the keys
    'one exponent': [(0.0, 1), (-5.6014175415, 70000), (-5.6014180183, None)],
}


def rows_of(kinds, V, dtype, seed):
    """[len(kinds)][1][V], each kind's values in random places"""
    import torch
    g = torch.Generator().manual_seed(seed)
    z = torch.empty((len(kinds), 1, V))
    for r, kind in enumerate(kinds):
        v, at = torch.empty(V), 0
        for value, many in ROWS[kind]:
            v[at:V if many is None else at + many] = value
            at = V if many is None else at + many
        z[r, 0] = v[torch.randperm(V, generator=g)]
    return z.to(dtype).cuda()


def check_draws(logits, copies, T, top_k, top_p, min_p, S=8):
    """Each row of logits [B][1][V] `copies` times in one call, with numbers of its own."""
    import torch
    import paper_2606_00722_gb300 as epic
    B = logits.shape[0]
    u = torch.rand((B, copies, S), generator=torch.Generator().manual_seed(3))
    u[:, 0, :4] = torch.tensor([0.0, 1.0, 1.0 - 2.0 ** -24, 0.5])
    u = u.cuda()
    pos = torch.zeros((B, copies), dtype=torch.int32, device='cuda')
    rules = [torch.tensor((x * B)[:B] if isinstance(x, list) else [x] * B, dtype=dt, device='cuda')
             for x, dt in ((T, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32))]
    tok = torch.full((B, copies, S), -7, dtype=torch.int32, device='cuda')
    prob = torch.full((B, copies, S), -7.0, device='cuda')
    epic.sample_tokens(logits, u, tok, prob, pos=pos, temperature=rules[0], top_k=rules[1], top_p=rules[2],
                       min_p=rules[3])
    for b in range(B):
        want_tok, want_prob, _ = sample_whole(logits[b:b + 1].float(), *(x[b:b + 1] for x in rules),
                                              u[b:b + 1].view(1, 1, copies * S))
        assert np.array_equal(tok[b].cpu().numpy().ravel(), want_tok.cpu().numpy().ravel())
        np.testing.assert_allclose(prob[b].cpu().numpy().ravel(), want_prob.cpu().numpy().ravel(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('top_p', [0.5, 0.8, 0.95, 0.99, 0.99999])
@pytest.mark.parametrize('kind,T,dtype', [('two in one bin', 1.0, 'bfloat16'), ('target in the last', 1.0, 'float16'),
                                          ('target in the last', 1.0, 'float32'),
                                          ('three in the first bin', 1000.0, 'bfloat16'),
                                          ('NaN in every warp', 1.0, 'bfloat16'), ('NaN in every warp', 1.0, 'float32'),
                                          ('one exponent', 1.0, 'float32')])
def test_masses_of_many_elements_of_one_bin(cuda, kind, T, dtype, top_p):
    import torch
    logits = rows_of([kind] * 2, 126000, getattr(torch, dtype), 11)
    check_draws(logits, 80, T, [0, 100000], top_p, [0.0, 1e-5])


@pytest.mark.parametrize('kind,T', [('two in one bin', 1.0), ('three in the first bin', 1000.0)])
def test_masses_of_many_elements_of_one_bin_in_a_cluster(cuda, kind, T):
    """Few rows of 1,000,000 tokens: eight slices of 125,000, most of them of one value."""
    import torch
    logits = rows_of([kind], 1000000, torch.float32, 12)
    check_draws(logits, 3, T, 0, 0.7, 0.0)


WIDE = [  # B, n, V, dtype, kind, pad, shift
    (32, 5, 126000, 'bf16', 'ties', 0, 0),
    (32, 5, 126000, 'bf16', 'peaked', 16, 0),
    (32, 5, 126000, 'bf16', 'specials', 0, 1),
    (32, 5, 125999, 'f32', 'specials', 1, 1),
    (32, 5, 126000, 'f16', 'normal', 3, 5),
    (32, 5, 150001, 'bf16', 'specials', 0, 0),  # two slices a row
]


@pytest.mark.parametrize('B,n,V,dtype,kind,pad,shift', WIDE)
def test_propose_wide_rows(cuda, B, n, V, dtype, kind, pad, shift):
    import torch
    import paper_2606_00722_gb300 as epic
    K = 32
    logits = make_logits(B, n, V, dtype, kind, V, pad, shift)
    T = torch.tensor([(0.7, 1.0, 1.9, 0.0, -1.0)[b % 5] for b in range(B)], device='cuda')
    cand = torch.full((B, n, K), -7, dtype=torch.int32, device='cuda')
    conf = torch.full((B, n, K), -7.0, device='cuda')
    epic.propose_topk(logits, cand, conf, temperature=T)
    want_cand, want_conf = propose64(rows64(logits, None), T.double().tolist(), K)
    assert np.array_equal(cand.cpu().numpy(), want_cand)
    np.testing.assert_allclose(conf.cpu().numpy(), want_conf, rtol=RTOL, atol=1e-30)


@pytest.mark.parametrize('rules', ['temperature', 'top-p', 'cold large top-k', 'min-p', 'large all', 'mixed'])
@pytest.mark.parametrize('B,n,V,dtype,kind,pad,shift', WIDE)
def test_sample_wide_rows(cuda, B, n, V, dtype, kind, pad, shift, rules):
    logits = make_logits(B, n, V, dtype, kind, V + 1, pad, shift)
    tok, prob, u, r = run_sample(logits, RULES[rules], 5)
    for b in range(0, B, 8):  # the reference sorts; eight sequences at a time
        want_tok, want_prob, _ = sample_whole(logits[b:b + 8].float(), *(x[b:b + 8] for x in r), u[b:b + 8])
        assert np.array_equal(tok[b:b + 8].cpu().numpy(), want_tok.cpu().numpy())
        np.testing.assert_allclose(prob[b:b + 8].cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('V,dtype,pad,shift', [(126000, 'bf16', 16, 0), (125999, 'f32', 0, 1), (150001, 'f16', 1, 3)])
def test_distill_wide_rows(cuda, V, dtype, pad, shift):
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, K, tau = 32, 5, 12, 1.5
    logits, ids, vals, valid, weight = distill.make(B, n, V, K, dtype, 'edges', V, pad, shift)
    up = (torch.rand((B, n), generator=torch.Generator().manual_seed(1)) + 0.2).cuda()
    want_loss, want_step = distill.distill64(logits, ids, vals, valid, weight, tau)
    want_grad = want_step * up.double().cpu().numpy()[..., None]
    loss, lse = torch.full((B, n), -7.0, device='cuda'), torch.full((B, n), -7.0, device='cuda')
    grad = torch.full((B, n, V), 7.0, dtype=logits.dtype, device='cuda')
    epic.distill_step(logits, ids, vals, loss, grad, tau=tau, weight=weight, valid=valid)
    distill.check(loss, grad, want_loss, want_step, ids, weight, tau, dtype)
    first = loss.clone()
    epic.distill_forward(logits, ids, vals, loss.fill_(-7.0), lse, tau=tau, weight=weight, valid=valid)
    assert torch.equal(loss, first)
    epic.distill_backward(logits, ids, vals, lse, up, grad.fill_(7.0), tau=tau, weight=weight, valid=valid)
    distill.check(loss, grad, want_loss, want_grad, ids, weight, tau, dtype, up)
