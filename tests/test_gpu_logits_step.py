"""From the model's logits to commits and back: the row calls together with the
constraint calls, as the example runs them, and the loss as a torch operation."""
import importlib.util
import math
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location('constrained_distillation',
                                                  os.path.join(ROOT, 'examples', 'constrained_distillation.py'))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_learns_and_commits(cuda):
    import oracle
    r = example().run(rounds=12, batch=2, n=32)
    w = r['workload']
    o = oracle.Oracle(w.grammar, w.vocab)
    assert np.array_equal(r['valid'], o.validate_batch(r['start'], w.pos, r['cand']))
    assert np.array_equal(r['drawn_valid'], o.validate_batch(r['start'], w.pos, r['drawn']))
    assert r['losses'][-1] < r['losses'][0]
    # what was committed is a drawn token of its position, and the rest is as it was
    changed = np.argwhere(r['x'] != r['start'])
    assert len(changed) == r['committed']
    for b, i in changed:
        j = int(np.flatnonzero(w.pos[b] == i)[0])
        assert r['start'][b, i] == -1 and r['x'][b, i] in r['drawn'][b, j]


def test_step_from_logits_is_propose_then_decode(cuda):
    """A padded vocabulary and positions read out of the whole output; candidates as the two calls give them."""
    import torch
    import paper_2606_00722_gb300 as epic
    from synth import make_workload
    w = make_workload('json-schema', 3, batch=3, n=40, k=4, vocab_size=1024)
    B, k, K, V = w.B, w.k, 6, len(w.vocab)
    g = epic.Grammar(w.grammar)
    t = epic.LexTable(g, w.vocab)
    pos = torch.from_numpy(w.pos).to(cuda)
    full = torch.randn((B, w.n, V + 64), generator=torch.Generator().manual_seed(4)).to(cuda)
    full[..., V:] = math.inf  # the padding must not be seen
    logits = full[..., :V]
    out = []
    for joint in (True, False):
        x = torch.from_numpy(w.x).to(cuda)
        bufs = dict(cand=torch.empty((B, k, K), dtype=torch.int32, device=cuda), cand_conf=torch.empty((B, k, K), device=cuda),
                    valid=torch.empty((B, k, K), dtype=torch.uint8, device=cuda),
                    tok=torch.empty((B, k), dtype=torch.int32, device=cuda), conf=torch.empty((B, k), device=cuda),
                    selected=torch.empty((B, k), dtype=torch.uint8, device=cuda),
                    filled=torch.empty((B, k), dtype=torch.int32, device=cuda))
        want = torch.full((B,), 2, dtype=torch.int32, device=cuda)
        if joint:
            epic.decode_step_from_logits(g, t, x, pos, logits, want, bufs)
        else:
            epic.propose_topk(logits, bufs['cand'], bufs['cand_conf'], pos)
            epic.decode_step(g, t, x, pos, bufs['cand'], bufs['cand_conf'], want, bufs)
        out.append([x.cpu()] + [v.cpu() for v in bufs.values()])
        assert (bufs['cand'] < V).all() and (bufs['cand_conf'][..., :-1] >= bufs['cand_conf'][..., 1:]).all()
    for a, b in zip(*out):
        assert (a == b).all()


def test_rows_without_candidates_are_no_valid_ones(cuda):
    """The -1 candidates of an empty row are rejected by the checks and never picked."""
    import torch
    import paper_2606_00722_gb300 as epic
    from synth import make_workload
    w = make_workload('expr-tiny', 5)
    g = epic.Grammar(w.grammar)
    t = epic.LexTable(g, w.vocab)
    B, k, K, V = w.B, w.k, 4, len(w.vocab)
    logits = torch.full((B, w.n, V), -math.inf, device=cuda)
    pos = torch.from_numpy(w.pos).to(cuda)
    cand = torch.empty((B, k, K), dtype=torch.int32, device=cuda)
    conf = torch.empty((B, k, K), device=cuda)
    valid = torch.full((B, k, K), 7, dtype=torch.uint8, device=cuda)
    tok, best = torch.empty((B, k), dtype=torch.int32, device=cuda), torch.empty((B, k), device=cuda)
    epic.propose_topk(logits, cand, conf, pos)
    epic.validate_batch(g, t, torch.from_numpy(w.x).to(cuda), pos, cand, valid)
    epic.pick_candidates(cand, conf, valid, tok, best)
    assert (cand == -1).all() and (valid == 0).all() and (tok == -1).all()


def test_loss_as_a_torch_operation(cuda):
    """loss and gradient of distill_loss through torch against the same in 64 bits; tolerances as derived in the
    distillation tests: 3.2e-5 w tau^2 of a loss, 6e-5 w tau g of a gradient element."""
    import torch
    import paper_2606_00722_gb300 as epic
    gen = torch.Generator().manual_seed(9)
    B, n, V, K, tau = 2, 3, 500, 7, 2.0
    z = (torch.randn((B, n, V), generator=gen) * 2).to(cuda).requires_grad_()
    ids = torch.stack([torch.randperm(V, generator=gen)[:K] for _ in range(B * n)]).view(B, n, K).to(torch.int32).to(cuda)
    vals = torch.randn((B, n, K), generator=gen).to(cuda)
    weight = torch.rand((B, n), generator=gen).to(cuda)
    up = torch.rand((B, n), generator=gen).to(cuda)
    loss = epic.distill_loss(z, ids, vals, tau, weight)
    (loss * up).sum().backward()
    z64 = z.detach().double().requires_grad_()
    p = torch.softmax(vals.double() / tau, -1)
    lq = torch.log_softmax(z64 / tau, -1).gather(-1, ids.long())
    want = weight.double() * tau ** 2 * (p * (p.log() - lq)).sum(-1)
    (want * up.double()).sum().backward()
    assert ((loss.double() - want).abs() <= 3.2e-5 * weight.double() * tau ** 2).all()
    assert ((z.grad.double() - z64.grad).abs() <= (6e-5 * tau * (weight * up).double())[..., None]).all()


def test_loss_keeps_what_its_gradient_needs(cuda):
    """Targets overwritten between the loss and its gradient are an error, not a wrong gradient; the gradient itself has no
    further one; without rows that need gradients there is none."""
    import torch
    import paper_2606_00722_gb300 as epic
    z = torch.randn((1, 2, 50), device=cuda, requires_grad=True)
    ids = torch.arange(3, dtype=torch.int32, device=cuda).repeat(1, 2, 1)
    vals = torch.zeros((1, 2, 3), device=cuda)
    loss = epic.distill_loss(z, ids, vals)
    vals.add_(1.0)
    with pytest.raises(RuntimeError):
        loss.sum().backward()
    loss = epic.distill_loss(z, ids, vals)
    grad, = torch.autograd.grad(loss.sum(), z, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
    assert not epic.distill_loss(z.detach(), ids, vals).requires_grad
