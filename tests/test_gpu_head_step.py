"""The head's calls together, as a program runs them: training a head, laying it out in 8 bits, decoding through it."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def workload(cuda, **kw):
    import torch
    import paper_2606_00722_gb300 as epic
    from synth import make_workload
    w = make_workload('json-schema', 3, batch=3, n=40, k=4, vocab_size=1024)
    g = epic.Grammar(w.grammar)
    return w, g, epic.LexTable(g, w.vocab), torch.from_numpy(w.pos).to(cuda)


def buffers(B, k, K, cuda):
    import torch
    return dict(cand=torch.empty((B, k, K), dtype=torch.int32, device=cuda), cand_conf=torch.empty((B, k, K), device=cuda),
                valid=torch.empty((B, k, K), dtype=torch.uint8, device=cuda),
                tok=torch.empty((B, k), dtype=torch.int32, device=cuda), conf=torch.empty((B, k), device=cuda),
                selected=torch.empty((B, k), dtype=torch.uint8, device=cuda),
                filled=torch.empty((B, k), dtype=torch.int32, device=cuda))


@pytest.mark.parametrize('draws', [False, True])
def test_step_from_hidden_states_is_its_calls(cuda, draws):
    import torch
    import paper_2606_00722_gb300 as epic
    w, g, t, pos = workload(cuda)
    B, k, K, V, d = w.B, w.k, 6, len(w.vocab), 96
    gen = torch.Generator().manual_seed(4)
    hidden = torch.randn((B, w.n, d), generator=gen).to(torch.bfloat16).to(cuda)
    head = (torch.randn((V + 24, d), generator=gen) / 5).to(torch.bfloat16).to(cuda)
    head_q, head_scale = torch.empty((V + 24, d), dtype=torch.int8, device=cuda), torch.empty(V + 24, device=cuda)
    epic.quantize_rows(head[None], head_q[None], head_scale[None])
    u = torch.rand((B, k, K), generator=gen).to(cuda) if draws else None
    want = torch.full((B,), 2, dtype=torch.int32, device=cuda)
    out = []
    for joint in (True, False):
        x, bufs = torch.from_numpy(w.x).to(cuda), buffers(B, k, K, cuda)
        bufs.update(q=torch.empty((B, k, d), dtype=torch.int8, device=cuda), scale=torch.empty((B, k), device=cuda),
                    logits=torch.empty((B, k, V + 24), device=cuda)[..., :V + 24])
        if joint:
            epic.decode_step_from_hidden(g, t, x, pos, hidden, head_q, head_scale, want, bufs, u=u)
        else:
            epic.quantize_rows(hidden, bufs['q'], bufs['scale'], pos)
            epic.int8_logits(bufs['q'], bufs['scale'], head_q, head_scale, bufs['logits'])
            if draws:
                epic.sample_tokens(bufs['logits'], u, bufs['cand'], bufs['cand_conf'])
            else:
                epic.propose_topk(bufs['logits'], bufs['cand'], bufs['cand_conf'])
            epic.decode_step(g, t, x, pos, bufs['cand'], bufs['cand_conf'], want, bufs)
        out.append([x.cpu()] + [v.cpu() for v in bufs.values()])
    for a, b in zip(*out):
        assert torch.equal(a, b)
    # logits are near those of the weights as they were: 8 bits are off by half of 1/127 of a row's largest, twice
    sel = hidden.double()[torch.arange(B, device=cuda)[:, None], pos.long()]
    exact = sel @ head.double().t()
    top, low = sel.abs().amax(-1)[..., None], head.double().abs().amax(-1)
    tol = (top / 254 * head.double().abs().sum(-1) + low / 254 * sel.abs().sum(-1)[..., None] + d * top * low / 254 ** 2)
    assert ((bufs['logits'].double() - exact).abs() <= tol * 1.001).all()


def test_training_then_decoding(cuda):
    """A head and hidden states trained by the loss's gradients propose their targets, also through 8 bits."""
    import torch
    import paper_2606_00722_gb300 as epic
    w, g, t, pos = workload(cuda)
    B, n, V, d = w.B, w.n, len(w.vocab), 128
    gen = torch.Generator().manual_seed(6)
    target = torch.randint(0, V, (B, n), generator=gen).to(torch.int32).to(cuda)
    hidden = torch.randn((B, n, d), generator=gen).to(cuda).to(torch.bfloat16)
    master = (torch.randn((V, d), generator=gen) / math.sqrt(d)).to(cuda)
    work = torch.empty(epic.head_loss_workspace('step', hidden, master.to(torch.bfloat16)), dtype=torch.uint8, device=cuda)
    loss, gh = torch.empty((B, n), device=cuda), torch.empty_like(hidden)
    gw = torch.empty((V, d), dtype=torch.bfloat16, device=cuda)
    for _ in range(3):
        head = master.to(torch.bfloat16)
        epic.head_loss_step(hidden, head, target, loss, gh, gw, workspace=work)
        # one step's gradients are those of torch's own graph in 64 bits, up to bf16 (three roundings of 2^-8 of the terms)
        x, m = hidden.double().requires_grad_(), head.double().requires_grad_()
        torch.nn.functional.cross_entropy((x @ m.t()).view(-1, V), target.view(-1).long(), reduction='sum').backward()
        p = torch.softmax((x @ m.t()).detach(), -1)
        p.scatter_add_(2, target.long()[..., None], torch.full((B, n, 1), -1.0, dtype=torch.float64, device=cuda))
        assert ((gh.double() - x.grad).abs() <= 2.0 ** -7 * 1.1 * (p.abs() @ m.abs().detach())).all()
        terms = p.abs().view(-1, V).t() @ x.abs().detach().view(-1, d)
        assert ((gw.double() - m.grad).abs() <= 3 * 2.0 ** -8 * 1.1 * terms).all()
        master -= 0.2 * gw.float()
    head = master.to(torch.bfloat16)
    head_q, head_scale = torch.empty((V, d), dtype=torch.int8, device=cuda), torch.empty(V, device=cuda)
    epic.quantize_rows(head[None], head_q[None], head_scale[None])
    bufs = buffers(B, w.k, 4, cuda)
    bufs.update(q=torch.empty((B, w.k, d), dtype=torch.int8, device=cuda), scale=torch.empty((B, w.k), device=cuda),
                logits=torch.empty((B, w.k, V), dtype=torch.bfloat16, device=cuda))
    x = torch.from_numpy(w.x).to(cuda)
    epic.decode_step_from_hidden(g, t, x, pos, hidden, head_q, head_scale,
                                 torch.full((B,), 2, dtype=torch.int32, device=cuda), bufs)
    best = bufs['logits'].float().argmax(-1)
    assert torch.equal(bufs['cand'][..., 0].long(), best)
    assert ((bufs['cand'] >= 0) & (bufs['cand'] < V)).all()
