"""Training by the loss's gradients, then decoding through the trained head in 8 bits: the loss falls, logits are those of the 8-bit
numbers, and the tokens proposed are the targets."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_trained_targets_are_proposed(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    from synth import make_workload
    w = make_workload('json-schema', 3, batch=3, n=40, k=4, vocab_size=1024)
    g = epic.Grammar(w.grammar)
    t = epic.LexTable(g, w.vocab)
    pos = torch.from_numpy(w.pos).to(cuda)
    B, n, k, V, d, K = w.B, w.n, w.k, len(w.vocab), 128, 4
    gen = torch.Generator().manual_seed(6)
    target = torch.randint(0, V, (B, n), generator=gen).to(torch.int32).to(cuda)
    hidden = torch.randn((B, n, d), generator=gen).to(torch.bfloat16).to(cuda)
    master = (torch.randn((V, d), generator=gen) / math.sqrt(d)).to(cuda)
    loss, gh = torch.empty((B, n), device=cuda), torch.empty_like(hidden)
    gw = torch.empty((V, d), dtype=torch.bfloat16, device=cuda)
    sums = []
    # 120 positions in 128 dimensions, |h|^2 about 128: a step of 0.02 moves a target's logit by 2.5, others' by 0.2
    for _ in range(8):
        epic.head_loss_step(hidden, master.to(torch.bfloat16), target, loss, gh, gw)
        sums.append(float(loss.double().sum()))
        master -= 0.02 * gw.float()
    assert all(b < a for a, b in zip(sums, sums[1:])), sums
    head = master.to(torch.bfloat16)
    head_q, head_scale = torch.empty((V, d), dtype=torch.int8, device=cuda), torch.empty(V, device=cuda)
    epic.quantize_rows(head[None], head_q[None], head_scale[None])
    bufs = dict(cand=torch.empty((B, k, K), dtype=torch.int32, device=cuda), cand_conf=torch.empty((B, k, K), device=cuda),
                valid=torch.empty((B, k, K), dtype=torch.uint8, device=cuda),
                tok=torch.empty((B, k), dtype=torch.int32, device=cuda), conf=torch.empty((B, k), device=cuda),
                selected=torch.empty((B, k), dtype=torch.uint8, device=cuda),
                filled=torch.empty((B, k), dtype=torch.int32, device=cuda),
                q=torch.empty((B, k, d), dtype=torch.int8, device=cuda), scale=torch.empty((B, k), device=cuda),
                logits=torch.empty((B, k, V), device=cuda))
    x = torch.from_numpy(w.x).to(cuda)
    epic.decode_step_from_hidden(g, t, x, pos, hidden, head_q, head_scale,
                                 torch.full((B,), 2, dtype=torch.int32, device=cuda), bufs)
    # logits are those of the 8-bit numbers: an exact sum, rounded as it is scaled, twice (and the number's own 2^-24)
    row = torch.arange(B, device=cuda)[:, None]
    h = hidden.double()[row, pos.long()]
    exact = (bufs['q'].double() @ head_q.double().t()) * bufs['scale'].double()[..., None] * head_scale.double()
    assert ((bufs['logits'].double() - exact).abs() <= 3 * 2.0 ** -24 * exact.abs()).all()
    # 8 bits are off by half of 1/127 of a row's largest, in either factor
    z = h @ head.double().t()
    top, low = h.abs().amax(-1)[..., None] / 254, head.double().abs().amax(-1) / 254
    off = 1.001 * (top * head.double().abs().sum(-1) + low * h.abs().sum(-1)[..., None] + d * top * low)
    assert ((bufs['logits'].double() - z).abs() <= off).all()
    # a target is proposed first wherever it leads by more than that: at nearly all positions
    want = target[row, pos.long()]
    at = want.long()[..., None]
    lead = z.gather(-1, at) - off.gather(-1, at) - (z + off).scatter(-1, at, -math.inf).amax(-1, keepdim=True)
    sure = lead[..., 0] > 0
    assert int(sure.sum()) >= B * k - 1
    assert torch.equal(bufs['cand'][..., 0][sure], want[sure])
