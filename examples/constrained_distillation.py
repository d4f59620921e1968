"""A student learns the tokens that a grammar allows, from a teacher that does
not know the grammar.

Each round takes a batch of partially masked JSON texts.  The teacher's logits
at the masked positions give its K best tokens (propose_topk); the grammar
checks every one of them in its place (validate_batch); the student's logits
are pulled towards the teacher's probabilities over the candidates that pass
(distill_step: loss and gradient in one call) and its weights take a step.
Then one denoising step decodes from the student's logits, with draws instead
of ranks (decode_step_from_logits).

Both models are a table of logits by the token to the left, random for the
teacher, zero for the student: stand-ins that need no data.

    python examples/constrained_distillation.py [--rounds 20] [--batch 4]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_00722_gb300 as epic  # noqa: E402
from synth import make_workload  # noqa: E402


def run(rounds=20, batch=4, n=48, K=8, seed=1, rate=0.5):
    dev = torch.device('cuda')
    w = make_workload('json-schema', seed, batch=batch, n=n, k=4, vocab_size=2048)
    V, (B, k) = len(w.vocab), w.pos.shape
    grammar = epic.Grammar(w.grammar)
    table = epic.LexTable(grammar, w.vocab)
    x = torch.from_numpy(w.x).to(dev)
    pos = torch.from_numpy(w.pos).to(dev)
    gen = torch.Generator(device=dev).manual_seed(seed)
    left = torch.roll(x, 1, dims=1).clamp_(min=0).long()  # the token to the left of every position (0: none or masked)
    teacher = torch.randn((V, V), generator=gen, device=dev) * 2.0
    student = torch.zeros((V, V), device=dev)
    # the teacher knows some of the language: the tokens of the text itself
    truth = torch.from_numpy(w.witness).to(dev)
    known = truth >= 0
    teacher[left[known], truth[known].long()] += 6.0

    at = pos.long()
    context = torch.gather(left, 1, at)                       # [B][k]
    cand = torch.empty((B, k, K), dtype=torch.int32, device=dev)
    conf = torch.empty((B, k, K), device=dev)
    valid = torch.empty((B, k, K), dtype=torch.uint8, device=dev)
    loss = torch.empty((B, k), device=dev)
    grad = torch.empty((B, k, V), device=dev)
    epic.propose_topk(teacher[context], cand, conf)
    epic.validate_batch(grammar, table, x, pos, cand, valid)
    target = torch.log(conf)                                  # -inf where there was no candidate: it does not count
    losses = []
    for _ in range(rounds):
        epic.distill_step(student[context], cand, target, loss, grad, valid=valid)
        student.index_put_((context,), -rate * grad, accumulate=True)
        losses.append(loss.sum())

    # one step of decoding from the student, with draws
    bufs = dict(cand=torch.empty_like(cand), cand_conf=torch.empty_like(conf), valid=torch.empty_like(valid),
                tok=torch.empty((B, k), dtype=torch.int32, device=dev), conf=torch.empty((B, k), device=dev),
                selected=torch.empty((B, k), dtype=torch.uint8, device=dev),
                filled=torch.empty((B, k), dtype=torch.int32, device=dev))
    u = torch.rand((B, k, K), generator=gen, device=dev)
    n_target = torch.full((B,), k, dtype=torch.int32, device=dev)
    top_p = torch.full((B,), 0.95, device=dev)
    before = int((x < 0).sum())
    epic.decode_step_from_logits(grammar, table, x, pos, student[left], n_target, bufs, u=u, top_p=top_p)
    torch.cuda.synchronize()
    return {'losses': [float(v) for v in losses], 'valid': valid.cpu().numpy(), 'cand': cand.cpu().numpy(),
            'x': x.cpu().numpy(), 'committed': before - int((x < 0).sum()), 'drawn': bufs['cand'].cpu().numpy(),
            'drawn_valid': bufs['valid'].cpu().numpy(), 'workload': w, 'start': np.asarray(w.x)}


if __name__ == '__main__':
    ap = argparse.ArgumentParser()
    ap.add_argument('--rounds', type=int, default=20)
    ap.add_argument('--batch', type=int, default=4)
    args = ap.parse_args()
    r = run(args.rounds, args.batch)
    print('loss %.3f -> %.3f; %d of %d teacher candidates valid, %d of %d drawn ones; %d tokens committed' % (
        r['losses'][0], r['losses'][-1], int((r['valid'] == 1).sum()), r['valid'].size,
        int((r['drawn_valid'] == 1).sum()), r['drawn_valid'].size, r['committed']))
