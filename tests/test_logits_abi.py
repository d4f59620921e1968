"""Refusals of the calls on rows of logits: found on the host before any device
work, so they need no GPU; empty calls are no-ops."""
import paper_2606_00722_gb300 as epic

P = 4096  # an address that nothing reads


def lib():
    return epic.load(epic.build())


def propose(base=P, dtype=2, B=2, n=3, V=100, sb=300, sn=100, pos=P, k=3, T=None, K=4, cand=P, conf=P):
    return lib().epic_propose_topk(base, dtype, B, n, V, sb, sn, pos, k, T, K, cand, conf, None)


def sample(base=P, dtype=2, B=2, n=3, V=100, sb=300, sn=100, pos=P, k=3, u=P, S=4, tok=P, prob=P):
    return lib().epic_sample_tokens(base, dtype, B, n, V, sb, sn, pos, k, None, None, None, None, u, S, tok, prob, None)


def step(base=P, dtype=2, B=2, n=3, V=100, sb=300, sn=100, ids=P, vals=P, K=4, tau=1.0, loss=P, grad=P, gb=300, gn=100):
    return lib().epic_distill_step(base, dtype, B, n, V, sb, sn, ids, vals, None, K, tau, None, loss, grad, gb, gn, None)


def forward(B=2, loss=P, lse=P):
    return lib().epic_distill_forward(P, 0, B, 3, 100, 300, 100, P, P, None, 4, 1.0, None, loss, lse, None)


def backward(B=2, lse=P, up=P, grad=P):
    return lib().epic_distill_backward(P, 0, B, 3, 100, 300, 100, P, P, None, 4, 1.0, None, lse, up, grad, 300, 100, None)


def test_bad_rows_are_refused():
    for call in (propose, sample, step):
        for bad in (dict(dtype=3), dict(dtype=-1), dict(B=-1), dict(n=-1), dict(V=-1), dict(sb=-1), dict(sn=-5),
                    dict(base=None), dict(base=P + 1), dict(base=P + 2, dtype=0)):
            assert call(**bad) == epic.epic.ERR_INVALID_ARG, (call, bad)
    for call in (propose, sample):
        for bad in (dict(k=-1), dict(pos=None, k=4)):
            assert call(**bad) == epic.epic.ERR_INVALID_ARG, (call, bad)


def test_bad_outputs_and_sizes_are_refused():
    for bad in (dict(K=-1), dict(cand=None), dict(conf=None)):
        assert propose(**bad) == epic.epic.ERR_INVALID_ARG, bad
    assert propose(K=257) == epic.epic.ERR_CAPACITY
    for call in (propose, sample):  # one more than the histograms of a row's slices take
        assert call(V=1047873, sn=1047873, sb=4000000) == epic.epic.ERR_CAPACITY
    assert step(V=0x7fffffff) == epic.epic.ERR_CAPACITY
    for bad in (dict(S=-1), dict(u=None), dict(tok=None), dict(prob=None)):
        assert sample(**bad) == epic.epic.ERR_INVALID_ARG, bad
    for bad in (dict(K=-1), dict(ids=None), dict(vals=None), dict(loss=None), dict(grad=None), dict(grad=P + 1),
                dict(gb=-1), dict(gn=-1), dict(tau=0.0), dict(tau=float('nan')), dict(tau=float('inf')), dict(tau=-2.0)):
        assert step(**bad) == epic.epic.ERR_INVALID_ARG, bad
    assert step(K=1025) == epic.epic.ERR_CAPACITY
    for bad in (dict(loss=None), dict(lse=None)):
        assert forward(**bad) == epic.epic.ERR_INVALID_ARG, bad
    for bad in (dict(lse=None), dict(up=None), dict(grad=None)):
        assert backward(**bad) == epic.epic.ERR_INVALID_ARG, bad


def test_empty_calls_touch_nothing():
    none = dict(base=None, B=0)
    assert propose(cand=None, conf=None, pos=None, k=3, **none) == 0
    assert propose(K=0, cand=None, conf=None) == 0
    assert sample(u=None, tok=None, prob=None, **none) == 0
    assert sample(S=0, u=None, tok=None, prob=None) == 0
    assert step(ids=None, vals=None, loss=None, grad=None, **none) == 0
    assert forward(B=0, loss=None, lse=None) == 0
    assert backward(B=0, lse=None, up=None, grad=None) == 0
