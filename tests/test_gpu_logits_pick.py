"""Candidates from logits (epic_propose_topk, epic_sample_tokens) against their
definitions: orders and draws exactly, probabilities against 64 bits.

Tolerance of a probability, from the arithmetic: the exponent y = (z - m) c has
two roundings, |y| 2^-23 of absolute error (|y| <= 60 where it matters), the
exponential 2 ulp, the sum of weights at most 2^-24 for each of the ~300
additions in one thread's chain: 60 ln2 2^-23 + 2^-22 + 300 2^-24 < 2.4e-5."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

RTOL = 2.4e-5
DT = ('f32', 'f16', 'bf16')


def _dtype(name):
    import torch
    return {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}[name]


def make_logits(B, n, V, dtype, kind, seed, pad=0, shift=0):
    """[B][n][V] view of a larger buffer whose other elements are NaN and inf."""
    import torch
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, n, V), generator=g) * 2.0
    if kind == 'peaked' and V > 4:
        z.scatter_(2, torch.randint(0, V, (B, n, 4), generator=g), 9.0)
    elif kind == 'ties':
        z = torch.randint(-2, 3, (B, n, V), generator=g).float()
        z[z == 0] = torch.where(torch.rand(int((z == 0).sum()), generator=g) < 0.5, -0.0, 0.0)
    elif kind == 'constant':
        z = torch.full((B, n, V), 1.5)
    elif kind == 'sorted':
        z = torch.sort(z, dim=2).values
    elif kind == 'specials':
        z[torch.rand(z.shape, generator=g) < 0.3] = -math.inf
        z[torch.rand(z.shape, generator=g) < 0.1] = math.nan
        z[torch.rand(z.shape, generator=g) < 0.1] = torch.finfo(_dtype(dtype)).min
        z[0, 0] = -math.inf                 # a row that the mask leaves empty
        if n > 1:
            z[0, 1] = torch.finfo(_dtype(dtype)).min   # a row at the type's lowest value
            z[-1, -1] = math.nan
        if n > 2:
            z[0, 2, ::3] = math.inf
    full = torch.full((B, n, V + pad), math.nan)
    full[..., V:].masked_fill_(torch.rand((B, n, pad), generator=g) < 0.5, math.inf)
    full[..., :V] = z
    flat = torch.full((shift + full.numel() + 16,), math.inf, dtype=_dtype(dtype), device='cuda')
    flat[shift:shift + full.numel()] = full.reshape(-1).to('cuda')
    return flat[shift:shift + full.numel()].view(B, n, V + pad)[..., :V]


def rows64(logits, pos):
    z = logits.double().cpu().numpy()
    B, n, V = z.shape
    if pos is None:
        return z
    out = np.full((B, pos.shape[1], V), -np.inf)
    for b in range(B):
        for j, i in enumerate(pos[b].tolist()):
            if 0 <= i < n:
                out[b, j] = z[b, i]
    return out


def propose64(z, T, K):
    """Row by row in 64 bits: (tokens, probabilities)."""
    B, k, V = z.shape
    cand = np.full((B, k, K), -1, np.int64)
    conf = np.zeros((B, k, K))
    for b in range(B):
        for j in range(k):
            if not T[b] >= 0:
                continue
            v = np.where(np.isnan(z[b, j]), -np.inf, z[b, j])
            order = np.argsort(-v, kind='stable')
            order = order[v[order] > -np.inf][:K]
            if not len(order):
                continue
            m = v.max()
            if T[b] == 0:
                w = np.zeros(V)
                w[order[0]] = 1
            elif m == np.inf:
                w = (v == m).astype(float)
            else:
                w = np.exp((v - m) / T[b])
            cand[b, j, :len(order)] = order
            conf[b, j, :len(order)] = w[order] / w.sum()
    return cand, conf


CASES = [  # B, n, k, V, K, dtype, kind, pad, shift
    (1, 1, 1, 1, 1, 'f32', 'normal', 0, 0),
    (2, 3, 3, 1, 5, 'bf16', 'specials', 1, 1),
    (1, 32, 8, 256, 8, 'f32', 'normal', 0, 0),
    (3, 5, 5, 7, 12, 'f16', 'ties', 0, 3),
    (2, 4, 4, 255, 256, 'bf16', 'specials', 0, 0),
    (2, 4, 2, 1000, 64, 'f32', 'ties', 3, 1),
    (2, 3, 3, 1021, 65, 'f16', 'constant', 0, 0),
    (3, 4, 3, 4099, 13, 'bf16', 'peaked', 5, 7),
    (2, 4, 4, 32768, 16, 'bf16', 'normal', 0, 0),
    (2, 4, 4, 32771, 16, 'f32', 'specials', 0, 2),
    (1, 3, 3, 50021, 53, 'f16', 'peaked', 0, 5),
    (1, 2, 2, 126000, 256, 'bf16', 'normal', 16, 0),
    (1, 2, 2, 126000, 32, 'bf16', 'constant', 0, 0),
    (1, 2, 2, 126000, 100, 'bf16', 'ties', 0, 0),
    (1, 2, 2, 126000, 32, 'f32', 'sorted', 1, 0),
    (1, 2, 2, 131071, 7, 'f32', 'ties', 0, 1),
    (1, 2, 2, 500009, 20, 'f32', 'normal', 0, 0),   # past the cluster's shared memory
    (1, 2, 2, 500009, 20, 'f32', 'ties', 0, 3),
    (1, 1, 1, 900001, 33, 'bf16', 'specials', 2, 1),
]


@pytest.mark.parametrize('B,n,k,V,K,dtype,kind,pad,shift', CASES)
def test_propose(cuda, B, n, k, V, K, dtype, kind, pad, shift):
    import torch
    import paper_2606_00722_gb300 as epic
    logits = make_logits(B, n, V, dtype, kind, V + K, pad, shift)
    g = torch.Generator().manual_seed(V)
    pos = None if k == n else torch.stack([torch.randperm(n, generator=g)[:k] for _ in range(B)]).to(torch.int32).cuda()
    T = torch.tensor([(0.7, 1.0, 1.9)[b % 3] for b in range(B)], device='cuda')
    cand = torch.full((B, k, K), -7, dtype=torch.int32, device='cuda')
    conf = torch.full((B, k, K), -7.0, device='cuda')
    epic.propose_topk(logits, cand, conf, pos=pos, temperature=T)
    want_cand, want_conf = propose64(rows64(logits, pos), T.double().tolist(), K)
    assert np.array_equal(cand.cpu().numpy(), want_cand)
    np.testing.assert_allclose(conf.cpu().numpy(), want_conf, rtol=RTOL, atol=1e-30)


def test_propose_temperatures_and_positions(cuda):
    """No temperature is 1; 0 is certain; below 0 and NaN give nothing; positions outside the row give nothing."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, V, K = 5, 6, 777, 9
    logits = make_logits(B, n, V, 'bf16', 'ties', 3)
    pos = torch.tensor([[0, 5, -1, 6]] * B, dtype=torch.int32, device='cuda')
    for temps in (None, [0.0, -1.0, math.nan, 1.3, 30.0]):
        T = None if temps is None else torch.tensor(temps, device='cuda')
        cand = torch.full((B, 4, K), -7, dtype=torch.int32, device='cuda')
        conf = torch.full((B, 4, K), -7.0, device='cuda')
        epic.propose_topk(logits, cand, conf, pos=pos, temperature=T)
        want_cand, want_conf = propose64(rows64(logits, pos), temps or [1.0] * B, K)
        assert np.array_equal(cand.cpu().numpy(), want_cand)
        np.testing.assert_allclose(conf.cpu().numpy(), want_conf, rtol=RTOL, atol=1e-30)


# Rows enough for every place on the GPU: a CTA takes several in a pipeline.
MANY = [  # B, n, V, dtype, kind, pad, shift
    (62, 5, 16411, 'bf16', 'normal', 0, 1),
    (62, 5, 16411, 'f16', 'specials', 3, 0),
    (103, 7, 8209, 'f32', 'specials', 0, 1),
    (64, 5, 16384, 'bf16', 'ties', 0, 0),
    (41, 8, 32771, 'bf16', 'peaked', 5, 0),
]


@pytest.mark.parametrize('B,n,V,dtype,kind,pad,shift', MANY)
def test_propose_many_rows(cuda, B, n, V, dtype, kind, pad, shift):
    import torch
    import paper_2606_00722_gb300 as epic
    logits = make_logits(B, n, V, dtype, kind, V, pad, shift)
    K = 12
    g = torch.Generator().manual_seed(V)
    pos = torch.stack([torch.randperm(n, generator=g) for _ in range(B)]).to(torch.int32)
    pos[3, 0], pos[B - 1, n - 1] = -1, n  # rows of nothing among the others
    pos = pos.cuda()
    T = torch.tensor([(0.7, 1.0, 1.9, 0.0, -1.0)[b % 5] for b in range(B)], device='cuda')
    for _ in range(2):
        cand = torch.full((B, n, K), -7, dtype=torch.int32, device='cuda')
        conf = torch.full((B, n, K), -7.0, device='cuda')
        epic.propose_topk(logits, cand, conf, pos=pos, temperature=T)
        want_cand, want_conf = propose64(rows64(logits, pos), T.double().tolist(), K)
        assert np.array_equal(cand.cpu().numpy(), want_cand)
        np.testing.assert_allclose(conf.cpu().numpy(), want_conf, rtol=RTOL, atol=1e-30)


# ---------------------------------------------------------------- draws

def share(a, q):
    return a * (q >> 24) + ((a * (q & 0xffffff)) >> 24)


def sample_whole(z, T, top_k, top_p, min_p, u):
    """The definition in whole numbers, with torch's 32-bit operations: z [B][k][V] float32 on the GPU, rules [B],
    u [B][k][S]; (tokens, probabilities, kept sets)."""
    import torch
    V = z.shape[-1]
    z = torch.where(torch.isnan(z), -math.inf, z)
    T, top_k, top_p, min_p = (x[:, None, None] for x in (T, top_k, top_p, min_p))
    m = z.amax(-1, keepdim=True)
    # a division: a number over a tensor would be torch's reciprocal times the number, with one more rounding
    c = torch.clamp(torch.full_like(T, 1.4426950408889634) / T, max=3.4028234663852886e38)
    w = torch.exp2((z - m) * c)
    w = torch.where(m == math.inf, (z == m).float(), w)
    w = torch.where(z > -math.inf, w, 0.0)
    q = torch.round(w * 2.0 ** 30).long()
    zs, order = torch.sort(z + 0.0, dim=-1, descending=True, stable=True)
    rank = torch.arange(V, device=z.device)
    best = rank < torch.where(T == 0, 1, torch.where(top_k <= 0, V, top_k))
    qs = torch.where(best, q.gather(-1, order), 0)
    upto = qs.cumsum(-1)
    part = share(torch.round(top_p.clamp(0, 1).double() * 2.0 ** 24).long(), upto[..., -1:])
    keep = (rank == 0) | (best & (upto - qs < part) & (w.gather(-1, order) >= min_p))
    keep = torch.zeros_like(keep).scatter_(-1, order, keep & (zs > -math.inf))
    upto = torch.where(keep, q, 0).cumsum(-1)
    mass = upto[..., -1:]
    t = torch.minimum(share(torch.floor(u.double() * 2.0 ** 24).long(), mass), mass - 1)
    tok = (upto[:, :, None, :] <= t[..., None]).sum(-1).clamp(max=V - 1)
    prob = w.gather(-1, tok) * 2.0 ** 30 / mass.float()
    ok = (mass > 0) & (T >= 0) & (u >= 0) & (u <= 1)
    return torch.where(ok, tok, -1).int(), torch.where(ok, prob, 0.0), keep


RULES = {  # temperature, top-k, top-p, min-p of the batch's sequences in turn; None: not given
    'temperature': ([0.7, 1.0, 2.5], None, None, None),
    'none': (None, None, None, None),
    'top-k': ([0.9, 1.4], [1, 50, 64, 3], None, None),
    'large top-k': ([1.0], [65, 300, 4000, 100000], None, None),
    'top-p': ([1.0, 0.8], None, [0.9, 0.5, 0.99, 0.0], None),
    'cold large top-k': ([0.05, 0.3], [300, 4000, 40000], [1.0, 0.9], None),
    'min-p': ([1.0], None, None, [0.05, 0.3, 1.0, 2.0]),
    'all': ([0.6, 1.1], [40, 64, 7], [0.95, 0.6], [0.02, 0.1]),
    'large all': ([1.3, 3.0], [500, 2000], [0.95, 0.7], [1e-4, 0.0]),
    'mixed': ([0.0, 1.0, 1.7, 0.5], [0, 50, 1000], [1.0, 0.9, 0.4, 1.5], [0.0, 0.05, -1.0]),
}


def run_sample(logits, rules, S, pos=None, seed=5, u=None):
    import torch
    import paper_2606_00722_gb300 as epic
    B = logits.shape[0]
    k = logits.shape[1] if pos is None else pos.shape[1]
    got = []
    for values, off, dt in zip(rules, (1.0, 0, 1.0, 0.0), (torch.float32, torch.int32, torch.float32, torch.float32)):
        given = None if values is None else torch.tensor([values[b % len(values)] for b in range(B)], dtype=dt, device='cuda')
        got.append((given, torch.full((B,), off, dtype=dt, device='cuda') if given is None else given))
    if u is None:
        u = torch.rand((B, k, S), generator=torch.Generator().manual_seed(seed))
        u.view(-1)[::7] = 0.0
        u.view(-1)[3::11] = 1.0
        u.view(-1)[5::13] = 1.0 - 2.0 ** -24
        u = u.cuda()
    tok = torch.full((B, k, S), -7, dtype=torch.int32, device='cuda')
    prob = torch.full((B, k, S), -7.0, device='cuda')
    epic.sample_tokens(logits, u, tok, prob, pos=pos, temperature=got[0][0], top_k=got[1][0], top_p=got[2][0],
                       min_p=got[3][0])
    return tok, prob, u, [x[1] for x in got]


SAMPLES = [  # B, n, V, S, dtype, kind, pad, shift
    (1, 1, 1, 3, 'f32', 'normal', 0, 0),
    (2, 3, 2, 2, 'bf16', 'specials', 1, 1),
    (4, 3, 256, 5, 'f32', 'peaked', 0, 0),
    (4, 3, 255, 33, 'f16', 'specials', 0, 3),
    (4, 2, 1000, 4, 'bf16', 'ties', 0, 0),
    (4, 3, 4099, 4, 'f32', 'specials', 5, 1),
    (4, 2, 4099, 9, 'bf16', 'constant', 0, 0),
    (4, 2, 32771, 8, 'bf16', 'peaked', 0, 3),
    (4, 1, 65521, 4, 'f16', 'normal', 1, 0),
    (4, 1, 65521, 4, 'f32', 'ties', 0, 0),
    (4, 1, 126000, 3, 'bf16', 'normal', 16, 0),
    (4, 1, 126000, 16, 'bf16', 'ties', 0, 0),
    (4, 1, 126000, 2, 'f32', 'sorted', 0, 1),
    (4, 1, 126000, 2, 'bf16', 'constant', 0, 1),
    (4, 1, 420001, 2, 'f32', 'peaked', 0, 1),   # past the cluster's shared memory
]


@pytest.mark.parametrize('rules', sorted(RULES))
@pytest.mark.parametrize('B,n,V,S,dtype,kind,pad,shift', SAMPLES)
def test_sample_is_the_definition(cuda, B, n, V, S, dtype, kind, pad, shift, rules):
    logits = make_logits(B, n, V, dtype, kind, V + S, pad, shift)
    tok, prob, u, r = run_sample(logits, RULES[rules], S)
    want_tok, want_prob, _ = sample_whole(logits.float(), *r, u)
    assert np.array_equal(tok.cpu().numpy(), want_tok.cpu().numpy())
    np.testing.assert_allclose(prob.cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('rules', ['large top-k', 'top-p', 'large all'])
@pytest.mark.parametrize('V', [700, 1900, 3500, 5120, 6500, 9000, 10235, 10245, 12000])
def test_sample_many_equal_values(cuda, V, rules):
    """Five values share the row, so the threshold falls among 140 to 2,400 equal ones: lists of every size that is sorted,
    full ones, and the first that are too long."""
    logits = make_logits(4, 2, V, 'f32', 'ties', V)
    tok, prob, u, r = run_sample(logits, RULES[rules], 12)
    want_tok, want_prob, _ = sample_whole(logits, *r, u)
    assert np.array_equal(tok.cpu().numpy(), want_tok.cpu().numpy())
    np.testing.assert_allclose(prob.cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('V,dtype,kind', [(1, 'f32', 'normal'), (700, 'bf16', 'specials'), (4099, 'f32', 'normal'),
                                          (5003, 'f16', 'specials'), (40001, 'bf16', 'specials')])
@pytest.mark.parametrize('rules', [(None, None, None), (None, [0.9, 0.3], None), ([300, 600], [1.0, 0.7], [0.5]),
                                   ([7], [0.9], None)])
def test_sample_at_infinite_temperature(cuda, V, dtype, kind, rules):
    """Every token that is one weighs 1; -inf and NaN, times an exponent's factor of 0, still weigh nothing."""
    logits = make_logits(2, 3, V, dtype, kind, V)
    tok, prob, u, r = run_sample(logits, ([math.inf],) + rules, 6)
    want_tok, want_prob, _ = sample_whole(logits.float(), *r, u)
    assert np.array_equal(tok.cpu().numpy(), want_tok.cpu().numpy())
    np.testing.assert_allclose(prob.cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('V,dtype', [(3, 'f32'), (700, 'bf16'), (40001, 'f16')])
def test_propose_at_infinite_temperature(cuda, V, dtype):
    import torch
    import paper_2606_00722_gb300 as epic
    K = 8
    logits = make_logits(2, 3, V, dtype, 'specials', V)
    pos = torch.arange(3, dtype=torch.int32).repeat(2, 1).cuda()
    cand = torch.full((2, 3, K), -7, dtype=torch.int32, device='cuda')
    conf = torch.full((2, 3, K), -7.0, device='cuda')
    epic.propose_topk(logits, cand, conf, temperature=torch.full((2,), math.inf, device='cuda'))
    z = rows64(logits, pos)
    want_cand, _ = propose64(z, [1.0, 1.0], K)  # the order does not depend on the temperature
    assert np.array_equal(cand.cpu().numpy(), want_cand)
    some = np.where(np.isposinf(z).any(-1), np.isposinf(z).sum(-1), (z > -np.inf).sum(-1))  # NaN is not above -inf
    want = np.where(want_cand >= 0, 1.0 / np.maximum(some, 1)[..., None], 0.0)
    want[np.isposinf(z).any(-1)[..., None] & ~np.isposinf(np.take_along_axis(z, want_cand.clip(0), -1))] = 0.0
    np.testing.assert_allclose(conf.cpu().numpy(), want, rtol=RTOL, atol=1e-30)


@pytest.mark.parametrize('rules', ['temperature', 'large all', 'mixed'])
@pytest.mark.parametrize('B,n,V,dtype,kind,pad,shift', MANY)
def test_sample_many_rows(cuda, B, n, V, dtype, kind, pad, shift, rules):
    logits = make_logits(B, n, V, dtype, kind, V + 1, pad, shift)
    tok, prob, u, r = run_sample(logits, RULES[rules], 5)
    want_tok, want_prob, _ = sample_whole(logits.float(), *r, u)
    assert np.array_equal(tok.cpu().numpy(), want_tok.cpu().numpy())
    np.testing.assert_allclose(prob.cpu().numpy(), want_prob.cpu().numpy(), rtol=2.0 ** -21, atol=0)


@pytest.mark.parametrize('rules', ['temperature', 'top-k', 'min-p', 'all'])
@pytest.mark.parametrize('V,dtype', [(300, 'f32'), (5003, 'bf16'), (40000, 'f16')])
def test_evenly_spread_numbers_give_the_distribution(cuda, V, dtype, rules):
    """S numbers spread evenly over [0, 1) draw every token S p times, within one draw and the sums' error in 64 bits:
    the kept mass is off by at most V 2^-31 + 2.4e-5 of itself, at either end of a token's interval."""
    import torch
    B, S = 2, 4096
    logits = make_logits(B, 1, V, dtype, 'peaked', 11)
    u = ((torch.arange(S) + 0.5) / S).float().cuda().expand(B, 1, S).contiguous()
    tok, prob, _, (T, top_k, top_p, min_p) = run_sample(logits, RULES[rules], S, u=u)
    for b in range(B):
        z = logits[b, 0].double().cpu().numpy()
        order = np.argsort(-z, kind='stable')
        p = np.exp((z - z.max()) / float(T[b]))
        kept = np.zeros(V, bool)
        many = int(top_k[b]) if top_k[b] > 0 else V
        first = order[:many]
        before = np.concatenate([[0], np.cumsum(p[first])[:-1]]) / p[first].sum()
        kept[first[(before < min(1.0, float(top_p[b]))) & (p[first] >= float(min_p[b]))]] = True
        p = np.where(kept, p, 0) / p[kept].sum()
        count = np.bincount(tok[b, 0].cpu().numpy(), minlength=V)
        assert (count[~kept] == 0).all()
        assert np.abs(count - S * p).max() <= 1 + 2 * S * (V * 2.0 ** -31 + 2.4e-5)
        np.testing.assert_allclose(prob[b, 0].cpu().numpy(), p[tok[b, 0].cpu().numpy()], rtol=2.4e-5 + V * 2.0 ** -31)


def test_sample_bad_rows_and_numbers(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    logits = make_logits(6, 2, 500, 'f32', 'normal', 1)
    pos = torch.tensor([[0, 2]] * 5 + [[-1, 1]], dtype=torch.int32, device='cuda')  # 2 and -1: no such position
    T = torch.tensor([1.0, -1.0, math.nan, 1.0, 1.0, 1.0], device='cuda')
    top_p = torch.tensor([0.9, 0.9, 0.9, math.nan, 0.9, 0.9], device='cuda')
    min_p = torch.tensor([0.0, 0.0, 0.0, 0.0, math.nan, 0.0], device='cuda')
    u = torch.tensor([0.3, -0.1, 1.1, math.nan], device='cuda').expand(6, 2, 4).contiguous()
    tok = torch.full((6, 2, 4), -7, dtype=torch.int32, device='cuda')
    prob = torch.full((6, 2, 4), -7.0, device='cuda')
    epic.sample_tokens(logits, u, tok, prob, pos=pos, temperature=T, top_p=top_p, min_p=min_p)
    good = torch.zeros((6, 2, 4), dtype=torch.bool)
    good[0, 0, 0] = good[5, 1, 0] = True
    assert (tok.cpu()[good] >= 0).all() and (prob.cpu()[good] > 0).all()
    assert (tok.cpu()[~good] == -1).all() and (prob.cpu()[~good] == 0).all()


def test_a_draw_depends_on_its_row_alone(cuda):
    """The same row and numbers in another batch, at another address and stride, draw the same tokens."""
    import torch
    a = make_logits(1, 1, 50021, 'bf16', 'peaked', 4)
    rules = ([1.1], None, [0.95], None)
    u = torch.rand((1, 1, 64), generator=torch.Generator().manual_seed(1)).cuda()
    tok, prob, _, _ = run_sample(a, rules, 64, u=u)
    wide = torch.zeros((200, 1, 50021 + 3), dtype=a.dtype, device='cuda')
    wide[:, :, 1:50022] = a
    tok2, prob2, _, _ = run_sample(wide[:, :, 1:50022], rules, 64, u=u.expand(200, 1, 64).contiguous())
    assert (tok2 == tok).all() and (prob2 == prob).all()


def test_rows_past_32_bit_offsets_and_odd_strides(cuda):
    """Elements past 2^32 bytes and 2^31 elements from the base; batch strides of 0 and transposed layouts."""
    import torch
    import paper_2606_00722_gb300 as epic
    V, K = 4096, 4
    far = (1 << 31) + 8
    flat = torch.empty((far + V,), dtype=torch.bfloat16, device='cuda')
    z = torch.randn((2, V), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    flat[:V], flat[far:] = z[0], z[1]
    cand = torch.empty((1, 2, K), dtype=torch.int32, device='cuda')
    conf = torch.empty((1, 2, K), device='cuda')
    epic.propose_topk(flat.as_strided((1, 2, V), (0, far, 1)), cand, conf)
    want, _ = propose64(z.double().cpu().numpy()[None], [1.0], K)
    assert np.array_equal(cand.cpu().numpy(), want)
    del flat
    many = torch.empty((3, 2, K), dtype=torch.int32, device='cuda')
    epic.propose_topk(z[None].expand(3, 2, V), many, torch.empty((3, 2, K), device='cuda'))
    assert (many == cand).all()
    turned = z[:, None, :].contiguous().transpose(0, 1)  # [1][2][V] with the strides of [2][1][V]
    epic.propose_topk(turned, cand, conf)
    assert np.array_equal(cand.cpu().numpy(), want)


def test_streams_and_graphs(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    logits = make_logits(2, 2, 30000, 'bf16', 'peaked', 8)
    u = torch.rand((2, 2, 8), generator=torch.Generator().manual_seed(3)).cuda()
    tok = torch.empty((2, 2, 8), dtype=torch.int32, device='cuda')
    prob = torch.empty((2, 2, 8), device='cuda')
    top_p = torch.full((2,), 0.9, device='cuda')
    epic.sample_tokens(logits, u, tok, prob, top_p=top_p)
    want = tok.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    tok.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        epic.sample_tokens(logits, u, tok, prob, top_p=top_p)
    side.synchronize()
    assert (tok == want).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        epic.sample_tokens(logits, u, tok, prob, top_p=top_p)
    other = make_logits(2, 2, 30000, 'bf16', 'peaked', 9)
    logits.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    replayed = tok.clone()
    epic.sample_tokens(other, u, tok, prob, top_p=top_p)
    assert (tok == replayed).all() and not (tok == want).all()


def test_refusals(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    z = torch.zeros((2, 3, 100), device='cuda')
    cand = torch.zeros((2, 3, 4), dtype=torch.int32, device='cuda')
    conf = torch.zeros((2, 3, 4), device='cuda')
    pos = torch.zeros((2, 3), dtype=torch.int32, device='cuda')
    for args, kw in [((z.double(), cand, conf), {}), ((z.cpu(), cand, conf), {}), ((z[0], cand, conf), {}),
                     ((z.transpose(1, 2), cand, conf), {}), ((z, cand.long(), conf), {}),
                     ((z, cand, conf[:, :, :3]), {}), ((z, cand.transpose(0, 1), conf), {}),
                     ((z, cand, conf), {'pos': pos.long()}), ((z, cand, conf), {'pos': pos[:, :2]}),
                     ((z, cand, conf), {'temperature': torch.ones(3, device='cuda')})]:
        with pytest.raises(ValueError):
            epic.propose_topk(*args, **kw)
    u = torch.zeros((2, 3, 4), device='cuda')
    with pytest.raises(ValueError):
        epic.sample_tokens(z, u, cand, conf, top_k=torch.ones(2, device='cuda'))
    with pytest.raises(ValueError):
        epic.sample_tokens(z, u.double(), cand, conf)
    big = torch.zeros((2, 3, 257), dtype=torch.int32, device='cuda')
    with pytest.raises(epic.EpicError) as e:
        epic.propose_topk(z, big, big.float())
    assert e.value.status == 6  # EPIC_ERR_CAPACITY
    five = torch.zeros((2, 5, 4), dtype=torch.int32, device='cuda')
    with pytest.raises(epic.EpicError) as e:  # five of three positions
        epic.propose_topk(z, five, five.float())
    assert e.value.status == 1
    # nothing to do
    epic.propose_topk(z[:, :0], cand[:, :0], conf[:, :0])
    epic.propose_topk(z, cand[..., :0].contiguous(), conf[..., :0].contiguous())
    epic.sample_tokens(z, u[..., :0].contiguous(), cand[..., :0].contiguous(), conf[..., :0].contiguous())
    # rows of no tokens
    epic.propose_topk(z[..., :0], cand, conf)
    assert (cand == -1).all() and (conf == 0).all()
    epic.sample_tokens(z[..., :0], u, cand.zero_(), conf)
    assert (cand == -1).all()
