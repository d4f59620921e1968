"""Performance cases of the operators between a model's logits and the constraint work.

Three operators: the K best tokens of each proposed position with their
softmax confidences (``propose_topk``), draws with temperature, top-k, top-p
and min-p from given uniform numbers (``sample_tokens``), and distillation
from a teacher's top logits (``distill_step``; ``distill_forward`` and
``distill_backward``).  A case is one call on device tensors as a decoding or
training loop makes it.

Sampling is defined on whole numbers: a token's weight is 2^((z - max) log2(e) / T)
in 32 bits, rounded to a multiple of 2^-30; sums of such weights are exact,
so a draw has one right answer whatever the order of the sums.
"""
import math

import torch

own = False

_DT = {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}
_LOG2E = 1.4426950408889634
_FMAX = 3.4028234663852886e38


# ---------------------------------------------------------------- cases

def _propose(name, B, n, k, V, K, dtype, pad=0):
    return {'name': name, 'op': 'propose', 'B': B, 'n': n, 'k': k, 'V': V, 'K': K, 'dtype': dtype, 'pad': pad}


def _sample(name, B, n, k, V, S, dtype, rules, pad=0):
    return {'name': name, 'op': 'sample', 'B': B, 'n': n, 'k': k, 'V': V, 'S': S, 'dtype': dtype, 'rules': rules,
            'pad': pad}


def _distill(name, form, B, n, V, K, dtype, active, pad=0):
    return {'name': name, 'op': 'distill', 'form': form, 'B': B, 'n': n, 'V': V, 'K': K, 'dtype': dtype,
            'active': active, 'pad': pad}


def listed():
    return [
        # the smallest decoding step there is: eight positions of one short row, 256 tokens; the launch is all of the time
        _propose('propose-expr', 1, 32, 8, 256, 8, 'f32'),
        # one step of schema-constrained JSON decoding: 4 of 256 positions of each row, read out of the model's whole output
        _propose('propose-json', 16, 256, 4, 32768, 16, 'bf16'),
        # an odd vocabulary, so that rows start at odd addresses; every masked position is proposed; many candidates
        _propose('propose-odd', 7, 37, 37, 50021, 53, 'f16'),
        # the largest decoding batch: 64 rows of 16 proposals, 126,000 tokens, rows padded to a multiple of 64
        _propose('propose-wide', 64, 16, 16, 126000, 32, 'bf16', pad=16),
        # one token for one interactive user, by the usual set of rules: latency alone
        _sample('sample-one', 1, 1, 1, 126000, 1, 'bf16', 'all'),
        # 16 drawn candidates for each proposal of the JSON batch, from the nucleus, logits in 32 bits
        _sample('sample-json', 16, 256, 4, 32768, 16, 'f32', 'top-p'),
        # requests with rules of their own in one batch, an odd vocabulary
        _sample('sample-mixed', 33, 5, 5, 65521, 4, 'f16', 'mixed'),
        # drawn candidates of a batch of 256 molecule strings: temperature alone
        _sample('sample-smiles', 256, 4, 4, 126000, 16, 'bf16', 'temperature'),
        # the widest batch from the nucleus with a floor on the probability
        _sample('sample-nucleus', 64, 16, 16, 126000, 8, 'bf16', 'top-p'),
        # fine-tuning a student on one short row, in 32 bits, an odd vocabulary: loss and gradient as two calls
        _distill('distill-small', 'train', 1, 32, 32771, 16, 'f32', 1.0),
        # a training micro-batch at the JSON configuration's sizes: loss and gradient in one call, half the positions masked
        _distill('distill-json', 'step', 16, 256, 32768, 16, 'bf16', 0.5),
        # the widest vocabulary, every position masked, loss and gradient as two calls under autograd
        _distill('distill-wide', 'train', 4, 256, 126000, 32, 'bf16', 1.0, pad=16),
    ]


_MOST = 126000 * 1024  # elements that one pass reads: the largest listed case's


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(['propose', 'sample', 'sample', 'distill'])
    dtype = rng.choice(['bf16', 'bf16', 'f16', 'f32'])
    V = _log(rng, 200, 126000)
    if rng.random() < 0.5:
        V = (V + 63) // 64 * 64
    V = min(V, 126000)
    pad = rng.choice([0, 0, 1, 24, 64])
    half = 2 if dtype == 'f32' else 1
    if op == 'distill':
        rows = _log(rng, 1, max(1, min(4096, _MOST // (half * V))))
        B = rng.randint(1, min(8, rows))
        return {'op': op, 'form': rng.choice(['step', 'train']), 'B': B, 'n': max(1, rows // B), 'V': V,
                'K': _log(rng, 1, 64), 'dtype': dtype, 'active': rng.choice([1.0, round(rng.uniform(0.3, 0.9), 2)]),
                'pad': pad}
    k = rng.randint(1, 16)
    B = _log(rng, 1, max(1, min(256, _MOST // (half * V * k))))
    n = k * rng.choice([1, 1, 2, 4])
    if B * n * V > 2 * _MOST:
        n = k
    if op == 'propose':
        return {'op': op, 'B': B, 'n': n, 'k': k, 'V': V, 'K': _log(rng, 1, 64), 'dtype': dtype, 'pad': pad}
    return {'op': op, 'B': B, 'n': n, 'k': k, 'V': V, 'S': _log(rng, 1, 32), 'dtype': dtype,
            'rules': rng.choice(['temperature', 'top-k', 'top-p', 'min-p', 'all', 'mixed']), 'pad': pad}


def _active_rows(case):
    return max(1, round(case['active'] * case['B'] * case['n']))


def work(case):
    size = 4 if case['dtype'] == 'f32' else 2
    V = case['V']
    if case['op'] == 'distill':
        rows, act, K = case['B'] * case['n'], _active_rows(case), case['K']
        return {'bytes': float((act + rows) * V * size + 9 * act * K + 8 * rows), 'flops': float(8 * act * V)}
    rows = case['B'] * case['k']
    if case['op'] == 'propose':
        return {'bytes': float(rows * V * size + 8 * rows * case['K']), 'flops': float(5 * rows * V)}
    return {'bytes': float(rows * V * size + 12 * rows * case['S']), 'flops': float(7 * rows * V)}


# ---------------------------------------------------------------- inputs

def _logits(gen, B, n, V, pad, dtype, dev):
    """A model's output: a broad bulk, a few dozen likely tokens of very different strength in each row, and the mask
    token (the last id) never allowed.  One row in eight is hard text (flat), one in eight nearly certain."""
    z = torch.randn((B * n, V), generator=gen, device=dev)
    kind = torch.randint(0, 8, (B * n, 1), generator=gen, device=dev)
    z *= torch.where(kind == 0, 0.8, 1.9)
    h = min(V, 24)
    at = torch.randint(0, V, (B * n, h), generator=gen, device=dev)
    up = torch.rand((B * n, h), generator=gen, device=dev) ** 2 * (math.log(V) + 1.0)
    up = torch.where(kind == 0, up * 0.3, torch.where(kind == 1, up * 1.8, up))
    z.scatter_add_(1, at, up)
    z[:, V - 1] = -math.inf
    full = torch.zeros((B, n, V + pad), dtype=_DT[dtype], device=dev)
    full[..., :V] = z.view(B, n, V)
    return full[..., :V]


def _rules(case, gen, dev):
    """Each request's rules, [B]; None where a program does not use the rule."""
    B, r = case['B'], case['rules']

    def among(*values):
        v = torch.tensor(values, device=dev)
        return v[torch.randint(0, len(values), (B,), generator=gen, device=dev)].contiguous()
    p = {'temperature': among(0.7, 0.8, 1.0, 1.0, 1.2), 'top_k': None, 'top_p': None, 'min_p': None}
    if r in ('top-k', 'all'):
        p['top_k'] = among(20, 40, 50, 64).to(torch.int32)
    if r in ('top-p', 'all'):
        p['top_p'] = among(0.8, 0.9, 0.95)
    if r in ('min-p', 'all'):
        p['min_p'] = among(0.02, 0.05, 0.1)
    if r == 'mixed':  # each request its own; 0 (1 for top-p) leaves a rule out, temperature 0 takes the likeliest
        p = {'temperature': among(0.0, 0.6, 1.0, 1.0, 1.5), 'top_k': among(0, 0, 1, 50, 1000).to(torch.int32),
             'top_p': among(1.0, 1.0, 0.9, 0.5), 'min_p': among(0.0, 0.0, 0.05)}
    return p


def prepare(case, seed):
    dev = torch.device('cuda')
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    B, n, V = case['B'], case['n'], case['V']
    s = {'case': case, 'logits': _logits(gen, B, n, V, case['pad'], case['dtype'], dev)}
    if case['op'] == 'distill':
        K, rows = case['K'], B * n
        ids = torch.randint(0, V - 1, (B, n, K), generator=gen, device=dev).to(torch.int32)
        vals = -torch.sort(torch.rand((B, n, K), generator=gen, device=dev) * 8.0, dim=-1).values
        # the student knows some of it: its logits lean towards the teacher's
        s['logits'].scatter_(2, ids.long(), (vals * 0.7 + math.log(V)).to(s['logits'].dtype))
        s['ids'], s['vals'] = ids, vals.contiguous()
        s['valid'] = (torch.rand((B, n, K), generator=gen, device=dev) < 0.8).to(torch.uint8)
        weight = 1.0 / (0.1 + 0.9 * torch.rand((rows,), generator=gen, device=dev))
        weight[torch.randperm(rows, generator=gen, device=dev)[_active_rows(case):]] = 0.0
        s['weight'] = weight.view(B, n)
        s['up'] = torch.rand((B, n), generator=gen, device=dev) + 0.5  # what autograd hands down
        s['loss'] = torch.empty((B, n), device=dev)
        s['lse'] = torch.empty((B, n), device=dev)
        s['grad'] = torch.empty((B, n, V), dtype=s['logits'].dtype, device=dev)
        return s
    k = case['k']
    s['pos'] = None if n == k else torch.rand((B, n), generator=gen, device=dev).argsort(1)[:, :k].sort(1).values.to(
        torch.int32).contiguous()
    if case['op'] == 'propose':
        s['temperature'] = 0.6 + 0.8 * torch.rand((B,), generator=gen, device=dev)
        s['cand'] = torch.empty((B, k, case['K']), dtype=torch.int32, device=dev)
        s['conf'] = torch.empty((B, k, case['K']), device=dev)
        return s
    s.update(_rules(case, gen, dev))
    s['u'] = torch.rand((B, k, case['S']), generator=gen, device=dev)
    s['tok'] = torch.empty((B, k, case['S']), dtype=torch.int32, device=dev)
    s['prob'] = torch.empty((B, k, case['S']), device=dev)
    return s


_TAU = 2.0


# ---------------------------------------------------------------- the operators in their plain form

def _rows(s):
    """The proposed positions' logits in 32 bits, [B][k][V]; NaN counts as -inf."""
    z = s['logits']
    if s['pos'] is not None:
        z = z[torch.arange(z.shape[0], device=z.device)[:, None], s['pos'].long()]
    z = z.float()
    return torch.where(torch.isnan(z), -math.inf, z)


def _weights(z, T):
    """2^((z - max) log2(e) / T), 0 where z is -inf."""
    m = z.amax(-1, keepdim=True)
    d = torch.where(z == m, 0.0, z - m)
    w = torch.exp2(d * torch.clamp(_LOG2E / T, max=_FMAX))
    return torch.where(z == -math.inf, 0.0, w)


def _plain_propose(s):
    z = _rows(s)
    K, V = s['case']['K'], z.shape[-1]
    w = _weights(z, s['temperature'][:, None, None])
    zs, order = torch.sort(z, dim=-1, descending=True, stable=True)
    there = zs[..., :min(K, V)] > -math.inf
    conf = torch.where(there, w.gather(-1, order[..., :K]) / w.sum(-1, keepdim=True), 0.0)
    cand = torch.where(there, order[..., :K], -1).to(torch.int32)
    more = K - cand.shape[-1]
    return [torch.nn.functional.pad(cand, (0, more), value=-1), torch.nn.functional.pad(conf, (0, more))]


def _share(a, q):
    """floor(a q / 2^24) of whole numbers, a up to 2^24, without passing 64 bits."""
    return a * (q >> 24) + ((a * (q & 0xffffff)) >> 24)


def _plain_sample(s):
    z = _rows(s)
    B, k, V = z.shape

    def rule(name, off):
        return torch.full((B, 1, 1), off, device=z.device) if s[name] is None else s[name][:, None, None]
    T, top_k, top_p, min_p = rule('temperature', 1.0), rule('top_k', 0), rule('top_p', 1.0), rule('min_p', 0.0)
    w = _weights(z, T)
    q = torch.round(w * 2.0 ** 30).long()
    zs, order = torch.sort(z, dim=-1, descending=True, stable=True)
    rank = torch.arange(V, device=z.device)
    best = rank < torch.where(T == 0, 1, torch.where(top_k <= 0, V, top_k))
    qs = torch.where(best, q.gather(-1, order), 0)
    upto = qs.cumsum(-1)
    nucleus = upto - qs < _share(torch.round(top_p.clamp(0.0, 1.0) * 2.0 ** 24).long(), upto[..., -1:])
    keep = (rank == 0) | (best & nucleus & (w.gather(-1, order) >= min_p))
    keep &= zs > -math.inf
    keep = torch.zeros_like(keep).scatter_(-1, order, keep)
    upto = torch.where(keep, q, 0).cumsum(-1)
    mass = upto[..., -1:]
    t = _share(torch.floor(s['u'] * 2.0 ** 24).long(), mass)
    tok = torch.searchsorted(upto, torch.minimum(t, mass - 1), right=True).clamp_(max=V - 1)
    prob = w.gather(-1, tok) * 2.0 ** 30 / mass.float()
    return [torch.where(mass > 0, tok, -1).to(torch.int32), torch.where(mass > 0, prob, 0.0)]


def _plain_distill(s):
    z = s['logits'].float() / _TAU
    V = z.shape[-1]
    m = z.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))
    ids = s['ids'].long()
    counts = (ids >= 0) & (ids < V) & (s['valid'] == 1) & (s['vals'] > -math.inf)
    some = counts.any(-1, keepdim=True)
    a = torch.where(counts, s['vals'] / _TAU, -math.inf)
    a = torch.where(some, a - a.amax(-1, keepdim=True), -math.inf)
    e = torch.exp(a)
    total = torch.where(some, e.sum(-1, keepdim=True), 1.0)
    p, lp = e / total, a - torch.log(total)
    ids = torch.where(counts, ids, 0)
    each = torch.where(p > 0, p * (lp - (z.gather(-1, ids) - lse)), 0.0)
    weight = s['weight']
    loss = torch.where(weight == 0, 0.0, weight * _TAU ** 2 * each.sum(-1))
    g = torch.where(some, torch.exp(z - lse), 0.0).scatter_add_(-1, ids, -p)
    coef = weight * _TAU * (s['up'] if s['case']['form'] == 'train' else 1.0)
    grad = torch.where(weight[..., None] == 0, 0.0, g * coef[..., None])
    return [loss, grad.to(s['logits'].dtype)]


def run(s):
    op = s['case']['op']
    if not own:
        return {'propose': _plain_propose, 'sample': _plain_sample, 'distill': _plain_distill}[op](s)
    import paper_2606_00722_gb300 as epic
    if op == 'propose':
        epic.propose_topk(s['logits'], s['cand'], s['conf'], pos=s['pos'], temperature=s['temperature'])
        return [s['cand'], s['conf']]
    if op == 'sample':
        epic.sample_tokens(s['logits'], s['u'], s['tok'], s['prob'], pos=s['pos'], temperature=s['temperature'],
                           top_k=s['top_k'], top_p=s['top_p'], min_p=s['min_p'])
        return [s['tok'], s['prob']]
    if s['case']['form'] == 'step':
        epic.distill_step(s['logits'], s['ids'], s['vals'], s['loss'], s['grad'], tau=_TAU, weight=s['weight'],
                          valid=s['valid'])
    else:
        epic.distill_forward(s['logits'], s['ids'], s['vals'], s['loss'], s['lse'], tau=_TAU, weight=s['weight'],
                             valid=s['valid'])
        epic.distill_backward(s['logits'], s['ids'], s['vals'], s['lse'], s['up'], s['grad'], tau=_TAU,
                              weight=s['weight'], valid=s['valid'])
    return [s['loss'], s['grad']]


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    """Row by row in 64 bits.  Tokens are whole numbers and have no 64-bit value."""
    s = prepare(case, seed)
    z = s['logits'].reshape(case['B'] * case['n'], -1)
    if case['op'] == 'distill':
        K = case['K']
        ids, valid = s['ids'].view(-1, K).long(), s['valid'].view(-1, K) == 1
        vals, weight, up = s['vals'].view(-1, K).double(), s['weight'].view(-1).double(), s['up'].view(-1).double()
        loss = torch.zeros(z.shape[0], dtype=torch.float64, device=z.device)
        grad = torch.zeros(z.shape, dtype=torch.float64, device=z.device)
        for r in torch.nonzero(weight).reshape(-1).tolist():
            use = torch.nonzero(valid[r]).reshape(-1)
            if not len(use):
                continue
            logq = torch.log_softmax(z[r].double() / _TAU, 0)
            logp = torch.log_softmax(vals[r, use] / _TAU, 0)
            loss[r] = weight[r] * _TAU ** 2 * (logp.exp() * (logp - logq[ids[r, use]])).sum()
            target = torch.zeros_like(logq).index_add_(0, ids[r, use], logp.exp())
            grad[r] = (logq.exp() - target) * weight[r] * _TAU * (up[r] if case['form'] == 'train' else 1.0)
        return [loss.view(case['B'], case['n']), grad.view(case['B'], case['n'], -1)]
    B, k = case['B'], case['k']
    rows = range(B * k) if s['pos'] is None else (s['pos'].long() + torch.arange(B, device=z.device)[:, None] * case['n']).view(-1).tolist()
    out = []
    for i, r in enumerate(rows):
        b = i // k
        T = float(s['temperature'][b])
        v = z[r].double()
        prob = torch.softmax(v / T, 0) if T > 0 else (torch.arange(len(v), device=v.device) == v.argmax()).double()
        if case['op'] == 'propose':
            top = torch.topk(prob, min(case['K'], int((v > -math.inf).sum()))).values
            out.append(torch.nn.functional.pad(top, (0, case['K'] - len(top))))
            continue
        order = torch.sort(v, descending=True, stable=True).indices
        p = prob[order]
        many = int(s['top_k'][b]) if s['top_k'] is not None else 0
        if many > 0:
            p[many:] = 0
            p = p / p.sum()
        if s['top_p'] is not None:
            p[p.cumsum(0) - p >= float(s['top_p'][b])] = 0
        if s['min_p'] is not None:
            p[p < float(s['min_p'][b]) * p[0]] = 0
        p = torch.zeros_like(p).scatter_(0, order, p / p.sum())
        upto = p.cumsum(0)
        at = torch.searchsorted(upto, s['u'].view(B * k, -1)[i].double() * upto[-1], right=True)
        out.append(p[at.clamp(max=len(p) - 1)])
    return [None, torch.stack(out).view(B, k, -1)]
