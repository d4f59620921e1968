"""Performance cases of the output head: from hidden states to a loss, and to rows of logits.

Two operators.  The loss of a masked diffusion LM's head: softmax cross
entropy of hidden states [B][n][d] through head weights [V][d], without
keeping the logits, with its gradients (``head_loss_forward``,
``head_loss_backward``, ``head_loss_step``).  The head in 8-bit integers for
decoding: the proposed positions' hidden states rounded to 8 bits with a scale
for each (``quantize_rows``), times a head of 8-bit weights with a scale for
each token of the vocabulary (``int8_logits``).  A case is what a training or
decoding loop calls, on device tensors.

The rounding to 8 bits is defined on 32-bit numbers: s = max|x| / 127 and
q = rint(x / s), quotients rounded to the nearest 32-bit number, halves to even.
"""
import math

import torch

own = False

_DT = {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}


# ---------------------------------------------------------------- cases

def _loss(name, form, B, n, d, V, dtype, active, pad=0):
    return {'name': name, 'op': 'loss', 'form': form, 'B': B, 'n': n, 'd': d, 'V': V, 'dtype': dtype, 'active': active,
            'pad': pad}


def _logits(name, B, n, k, d, V, dtype, pad=0):
    return {'name': name, 'op': 'logits', 'B': B, 'n': n, 'k': k, 'd': d, 'V': V, 'dtype': dtype, 'pad': pad}


def listed():
    return [
        # the smallest training step: one row of 32 expression tokens, a toy model; launches are all of the time
        _loss('loss-expr', 'step', 1, 32, 128, 256, 'bf16', 0.5),
        # one short row through the widest head: the head's weights and their gradient are all of the traffic
        _loss('loss-row', 'step', 1, 32, 4096, 126000, 'bf16', 1.0),
        # odd sizes, so that rows of the head start at odd addresses; loss and gradients as two calls, fp16
        _loss('loss-odd', 'train', 7, 37, 771, 50021, 'f16', 0.8),
        # validation loss of a JSON batch: no gradient, half the positions masked
        _loss('loss-eval', 'forward', 16, 256, 2048, 32768, 'bf16', 0.5),
        # a training micro-batch at the C-like configuration's sizes, half the positions masked, loss and gradients in one call
        _loss('loss-clike', 'step', 32, 512, 2048, 65536, 'bf16', 0.5),
        # the widest head, every position counts, loss and gradients as two calls under autograd
        _loss('loss-wide', 'train', 4, 1024, 4096, 126000, 'bf16', 1.0),
        # the smallest decoding step: eight positions of an expression, a toy model; latency alone
        _logits('logits-expr', 1, 32, 8, 128, 256, 'bf16'),
        # one position for one interactive user through the widest head: the weights are read once
        _logits('logits-one', 1, 1, 1, 4096, 126000, 'bf16'),
        # one step of schema-constrained JSON decoding: 4 of 256 positions of each row
        _logits('logits-json', 16, 256, 4, 2048, 32768, 'bf16'),
        # odd sizes everywhere, hidden states and logits in fp16
        _logits('logits-odd', 33, 5, 5, 1003, 50021, 'f16'),
        # the largest decoding batch: 64 rows of 16 proposals, rows of logits padded to a multiple of 64
        _logits('logits-wide', 64, 16, 16, 4096, 126000, 'bf16', pad=16),
        # 16 proposals for each of 256 molecule strings, hidden states and logits in 32 bits
        _logits('logits-smiles', 256, 16, 16, 2048, 126000, 'f32'),
    ]


_MOST_LOSS = 8.0 * 4096 * 4096 * 126000  # operations of the largest listed case of each operator
_MOST_LOGITS = 2.0 * 4096 * 2048 * 126000
_MOST_CELLS = 4096 * 126000              # (position, token) pairs of the largest listed case


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(['loss', 'loss', 'logits'])
    V = _log(rng, 200, 126000)
    if rng.random() < 0.5:
        V = min((V + 63) // 64 * 64, 126000)
    d = _log(rng, 32, 4096)
    if rng.random() < 0.7:
        d = min((d + 31) // 32 * 32, 4096)
    pad = rng.choice([0, 0, 8, 24, 3])
    if op == 'loss':
        rows = _log(rng, 1, max(1, min(16384, _MOST_CELLS // V, int(_MOST_LOSS / (8.0 * V * d)))))
        B = rng.randint(1, min(16, rows))
        return {'op': op, 'form': rng.choice(['forward', 'train', 'step', 'step']), 'B': B, 'n': max(1, rows // B), 'd': d,
                'V': V, 'dtype': rng.choice(['bf16', 'bf16', 'f16']),
                'active': rng.choice([1.0, round(rng.uniform(0.2, 0.9), 2)]), 'pad': pad}
    k = rng.randint(1, 16)
    B = _log(rng, 1, max(1, min(1024, _MOST_CELLS // (V * k), int(_MOST_LOGITS / (2.0 * V * d * k)))))
    n = k * rng.choice([1, 1, 2, 4, 16])
    return {'op': op, 'B': B, 'n': n, 'k': k, 'd': d, 'V': V, 'dtype': rng.choice(['bf16', 'bf16', 'f16', 'f32']),
            'pad': pad}


def _active_rows(case):
    return max(1, round(case['active'] * case['B'] * case['n']))


def work(case):
    size = 4 if case['dtype'] == 'f32' else 2
    V, d = case['V'], case['d']
    if case['op'] == 'logits':
        rows = case['B'] * case['k']
        return {'bytes': float(rows * d * size + V * d + 4 * V + rows * V * size), 'flops': 2.0 * rows * V * d}
    rows, act = case['B'] * case['n'], _active_rows(case)
    read = (act * d + V * d) * size + 12 * rows
    if case['form'] == 'forward':
        return {'bytes': float(read), 'flops': 2.0 * act * V * d}
    # logits are not kept from one call to the other: two calls make them twice
    return {'bytes': float(read + (rows * d + V * d) * size), 'flops': (8.0 if case['form'] == 'train' else 6.0) * act * V * d}


# ---------------------------------------------------------------- inputs

def _head(gen, V, d, dev):
    """Rows of a trained head: lengths differ, a few coordinates are larger than the rest."""
    w = torch.randn((V, d), generator=gen, device=dev)
    w *= (0.7 + 0.6 * torch.rand((V, 1), generator=gen, device=dev)) * (2.0 / math.sqrt(d))
    w *= 1.0 + 2.0 * (torch.rand((d,), generator=gen, device=dev) < 0.02)
    return w


def _padded(x, pad, dtype):
    """x in that type, its rows `pad` elements apart in memory."""
    full = torch.zeros(x.shape[:-1] + (x.shape[-1] + pad,), dtype=_DT[dtype], device=x.device)
    full[..., :x.shape[-1]] = x
    return full[..., :x.shape[-1]]


def prepare(case, seed):
    dev = torch.device('cuda')
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    B, n, d, V = case['B'], case['n'], case['d'], case['V']
    head = _head(gen, V, d, dev)
    h = torch.randn((B, n, d), generator=gen, device=dev)
    s = {'case': case}
    # the model knows the text in part: hidden states lean towards the right token's row by amounts of every size
    target = torch.randint(0, V, (B, n), generator=gen, device=dev).to(torch.int32)
    sure = torch.rand((B, n, 1), generator=gen, device=dev) * 3.5
    h += sure * head[target.view(-1).long()].view(B, n, d)
    if case['op'] == 'loss':
        rows = B * n
        off = torch.randperm(rows, generator=gen, device=dev)[_active_rows(case):]
        target.view(-1)[off] = -1  # positions that were not masked have no loss
        s['target'] = target
        s['weight'] = 1.0 / (0.1 + 0.9 * torch.rand((B, n), generator=gen, device=dev))
        s['up'] = torch.rand((B, n), generator=gen, device=dev) + 0.5  # what autograd hands down
        s['hidden'] = _padded(h, case['pad'], case['dtype'])
        s['head'] = _padded(head, case['pad'], case['dtype'])
        s['loss'] = torch.empty((B, n), device=dev)
        s['lse'] = torch.empty((B, n), device=dev)
        if case['form'] != 'forward':
            s['grad_hidden'] = torch.empty((B, n, d), dtype=_DT[case['dtype']], device=dev)
            s['grad_head'] = torch.empty((V, d), dtype=_DT[case['dtype']], device=dev)
        return s
    k = case['k']
    s['hidden'] = h.to(_DT[case['dtype']])
    s['pos'] = None if n == k else torch.rand((B, n), generator=gen, device=dev).argsort(1)[:, :k].sort(1).values.to(
        torch.int32).contiguous()
    s['head_q'], s['head_scale'] = _quantized(head)
    s['q'] = torch.empty((B, k, d), dtype=torch.int8, device=dev)
    s['scale'] = torch.empty((B, k), device=dev)
    s['logits'] = torch.empty((B, k, V + case['pad']), dtype=_DT[case['dtype']], device=dev)[..., :V]
    return s


# ---------------------------------------------------------------- the operators in their plain form

def _quantized(x):
    """(q int8, s) of rows in 32 bits.  Both divisions take tensors: by a Python number torch multiplies by its reciprocal."""
    x = x.float()
    s = x.abs().amax(-1) / torch.full((1,), 127.0, device=x.device)
    q = torch.where(s[..., None] > 0, x / s[..., None], 0.0)
    return torch.round(q).clamp_(-127, 127).to(torch.int8), s


def _plain_logits(s):
    h = s['hidden']
    if s['pos'] is not None:
        h = h[torch.arange(h.shape[0], device=h.device)[:, None], s['pos'].long()]
    q, scale = _quantized(h)
    B, k, d = q.shape
    # whole numbers: sums below 2^24 are exact in 32 bits whatever their order
    z = (q.view(B * k, d).float() @ s['head_q'].float().t()).view(B, k, -1)
    return [(z * scale[..., None] * s['head_scale']).to(h.dtype), scale]


def _plain_loss(s):
    form, dtype = s['case']['form'], s['hidden'].dtype
    B, n, d = s['hidden'].shape
    w = s['head'].float()
    V = w.shape[0]
    target, weight = s['target'].reshape(-1).long(), s['weight'].reshape(-1)
    at = torch.nonzero((target >= 0) & (target < V) & (weight != 0)).reshape(-1)
    h, y, weight = s['hidden'].reshape(B * n, d)[at].float(), target[at], weight[at]
    z = h @ w.t()
    m = z.amax(-1)
    lse = m + torch.log(torch.exp(z - m[:, None]).sum(-1))
    loss = weight * (lse - z.gather(1, y[:, None])[:, 0])

    def whole(rows, like):
        out = torch.zeros((B * n,) + rows.shape[1:], device=rows.device)
        out[at] = rows
        return out.view((B, n) + rows.shape[1:]).to(like)
    if form == 'forward':
        return [whole(loss, torch.float32), whole(lse, torch.float32)]
    p = z.sub_(lse[:, None]).exp_()
    p[torch.arange(len(y), device=p.device), y] -= 1.0
    p *= (weight * s['up'].reshape(-1)[at] if form == 'train' else weight)[:, None]
    return [whole(loss, torch.float32), whole(p @ w, dtype), (p.t() @ h).to(dtype)]


def run(s):
    loss = s['case']['op'] == 'loss'
    if not own:
        return _plain_loss(s) if loss else _plain_logits(s)
    import paper_2606_00722_gb300 as epic
    if not loss:
        epic.quantize_rows(s['hidden'], s['q'], s['scale'], pos=s['pos'])
        epic.int8_logits(s['q'], s['scale'], s['head_q'], s['head_scale'], s['logits'])
        return [s['logits'], s['scale']]
    if s['case']['form'] == 'step':
        epic.head_loss_step(s['hidden'], s['head'], s['target'], s['loss'], s['grad_hidden'], s['grad_head'],
                            weight=s['weight'])
        return [s['loss'], s['grad_hidden'], s['grad_head']]
    epic.head_loss_forward(s['hidden'], s['head'], s['target'], s['loss'], s['lse'], weight=s['weight'])
    if s['case']['form'] == 'forward':
        return [s['loss'], s['lse']]
    epic.head_loss_backward(s['hidden'], s['head'], s['target'], s['lse'], s['up'], s['grad_hidden'], s['grad_head'],
                            weight=s['weight'])
    return [s['loss'], s['grad_hidden'], s['grad_head']]


# ---------------------------------------------------------------- in 64 bits, from the definitions

def exact(case, seed):
    """In 64 bits.  The rounding to 8 bits is defined on 32-bit numbers and taken as that."""
    if work(case)['flops'] > 7e12:  # 64-bit products are slow on this card
        return None
    s = prepare(case, seed)
    V, d = case['V'], case['d']
    if case['op'] == 'logits':
        B, k = case['B'], case['k']
        rows = s['hidden'].float()
        if s['pos'] is not None:
            rows = rows.gather(1, s['pos'].long()[..., None].expand(B, k, d))
        scale = rows.abs().max(dim=2).values.div(torch.tensor([127.0], device=rows.device))
        q = (rows / scale.clamp(min=1e-45)[..., None]).round().double()
        value = q.view(B * k, d) * scale.view(-1, 1).double()
        out = torch.empty((B * k, V), dtype=torch.float64, device=rows.device)
        for v in range(0, V, 16384):
            part = s['head_q'][v:v + 16384].double() * s['head_scale'][v:v + 16384, None].double()
            torch.mm(value, part.t(), out=out[:, v:v + 16384])
        return [out.view(B, k, V), scale]
    form = case['form']
    H, W = s['hidden'].reshape(-1, d), s['head'].double()
    target, weight, up = s['target'].view(-1), s['weight'].view(-1).double(), s['up'].view(-1).double()
    R = H.shape[0]
    loss = torch.zeros(R, dtype=torch.float64, device=H.device)
    lse = torch.zeros_like(loss)
    gh = torch.zeros((R, d), dtype=torch.float64, device=H.device) if form != 'forward' else None
    gw = torch.zeros((V, d), dtype=torch.float64, device=H.device) if form != 'forward' else None
    for r0 in range(0, R, 1024):
        use = r0 + torch.nonzero(target[r0:r0 + 1024] >= 0).view(-1)
        if not len(use):
            continue
        x, y = H[use].double(), target[use].long()
        logp = x @ W.t()
        lse[use] = torch.logsumexp(logp, 1)
        logp -= lse[use][:, None]
        loss[use] = -weight[use] * logp.gather(1, y[:, None]).view(-1)
        if form == 'forward':
            continue
        g = logp.exp_().scatter_add_(1, y[:, None], torch.full((len(use), 1), -1.0, dtype=torch.float64, device=H.device))
        g *= (weight[use] * (up[use] if form == 'train' else 1.0))[:, None]
        gh[use] = g @ W
        gw += g.t() @ x
    shape = (case['B'], case['n'])
    if form == 'forward':
        return [loss.view(shape), lse.view(shape)]
    return [loss.view(shape), gh.view(shape + (d,)), gw]
