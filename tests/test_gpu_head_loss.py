"""The loss of a head from hidden states against its formulas in 64 bits, and against differences.

Tolerances, from the arithmetic, with u = eps / 2 of the type (bf16 2^-8, fp16 2^-11):
- A logit is a sum of d exact products in 32 bits, in any order: off by at most (d + 4) 2^-24 A, A the sum of the products'
  sizes; tensor units cut what they add to 2^-23 of the running sum, but only once for 8 products or more.
- lse is off by the largest error of a logit, its power's argument and value (|z| 2^-23 + 2^-21), sums of V terms
  (2^-24 for each of at most 400 in a chain: 2^-15), so a loss by w (2 dz + 2^-15 + 2^-20 |lse|).
- A probability is off by e = 2 dz + 2^-14 + |lse| 2^-21 of itself, and u by its rounding (fp16: a gradient of a logit also
  by 2^-38 of the largest factor: half of 2^-24 at a scale of 2^14 over the power of two above it); hidden states times a
  factor by u.  So with
  a = |dz| |W| summed over tokens, a gradient of hidden states is off by (u + e + 2^-12) a and one last rounding, u of the
  value; with b = |dz| |h| summed over positions, one of the head by (2 u + u^2 + e + 2^-12) b and u of the value.  2^-12 is
  for the chains of these sums: they are cut to 2^-23 at each step of 8 or more products, of at most 2^14 (V = 126,000); a
  rounding of halves may be of a subnormal, 2^-25."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _dtype(name):
    import torch
    return {'f16': torch.float16, 'bf16': torch.bfloat16}[name]


def put(x, dtype, pad=0, shift=0, fill=math.nan):
    """x in that type on the GPU, rows `pad` elements apart, the first `shift` elements into its storage."""
    import torch
    full = torch.full(x.shape[:-1] + (x.shape[-1] + pad,), fill, dtype=_dtype(dtype))
    full[..., :x.shape[-1]] = x.to(_dtype(dtype))
    flat = torch.full((shift + full.numel() + 16,), fill, dtype=_dtype(dtype), device='cuda')
    flat[shift:shift + full.numel()] = full.reshape(-1).cuda()
    return flat[shift:shift + full.numel()].view(full.shape)[..., :x.shape[-1]]


def make(B, n, d, V, dtype, seed, pad=0, shift=0, scale=1.0, edges=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((V, d), generator=g) * (2.0 * scale / math.sqrt(d))
    h = torch.randn((B, n, d), generator=g)
    target = torch.randint(0, max(V, 1), (B, n), generator=g).to(torch.int32)
    weight = torch.rand((B, n), generator=g) * 2.0 + 0.1
    sure = torch.rand((B, n, 1), generator=g) * 3.0
    if V:
        h += sure * W[target.long()] / scale
    if edges and B * n > 3:
        off = torch.rand((B, n), generator=g) < 0.4
        target[off] = torch.where(torch.rand((B, n), generator=g) < 0.5, -1, V)[off].to(torch.int32)
        weight[torch.rand((B, n), generator=g) < 0.1] = 0.0
        none = (target < 0) | (target >= V) | (weight == 0)
        h[none] = torch.tensor([math.nan, math.inf, 3.0])[torch.randint(0, 3, (int(none.sum()),), generator=g)][:, None]
    return (put(h, dtype, pad, shift), put(W, dtype, pad, shift), target.cuda(), weight.cuda(),
            (torch.rand((B, n), generator=g) * 2.0 - 0.5).cuda())


def head64(h, W, target, weight, up=None):
    """The formulas in 64 bits, and what the tolerances need."""
    import torch
    B, n, d = h.shape
    V = W.shape[0]
    w = torch.ones((B, n), device=h.device) if weight is None else weight
    at = torch.nonzero(((target >= 0) & (target < V) & (w != 0)).view(-1)).view(-1)
    x, y, w = h.reshape(-1, d)[at].double(), target.view(-1)[at].long(), w.view(-1)[at].double()
    W = W.double()
    z = x @ W.t()
    dz = ((x.abs() @ W.abs().t()).amax(1) if V else x.new_zeros(len(at))) * (d + 4) * 2.0 ** -24
    lse = torch.logsumexp(z, 1)
    arange = torch.arange(len(at), device=h.device)
    others = z.clone()
    others[arange, y] = -math.inf
    loss = w * torch.nn.functional.softplus(torch.logsumexp(others, 1) - z[arange, y], threshold=700)
    g = w if up is None else w * up.view(-1)[at].double()
    p = torch.exp(z - lse[:, None])
    p[arange, y] = 0.0
    p[arange, y] = -p.sum(1)
    p *= g[:, None]
    e = 2 * dz + 2.0 ** -14 + lse.abs() * 2.0 ** -21

    gtop = float(g.abs().max()) if len(at) else 0.0

    def whole(rows):
        out = torch.zeros((B * n,) + rows.shape[1:], dtype=rows.dtype, device=rows.device)
        out[at] = rows
        return out.view((B, n) + rows.shape[1:])
    a = p.abs()
    return dict(loss=whole(loss), lse=whole(lse), gh=whole(p @ W), gw=p.t() @ x,
                loss_tol=whole(w * (2 * dz + 2.0 ** -15 + lse.abs() * 2.0 ** -20)),
                lse_tol=whole(2 * dz + 2.0 ** -15 + lse.abs() * 2.0 ** -20),
                a=whole(a @ W.abs()), ae=whole((a * e[:, None]) @ W.abs()), sw=gtop * W.abs().sum(0), sx=gtop * x.abs().sum(0),
                b=a.t() @ x.abs(), be=(a * e[:, None]).t() @ x.abs())


def close(got, want, tol):
    assert got.isfinite().all()
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (got.double()[bad][:4], want[bad][:4], tol[bad][:4], int(bad.sum()))


def check_grads(gh, gw, r, dtype):
    u = {'f16': 2.0 ** -11, 'bf16': 2.0 ** -8}[dtype]
    low = 2.0 ** -25 if dtype == 'f16' else 0.0
    f16 = dtype == 'f16'
    if gh is not None:
        tol = (u + 2.0 ** -12) * r['a'] + r['ae'] + u * r['gh'].abs() + low + 1e-30
        close(gh, r['gh'], tol + (2.0 ** -38 * r['sw'] if f16 else 0.0))
    if gw is not None:
        tol = (2 * u + u * u + 2.0 ** -12) * r['b'] + r['be'] + u * r['gw'].abs() + low + 1e-30
        close(gw, r['gw'], tol + (2.0 ** -38 * r['sx'] if f16 else 0.0))


SIZES = [  # B, n, d, V, dtype, pad, shift
    (1, 1, 1, 1, 'bf16', 0, 0),
    (1, 1, 8, 2, 'f16', 0, 0),
    (2, 3, 7, 33, 'bf16', 1, 1),
    (1, 32, 128, 256, 'bf16', 0, 0),
    (3, 7, 100, 1000, 'f16', 4, 0),
    (2, 130, 128, 517, 'bf16', 0, 8),
    (1, 257, 72, 4099, 'f16', 3, 5),
    (5, 103, 200, 1024, 'bf16', 24, 0),
    (7, 37, 771, 5021, 'f16', 0, 0),
    (3, 300, 264, 2050, 'bf16', 0, 0),
    (1, 3, 4096, 9001, 'bf16', 0, 0),
    (2, 5, 1003, 50021, 'bf16', 8, 0),
    (1, 900, 65, 130, 'f16', 0, 0),
    (1, 1500, 40, 300, 'bf16', 0, 0),    # more positions than one scan counts
    (2, 2100, 72, 513, 'f16', 1, 3),
    (1, 200, 320, 3000, 'bf16', 3, 2),   # rows of the head and of gradients at odd places, sums in parts
    (1, 5000, 64, 260, 'bf16', 0, 0),
]


@pytest.mark.parametrize('B,n,d,V,dtype,pad,shift', SIZES)
def test_loss_and_gradients(cuda, B, n, d, V, dtype, pad, shift):
    import torch
    import paper_2606_00722_gb300 as epic
    h, W, target, weight, up = make(B, n, d, V, dtype, V + d, pad, shift)
    gstore = torch.full((B, n, d + pad + 2), 7.0, dtype=h.dtype, device=cuda)
    wstore = torch.full((V, d + 8), 7.0, dtype=h.dtype, device=cuda)
    gh, gw = gstore[..., :d], wstore[:, :d]
    loss, lse = torch.full((B, n), -7.0, device=cuda), torch.full((B, n), -7.0, device=cuda)
    want, step = head64(h, W, target, weight, up), head64(h, W, target, weight)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    close(loss, want['loss'], want['loss_tol'])
    close(lse, want['lse'], want['lse_tol'])
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    check_grads(gh, gw, want, dtype)
    first = gh.clone(), gw.clone()
    gh.fill_(7.0), gw.fill_(7.0)
    epic.head_loss_backward(h, W, target, lse, up, gh, None, weight=weight)  # either alone, and the same bits
    epic.head_loss_backward(h, W, target, lse, up, None, gw, weight=weight)
    assert torch.equal(gh, first[0]) and torch.equal(gw, first[1])
    gh.fill_(7.0), gw.fill_(7.0), loss.fill_(7.0)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    close(loss, step['loss'], step['loss_tol'])
    check_grads(gh, gw, step, dtype)
    assert (gstore[..., d:] == 7).all() and (wstore[:, d:] == 7).all()
    # without weights all count alike
    one = head64(h, W, target, torch.ones_like(weight))
    if not (torch.isfinite(h.float()).all(-1) | (target < 0) | (target >= V)).all():
        return  # rows of weight 0 above hold NaN
    epic.head_loss_step(h, W, target, loss, gh, gw)
    close(loss, one['loss'], one['loss_tol'])
    check_grads(gh, gw, one, dtype)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('rows', [257, 520, 800])
def test_pieces_add_up(cuda, monkeypatch, rows, dtype):
    """Two to four pieces of 256 positions; one of them has none that count."""
    import torch
    import paper_2606_00722_gb300 as epic
    monkeypatch.setenv('EPIC_HEAD_PIECE_MB', '1')
    d, V = 96 if rows != 520 else 97, 2051
    h, W, target, weight, up = make(1, rows, d, V, dtype, rows)
    target[:, 256:512] = -1 if rows > 512 else target[:, 256:512]
    want, step = head64(h, W, target, weight, up), head64(h, W, target, weight)
    loss, lse = torch.empty((1, rows), device=cuda), torch.empty((1, rows), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty((V, d), dtype=h.dtype, device=cuda)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    close(loss, want['loss'], want['loss_tol'])
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    check_grads(gh, gw, want, dtype)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    close(loss, step['loss'], step['loss_tol'])
    check_grads(gh, gw, step, dtype)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('scale', [20.0, 60.0])
def test_targets_far_below_the_largest_logit(cuda, dtype, scale):
    """Logits apart by hundreds: exponentials relative to the target's would pass 32 bits.  At the smaller scale some rows
    do and some do not."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 2, 70, 128, 700
    h, W, target, weight, up = make(B, n, d, V, dtype, 11, scale=scale)
    step = head64(h, W, target, weight)
    loss = torch.empty((B, n), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    close(loss, step['loss'], step['loss_tol'])
    # a power's argument is rounded to 2^-24 of up to |z| log2 e
    z = 2.0 ** -21 * float((h.double().nan_to_num(0, 0, 0) @ W.double().t()).abs().max())
    step['ae'] += z * step['a']
    step['be'] += z * step['b']
    check_grads(gh, gw, step, dtype)
    lse = torch.empty((B, n), device=cuda)
    want = head64(h, W, target, weight, up)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    want['ae'] += z * want['a']
    want['be'] += z * want['b']
    check_grads(gh, gw, want, dtype)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_sure_rows_keep_small_gradients(cuda, dtype):
    """Where the model is sure, the gradient is of the others' probabilities alone, a millionth and less: it keeps their
    precision."""
    import torch
    import paper_2606_00722_gb300 as epic
    d, V = 64, 64
    W = put(torch.eye(64) * 16.0, dtype)
    h = put(torch.eye(64)[None, :8], dtype)  # the target's logit is 16, the others' 0
    target = torch.arange(8, dtype=torch.int32, device=cuda)[None]
    step = head64(h, W, target, None)
    loss = torch.empty((1, 8), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw)
    assert (step['loss'] < 1e-5).all()
    assert ((loss.double() - step['loss']).abs() <= 2.0 ** -15 * step['loss'] + 1e-12).all()
    if dtype == 'bf16':  # as numbers of fp16, gradients of 1e-7 are subnormal
        check_grads(gh, gw, step, dtype)
        assert (gh[0, 0, 1:] > 0).all() and (gh[0, 0, 0] < 0)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_nan_and_infinite_logits(cuda, dtype):
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 1, 6, 16, 300
    for bad in (math.nan, math.inf):
        h, W, target, weight, up = make(B, n, d, V, dtype, 3, edges=False)
        h[0, 2, 5] = bad
        loss, lse = torch.empty((B, n), device=cuda), torch.empty((B, n), device=cuda)
        gh, gw = torch.empty_like(h), torch.empty_like(W)
        for form in ('step', 'two'):
            if form == 'step':
                epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
            else:
                epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
                epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
            assert loss[0, 2].isnan() and gh[0, 2].isnan().all() and gw.isnan().all()
            rest = [0, 1, 3, 4, 5]
            assert loss[0, rest].isfinite().all() and gh[0, rest].isfinite().all()
    # a target that has no probability: the loss is infinite, gradients are those of the others
    W = put(torch.tensor([[1.0], [2.0], [-math.inf]]), dtype)
    h = put(torch.ones((1, 2, 1)), dtype)
    target = torch.tensor([[2, 0]], dtype=torch.int32, device=cuda)
    loss, lse = torch.empty((1, 2), device=cuda), torch.empty((1, 2), device=cuda)
    epic.head_loss_forward(h, W, target, loss, lse)
    assert loss[0, 0] == math.inf and abs(float(lse[0, 0]) - math.log(math.e + math.e ** 2)) < 1e-5
    assert loss[0, 1].isfinite()
    # one token: it is certain
    W = put(torch.tensor([[3.0]]), dtype)
    target = torch.zeros((1, 2), dtype=torch.int32, device=cuda)
    gh, gw = torch.full_like(h, 7.0), torch.full_like(W, 7.0)
    epic.head_loss_step(h, W, target, loss, gh, gw)
    assert (loss == 0).all() and (gh == 0).all() and (gw == 0).all()


@pytest.mark.parametrize('rows,V', [(0, 40), (5, 0), (5, 40)])
def test_nothing_counts(cuda, rows, V):
    """No positions, no tokens, no targets: losses and gradients of 0, written whole."""
    import torch
    import paper_2606_00722_gb300 as epic
    d = 24
    h = torch.full((1, rows, d), math.nan, dtype=torch.bfloat16, device=cuda)
    W = torch.ones((V, d), dtype=torch.bfloat16, device=cuda)
    target = torch.full((1, rows), -1 if V else 0, dtype=torch.int32, device=cuda)
    loss, lse = torch.full((1, rows), 7.0, device=cuda), torch.full((1, rows), 7.0, device=cuda)
    gh, gw = torch.full_like(h, 7.0), torch.full_like(W, 7.0)
    epic.head_loss_step(h, W, target, loss, gh, gw)
    assert (loss == 0).all() and (gh == 0).all() and (gw == 0).all()
    loss.fill_(7.0), gh.fill_(7.0), gw.fill_(7.0)
    epic.head_loss_forward(h, W, target, loss, lse)
    epic.head_loss_backward(h, W, target, lse, torch.ones_like(loss), gh, gw)
    assert (loss == 0).all() and (lse == 0).all() and (gh == 0).all() and (gw == 0).all()


def test_hidden_states_of_any_strides(cuda):
    """Positions transposed in memory, and one sequence's hidden states broadcast to all."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 3, 20, 40, 333
    h, W, target, weight, up = make(B, n, d, V, 'bf16', 5, edges=False)
    loss = torch.empty((B, n), device=cuda)
    for x in (h.transpose(0, 1).contiguous().transpose(0, 1), h[:1].expand(B, n, d), h[:, :1].expand(B, n, d)):
        store = torch.empty((n, B, d), dtype=h.dtype, device=cuda)
        gh, gw = store.transpose(0, 1), torch.empty_like(W)
        step = head64(x, W, target, weight)
        epic.head_loss_step(x, W, target, loss, gh, gw, weight=weight)
        close(loss, step['loss'], step['loss_tol'])
        check_grads(gh, gw, step, 'bf16')


def test_gradient_against_differences(cuda):
    """(L(h + s e) - L(h - s e)) / 2s of the kernel's own losses, s = 1/32 so that both points are numbers of fp16 (h a
    multiple of 1/32 below 16).  It is off by s^2/6 of a third moment, at most (2 max|w|)^3, and by the losses' 2^-15 ... / s."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 1, 9, 32, 200
    h, W, target, weight, _ = make(B, n, d, V, 'f16', 21, edges=False)
    h.copy_((h.float() * 32).round() / 32)
    s = 1.0 / 32
    loss, lse = torch.empty((B, n), device=cuda), torch.empty((B, n), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    r = head64(h, W, target, weight)
    for c in (0, 13, 31):
        far = []
        for sign in (1.0, -1.0):
            x = h.clone()
            x[..., c] += sign * s
            epic.head_loss_forward(x, W, target, loss, lse, weight=weight)
            far.append(loss.double().clone())
        moment = (2 * float(W[:, c].abs().max())) ** 3
        tol = weight.double() * s * s / 6 * moment + r['loss_tol'] / s + 2.0 ** -10 * r['a'][..., c] + r['ae'][..., c]
        assert (((far[0] - far[1]) / (2 * s) - gh[..., c].double()).abs() <= tol).all()
    # the head: a weight of one token moves every position's logit by s h
    W.copy_((W.float() * 64).round() / 64)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    for v, c in ((int(target[0, 0]), 3), (int(target[0, 4]), 30), (100, 7)):
        far = []
        for sign in (1.0, -1.0):
            x = W.clone()
            x[v, c] += sign / 64
            epic.head_loss_forward(h, x, target, loss, lse, weight=weight)
            far.append(loss.double().sum())
        moment = float((weight.double() * (2 * h[..., c].double().abs()) ** 3).sum())
        tol = moment / 64 ** 2 / 6 + float(r['loss_tol'].sum()) * 64 + 2.0 ** -9 * float(r['b'][v, c] + 1)
        assert abs(float((far[0] - far[1]) * 32) - float(gw[v, c])) <= tol


def test_same_bits_streams_and_graphs(cuda):
    """The same call twice, beside another on a second stream, and captured and replayed on other inputs."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 2, 150, 136, 3001
    sets = [make(B, n, d, V, 'bf16', s) for s in (1, 2)]
    outs = []
    for h, W, target, weight, up in sets:
        o = [torch.empty((B, n), device=cuda), torch.empty_like(h), torch.empty_like(W)]
        epic.head_loss_step(h, W, target, *o, weight=weight)
        outs.append([t.clone() for t in o])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [[torch.empty((B, n), device=cuda), torch.empty_like(s[0]), torch.empty_like(s[1])] for s in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        epic.head_loss_step(sets[0][0], sets[0][1], sets[0][2], *got[0], weight=sets[0][3])
        epic.head_loss_step(sets[1][0], sets[1][1], sets[1][2], *got[1], weight=sets[1][3], stream=side)
    torch.cuda.synchronize()
    for a, b in zip(outs, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    h, W, target, weight = [t.clone() for t in sets[0][:4]]
    need = epic.head_loss_workspace('step', h, W)
    work = torch.empty(need, dtype=torch.uint8, device=cuda)
    loss, gh, gw = torch.empty((B, n), device=cuda), torch.empty_like(h), torch.empty_like(W)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight, workspace=work)
    for s, want in zip(sets, outs):
        for t, x in zip((h, W, target, weight), s):
            t.copy_(x)
        work.fill_(255)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip((loss, gh, gw), want))


def test_as_a_torch_operation(cuda):
    """Loss and gradients through autograd; only what asks for a gradient gets one; inputs that change are an error."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 2, 33, 56, 400
    h, W, target, weight, up = make(B, n, d, V, 'bf16', 8)
    want = head64(h, W, target, weight, up)
    x, w = h.clone().requires_grad_(), W.clone().requires_grad_()
    (epic.head_loss(x, w, target, weight) * up).sum().backward()
    check_grads(x.grad, w.grad, want, 'bf16')
    x.grad = w.grad = None
    (epic.head_loss(x, W, target, weight) * up).sum().backward()
    check_grads(x.grad, None, want, 'bf16')
    (epic.head_loss(h, w, target, weight) * up).sum().backward()
    check_grads(None, w.grad, want, 'bf16')
    assert not epic.head_loss(h, W, target, weight).requires_grad
    loss = epic.head_loss(x, w, target, weight)
    target.add_(1)
    with pytest.raises(RuntimeError):
        loss.sum().backward()


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('R,d,V', [(40, 64, 300), (300, 97, 2100)])
def test_what_a_workspace_holds_does_not_matter(cuda, dtype, R, d, V):
    """All forms with workspaces of NaNs, infinities and numbers give the same bits; a workspace of the size that is asked
    for is enough, and nothing behind it is written."""
    import torch
    import paper_2606_00722_gb300 as epic
    h, W, target, weight, up = make(1, R, d, V, dtype, R + d)
    results = []
    for fill in (0, 0x7f, 0xff, 0x80):
        loss, lse = torch.empty((1, R), device=cuda), torch.empty((1, R), device=cuda)
        outs = [loss, lse]
        for form in ('forward', 'backward', 'step'):
            need = epic.head_loss_workspace(form, h, W)
            store = torch.full((need + 512,), fill, dtype=torch.uint8, device=cuda)
            store[need:] = 77
            work = store[:need]
            gh, gw = torch.empty_like(h), torch.empty((V, d), dtype=h.dtype, device=cuda)
            if form == 'forward':
                epic.head_loss_forward(h, W, target, loss, lse, weight=weight, workspace=work)
            elif form == 'backward':
                epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight, workspace=work)
                outs += [gh, gw]
            else:
                again = torch.empty_like(loss)
                epic.head_loss_step(h, W, target, again, gh, gw, weight=weight, workspace=work)
                outs += [again, gh, gw]
            assert (store[need:] == 77).all()
        results.append(outs)
    for outs in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], outs))


def test_positions_far_apart(cuda):
    """Sequences 2^31 elements apart, in hidden states and in their gradient."""
    import torch
    import paper_2606_00722_gb300 as epic
    n, d, V, far = 3, 24, 90, (1 << 31) + 16
    h, W, target, weight, up = make(2, n, d, V, 'bf16', 5, edges=False)
    big, grad = [torch.zeros(far + n * d, dtype=h.dtype, device=cuda) for _ in range(2)]
    x, gh = [t.as_strided((2, n, d), (far, d, 1)) for t in (big, grad)]
    x.copy_(h)
    loss, gw = torch.empty((2, n), device=cuda), torch.empty_like(W)
    epic.head_loss_step(x, W, target, loss, gh, gw, weight=weight)
    step = head64(h, W, target, weight)
    close(loss, step['loss'], step['loss_tol'])
    check_grads(gh, gw, step, 'bf16')
    assert int((grad != 0).sum()) <= 2 * n * d


def test_a_head_past_32_bits(cuda):
    """2.3e9 weights, all 0 but those of the last token: lse = log(V - 1 + exp z), and gradients by hand."""
    import torch
    import paper_2606_00722_gb300 as epic
    V, d = 70000, 32768
    W = torch.zeros((V, d), dtype=torch.bfloat16, device=cuda)
    W[-1, ::2] = 2.0 ** -10
    h = torch.ones((1, 2, d), dtype=torch.bfloat16, device=cuda) * 0.5  # z of the last token: 16384 / 1024 / 2 = 8
    target = torch.tensor([[V - 1, 7]], dtype=torch.int32, device=cuda)
    loss, lse = torch.empty((1, 2), device=cuda), torch.empty((1, 2), device=cuda)
    want = math.log(V - 1 + math.exp(8.0))
    epic.head_loss_forward(h, W, target, loss, lse)
    assert ((lse - want).abs() < 1e-4).all() and abs(float(loss[0, 0]) - (want - 8.0)) < 1e-4
    assert abs(float(loss[0, 1]) - want) < 1e-4
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    epic.head_loss_step(h, W, target, loss, gh, gw)
    p, rest = math.exp(8.0 - want), math.exp(-want)
    u = 2.0 ** -8  # three roundings of terms that do not cancel but at the two targets, there of sums of 2
    assert ((gw[-1].double() - 0.5 * (2 * p - 1)).abs() < 3.1 * u * 0.5 * (1 + 2 * p)).all()
    assert ((gw[7].double() - 0.5 * (2 * rest - 1)).abs() < 3.1 * u * 0.5 * (1 + 2 * rest)).all()
    assert ((gw[1000].double() - rest).abs() < 3.1 * u * rest).all()
    assert ((gh[0, 1, ::2].double() - p * 2.0 ** -10).abs() < 2.1 * u * p * 2.0 ** -10).all() and (gh[0, 1, 1::2] == 0).all()
    assert ((gh[0, 0, ::2].double() - (p - 1) * 2.0 ** -10).abs() < 2.1 * u * 2.0 ** -10).all()


def test_gradients_of_broadcast_hidden_states(cuda):
    """One sequence's hidden states for all: torch adds up what each position's gradient is."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 3, 10, 32, 100
    h, W, target, weight, up = make(B, n, d, V, 'bf16', 2, edges=False)
    one = h[:1].clone().requires_grad_()
    (epic.head_loss(one.expand(B, n, d), W, target, weight) * up).sum().backward()
    r = head64(h[:1].expand(B, n, d), W, target, weight, up)
    u = 2.0 ** -8
    tol = ((u + 2.0 ** -12) * r['a'] + r['ae'] + u * r['gh'].abs()).sum(0) + 3 * u * r['gh'].abs().sum(0)
    assert one.grad.shape == (1, n, d) and ((one.grad[0].double() - r['gh'].sum(0)).abs() <= tol).all()


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_weights_of_all_sizes(cuda, dtype):
    """Weights from 1e-4 to 1e4: in bf16 a small row keeps its precision, in fp16 what is left of the largest one's."""
    import torch
    import paper_2606_00722_gb300 as epic
    B, n, d, V = 2, 60, 72, 400
    h, W, target, weight, up = make(B, n, d, V, dtype, 17)
    weight *= 10.0 ** (torch.arange(B * n, device=cuda) % 9 - 4).view(B, n)
    h *= 0.1  # so that gradients are within fp16
    loss, lse = torch.empty((B, n), device=cuda), torch.empty((B, n), device=cuda)
    gh, gw = torch.empty_like(h), torch.empty_like(W)
    step, want = head64(h, W, target, weight), head64(h, W, target, weight, up)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    close(loss, step['loss'], step['loss_tol'])
    check_grads(gh, gw, step, dtype)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    check_grads(gh, gw, want, dtype)


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
@pytest.mark.parametrize('d,V', [(64, 300), (200, 9000)])
def test_targets_that_many_positions_share(cuda, dtype, d, V):
    """One target for a third of 700 positions, a few for the rest, in all forms; also with rows that leave the window."""
    import torch
    import paper_2606_00722_gb300 as epic
    for scale in (1.0, 30.0):
        h, W, target, weight, up = make(1, 700, d, V, dtype, d, scale=scale)
        target[0, ::3] = torch.where((target[0, ::3] >= 0) & (target[0, ::3] < V), 7, target[0, ::3])
        target[0, 1::3] = torch.where((target[0, 1::3] >= 0) & (target[0, 1::3] < V), target[0, 1::3] % 60, target[0, 1::3])
        step, want = head64(h, W, target, weight), head64(h, W, target, weight, up)
        z = 2.0 ** -21 * float((h.double().nan_to_num(0, 0, 0) @ W.double().t()).abs().max())  # a power's argument
        for r in (step, want):
            r['ae'] += z * r['a']
            r['be'] += z * r['b']
        loss, lse = torch.empty((1, 700), device=cuda), torch.empty((1, 700), device=cuda)
        gh, gw = torch.empty_like(h), torch.empty_like(W)
        epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
        close(loss, step['loss'], step['loss_tol'])
        check_grads(gh, gw, step, dtype)
        epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
        epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
        check_grads(gh, gw, want, dtype)
