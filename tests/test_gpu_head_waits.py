"""What a kernel of the head leaves when a wait inside it gives up: NaN wherever its result would have gone, nowhere else, and the
next call is as ever.  EPIC_HEAD_WAIT_MS = 0 lets every wait give up before it begins."""
import pytest

pytestmark = pytest.mark.gpu


def inputs(B, n, d, V, dtype, pad=0):
    import torch
    t = {'f16': torch.float16, 'bf16': torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(d + V)
    h = torch.randn((B, n, d), generator=g).to(t).cuda()
    store = torch.empty((V, d + pad), dtype=t, device='cuda')
    store[:, :d] = (torch.randn((V, d), generator=g) / d ** 0.5).to(t)
    target = torch.randint(-V // 2, V, (B, n), generator=g).to(torch.int32).cuda()
    return h, store[:, :d], target


@pytest.mark.parametrize('B,n,d,V,dtype,pad,piece', [
    (1, 5, 64, 300, 'bf16', 0, None),
    (2, 150, 136, 3001, 'bf16', 0, None),    # sums in parts
    (1, 300, 97, 2051, 'f16', 3, None),      # rows of the head at odd places
    (1, 700, 96, 2051, 'f16', 0, '1'),       # three pieces
    (3, 250, 264, 2050, 'bf16', 0, '1'),
])
def test_losses_and_gradients(cuda, monkeypatch, B, n, d, V, dtype, pad, piece):
    import torch
    import paper_2606_00722_gb300 as epic
    if piece:
        monkeypatch.setenv('EPIC_HEAD_PIECE_MB', piece)
    h, W, target = inputs(B, n, d, V, dtype, pad)
    up = torch.ones((B, n), device=cuda)

    def run(lse=None):
        loss, keep, again = [torch.full((B, n), 7.0, device=cuda) for _ in range(3)]
        gs = [torch.full((B, n, d + 2), 7.0, dtype=h.dtype, device=cuda) for _ in range(2)]
        ws = [torch.full((V, d + 8), 7.0, dtype=h.dtype, device=cuda) for _ in range(2)]
        epic.head_loss_forward(h, W, target, loss, keep)
        epic.head_loss_backward(h, W, target, keep if lse is None else lse, up, gs[0][..., :d], ws[0][:, :d])
        epic.head_loss_step(h, W, target, again, gs[1][..., :d], ws[1][:, :d])
        for t in gs + ws:
            assert (t[..., d:] == 7).all()
        return loss, keep, again, gs[0][..., :d], gs[1][..., :d], ws[0][:, :d], ws[1][:, :d]

    want = run()
    assert all(t.isfinite().all() for t in want)
    monkeypatch.setenv('EPIC_HEAD_WAIT_MS', '0')
    got = run(want[1])
    counts = target >= 0
    assert counts.any() and not counts.all()
    for t in got[:5]:
        assert t[counts].isnan().all() and (t[~counts] == 0).all()
    assert all(t.isnan().all() for t in got[5:])
    monkeypatch.delenv('EPIC_HEAD_WAIT_MS')
    assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize('dtype', ['f32', 'f16', 'bf16'])
@pytest.mark.parametrize('B,k,d,V,pad', [(1, 20, 64, 300, 0), (3, 20, 1100, 2050, 0), (33, 5, 203, 1021, 5),
                                         (7, 40, 2100, 600, 12), (1, 300, 160, 90, 0), (1, 9, 33, 1, 0)])
def test_integer_logits(cuda, monkeypatch, B, k, d, V, pad, dtype):
    import torch
    import paper_2606_00722_gb300 as epic
    t = {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(d + V)
    q = torch.randint(-20, 21, (B, k, d), generator=g).to(torch.int8).to(cuda)
    head = torch.randint(-20, 21, (V, d + pad), generator=g).to(torch.int8).to(cuda)[:, :d]
    scale, head_scale = [(torch.rand(s, generator=g) * 0.01).to(cuda) for s in ((B, k), (V,))]

    def run():
        z = torch.full((B, k, V + 3), 7.0, dtype=t, device=cuda)
        epic.int8_logits(q, scale, head, head_scale, z[..., :V])
        assert (z[..., V:] == 7).all()
        return z[..., :V]

    want = run()
    assert want.isfinite().all()
    monkeypatch.setenv('EPIC_HEAD_WAIT_MS', '0')
    assert run().isnan().all()
    monkeypatch.delenv('EPIC_HEAD_WAIT_MS')
    assert torch.equal(run(), want)


def test_a_limit_that_is_no_number_is_left_out(cuda, monkeypatch):
    import torch
    import paper_2606_00722_gb300 as epic
    h, W, target = inputs(1, 40, 64, 300, 'bf16')
    loss, lse = torch.empty((1, 40), device=cuda), torch.empty((1, 40), device=cuda)
    for limit, finite in (('', True), ('x', True), ('1000', True), ('-5', False)):
        monkeypatch.setenv('EPIC_HEAD_WAIT_MS', limit)
        epic.head_loss_forward(h, W, target, loss, lse)
        assert bool(loss.isfinite().all()) == finite
