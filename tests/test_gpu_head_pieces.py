"""A forward call of several pieces against 64 bits, beside the same call in one."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_forward_pieces(cuda, monkeypatch, dtype):
    import torch
    import paper_2606_00722_gb300 as epic
    t = {'f16': torch.float16, 'bf16': torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(1)
    B, n, d, V = 3, 250, 40, 66000  # 4,128 bytes of records a position: pieces of 256
    h = torch.randn((B, n, d), generator=g).to(t).to(cuda)
    W = (torch.randn((V, d), generator=g) / d ** 0.5).to(t).to(cuda)
    target = torch.randint(-V // 3, V, (B, n), generator=g).to(torch.int32).to(cuda)
    out = []
    for piece in (None, '1'):
        if piece:
            monkeypatch.setenv('EPIC_HEAD_PIECE_MB', piece)
        loss, lse = torch.full((B, n), 7.0, device=cuda), torch.full((B, n), 7.0, device=cuda)
        need = epic.head_loss_workspace('forward', h, W)
        epic.head_loss_forward(h, W, target, loss, lse)
        out.append((need, loss, lse))
    assert out[1][0] < out[0][0]
    counts = target >= 0
    z = h.double() @ W.double().t()
    want = torch.logsumexp(z, -1)
    cost = want - z.gather(-1, target.clamp(min=0).long()[..., None])[..., 0]
    for _, loss, lse in out:
        # a logit is off by 44 2^-24 of sum |h| |W| (some 40), twice in a loss; 2^-15 for the sums, 2^-20 of itself
        assert ((lse.double() - want)[counts].abs() < 2.0 ** -11).all() and (lse[~counts] == 0).all()
        assert ((loss.double() - cost)[counts].abs() < 2.0 ** -10).all() and (loss[~counts] == 0).all()


@pytest.mark.parametrize('dtype', ['bf16', 'f16'])
def test_more_positions_than_a_piece_has(cuda, dtype):
    """17,000 positions at the default size of pieces: one of 16,384 and the rest.  Tolerances are those of the loss's own test,
    whose chains of 2^14 steps of 8 these sums do not pass."""
    import torch
    import paper_2606_00722_gb300 as epic
    from test_gpu_head_loss import check_grads, close, head64, make
    B, n, d, V = 1, 17000, 40, 300
    h, W, target, weight, up = make(B, n, d, V, dtype, 12)
    loss, lse = torch.full((B, n), 7.0, device=cuda), torch.full((B, n), 7.0, device=cuda)
    gh, gw = torch.full_like(h, 7.0), torch.full((V, d), 7.0, dtype=h.dtype, device=cuda)
    epic.head_loss_step(h, W, target, loss, gh, gw, weight=weight)
    want = head64(h, W, target, weight)
    close(loss, want['loss'], want['loss_tol'])
    check_grads(gh, gw, want, dtype)
    want = head64(h, W, target, weight, up)
    epic.head_loss_forward(h, W, target, loss, lse, weight=weight)
    close(lse, want['lse'], want['lse_tol'])
    epic.head_loss_backward(h, W, target, lse, up, gh, gw, weight=weight)
    check_grads(gh, gw, want, dtype)
