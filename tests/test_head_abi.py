"""Refusals of the head's calls: found on the host before any device work, so they need no GPU; empty calls are no-ops;
workspaces grow with their calls."""
import ctypes as C

import paper_2606_00722_gb300 as epic

P = 4096  # an address that nothing reads
BIG = 1 << 40
BAD, CAPACITY = 1, 6


def lib():
    return epic.load(epic.build())


def forward(h=P, dtype=2, B=2, n=3, d=64, sb=192, sn=64, W=P, V=100, sw=64, target=P, loss=P, lse=P, ws=P, size=BIG):
    return lib().epic_head_loss_forward(h, dtype, B, n, d, sb, sn, W, V, sw, target, None, loss, lse, ws, size, None)


def backward(h=P, dtype=2, B=2, n=3, d=64, sb=192, sn=64, W=P, V=100, sw=64, target=P, lse=P, up=P, gh=P, gb=192, gn=64,
             gw=P, gs=64, ws=P, size=BIG):
    return lib().epic_head_loss_backward(h, dtype, B, n, d, sb, sn, W, V, sw, target, None, lse, up, gh, gb, gn, gw, gs, ws,
                                         size, None)


def step(h=P, dtype=2, B=2, n=3, d=64, sb=192, sn=64, W=P, V=100, sw=64, target=P, loss=P, gh=P, gb=192, gn=64, gw=P, gs=64,
         ws=P, size=BIG):
    return lib().epic_head_loss_step(h, dtype, B, n, d, sb, sn, W, V, sw, target, None, loss, gh, gb, gn, gw, gs, ws, size,
                                     None)


def quantize(x=P, dtype=2, B=2, n=3, d=64, sb=192, sn=64, pos=P, k=2, q=P, s=P):
    return lib().epic_quantize_rows(x, dtype, B, n, d, sb, sn, pos, k, q, s, None)


def logits(q=P, s=P, B=2, k=3, d=64, W=P, S=P, V=100, sw=64, z=P, dtype=2, zb=300, zn=100, ws=P, size=BIG):
    return lib().epic_int8_logits(q, s, B, k, d, W, S, V, sw, z, dtype, zb, zn, ws, size, None)


def loss_bytes(form=0, dtype=2, B=2, n=3, d=64, V=100, W=P, sw=64):
    size = C.c_size_t(12345)
    status = lib().epic_head_loss_workspace(form, dtype, B, n, d, V, W, sw, C.byref(size))
    return size.value if status == 0 else -status


def logits_bytes(B=2, k=3, d=64, V=100, W=P, sw=64):
    size = C.c_size_t(12345)
    status = lib().epic_int8_logits_workspace(B, k, d, V, W, sw, C.byref(size))
    return size.value if status == 0 else -status


def test_bad_losses_are_refused():
    for call in (forward, backward, step):
        for bad in (dict(dtype=0), dict(dtype=3), dict(B=-1), dict(n=-1), dict(d=0), dict(V=-1), dict(sb=-1), dict(sn=-1),
                    dict(h=None), dict(h=P + 1), dict(W=None), dict(W=P + 1), dict(sw=63), dict(target=None),
                    dict(ws=None), dict(ws=P + 128), dict(size=100), dict(size=0)):
            assert call(**bad) == BAD, (call, bad)
        assert call(V=0x7fffffff) == CAPACITY
        assert call(d=(1 << 20) + 1, sw=1 << 21) == CAPACITY
    for bad in (dict(loss=None), dict(lse=None)):
        assert forward(**bad) == BAD, bad
    for bad in (dict(lse=None), dict(up=None), dict(gh=P + 1), dict(gw=P + 1), dict(gb=-1), dict(gn=-1), dict(gs=63)):
        assert backward(**bad) == BAD, bad
    for bad in (dict(loss=None), dict(gh=P + 1), dict(gw=P + 1), dict(gb=-1), dict(gn=-1), dict(gs=63)):
        assert step(**bad) == BAD, bad


def test_workspaces_of_the_loss():
    for bad in (dict(form=-1), dict(form=3), dict(dtype=0), dict(B=-1), dict(n=-2), dict(d=0), dict(V=-1), dict(sw=5)):
        assert loss_bytes(**bad) == -BAD, bad
    assert lib().epic_head_loss_workspace(0, 2, 2, 3, 64, 100, P, 64, None) == BAD
    assert loss_bytes(V=0x7fffffff) == -CAPACITY
    for form in range(3):
        small = loss_bytes(form=form)
        assert 0 < small <= loss_bytes(form=form, V=50000) <= loss_bytes(form=form, V=50000, B=1000)
        call = (forward, backward, step)[form]
        assert call(size=small - 1) == BAD
    # exponentials of a piece are bounded: 2 GB by default, beside a gradient in 32 bits and 2 % for the rest
    most = loss_bytes(form=2, B=1 << 20, n=1 << 20, V=126000, d=4096, sw=4096)
    assert most < (2 << 30) + 4 * 126000 * 4096 + (1 << 29) + 2 * 126000 * 4096


def test_piece_size_is_an_environment_knob(monkeypatch):
    big = loss_bytes(form=2, B=64, n=64, V=50000)
    monkeypatch.setenv('EPIC_HEAD_PIECE_MB', '64')
    assert loss_bytes(form=2, B=64, n=64, V=50000) < big


def test_bad_rows_in_8_bits_are_refused():
    for bad in (dict(dtype=3), dict(dtype=-1), dict(B=-1), dict(n=-1), dict(d=0), dict(sb=-1), dict(sn=-1), dict(k=-1),
                dict(pos=None, k=4), dict(x=None), dict(x=P + 1), dict(x=P + 2, dtype=0), dict(q=None), dict(s=None),
                dict(s=P + 2), dict(pos=P + 2)):
        assert quantize(**bad) == BAD, bad
    assert quantize(B=1 << 20, k=1 << 11) == CAPACITY


def test_bad_integer_logits_are_refused():
    for bad in (dict(B=-1), dict(k=-1), dict(d=0), dict(V=-1), dict(sw=63), dict(dtype=3), dict(zb=-1), dict(zn=-1),
                dict(q=None), dict(s=None), dict(W=None), dict(S=None), dict(z=None), dict(z=P + 1),
                dict(z=P + 2, dtype=0), dict(s=P + 2), dict(S=P + 1), dict(ws=None), dict(ws=P + 64), dict(size=0)):
        assert logits(**bad) == BAD, bad
    for big in (dict(d=131072, sw=131072), dict(V=0x7fffffff), dict(B=1 << 11, k=(1 << 10) + 1)):
        assert logits(**big) == CAPACITY, big
        assert logits_bytes(**big) == -CAPACITY, big
    for bad in (dict(B=-1), dict(k=-1), dict(d=0), dict(V=-1), dict(sw=2)):
        assert logits_bytes(**bad) == -BAD, bad
    assert lib().epic_int8_logits_workspace(2, 3, 64, 100, P, 64, None) == BAD


def test_empty_calls_touch_nothing():
    none = dict(B=0, target=None, ws=None, size=0, h=None)
    assert forward(loss=None, lse=None, **none) == 0
    assert backward(lse=None, up=None, gh=None, gw=None, **none) == 0
    assert step(loss=None, gh=None, gw=None, **none) == 0
    assert step(loss=None, V=0, W=None, gw=None, **none) == 0
    assert quantize(B=0, x=None, pos=None, q=None, s=None) == 0
    assert quantize(k=0, q=None, s=None) == 0
    assert logits(B=0, q=None, s=None, z=None, ws=None, size=0) == 0
    assert logits(V=0, W=None, S=None, z=None, ws=None, size=0) == 0
