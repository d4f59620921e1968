"""How much of a loss's call exists at a time, without a GPU: from the workspaces' sizes."""
import ctypes as C

import pytest

import paper_2606_00722_gb300 as epic

FORWARD, BACKWARD, STEP = range(3)


def size(form, rows, V, d=64):
    n = C.c_size_t()
    lib = epic.load(epic.build())
    assert lib.epic_head_loss_workspace(form, 2, 1, rows, d, V, 4096, d, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize('V', [2000, 50000, 126000])
def test_a_forward_call_is_cut_by_what_it_keeps(monkeypatch, V):
    """Exponentials, which only gradients need, do not cut it: 16,384 positions stay one piece where their records fit."""
    whole = size(FORWARD, 16384, V)
    records = 16384 * ((V + 127) // 128) * 8
    assert records <= whole < records + 16384 * (2 * 64 + 200)  # records, hidden states, a few numbers each
    monkeypatch.setenv('EPIC_HEAD_PIECE_MB', str(records // (1 << 20) + 1))
    assert size(FORWARD, 16384, V) == whole
    monkeypatch.setenv('EPIC_HEAD_PIECE_MB', '1')
    assert size(FORWARD, 16384, V) < whole


@pytest.mark.parametrize('form', [BACKWARD, STEP])
def test_exponentials_are_bounded_down_to_256_positions(monkeypatch, form):
    V, rest = 126000, 126000 * 64 * 4 + 126000 * 16 + (1 << 23)  # the head's gradient in 32 bits, lists, records
    row = (V + 63) // 64 * 64 * 2
    for mb in (1, 64, 100, 500):
        monkeypatch.setenv('EPIC_HEAD_PIECE_MB', str(mb))
        positions = max(256, (mb << 20) // row // 256 * 256)
        assert 0 < size(form, 4096, V) - positions * row < rest + positions * 9000  # (records 8 x 985, hidden states, numbers)


def test_a_huge_vocabulary():
    """More than the default 2 GB from some 4 million tokens on: 256 positions are the least."""
    V = 8 << 20
    assert size(BACKWARD, 4096, V) > 256 * V * 2
    assert size(FORWARD, 4096, V) < (2 << 30) + (1 << 26)
