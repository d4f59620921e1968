"""Rows in 8 bits and logits of 8-bit hidden states and heads, against whole-number arithmetic.

A sum of products is a whole number and exact; as 32-bit number (2^-24), times two scales (2^-24 each) and as the logits'
type (u = eps / 2: bf16 2^-8, fp16 2^-11, fp32 2^-24) it is off by at most 3 2^-24 + u of itself, more in fp16 below its
normal numbers (2^-25)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _dtype(name):
    import torch
    return {'f32': torch.float32, 'f16': torch.float16, 'bf16': torch.bfloat16}[name]


def quantized(x):
    """(q, s) of rows of 32-bit numbers, by numpy's IEEE arithmetic."""
    s = (np.abs(x).max(-1) / np.float32(127)).astype(np.float32)
    with np.errstate(all='ignore'):
        q = np.rint(x / s[..., None])
    return np.where(s[..., None] > 0, np.clip(q, -127, 127), 0).astype(np.int8), s


@pytest.mark.parametrize('B,n,d,k,dtype,pad', [(1, 1, 1, 1, 'f32', 0), (2, 5, 7, 3, 'bf16', 1), (3, 9, 100, 9, 'f16', 4),
                                               (2, 40, 4096, 16, 'bf16', 8), (1, 3, 1003, 2, 'f32', 5),
                                               (1, 2, 20001, 2, 'f16', 0), (700, 2, 72, 1, 'bf16', 0)])
def test_rows_in_8_bits(cuda, B, n, d, k, dtype, pad):
    import torch
    import paper_2606_00722_gb300 as epic
    g = torch.Generator().manual_seed(d)
    x = torch.randn((B, n, d + pad), generator=g) * torch.exp(torch.randn((B, n, 1), generator=g) * 3)
    x[..., 0] *= 5.0
    x[0, 0] = 0.0                       # a row of zeros has scale 0
    x[-1, -1, :] = 2.0 ** -20 if dtype == 'f16' else 1e-41  # subnormals of 32 bits
    x = x.to(_dtype(dtype)).cuda()[..., :d]
    pos = torch.stack([torch.randperm(n, generator=g)[:k] for _ in range(B)]).to(torch.int32).cuda()
    for p in (pos, None):
        q = torch.full((B, k, d), 99, dtype=torch.int8, device=cuda)
        s = torch.full((B, k), 7.0, device=cuda)
        epic.quantize_rows(x, q, s, pos=p)
        rows = x.float().cpu().numpy()
        at = np.arange(k)[None].repeat(B, 0) if p is None else p.cpu().numpy()
        wq, ws = quantized(rows[np.arange(B)[:, None], at])
        np.testing.assert_array_equal(s.cpu().numpy(), ws)
        np.testing.assert_array_equal(q.cpu().numpy(), wq)


def test_rows_without_a_scale(cuda):
    """NaN, infinities and positions out of range: their rows have no finite logits; the others are as they were."""
    import torch
    import paper_2606_00722_gb300 as epic
    for dtype in ('f32', 'f16', 'bf16'):
        x = torch.randn((1, 5, 600), generator=torch.Generator().manual_seed(1)).to(_dtype(dtype)).cuda()
        x[0, 1, 599] = math.nan
        x[0, 2, 300] = -math.inf
        x[0, 3, :] = math.nan
        x[0, 3, 5] = math.inf
        pos = torch.tensor([[0, 1, 2, 3, 4, -1, 5]], dtype=torch.int32, device=cuda)
        q, s = torch.full((1, 7, 600), 99, dtype=torch.int8, device=cuda), torch.zeros((1, 7), device=cuda)
        epic.quantize_rows(x, q, s, pos=pos)
        assert s[0, [1, 3, 5, 6]].isnan().all() and s[0, 2] == math.inf and s[0, [0, 4]].isfinite().all()
        assert (q[0, 5:] == 0).all()
        head = torch.randint(-127, 128, (90, 600), dtype=torch.int8, device=cuda)
        z = torch.zeros((1, 7, 90), dtype=_dtype(dtype), device=cuda)
        epic.int8_logits(q, s, head, torch.ones(90, device=cuda), z)
        assert not z[0, [1, 2, 3, 5, 6]].isfinite().any() and z[0, [0, 4]].isfinite().all()
        cand, conf = torch.zeros((1, 7, 3), dtype=torch.int32, device=cuda), torch.zeros((1, 7, 3), device=cuda)
        epic.propose_topk(z, cand, conf)
        assert (cand[0, 5:] == -1).all()


SIZES = [  # B, k, d, V, dtype, pad of the logits, head: pad and shift
    (1, 1, 1, 1, 'f32', 0, 0, 0),
    (1, 8, 128, 256, 'bf16', 0, 0, 0),
    (1, 1, 4096, 5003, 'bf16', 0, 0, 0),
    (1, 3, 1003, 777, 'f16', 3, 0, 0),
    (2, 2, 512, 3000, 'f32', 0, 16, 16),
    (3, 3, 130, 1000, 'bf16', 1, 5, 3),
    (1, 13, 96, 1001, 'f16', 0, 0, 0),
    (16, 4, 2048, 2000, 'bf16', 0, 0, 0),
    (33, 5, 1003, 3001, 'f16', 0, 0, 0),
    (1, 257, 64, 517, 'bf16', 7, 0, 0),
    (5, 103, 1040, 650, 'f32', 4, 0, 0),
    (9, 100, 2056, 1300, 'bf16', 16, 8, 0),
    (1, 40, 5000, 300, 'f32', 0, 0, 1),
]


def int8_case(B, k, d, V, seed, extreme=False, hpad=0, hshift=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(-128, 128, (B, k, d), generator=g).to(torch.int8)
    w = torch.randint(-128, 128, (V, d + hpad), generator=g).to(torch.int8)
    if extreme:  # sums that grow as far as they can, odd ones too
        q.fill_(-128)
        q[:, 1::2] = 127
        w[::3] = -128
        w[1::3] = 127
    flat = torch.zeros(hshift + w.numel() + 64, dtype=torch.int8, device='cuda')
    flat[hshift:hshift + w.numel()] = w.reshape(-1).cuda()
    head = flat[hshift:hshift + w.numel()].view(V, d + hpad)[:, :d]
    return (q.cuda(), head, (torch.rand((B, k), generator=g) * 0.02 + 0.001).cuda(),
            (torch.rand(V, generator=g) * 0.002 + 1e-4).cuda())


def check_logits(z, q, head, s, S, dtype):
    sums = (q.reshape(-1, q.shape[2]).double() @ head.double().t()).view(z.shape)  # exact: below 2^53
    want = sums * s[..., None].double() * S.double()
    u = {'f32': 2.0 ** -24, 'f16': 2.0 ** -11, 'bf16': 2.0 ** -8}[dtype]
    tol = want.abs() * (3 * 2.0 ** -24 * 1.001 + u * 1.001) + (2.0 ** -25 if dtype == 'f16' else 0.0)
    bad = (z.double() - want).abs() > tol
    assert not bad.any(), (int(bad.sum()), z[bad][:4], want[bad][:4])


@pytest.mark.parametrize('extreme', [False, True])
@pytest.mark.parametrize('B,k,d,V,dtype,pad,hpad,hshift', SIZES)
def test_logits(cuda, B, k, d, V, dtype, pad, hpad, hshift, extreme):
    import torch
    import paper_2606_00722_gb300 as epic
    q, head, s, S = int8_case(B, k, d, V, d + V, extreme, hpad, hshift)
    if extreme and dtype == 'f16':
        s *= 0.01  # within fp16's range
    store = torch.full((B, k, V + pad + 1), 7.0, dtype=_dtype(dtype), device=cuda)
    z = store[..., :V]
    epic.int8_logits(q, s, head, S, z)
    check_logits(z, q, head, s, S, dtype)
    assert (store[..., V:] == 7).all()
    again = torch.empty((k, B, V), dtype=_dtype(dtype), device=cuda).transpose(0, 1)
    epic.int8_logits(q, s, head, S, again)
    assert torch.equal(again, z)


@pytest.mark.parametrize('rows', [1, 5, 70])
def test_sums_past_24_bits_are_exact(cuda, rows):
    """32-bit logits with scales of 1 show whole sums: up to 2^24 to the last bit, above as 32 bits round them once."""
    import torch
    import paper_2606_00722_gb300 as epic
    d, V = 131071, 70
    q, head, s, S = int8_case(1, rows, d, V, 3, True)
    g = torch.Generator().manual_seed(4)
    head[2::3] = torch.randint(-128, 128, head[2::3].shape, generator=g).to(torch.int8).cuda()
    q[:, ::2, d // 2:] *= -1  # -128 stays: sums rise far, and fall for the rest of the row
    q[:, ::2, d // 2:] = torch.where(q[:, ::2, d // 2:] == -128, 127, q[:, ::2, d // 2:])
    z = torch.empty((1, rows, V), device=cuda)
    epic.int8_logits(q, torch.ones_like(s), head, torch.ones_like(S), z)
    want = (q.double() @ head.double().t()).float()
    assert torch.equal(z, want)


def test_streams_and_graphs(cuda):
    import torch
    import paper_2606_00722_gb300 as epic
    q, head, s, S = int8_case(2, 30, 515, 1200, 5)
    x = torch.randn((2, 64, 515), generator=torch.Generator().manual_seed(2)).cuda().to(torch.bfloat16)
    z = torch.empty((2, 30, 1200), dtype=torch.bfloat16, device=cuda)
    pos = torch.arange(30, dtype=torch.int32, device=cuda).repeat(2, 1) * 2
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    epic.quantize_rows(x, q, s, pos, stream=side)
    epic.int8_logits(q, s, head, S, z, stream=side)
    torch.cuda.synchronize()
    check_logits(z, q, head, s, S, 'bf16')
    want = z.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        epic.quantize_rows(x, q, s, pos)
        epic.int8_logits(q, s, head, S, z)
    keep = x.clone()
    x.zero_()
    graph.replay()
    assert (z == 0).all()
    x.copy_(keep)
    graph.replay()
    assert torch.equal(z, want)


@pytest.mark.parametrize('size,d', [(64, 2048), (65, 2048), (32, 4096), (33, 4096), (127, 1024), (16, 8200), (3, 40000)])
def test_sums_at_the_border_of_what_is_exact(cuda, size, d):
    """Rows of one size against weights of -128 and 127: 128 times 2,048 times 64 is 2^24 to the bit.  Odd weights in between
    show a sum that lost its last bit."""
    import torch
    import paper_2606_00722_gb300 as epic
    rows, V = 40, 300
    g = torch.Generator().manual_seed(size)
    q = torch.full((1, rows, d), size, dtype=torch.int8)
    q[:, 1::3] *= -1
    q[:, 2::3] = torch.randint(-size, size + 1, (rows // 3, d), generator=g).to(torch.int8)
    w = torch.randint(-128, 128, (V, d), generator=g).to(torch.int8)
    w[::3] = -128
    w[1::3] = 127
    q, w = q.cuda(), w.cuda()
    z = torch.empty((1, rows, V), device=cuda)
    epic.int8_logits(q, torch.ones((1, rows), device=cuda), w, torch.ones(V, device=cuda), z)
    assert torch.equal(z, (q.double() @ w.double().t()).float())


def test_logits_do_not_depend_on_the_other_rows(cuda):
    """A row's logits have the same bits alone, among few rows and among many: whatever way they are made, sums are exact."""
    import torch
    import paper_2606_00722_gb300 as epic
    q, head, s, S = int8_case(1, 300, 1536, 700, 9)
    z = torch.empty((1, 300, 700), dtype=torch.bfloat16, device=cuda)
    epic.int8_logits(q, s, head, S, z)
    for n in (1, 2, 3, 7, 8, 9, 33, 100):
        part = torch.empty((1, n, 700), dtype=torch.bfloat16, device=cuda)
        epic.int8_logits(q[:, :n].contiguous(), s[:, :n].contiguous(), head, S, part)
        assert torch.equal(part, z[:, :n])


def test_far_apart_and_past_32_bits(cuda):
    """Rows of logits 2^31 elements apart; a head of 2.3e9 bytes, seen at its last tokens; workspaces of other contents."""
    import torch
    import paper_2606_00722_gb300 as epic
    q, head, s, S = int8_case(2, 6, 256, 500, 3)
    far = (1 << 31) + 64
    store = torch.zeros(far + 6 * 500, dtype=torch.bfloat16, device=cuda)
    z = store.as_strided((2, 6, 500), (far, 500, 1))
    epic.int8_logits(q, s, head, S, z)
    check_logits(z, q, head, s, S, 'bf16')
    del store, z
    d, V = 32768, 70000
    big = torch.zeros((V, d), dtype=torch.int8, device=cuda)
    big[-2:] = torch.randint(-128, 128, (2, d), generator=torch.Generator().manual_seed(1)).to(torch.int8).cuda()
    S = torch.ones(V, device=cuda)
    for rows in (1, 20):
        q = torch.randint(-128, 128, (1, rows, d), generator=torch.Generator().manual_seed(2)).to(torch.int8).cuda()
        z = torch.empty((1, rows, V), device=cuda)
        for fill in (0, 255):
            work = torch.full((rows * (d * 2 + 4 * 32) + 4096,), fill, dtype=torch.uint8, device=cuda)
            epic.int8_logits(q, torch.ones((1, rows), device=cuda), big, S, z, workspace=work)
            assert torch.equal(z[..., -2:], (q.double() @ big[-2:].double().t()).float()) and (z[..., :-2] == 0).all()
