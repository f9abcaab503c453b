"""Large differences of scores beside value exponents at both limits, 2^96 apart: what a weight loses stays within the stated bound.

A weight times its block's scale is off by 2^-11 of itself and by 2^-29 of the row's largest such product; a code is 448 at most.  So a column is off by
n 2^-29 448 of that product over the sum of the weights, beside what test_gpu_paged8 counts with (sums, scores, the weights' rounding, the output's).
"""
import numpy as np
import pytest
import torch

import paged8_ref as ref
from gpu_helpers import np64
from test_gpu_paged8 import Cache, bytes_of, query, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [[-56.0, -72.0, -80.0, -88.0, -96.0], [-88.0, -96.0]], ids=["far_blocks_decide", "far_weights_below_2^-126"])
@pytest.mark.parametrize("T", [1, 3])
@pytest.mark.parametrize("n", [640, 9000])                       # in a few warps; over all SMs, so that whole states lie far below others
@pytest.mark.parametrize("code", [ref.E4M3, ref.S8])
@pytest.mark.parametrize("d", [64, 128])
def test_far_weights_in_far_blocks(d, code, n, T, steps):
    import paper_2603_20586_b200 as mka
    B, H, Hkv = 1, 4, 1
    c = Cache(21, B, Hkv, d, [n], 16, 16, code)
    g = torch.Generator().manual_seed(d + n)
    # keys: one column counts, score = code; the blocks with the largest scores have the smallest value scales
    value = ref.code_values(code)
    byte = [int(np.flatnonzero(value == x)[0]) for x in steps]
    zero = int(np.flatnonzero(value == 0)[0])
    keys = torch.full((c.k.shape[0], Hkv, 16, d), zero, dtype=torch.uint8)
    ev = torch.full((c.k.shape[0], Hkv, 1), 127 - 48, dtype=torch.uint8)
    near = 3                                                     # its rows score 0
    for i in range(-(-n // 16)):
        if i == near:
            continue
        page = int(c.table[0, i])
        keys[page, 0, :, 0] = torch.tensor(byte, dtype=torch.uint8)[torch.randint(0, len(byte), (16,), generator=g)]
        ev[page] = 127 + 48
    c.k.view(torch.uint8).copy_(keys)
    c.ek.fill_(127)
    c.ev.copy_(ev)
    v = c.v.view(torch.uint8)
    v[int(c.table[0, near]), 0, :, :8] = zero                    # columns that only the far blocks have anything in
    c.vk, c.vv = (np.nan_to_num(ref.values(bytes_of(x), e.cpu().numpy(), code)) for x, e in ((c.k, c.ek), (c.v, c.ev)))
    q = torch.zeros(B, H, T, d, dtype=torch.bfloat16)
    q[..., 0] = 1
    q = q.cuda()
    gate = torch.tensor([[[0.0, 1.0, 0.0]] * T] * B)
    one = lambda x: [None, x, None]                              # noqa: E731
    shape = mka.make_shape(B, H, T, d, window=1, q_offset=n - T, scale=1.0)
    call = mka.mka_decode_paged8 if T == 1 else mka.mka_fwd_paged8
    x = q[:, :, 0].contiguous() if T == 1 else q
    O, LSE = call(shape, Hkv, x, one(c.k), one(c.v), one(c.ek), one(c.ev), one(c.tab), (0, n, 0), (gate[:, 0].contiguous() if T == 1 else gate).cuda())
    Or, Lr, A, S = reference(q, one(c), gate, scale=1.0, **({} if T == 1 else dict(window=1, q_offset=n - T)))
    k0 = ref.rows_of(c.vk, c.table.numpy(), 0, 0, n)[:, 0]
    scale = np.exp2(ref.byte_exponent(np.repeat(ev.numpy()[c.table[0].numpy(), 0, 0], 16)[:n]).astype(float))
    w = np.exp(k0)
    largest = (w * scale).max() / w[:n - T + 1].sum()            # (the first token's sum is the smallest)
    E, K = (d + 8) * 2.0 ** -23 * S + 2.0 ** -21, (n / 64 + 400) * 2.0 ** -22
    O, LSE = np64(O).reshape(Or.shape), np64(LSE).reshape(Lr.shape)
    tol = 2.0 ** -8 * np.abs(Or) + A * (2 * E[..., None] + 2 * K + 2.0 ** -11) + n * 2.0 ** -29 * 448 * largest
    over = np.abs(O - Or) / tol
    assert over.max() <= 1, f"O at {over.max():.3g} of its bound"
    assert (np.abs(LSE - Lr) <= E + K + 2.0 ** -22 * np.abs(Lr)).all()
    assert (np.abs(Or[..., :8]) > 0).all()
