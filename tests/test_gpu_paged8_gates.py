"""Gates that are not above 0 (negative, NaN, -0) close a level, whichever way a chunk goes: the same bits as with 0."""
import pytest
import torch

import paged8_ref as ref
from test_gpu_paged8 import Cache, args, check, gates, query, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 4, 11, 400])
@pytest.mark.parametrize("d,code", [(64, ref.S8), (128, ref.E4M3)])
def test_gates_that_are_not_above_zero(d, code, T):
    import paper_2603_20586_b200 as mka
    B, H, Hkv, n = 2, 8, 2, 500
    levels = [Cache(70 + l, B, Hkv, d, [m] * B, 16, 16, code) for l, m in enumerate((n + T, n + T, 40))]
    q, gate = query(7, B, H, T, d), gates(8, B, T)
    gate[0, ::2, 1] = 0                                          # some tokens close a level,
    gate[1, :, 2] = 0                                            # a sequence one for all of its tokens,
    gate[1, T // 2] = 0                                          # a token all three
    k, v, ek, ev, tab, most = args(levels)
    shape = mka.make_shape(B, H, T, d, window=90, q_offset=n)
    call = lambda g: mka.mka_fwd_paged8(shape, Hkv, q, k, v, ek, ev, tab, most, g.cuda())                            # noqa: E731
    O, LSE = call(gate)
    check(O, LSE, reference(q, levels, gate, window=90, q_offset=n), d, 2 * (n + T) + 40, 2.0 ** -8)
    for closed in (-1e-9, float("nan"), -0.0, float("-inf"), -3.0):
        other = torch.where(gate == 0, torch.full_like(gate, closed), gate)
        a, b = call(other)
        assert torch.equal(a, O) and torch.equal(b, LSE), closed
        if T == 1:
            one = mka.make_shape(B, H, 1, d)
            want = mka.mka_decode_paged8(one, Hkv, q[:, :, 0].contiguous(), k, v, ek, ev, tab, most, gate[:, 0].contiguous().cuda())
            got = mka.mka_decode_paged8(one, Hkv, q[:, :, 0].contiguous(), k, v, ek, ev, tab, most, other[:, 0].contiguous().cuda())
            assert all(torch.equal(x, y) for x, y in zip(got, want)), closed
