"""Groups of 9 to 16 query heads over an 8-bit cache (two products of eight heads to a KV head), at both widths, both codes and every layout; and few tokens of them."""
import pytest

import paged8_ref as ref
from test_gpu_paged8 import _chunk, _levels, check, decode, gates, query, reference

pytestmark = pytest.mark.gpu

GROUPS = [
    # B, H, H_kv, rows of the three levels (per sequence), page, block
    (2, 16, 1, [[70, 5], [300, 1500], [129, 0]], 16, 16),
    (3, 18, 2, [[64, 65, 1], [15, 700, 259], None], 32, 16),                              # nine
    (1, 60, 5, [None, [4099], [33]], 64, 32),                                             # twelve
    (40, 26, 2, [[(7 * b) % 90 for b in range(40)], [(131 * b) % 700 for b in range(40)], [b % 3 for b in range(40)]], 16, 16),       # thirteen, more sequences than lanes
    (90, 32, 2, [None, [(53 * b) % 330 for b in range(90)], [b % 2 for b in range(90)]], 128, 128),       # many lists of few partials
    (2, 64, 4, [[1, 16], [9000, 3], [500, 17]], 256, 256),
]


@pytest.mark.parametrize("layout", ["page", "row", "padded"])
@pytest.mark.parametrize("code", [ref.E4M3, ref.S8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", GROUPS, ids=lambda c: f"B{c[0]}_{c[1]}on{c[2]}_p{c[4]}_b{c[5]}")
def test_wide_groups(case, d, code, layout):
    import paper_2603_20586_b200 as mka
    B, H, Hkv, rows, page, block = case
    levels = _levels((B, H, Hkv, d, rows, page, block, code), layout=layout, per_head=layout == "padded")
    q, gate = query(5, B, H, d), gates(6, B, 1)
    O, LSE = decode(mka, q, levels, gate.cuda())
    check(O, LSE, reference(q[:, :, None], levels, gate), d, sum(x.n for x in levels if x), 2.0 ** -11)


@pytest.mark.parametrize("layout", ["page", "row", "padded"])
@pytest.mark.parametrize("code", [ref.E4M3, ref.S8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,T", [(28, 4, 4), (28, 4, 16), (8, 1, 33), (16, 16, 7), (16, 16, 24), (18, 2, 3), (16, 1, 1), (16, 16, 100), (28, 4, 73)])
def test_few_tokens_of_every_group(H, Hkv, T, d, code, layout):
    """Sizes on both sides of where a chunk goes through the forward instead."""
    import paper_2603_20586_b200 as mka
    _chunk(mka, (2, H, Hkv, d, T, 400, 130, (400 + T, 400 + T, 50), 32, 16, code), layout=layout)


@pytest.mark.parametrize("code", [ref.E4M3, ref.S8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,spare", [(16, 3), (64, 0)])
def test_pools_with_the_heads_outermost(d, code, page, spare):
    """[heads, pages, rows, d] in memory, exponents too; and pools of a single page."""
    import torch

    import paper_2603_20586_b200 as mka
    from test_gpu_paged8 import Cache, args, bytes_of
    B, H, Hkv, T, n = (2, 16, 2, 5, 150) if spare else (1, 6, 3, 5, 60)
    c = Cache(17, B, Hkv, d, [n] * B, page, 16, code, spare=spare)
    assert spare or c.k.shape[0] == 1
    plain = args([None, c, None])
    turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)                                                 # noqa: E731
    k, v, ek, ev = ([None, turned(x[1].view(torch.uint8)).view(x[1].dtype), None] for x in plain[:4])
    tab, most = plain[4:]
    q, gate = query(5, B, H, d), gates(6, B, 1, (0, 2)).cuda()
    O, LSE = mka.mka_decode_paged8(mka.make_shape(B, H, 1, d), Hkv, q, k, v, ek, ev, tab, most, gate)
    check(O, LSE, reference(q[:, :, None], [None, c, None], gate.cpu()), d, n, 2.0 ** -11)
    for t in (T, 90):
        Q, gateT = query(7, B, H, t, d), gates(8, B, t, (0, 2))
        shape = mka.make_shape(B, H, t, d, window=1, q_offset=max(0, n - t))
        O, LSE = mka.mka_fwd_paged8(shape, Hkv, Q, k, v, ek, ev, tab, most, gateT.cuda())
        check(O, LSE, reference(Q, [None, c, None], gateT, window=1, q_offset=max(0, n - t)), d, n, 2.0 ** -8)
    new = [query(20 + i, B, Hkv, 9, d) for i in range(2)]
    at = torch.tensor([n - 9] * B, dtype=torch.int32).cuda()
    mka.mka_append_kv_paged8(*new, k[1], v[1], ek[1], ev[1], tab[1], dst_offsets=at)
    mka.mka_append_kv_paged8(*new, c.k, c.v, c.ek, c.ev, c.tab, dst_offsets=at)
    for a, b in zip((k[1], v[1], ek[1], ev[1]), (c.k, c.v, c.ek, c.ev)):
        assert (bytes_of(a) == bytes_of(b)).all()
