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
