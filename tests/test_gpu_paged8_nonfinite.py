"""A chunk over an 8-bit cache: a row that sees a score of NaN or +inf ends as O = 0 with LSE = -inf, through the single-token kernel (few tokens) as through the
tensor-core forward, and as mka_fwd_paged ends it on the same values; rows that do not see it are as they are without."""
import pytest
import torch

import paged8_ref as ref
from test_gpu_paged8 import Cache, args, gates, query

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mka():
    import paper_2603_20586_b200 as m
    return m


@pytest.mark.parametrize("value", ["nan", "inf"])
@pytest.mark.parametrize("B,n", [(2, 400), (60, 330), (1, 9000)])        # partials added up by a CTA and by a warp; over all SMs
@pytest.mark.parametrize("T", [1, 3, 6, 260])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_the_score(mka, d, T, B, n, value):
    H, Hkv = 8, 2
    c = Cache(51, B, Hkv, d, [n] * B, 16, 16, ref.E4M3)
    q, gate = query(2, B, H, T, d), gates(3, B, T, (0, 2)).cuda()
    q[..., 0] = 1                                                # (the score of the infinite key is then +inf)
    shape = mka.make_shape(B, H, T, d, window=1, q_offset=n - T)
    k, v, ek, ev, tab, most = args([None, c, None])
    run = lambda: mka.mka_fwd_paged8(shape, Hkv, q, k, v, ek, ev, tab, most, gate)                                    # noqa: E731
    O0, L0 = run()
    assert torch.isfinite(O0).all() and torch.isfinite(L0).all()
    at, b, h = n - 1 - T // 2, B - 1, 1                          # half of the tokens see it
    page, row = int(c.table[b, at // 16]), at % 16
    codes = c.k.view(torch.uint8)
    if value == "nan":
        codes[page, h, row, 5] = 0x7f
    else:                                                        # 448 x 2^48 x 2^127 / sqrt(d): past fp32
        codes[page, h, row] = 0
        codes[page, h, row, 0] = 0x7e
        c.ek[page, h] = 127 + 48
        codes[page, h, :row, :] = 0                              # (its block's other rows count for nothing then)
        codes[page, h, row + 1:, :] = 0
        q[b, h * 4:(h + 1) * 4, :, 0] = 2.0 ** 127
    O, L = run()
    sees = torch.arange(T, device="cuda") + n - T >= at
    mine = (O[b, h * 4:(h + 1) * 4], L[b, h * 4:(h + 1) * 4])
    assert (mine[0][:, sees] == 0).all() and torch.isneginf(mine[1][:, sees]).all()
    if value == "nan":
        assert torch.isfinite(mine[0][:, ~sees]).all() and torch.isfinite(mine[1][:, ~sees]).all()
        assert torch.equal(mine[0][:, ~sees], O0[b, h * 4:(h + 1) * 4][:, ~sees]) and torch.equal(mine[1][:, ~sees], L0[b, h * 4:(h + 1) * 4][:, ~sees])
    other = torch.ones(B, H, dtype=torch.bool, device="cuda")
    other[b, h * 4:(h + 1) * 4] = False
    assert torch.equal(O[other], O0[other]) and torch.equal(L[other], L0[other])
    # the same values as bf16 pools
    wide = lambda x, e: (x.float() * torch.exp2((e.float() - 127).clamp(-48, 48)).repeat_interleave(16, 2)[..., None]).to(torch.bfloat16)     # noqa: E731
    P, Lp = mka.mka_fwd_paged(shape, Hkv, q, [None, wide(c.k, c.ek), None], [None, wide(c.v, c.ev), None], tab, most, gate)
    assert torch.isneginf(Lp[b, h * 4:(h + 1) * 4][:, sees]).all() and (P[b, h * 4:(h + 1) * 4][:, sees] == 0).all()
    if value == "nan":                                           # (queries of 2^127: there a product before the scale passes fp32 with ordinary keys too)
        assert torch.equal(torch.isneginf(L), torch.isneginf(Lp))
