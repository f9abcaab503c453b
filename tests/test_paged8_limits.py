"""Sizes whose tiles the decode over an 8-bit cache cannot number in 32 bits are refused (host checks: nothing is launched)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def mka():
    from paper_2603_20586_b200 import build
    build.build()
    import paper_2603_20586_b200 as m
    return m


def _level(mka, n, d, page=512):
    return mka.binding.mka_paged_level8(k=256, v=512, k_exp=8, v_exp=16, page_table=4, rows=None, n=n, table_stride=-(-n // page), table_head_stride=0,
                                        stride_page=page * 64 * d, stride_h=page * d, stride_n=d, exp_stride_page=128, exp_stride_h=2, pool_pages=9, page_rows=page,
                                        block_rows=256, code=0, reserved=0)


@pytest.mark.parametrize("d,B,H_kv,n", [
    (128, 65535, 8, (1 << 20) + 32),           # one list's tiles of all sequences: a prefix of a million rows that all of them share
    (64, 65535, 1, (1 << 21) + 64),
    (128, 1, 64, (1 << 31) - 1),        # all lists of a sequence
    (64, 2, 65535, (1 << 21) + 64),
    (128, 60000, 60000, 1 << 15),       # a share of a CTA
])
def test_tiles_past_32_bits_are_refused(mka, d, B, H_kv, n):
    L = (mka.binding.mka_paged_level8 * 3)()
    L[1] = _level(mka, n, d)
    shape = mka.make_shape(B, H_kv, 1, d)
    assert mka.lib.mka_decode_paged8(ctypes.byref(shape), H_kv, 16, L, 16, 16, None, 256, 1 << 62, None) == 2
