"""Pools and levels of a type that an entry point would read as another one (8-bit pools as bf16: twice their bytes) are refused (no GPU)."""
import pytest
import torch

import paper_2603_20586_b200 as mka
from paper_2603_20586_b200 import binding as b

EIGHT = [torch.int8, torch.uint8, torch.float8_e4m3fn]


def _zeros(dtype, *shape):
    return torch.zeros(*shape, dtype=torch.uint8).view(dtype) if dtype in EIGHT else torch.zeros(*shape, dtype=dtype)


TABLE = torch.zeros(3, 4, dtype=torch.int32)


@pytest.mark.parametrize("dtype", EIGHT + [torch.float16, torch.float32, torch.int16])
def test_paged_levels_are_bf16(dtype):
    good, bad = _zeros(torch.bfloat16, 9, 2, 16, 64), _zeros(dtype, 9, 2, 16, 64)
    b._paged_levels([good, None, None], [good, None, None], [TABLE, None, None], None, [60, 0, 0])
    for k, v in ((bad, bad), (good, bad), (bad, good)):
        with pytest.raises(AssertionError):
            b._paged_levels([k, None, None], [v, None, None], [TABLE, None, None], None, [60, 0, 0])
    b._paged_levels([bad, None, None], [bad, None, None], [TABLE, None, None], None, [0, 0, 0])          # (no rows: not looked at)
    q, gate = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 3)
    with pytest.raises(AssertionError):
        mka.mka_decode_paged(mka.make_shape(3, 4, 1, 64), 2, q, [bad] * 3, [bad] * 3, [TABLE] * 3, (60, 60, 60), gate, ws=gate)
    with pytest.raises(AssertionError):
        mka.mka_fwd_paged(mka.make_shape(3, 4, 1, 64), 2, q[:, :, None], [bad] * 3, [bad] * 3, [TABLE] * 3, (60, 60, 60), gate[:, None], ws=gate)


@pytest.mark.parametrize("dtype", EIGHT + [torch.float16])
def test_levels_and_gradients_are_bf16_or_f32(dtype):
    bad = _zeros(dtype, 2, 3, 40, 64)
    for good in (_zeros(torch.bfloat16, 2, 3, 40, 64), _zeros(torch.float32, 2, 3, 40, 64)):
        for k, v in ((bad, bad), (good, bad), (bad, good)):
            with pytest.raises(AssertionError):
                b._levels([None, k, None], [None, v, None])
            with pytest.raises(AssertionError):
                b._host_args.grads([good, None, None], [k, None, None], [v, None, None])
        other = good.to(torch.float32 if good.dtype == torch.bfloat16 else torch.bfloat16)
        for k, v in (([good, other, None], [good, other, None]), ([good, None, None], [other, None, None])):
            with pytest.raises(AssertionError):
                b._levels(k, v)
        b._levels([good, None, good], [good, None, good])
        with pytest.raises(AssertionError):
            b._host_args.grads([good, None, None], [other, None, None], [other, None, None])


@pytest.mark.parametrize("dtype", EIGHT + [torch.float16])
def test_fused_rows_go_into_pools_of_their_own_type(dtype):
    x, gate = _zeros(torch.bfloat16, 3, 2, 5, 64), torch.zeros(3, 5, 3)
    good, bad = _zeros(torch.bfloat16, 9, 2, 16, 64), _zeros(dtype, 9, 2, 16, 64)
    for k, v in ((bad, bad), (good, bad), (bad, good)):
        with pytest.raises(AssertionError):
            mka.mka_fuse_kv_paged([x, None, None], [x, None, None], gate, k, v, TABLE)


@pytest.mark.parametrize("dtype", EIGHT + [torch.float16, torch.float32])
def test_the_recall_index_is_of_bf16_keys(dtype):
    with pytest.raises(AssertionError):
        mka.mka_l3_index(_zeros(dtype, 9, 2, 16, 64), torch.zeros(64, 64))
