"""Calls over an 8-bit cache in a workspace that was sized for larger ones, and in one without room for the forward's scratch."""
import pytest
import torch

import paged8_ref as ref
from test_gpu_paged8 import Cache, args, check, gates, query, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,d,most_T,most_n,W,sizes", [
    (32, 8, 64, 200, 1250, 4096, [(200, 1000), (200, 1050), (130, 400), (16, 1234), (3, 900), (1, 0), (200, 0)]),
    (8, 1, 128, 64, 364, 300, [(64, 150), (64, 300), (64, 200), (17, 127), (2, 200), (64, 0)]),
    (16, 16, 128, 100, 900, 64, [(100, 800), (33, 100), (32, 128), (31, 129), (7, 777)]),
])
def test_one_workspace_for_all_chunks(H, Hkv, d, most_T, most_n, W, sizes):
    """What lies behind the workspace stays as it is, and the results are those of a workspace of the call's own."""
    import paper_2603_20586_b200 as mka
    B, n3 = 2, 40
    levels = [Cache(30 + l, B, Hkv, d, [m] * B, 32, 16, ref.E4M3) for l, m in enumerate((most_n, most_n, n3))]
    k, v, ek, ev, tab, _ = args(levels)
    size = mka.mka_fwd_paged8_workspace_bytes(mka.make_shape(B, H, most_T, d, window=W, q_offset=most_n - most_T), Hkv, (most_n, most_n, n3))
    room = torch.full((size + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    for T, at in sizes:
        n = (at + T, at + T, n3)
        shape = mka.make_shape(B, H, T, d, window=W, q_offset=at)
        q, gate = query(T, B, H, T, d), gates(at, B, T)
        call = lambda ws: mka.mka_fwd_paged8(shape, Hkv, q, k, v, ek, ev, tab, n, gate.cuda(), ws=ws)                 # noqa: E731
        O, LSE = call(room[:size])
        assert (room[size:] == 0xa5).all()
        a, b = call(None)
        assert torch.equal(O, a) and torch.equal(LSE, b), (T, at)
        part = [0 if x is None else [m] * B for x, m in zip(levels, n)]
        check(O, LSE, reference(q, levels, gate, window=W, q_offset=at, rows=dict(enumerate(part))), d, sum(n), 2.0 ** -8, f"T {T} at {at}")


@pytest.mark.parametrize("d", [64, 128])
def test_without_room_for_the_forwards_scratch(d):
    """Header, tables and expanded rows are enough; one byte less is refused."""
    import paper_2603_20586_b200 as mka
    B, H, Hkv, T, n = 1, 28, 4, 300, 4000
    c = Cache(33, B, Hkv, d, [n], 16, 16, ref.S8)
    k, v, ek, ev, tab, most = args([None, c, None])
    q, gate = query(3, B, H, T, d), gates(4, B, T, (0, 2))
    pages = -(-n // 128)
    need = 256 + -(-pages * 4 // 256) * 256 + pages * 128 * Hkv * 4 * d
    room = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    shape = mka.make_shape(B, H, T, d, window=1, q_offset=n - T)
    call = lambda ws: mka.mka_fwd_paged8(shape, Hkv, q, k, v, ek, ev, tab, most, gate.cuda(), ws=ws)                  # noqa: E731
    O, LSE = call(room[:need])
    assert (room[need:] == 0xa5).all()
    check(O, LSE, reference(q, [None, c, None], gate, window=1, q_offset=n - T), d, n, 2.0 ** -8)
    with pytest.raises(mka.MkaError):
        call(room[:need - 1])
