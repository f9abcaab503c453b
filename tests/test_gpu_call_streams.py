"""Calls on a stream of their own, beside torch's current one: what a call allocates (outputs that the caller drops, workspaces) is not handed out again before
that stream is done with it."""
import ctypes

import pytest
import torch

from test_gpu_paged8 import Cache, args, gates, query

pytestmark = pytest.mark.gpu
B, H, HKV, D, N, T = 2, 8, 2, 64, 300, 5


@pytest.fixture(scope="module")
def mka():
    import paper_2603_20586_b200 as m
    return m


def bf16(*shape):
    return torch.randn(*shape, device="cuda").to(torch.bfloat16)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls(mka):
    """Name -> (call of a stream)."""
    levels = [Cache(20 + l, B, HKV, D, [N] * B) for l in range(3)]
    k, v, ek, ev, tab, n = args(levels)
    q, Q, gate, gateT = query(1, B, H, D), query(2, B, H, T, D), gates(3, B, 1).cuda(), gates(4, B, T).cuda()
    one, few, many = mka.make_shape(B, H, 1, D), mka.make_shape(B, H, T, D, window=50, q_offset=N - T), mka.make_shape(B, H, 200, D, window=50, q_offset=N - 200)
    gate1, bank_len = gate[:, 0].contiguous(), i32([3, 2])
    Qm, gatem = query(5, B, H, 200, D), gates(6, B, 200).cuda()
    pool_k, pool_v = [bf16(60, HKV, 16, D) for _ in range(3)], [bf16(60, HKV, 16, D) for _ in range(3)]
    K, V = [bf16(B, H, N, D) for _ in range(3)], [bf16(B, H, N, D) for _ in range(3)]
    Kt, Vt = [bf16(B, H, T, D) for _ in range(3)], [bf16(B, H, T, D) for _ in range(3)]
    R, Wr, X = bf16(B, T, 64), torch.randn(64, 3, device="cuda"), bf16(B, 64, 64)
    proj, bank = torch.randn(64, D, device="cuda"), i32([[3, 1, 2]] * B)
    codes = mka.mka_l3_index(pool_k[0], proj)
    O, LSE = mka.mka_fwd(few, Q, K, V, gateT)
    refs, table, rows = i32([1, 0, 1, 1, 0, 0]), i32([[0, 3], [2, 5]]), i32([20, 3])
    new = i32([30, 3])
    return {
        "router": lambda s: mka.mka_router(R, Wr, None, stream=s),
        "fwd": lambda s: mka.mka_fwd(few, Q, K, V, gateT, stream=s),
        "decode": lambda s: mka.mka_decode(one, q, K, V, gate1, stream=s),
        "bwd": lambda s: list(mka.mka_bwd(few, Q, K, V, gateT, O, LSE, Q, stream=s).values()),
        "fuse": lambda s: mka.mka_fuse_kv(Kt, Vt, gateT, stream=s),
        "summary": lambda s: mka.mka_l2_summary(X, stream=s),
        "index": lambda s: mka.mka_l3_index(pool_k[0], proj, stream=s),
        "retrieve": lambda s: mka.mka_l3_retrieve(q, HKV, proj, codes, bank, bank_len, 2, 16, stream=s),
        "fwd_paged": lambda s: mka.mka_fwd_paged(few, HKV, Q, pool_k, pool_v, tab, n, gateT, stream=s),
        "decode_paged": lambda s: mka.mka_decode_paged(one, HKV, q, pool_k, pool_v, tab, n, gate1, stream=s),
        "decode_paged8": lambda s: mka.mka_decode_paged8(one, HKV, q, k, v, ek, ev, tab, n, gate, stream=s),
        "fwd_paged8_few": lambda s: mka.mka_fwd_paged8(few, HKV, Q, k, v, ek, ev, tab, n, gateT, stream=s),
        "fwd_paged8": lambda s: mka.mka_fwd_paged8(many, HKV, Qm, k, v, ek, ev, tab, n, gatem, stream=s),
        "resize": lambda s: mka.mka_pages_resize([], refs, table, rows, new, 16, stream=s),
        "compact": lambda s: mka.mka_pages_compact([], refs, table, rows, 16, stream=s),
    }


NAMES = ["router", "fwd", "decode", "bwd", "fuse", "summary", "index", "retrieve", "fwd_paged", "decode_paged", "decode_paged8", "fwd_paged8_few", "fwd_paged8", "resize", "compact"]


@pytest.mark.parametrize("name", NAMES)
def test_dropped_memory_is_not_handed_out_early(mka, name):
    call = calls(mka)[name]
    stream = torch.cuda.Stream()
    call(stream)
    fill = lambda ts: (torch._foreach_zero_(ts), torch._foreach_add_(ts, 0x5a))                                        # noqa: E731
    fill([torch.empty(512, dtype=torch.uint8, device="cuda") for _ in range(300)])         # (loads what is needed below: that waits for the GPU)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(2_000_000_000)                         # the call's kernels come a second later
    call(stream)                                                 # (its outputs are dropped)
    assert not stream.query()
    # what the allocator has to give on the current stream, piece by piece, until it asks for more
    taken, reserved = [], torch.cuda.memory_reserved()
    while torch.cuda.memory_reserved() == reserved and len(taken) < 50000:
        taken += [torch.empty(512, dtype=torch.uint8, device="cuda") for _ in range(512)]
    fill(taken)
    assert not stream.query()
    torch.cuda.synchronize()
    assert bool((torch.stack(taken) == 0x5a).all()), name


class Handle:
    """What has a cuda_stream is a stream: a number, or a c_void_p."""

    def __init__(self, value):
        self.cuda_stream = value


@pytest.mark.parametrize("wrap", [int, ctypes.c_void_p])
@pytest.mark.parametrize("name", ["decode", "fwd_paged", "decode_paged8", "fwd_paged8", "compact"])
def test_streams_of_other_kinds(mka, name, wrap):
    call = calls(mka)[name]
    want, stream = call(None), torch.cuda.Stream()
    torch.cuda.synchronize()
    if name == "compact":                                        # (nothing moves the second time)
        want = call(None)
        torch.cuda.synchronize()
    for s in (Handle(wrap(stream.cuda_stream)), Handle(wrap(torch.cuda.current_stream().cuda_stream))):
        got = call(s)
        torch.cuda.synchronize()
        pairs = zip(want, got) if isinstance(want, tuple) else [(want, got)]
        assert all(torch.equal(a, b) for a, b in pairs)
