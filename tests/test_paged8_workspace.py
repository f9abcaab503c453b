"""The chunk's workspace over an 8-bit cache: the size for an upper bound serves every smaller call (host function, no GPU)."""
import random

import pytest


@pytest.fixture(scope="module")
def size():
    from paper_2603_20586_b200 import build
    build.build()
    import paper_2603_20586_b200 as mka

    def size(B, H, Hkv, d, T, at, W, n):
        return mka.mka_fwd_paged8_workspace_bytes(mka.make_shape(B, H, T, d, window=W, q_offset=at), Hkv, n)
    return size


@pytest.mark.parametrize("H,Hkv,d,T,longer,shorter", [
    (32, 8, 64, 200, 1050, 1000), (28, 4, 64, 1000, 1800, 1700), (8, 1, 128, 64, 300, 150), (8, 1, 128, 64, 200, 150)])
def test_a_shorter_context_needs_no_more(size, H, Hkv, d, T, longer, shorter):
    """The forward's form, or the way of the chunk, changes between the two."""
    a, b = (size(1, H, Hkv, d, T, at, 4096, (at + T, at + T, 0)) for at in (longer, shorter))
    assert 0 < b <= a


HEADS = [(28, 4), (32, 8), (12, 4), (16, 16), (8, 1), (64, 4), (4, 4), (18, 2), (128, 128)]


@pytest.mark.parametrize("seed", range(8))
def test_smaller_calls_need_no_more(size, seed):
    rng = random.Random(seed)
    log = lambda lo, hi: int(lo * (hi / lo) ** rng.random())                       # noqa: E731
    for _ in range(400):
        H, Hkv = rng.choice(HEADS)
        d, B, T, at, W = rng.choice([64, 128]), log(1, 64), log(1, 3000), log(1, 100000) - 1, log(1, 8192)
        n = [rng.choice([0, at + T, log(1, 100000)]) for _ in range(2)] + [rng.choice([0, log(1, 8192)])]
        most = size(B, H, Hkv, d, T, at, W, n)
        assert most > 0
        for _ in range(25):
            part = lambda x, lo: rng.choice([x, max(lo, x - rng.randint(0, 200)), rng.randint(lo, max(lo, x))])      # noqa: E731
            less = (part(B, 1), H, Hkv, d, part(T, 1), part(at, 0), part(W, 1), [part(x, 0) for x in n])
            assert size(*less) <= most, ((B, H, Hkv, d, T, at, W, n), less)


def test_few_tokens_take_little(size):
    """Partial results only, not the cache's rows: four tokens at 100,000 rows of eight KV heads of 128 would take 820 MB."""
    assert size(1, 32, 8, 128, 4, 100000, 4096, (100004, 100004, 0)) < 16 << 20
