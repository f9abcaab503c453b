"""Page tables whose sequences ask for more pages together than 32 bits hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("seqs", [7, 70])
def test_demands_past_32_bits(copies, seqs):
    """Four sequences ask for 2^29 pages each of a pool of 100: those in front are served, nobody behind is, whatever the sum wraps to."""
    import paper_2603_20586_b200 as mka
    W, P = 1 << 29, 100
    if seqs == 70:
        W, want, behind = 1 << 25, [10] + [1 << 25] * 64, [500, 5, 0, -1, 7]          # 64 of 2^25
    else:
        want, behind = [10] + [W] * 4, [500, 5]
    table = torch.empty(seqs, W, dtype=torch.int32, device="cuda")                   # 9 to 15 GB, of which a few entries are touched
    table[:, :200] = -1
    refs, rows, missing = i32([0] * P), i32([0] * seqs), i32([-1])
    planes = [torch.zeros(P, 64, dtype=torch.uint8, device="cuda")] if copies else []
    new = want + behind
    assert len(new) == seqs and sum(want) > 1 << 31
    mka.mka_pages_resize(planes, refs, table, rows, i32(new), 1, missing=missing)
    assert rows.tolist() == [10] + [0] * (seqs - 1)
    assert refs.tolist() == [1] * 10 + [0] * 90
    assert table[0, :12].tolist() == list(range(10)) + [-1] * 2 and (table[1:, :200] == -1).all()
    assert int(missing) == 2 ** 31 - 1                           # 2^31 + 10 + ... - 100, as far as an int32 goes
    # one page less than 2^31 is counted exactly; a sequence that needs none is served among those that wait
    new = [5] + want[1:] + [0] * len(behind)
    mka.mka_pages_resize(planes, refs, table, rows, i32(new), 1, missing=missing)
    assert rows.tolist() == [5] + [0] * (seqs - 1) and refs.tolist() == [1] * 5 + [0] * 95
    assert int(missing) == 2 ** 31 - 95
