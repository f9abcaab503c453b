"""Compaction of a pool without pages: tables that hold entries all the same (none of them a page) come out as they were."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("planes", [0, 2])
def test_tables_of_an_empty_pool(planes):
    import paper_2603_20586_b200 as mka
    refs, rows, live = i32([]), i32([40, 0, 16]), i32([7])
    table, out = i32([[3, -1, 9, 5], [1, 2, 3, 4], [0, 8, 8, 8]]), i32([[70] * 4] * 3)
    pools = [torch.empty(0, 2, 16, dtype=torch.uint8, device="cuda")] * planes
    mka.mka_pages_compact(pools, refs, table, rows, 16, table_out=out, live=live)
    assert int(live) == 0
    # the entries in use (three, none, one); those behind a sequence's last page are left as they were
    assert out.tolist() == [[3, -1, 9, 70], [70] * 4, [0, 70, 70, 70]]
    mka.mka_pages_compact(pools, refs, table, rows, 16)
    assert table.tolist() == [[3, -1, 9, 5], [1, 2, 3, 4], [0, 8, 8, 8]]
    none = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    mka.mka_pages_compact(pools, refs, none, i32([]), 16, live=live.fill_(7))
    assert int(live) == 0
