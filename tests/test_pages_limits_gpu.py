"""Page operations at the ends of their ranges."""
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests.test_pages_gpu import DEV, State, config, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,first", [(2051, 1), (2051, 0), (4100, 1)])
def test_requests_for_more_pages_than_32_bits_count_are_left_out(n, first):
    """Rows of 2^20 entries that all ask for 2^20 pages: the needs of 2048 of them add up to 2^31, of 4096 to 2^32. The first request is for one page, which
    it gets; with it the sums in front of the others are 1 or 0 past a multiple of 2^20."""
    width, pages = 1 << 20, 64
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=1, dtype="fp32")
    lib = binding.DFlash(cfg)
    s = State(cfg, pages, 1, 1, [1], seed=1)
    table = torch.full((n + 1, width), -1, dtype=torch.int32, device=DEV)
    table[n, 0] = int(s.table[0, 0])                         # a row that is not listed holds a page
    rows = torch.arange(n, dtype=torch.int32, device=DEV)
    keep, cap = torch.zeros_like(rows), torch.full_like(rows, width)
    if first:
        cap[0] = 1
    copies = tuple(torch.full((n,), -7, dtype=torch.int32, device=DEV) for _ in range(3))
    lib.dflash_pages_resize(rows, keep, cap, table, s.d_ref, s.d_pool, copies=copies)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == binding.DEV_POOL_FULL
    want = s.ref.copy()
    if first:
        free = int((s.ref == 0).argmax())                    # the lowest free page
        assert int(table[0, 0]) == free
        want[free] = 1
        table[0, 0] = -1
    assert s.d_ref.tolist() == want.tolist()
    assert int(table[n, 0]) == int(s.table[0, 0])
    table[n, 0] = -1
    assert int(table.max()) == int(table.min()) == -1
    assert all(int(c.max()) <= 0 for c in copies) and int(copies[1].max()) == -1
    assert torch.equal(s.d_pool.cpu().view(torch.int32), torch.from_numpy(s.pool))


@pytest.mark.parametrize("used", [0, 1])
def test_compacting_a_pool_of_one_page_reports_its_moves_too(used):
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=1, dtype="fp32")
    lib = binding.DFlash(cfg)
    s = State(cfg, 1, 1, 2, [used])
    n_live, none = i32([-1]), torch.zeros(0, dtype=torch.int32, device=DEV)
    moved = i32([-7])
    lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool, n_live=n_live, copies=(none, none.clone(), moved))
    s.same(lib, 0)
    assert int(n_live) == used and int(moved) == 0
