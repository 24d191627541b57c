"""Page operations on two streams at once, and compaction of tables with entries that name pages not in use."""
import random

import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests import pages_model as model
from tests.test_pages_gpu import State, bits_of, config, i32

pytestmark = pytest.mark.gpu
HOLD = 4_000_000                 # clocks for which a stream is held: about 2 ms, longer than the host takes for the calls of a round


def test_calls_queued_on_two_streams_run_together():
    """Both streams are held until all calls are queued, so that they run side by side. Each has a workspace of its own."""
    cfg = config(hq=4, hkv=2, hd=64, page=16, layers=1)
    lib = binding.DFlash(cfg)
    rows, width, pages = 96, 160, 9000
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    states, alone, lists = [], [], []
    for k in range(2):
        r = random.Random(k)
        lens = [r.randint(1, 40 * 16) for _ in range(rows // 3)] + [0] * (rows - rows // 3)
        child = list(range(rows // 3, rows))
        parent = [r.randrange(rows // 3) for _ in child]
        keep = [r.randint(1, lens[p]) for p in parent]
        room = [n + r.randint(0, 60 * 16) for n in keep]
        lists.append(tuple(i32(v) for v in (parent, child, keep, room)))
        states.append([State(cfg, pages, rows, width, lens, seed=60 + k) for _ in range(3)])
        alone.append(State(cfg, pages, rows, width, lens, seed=60 + k))

    def work(s, l, stream):
        parent, child, keep, room = l
        lib.dflash_pages_fork(parent, child, keep, s.d_table, s.d_ref, s.d_pool, stream=stream)
        lib.dflash_pages_resize(child, keep, room, s.d_table, s.d_ref, s.d_pool, stream=stream)
        lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool, stream=stream)

    for s, l in zip(alone, lists):
        work(s, l, None)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    for s in streams:                                        # the workspaces exist before the streams are held
        lib.dflash_pages_compact(alone[0].d_table.clone(), alone[0].d_ref.clone(), alone[0].d_pool.clone(), stream=s)
        s.synchronize()
    for k in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                torch.cuda._sleep(HOLD)
        for st, l, s in zip(states, lists, streams):
            work(st[k], l, s)
        torch.cuda.synchronize()
        for st, one in zip(states, alone):
            assert torch.equal(st[k].d_table, one.d_table) and torch.equal(st[k].d_ref, one.d_ref)
            np.testing.assert_array_equal(bits_of(st[k].d_pool), bits_of(one.d_pool))
    assert int(lib.status.item()) == 0
    held = [lib._scratches["pages", s.cuda_stream] for s in streams]
    (a, n), (b, m) = [(address, size) for _, address, size in held]
    assert a + n <= b or b + m <= a


@pytest.mark.parametrize("seed", range(6))
def test_compact_flags_every_entry_whose_page_is_not_in_use(seed):
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=2, dtype="fp32")
    lib = binding.DFlash(cfg)
    r = random.Random(seed)
    pages = r.choice([7, 60, 5000])
    rows, width = 6, pages // 3 + 2
    s = State(cfg, pages, rows, width, [r.randint(0, pages // 8) for _ in range(rows)], seed=seed)
    live = int((s.ref > 0).sum())
    free = np.flatnonzero(s.ref == 0)
    below, behind = free[free < live], free[free >= live]
    named = [int(x[r.randrange(len(x))]) for x in (below, behind) for _ in range(r.randint(0, 3)) if len(x)] + r.choice([[], [pages], [2 ** 31 - 1]])
    s.ref[free[::2]] = -3
    for i, page in enumerate(named):
        s.table[i % rows, width - 1 - i // rows] = page
    s.d_table.copy_(torch.from_numpy(s.table))
    s.d_ref.copy_(torch.from_numpy(s.ref))
    lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool)
    model.compact(s.table, s.ref, s.pool)                    # leaves such entries alone, and tells of those behind the border
    s.same(lib, binding.DEV_BAD_PAGE if named else 0)
