"""Shared-prefix attention of groups whose sequences have not got as far as their prefix: nothing of the prefix is looked at."""
import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests.test_prefix_attention_gpu import Batch, config

pytestmark = pytest.mark.gpu


def unshared(cfg, rows, lens, seed):
    """A batch of sequences with pages of their own: table entries behind a sequence's length name a page that does not exist."""
    x = Batch(cfg, rows, [0], [], lens, seed=seed)
    return x, x.cuda()


def run(lib, x, d, starts, prefix, mode=1):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")
    out, lse = torch.full_like(d["q"], float("nan")), torch.full(d["q"].shape[:3], float("nan"), device="cuda:0")
    lib.dflash_prefix_attention(mode, d["q"], d["k"], d["v"], i32(starts), i32(prefix), d["lens"], max(x.lens + prefix), d["table"], d["pool"], x.layer, out,
                                lse_out=lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("shape", [{}, dict(hq=6, hkv=2, hd=64, page=16), dict(hq=4, hkv=2, hd=64, dtype="fp32")], ids=["hd128", "hd64", "fp32"])
def test_a_group_that_has_not_reached_its_prefix_reads_nothing_of_it(shape):
    cfg = config(**shape)
    lib = binding.DFlash(cfg)
    for starts, prefix in (([0, 4], [1000]), ([0, 1, 4], [301, 1000]), ([1, 3], [2000]), ([0, 0, 4, 4], [50, 302, 300])):
        x, d = unshared(cfg, 5, [300, 10, 0, 260], seed=3)
        out, lse = run(lib, x, d, starts, prefix)
        assert int(lib.status.item()) == 0
        x.check(out, lse, True)


def test_groups_that_reach_their_prefix_beside_groups_that_do_not():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 9, [2, 5], [131], [200, 90, 100, 131, 400, 150], seed=5)      # the group's first sequence is shorter than its prefix
    d = x.cuda()
    out, lse = run(lib, x, d, [0, 2, 5, 6], [900, 131, 151])
    assert int(lib.status.item()) == 0
    x.check(out, lse, True)


def test_many_groups_that_do_not_reach_their_prefix():
    cfg = config(hq=4, hkv=2, hd=64, page=16, layers=1)                          # more entries than the plan keeps in shared memory
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 2, [0], [], [(7 * b) % 90 for b in range(700)], seed=6, layer=0)
    d = x.cuda()
    out, lse = run(lib, x, d, list(range(0, 701, 2)), [91 + g % 300 for g in range(350)])
    assert int(lib.status.item()) == 0
    x.check(out, lse, True, seqs=range(0, 700, 23))


def test_a_replayed_call_with_shorter_lengths():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 5, [0, 3], [300], [300, 400, 500], seed=7)
    d = x.cuda()
    x.run(lib, 1, d)
    torch.cuda.synchronize()
    out, lse = torch.zeros_like(d["q"]), torch.zeros(d["q"].shape[:3], device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.run(lib, 1, d, out, lse)
    graph.replay()
    torch.cuda.synchronize()
    x.check(out, lse, True)
    y = Batch(cfg, 5, [0], [], [130, 10, 120], seed=8)                           # the same buffers, other sequences
    y.q, y.k, y.v = x.q, x.k, x.v
    table = np.full(x.table.shape, 10 ** 6, dtype=np.int32)
    table[:, :y.table.shape[1]] = y.table[:, :x.table.shape[1]]
    y.table = table
    assert y.pages <= x.pages
    pool = torch.full_like(x.pool, float("nan"))
    pool[:, :y.pages] = y.pool
    y.pool = pool
    d["table"].copy_(torch.from_numpy(table))
    d["pool"].copy_(pool)
    d["lens"].copy_(torch.tensor(y.lens, dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    y.check(out, lse, True)
