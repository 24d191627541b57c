"""GPU parity of the page operations (copy, fork, resize, compact) with the host model, bit for bit: tables, counts, pool
contents and status bits, on sound states and on requests that have to be left out."""
import random

import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding, synth
from tests import pages_model as model
from tests.test_prefix_attention_gpu import config

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def pool_of(cfg, pages, seed=0):
    """Bit patterns of every kind, NaN among them, as integers of the element's size."""
    kind = torch.int16 if cfg.dtype == "bf16" else torch.int32
    g = torch.Generator().manual_seed(seed)
    bits = torch.randint(-2 ** 15, 2 ** 15, synth.kv_pool_shape(cfg, pages), generator=g, dtype=torch.int32).to(kind)
    return bits.numpy(), bits.to(DEV).view(cfg.torch_dtype)


def bits_of(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy()


class State:
    def __init__(self, cfg, pages, rows, width, lens, seed=0, shared=()):
        """Rows of the given lengths over scattered pages; (a, b, n): row b shares the first n pages of row a."""
        self.cfg, ps = cfg, cfg.page_size
        r = random.Random(seed)
        ids = list(range(pages))
        r.shuffle(ids)
        self.table = np.full((rows, width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(lens):
            have = -(-n // ps)
            self.table[b, :have] = ids[at:at + have]
            at += have
        for a, b, n in shared:
            self.table[b, :n] = self.table[a, :n]
        held = self.table[self.table >= 0]
        self.ref = np.bincount(held, minlength=pages).astype(np.int32)
        self.pool, self.d_pool = pool_of(cfg, pages, seed)
        self.d_table, self.d_ref = torch.from_numpy(self.table.copy()).to(DEV), torch.from_numpy(self.ref.copy()).to(DEV)

    def same(self, lib, status):
        torch.cuda.synchronize()
        np.testing.assert_array_equal(self.d_table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.d_ref.cpu().numpy(), self.ref)
        np.testing.assert_array_equal(bits_of(self.d_pool), self.pool)
        assert int(lib.status.item()) == status
        lib.status.zero_()


SHAPES = [dict(hq=4, hkv=2, hd=64, page=16, dtype="fp32"), dict(hq=8, hkv=2, hd=128, page=64), dict(hq=6, hkv=6, hd=64, page=8), dict(hq=4, hkv=4, hd=64, page=1, dtype="fp32")]


@pytest.mark.parametrize("shape", SHAPES)
def test_copy(shape):
    cfg = config(layers=3, **shape)
    lib = binding.DFlash(cfg)
    r = random.Random(7)
    pages, ps = 29, cfg.page_size
    for trial in range(8):
        bits, pool = pool_of(cfg, pages, trial)
        ids = list(range(pages))
        r.shuffle(ids)
        n = r.choice([1, 2, 5, 14])
        src, dst = ids[:n], ids[n:2 * n]
        slots = [r.choice([0, 1, ps - 1, ps, r.randint(0, ps), ps + 5, -2]) for _ in range(n)] if trial % 2 else None
        if trial >= 3:                          # twice the same destination, a source that is a destination, indices outside, nothing to do
            for _ in range(3):
                what, i = r.randint(0, 4), r.randrange(n)
                if what == 0: dst[i] = dst[r.randrange(n)]
                elif what == 1: src[i] = dst[r.randrange(n)]
                elif what == 2: dst[i] = r.choice([-1, pages, 2 ** 31 - 1])
                elif what == 3: src[i] = r.choice([-1, pages, 2 ** 31 - 1, -2 ** 31])
                else: src[i] = dst[i]
        count = r.choice([None, n, n - 1, 0, n + 5])
        status = model.copy(bits, src, dst, slots, count)
        lib.dflash_pages_copy(i32(src), i32(dst), pool, n_slots=None if slots is None else i32(slots), count=None if count is None else i32([count]))
        torch.cuda.synchronize()
        np.testing.assert_array_equal(bits_of(pool), bits)
        assert int(lib.status.item()) == status
        lib.status.zero_()


def test_copy_of_many_pages():
    cfg = config(hq=8, hkv=2, layers=2)
    lib = binding.DFlash(cfg)
    pages = 700
    bits, pool = pool_of(cfg, pages, 1)
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).tolist()
    src, dst = ids[:340], ids[340:680]
    assert model.copy(bits, src, dst) == 0
    lib.dflash_pages_copy(i32(src), i32(dst), pool)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(bits_of(pool), bits)


@pytest.mark.parametrize("shape", SHAPES)
def test_fork(shape):
    cfg = config(layers=2, **shape)
    lib = binding.DFlash(cfg)
    ps = cfg.page_size
    r = random.Random(3)
    for trial in range(10):
        lens = [5 * ps, 3 * ps + max(1, ps // 2), 0, 1, 7 * ps - 1, 2 * ps] + [0] * 8
        s = State(cfg, 40, 14, 8, lens, seed=trial, shared=[(0, 12, 3)] if trial % 2 else ())
        n = r.choice([1, 3, 8])
        parent = [r.choice([0, 1, 2, 3, 4, 5]) for _ in range(n)]
        child = r.sample(range(6, 12), 6)[:n] + [13] * max(0, n - 6)
        length = [r.choice([lens[p], r.randint(0, lens[p]), lens[p] // ps * ps, -1]) for p in parent]
        if trial >= 4:
            for _ in range(2):
                what, i = r.randint(0, 5), r.randrange(n)
                if what == 0: parent[i] = r.choice([-1, 14, child[0]])
                elif what == 1: child[i] = r.choice([-5, 14, 0, 12, child[0]])
                elif what == 2: length[i] = 8 * ps + 1
                elif what == 3: length[i] = 8 * ps          # more pages than the parent has
                elif what == 4: child[i] = parent[i]
                else: length[i] = 2 ** 31 - 1
        if trial == 9:                                  # next to no free page
            s.ref[np.flatnonzero(s.ref == 0)[2:]] = 1
            s.d_ref.copy_(torch.from_numpy(s.ref))
        copies = tuple(torch.full((n,), -7, dtype=torch.int32, device=DEV) for _ in range(3))
        lib.dflash_pages_fork(i32(parent), i32(child), i32(length), s.d_table, s.d_ref, s.d_pool, copies=copies)
        status, made = model.fork(s.table, s.ref, s.pool, parent, child, length)
        s.same(lib, status)
        assert list(zip(*(c.tolist() for c in copies))) == made


@pytest.mark.parametrize("shape", SHAPES)
def test_resize(shape):
    cfg = config(layers=2, **shape)
    lib = binding.DFlash(cfg)
    ps = cfg.page_size
    r = random.Random(5)
    for trial in range(14):
        lens = [5 * ps, 3 * ps + max(1, ps // 2), 0, 1, 7 * ps, 2 * ps, 0, 0]
        shared = [(4, 6, 5), (4, 7, 3)] if trial % 2 else [(1, 6, 4), (1, 7, 4), (0, 2, 5)]
        s = State(cfg, 60, 8, 9, lens, seed=trial, shared=shared)
        rows = r.sample(range(8), r.choice([1, 4, 8]))
        have = [int((s.table[x] >= 0).sum()) * ps for x in rows]
        keep = [r.choice([h, max(0, h - 1), h // 2, r.randint(0, h), 0]) for h in have]
        cap = [r.choice([0, k, k + 1, k + 2 * ps, r.randint(0, 9 * ps), 9 * ps, -4]) for k in keep]
        if trial >= 6:
            for _ in range(2):
                what, i = r.randint(0, 4), r.randrange(len(rows))
                if what == 0: rows[i] = r.choice([-1, 8, rows[0]])
                elif what == 1: cap[i] = 9 * ps + 1
                elif what == 2: keep[i], cap[i] = 9 * ps, 9 * ps          # pages of kept positions are missing
                elif what == 3: s.table[rows[0] % 8, 8] = 60
                else: keep[i] = cap[i] = 2 ** 31 - 1
            s.d_table.copy_(torch.from_numpy(s.table))
        if trial in (5, 13):
            s.ref[np.flatnonzero(s.ref == 0)[3:]] = 1
            s.d_ref.copy_(torch.from_numpy(s.ref))
        copies = tuple(torch.full((len(rows),), -7, dtype=torch.int32, device=DEV) for _ in range(3))
        lib.dflash_pages_resize(i32(rows), i32(keep), i32(cap), s.d_table, s.d_ref, s.d_pool, copies=copies)
        status, made = model.resize(s.table, s.ref, s.pool, rows, keep, cap)
        s.same(lib, status)
        assert list(zip(*(c.tolist() for c in copies))) == made


def test_resize_of_long_rows_in_a_large_pool():
    # rows of more entries than a CTA has threads, counts in several stretches of the scan, free pages with negative counts
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=1, dtype="fp32")
    lib = binding.DFlash(cfg)
    pages, width = 9001, 1100
    s = State(cfg, pages, 6, width, [700, 0, 1100, 300, 0, 1], seed=1, shared=[(2, 4, 1000)])
    s.ref[np.flatnonzero(s.ref == 0)[::3]] = -2
    s.d_ref.copy_(torch.from_numpy(s.ref))
    rows, keep, cap = [4, 1, 0, 2, 5, 3], [600, 0, 700, 5, 1, 300], [1100, 1100, 1099, 10, 1000, 0]
    lib.dflash_pages_resize(i32(rows), i32(keep), i32(cap), s.d_table, s.d_ref, s.d_pool)
    status, _ = model.resize(s.table, s.ref, s.pool, rows, keep, cap)
    s.same(lib, status)


@pytest.mark.parametrize("pages", [1, 2, 3, 33, 4096, 4097, 12345])
def test_compact(pages):
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=2, dtype="fp32")
    lib = binding.DFlash(cfg)
    for trial, share in enumerate((0.0, 0.3, 0.7, 1.0)):
        r = random.Random(trial)
        want = int(pages * share)
        rows, width = 5, pages // 4 + 1
        s = State(cfg, pages, rows, width, [min(width, max(0, want - b * width)) for b in range(rows)], seed=trial)
        s.table[4, 0] = s.table[0, 0]                 # shared by two rows
        held = s.table[s.table >= 0]
        s.ref = np.bincount(held, minlength=pages).astype(np.int32)
        if trial == 2 and pages > 3:                  # an entry that names a free page behind the border
            free = np.flatnonzero(s.ref == 0)
            if len(free):
                s.table[3, width - 1] = free[-1]
        if trial == 1:
            s.ref[s.ref == 0] = -1
        s.d_table.copy_(torch.from_numpy(s.table))
        s.d_ref.copy_(torch.from_numpy(s.ref))
        n_live = i32([-1])
        copies = (torch.full((pages // 2,), -7, dtype=torch.int32, device=DEV), torch.full((pages // 2,), -7, dtype=torch.int32, device=DEV), i32([-7]))
        lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool, n_live=n_live, copies=copies if pages > 1 else None)
        status, live, moves = model.compact(s.table, s.ref, s.pool)
        s.same(lib, status)
        assert int(n_live) == live
        if pages > 1:
            assert int(copies[2]) == len(moves)
            assert list(zip(copies[0].tolist(), copies[1].tolist())) == moves + [(-1, -1)] * (pages // 2 - len(moves))


def test_compact_flags_entries_whose_page_is_not_in_use():
    # pages 0 2 5 in use, border 3: page 1 is the hole that 5 moves to, and an entry that names it would come by 5's contents
    cfg = config(hq=2, hkv=2, hd=64, page=1, layers=1, dtype="fp32")
    lib = binding.DFlash(cfg)
    s = State(cfg, 6, 3, 4, [0, 0, 0])
    s.table[0, :3] = [0, 2, 5]
    s.table[1, :4] = [1, 4, -5, 2]
    s.table[2, :2] = [6, 2 ** 31 - 1]
    s.ref[:] = [1, 0, 2, 0, -3, 1]
    s.d_table.copy_(torch.from_numpy(s.table))
    s.d_ref.copy_(torch.from_numpy(s.ref))
    lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool)
    s.table[0, 2] = 1
    s.ref[:] = [1, 1, 2, 0, -3, 0]
    s.pool[:, 1] = s.pool[:, 5]
    s.same(lib, binding.DEV_BAD_PAGE)


def test_a_second_pool_follows_the_reported_copies():
    cfg, other = config(hq=8, hkv=2, layers=2), config(hq=4, hkv=4, hd=64, layers=3)
    lib, lib2 = binding.DFlash(cfg), binding.DFlash(other)
    s = State(cfg, 30, 6, 6, [200, 100, 0, 0, 0, 0], seed=2)
    bits2, pool2 = pool_of(other, 30, 9)
    copies = tuple(torch.empty(3, dtype=torch.int32, device=DEV) for _ in range(3))
    lib.dflash_pages_fork(i32([0, 0, 1]), i32([2, 3, 4]), i32([200, 128, 100]), s.d_table, s.d_ref, s.d_pool, copies=copies)
    lib2.dflash_pages_copy(copies[0], copies[1], pool2, n_slots=copies[2])
    _, made = model.fork(s.table, s.ref, s.pool, [0, 0, 1], [2, 3, 4], [200, 128, 100])
    s.same(lib, 0)
    assert model.copy(bits2, [m[0] for m in made], [m[1] for m in made], [m[2] for m in made]) == 0
    np.testing.assert_array_equal(bits_of(pool2), bits2)
    mv = (torch.empty(15, dtype=torch.int32, device=DEV), torch.empty(15, dtype=torch.int32, device=DEV), i32([0]))
    lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool, copies=mv)
    lib2.dflash_pages_copy(mv[0], mv[1], pool2, count=mv[2])
    _, _, moves = model.compact(s.table, s.ref, s.pool)
    s.same(lib, 0)
    assert model.copy(bits2, [m[0] for m in moves], [m[1] for m in moves]) == 0
    np.testing.assert_array_equal(bits_of(pool2), bits2)
    assert int(lib2.status.item()) == 0


def test_serving_round_captured_into_a_graph():
    """A prompt is forked, its continuations get room and are attended to together; the pool is compacted, which leaves the
    attention as it was, bit for bit; one of them is released and the pool compacted again. A replayed graph of the round does what the eager calls do."""
    cfg = config(hq=8, hkv=2, layers=1)
    lib = binding.DFlash(cfg)
    L, S, R = 300, 4, 16
    g = torch.Generator().manual_seed(4)
    mk = lambda *shape: torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)
    q, k, v = mk(S, R, 8, 128), mk(S, R, 2, 128), mk(S, R, 2, 128)
    pool0 = mk(*synth.kv_pool_shape(cfg, 40))
    start, prefix = i32([0, S]), i32([L])

    def fresh():
        s = State(cfg, 40, S, 12, [L] + [0] * (S - 1), seed=6)
        return s.d_table, s.d_ref, pool0.clone()

    def round_(table, ref, pool, outs):
        lib.dflash_pages_fork(i0, i1, il, table, ref, pool)
        lib.dflash_pages_resize(rows, keep, cap, table, ref, pool)
        lib.dflash_prefix_attention(1, q, k, v, start, prefix, lens, 400, table, pool, 0, outs[0])
        lib.dflash_pages_compact(table, ref, pool)
        lib.dflash_prefix_attention(1, q, k, v, start, prefix, lens, 400, table, pool, 0, outs[1])
        lib.dflash_pages_resize(last, zero, zero, table, ref, pool)
        lib.dflash_pages_compact(table, ref, pool, n_live=n_live)

    i0, i1, il = i32([0] * (S - 1)), i32([1, 2, 3]), i32([L] * (S - 1))
    rows, keep, cap = i32([0, 1, 2, 3]), i32([L] * S), i32([L + 17] * S)
    lens, last, zero, n_live = i32([L] * S), i32([3]), i32([0]), i32([0])
    eager = fresh()
    outs = [torch.zeros_like(q), torch.zeros_like(q)]
    round_(*eager, outs)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    assert torch.equal(outs[0], outs[1]) and float(outs[0].float().abs().max()) > 0
    # one whole prompt, its four whole pages shared by three rows, a partial page each
    assert int(n_live) == 4 + 3 and sorted(eager[1].tolist(), reverse=True)[:5] == [3, 3, 3, 3, 1]
    state = fresh()
    start_state = [t.clone() for t in state]
    outs2 = [torch.zeros_like(q), torch.zeros_like(q)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_(*state, outs2)
    for _ in range(2):
        for t, t0 in zip(state, start_state):
            t.copy_(t0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(state, eager):
            assert torch.equal(a, b)
        assert torch.equal(outs2[0], outs[0]) and torch.equal(outs2[1], outs[1])


def test_calls_on_two_streams_overlap():
    """Two tables over two pools, worked on from two streams with one handle: each stream has its own workspace."""
    cfg = config(hq=4, hkv=2, hd=64, page=16)
    lib = binding.DFlash(cfg)
    kinds = [([100, 0, 0, 0, 37], [0, 4], [1, 2], [90, 37]), ([64, 50, 0, 0], [1, 0, 1], [2, 3, 2], [33, 64, 5])]
    states, alone, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]

    def work(s, parent, child, keep, rows, room, stream):
        lib.dflash_pages_fork(parent, child, keep, s.d_table, s.d_ref, s.d_pool, stream=stream)
        lib.dflash_pages_resize(rows, keep, room, s.d_table, s.d_ref, s.d_pool, stream=stream)
        lib.dflash_pages_compact(s.d_table, s.d_ref, s.d_pool, stream=stream)

    for k, (lens, parent, child, keep) in enumerate(kinds):
        lists = (i32(parent), i32(child), i32(keep), i32(child), i32([n + 20 for n in keep]))
        one, two = (State(cfg, 60, len(lens), 9, lens, seed=40 + k) for _ in range(2))
        work(one, *lists, None)
        torch.cuda.synchronize()
        first = int(lib.status.item())
        lib.status.zero_()
        states.append((two, lists, first))
        alone.append(one)
    torch.cuda.synchronize()
    for (two, lists, _), stream in zip(states, streams):
        work(two, *lists, stream)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == states[0][2] | states[1][2]
    for one, (two, _, _) in zip(alone, states):
        assert torch.equal(one.d_table, two.d_table) and torch.equal(one.d_ref, two.d_ref)
        np.testing.assert_array_equal(bits_of(one.d_pool), bits_of(two.d_pool))


def test_refusals():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    s = State(cfg, 10, 3, 4, [100, 0, 0])
    with pytest.raises(AssertionError):
        lib.dflash_pages_copy(i32([0]), i32([1]), s.d_pool.float())
    with pytest.raises(AssertionError):
        lib.dflash_pages_copy(i32([0]).long(), i32([1]), s.d_pool)
    with pytest.raises(AssertionError):
        lib.dflash_pages_fork(i32([0]), i32([1]), i32([5]), s.d_table, s.d_ref[:9].contiguous(), s.d_pool)
    with pytest.raises(AssertionError):
        lib.dflash_pages_fork(i32([0]), i32([1, 2]), i32([5]), s.d_table, s.d_ref, s.d_pool)
    with pytest.raises(AssertionError):
        lib.dflash_pages_resize(i32([0]), i32([1]), i32([5]), s.d_table.t(), s.d_ref, s.d_pool)
    empty = torch.zeros(0, dtype=torch.int32, device=DEV)
    lib.dflash_pages_copy(empty, empty, s.d_pool)
    lib.dflash_pages_fork(empty, empty, empty, s.d_table, s.d_ref, s.d_pool)
    lib.dflash_pages_resize(empty, empty, empty, s.d_table, s.d_ref, s.d_pool)
    s.same(lib, 0)
