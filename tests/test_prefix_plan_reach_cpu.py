"""The work split of the shared-prefix attention has no items for a prefix that none of its sequences reads."""
import random

import pytest

from tests.test_prefix_plan_cpu import SHAPES, _check, _handle, lib  # noqa: F401  (lib: the fixture)


def test_a_prefix_that_none_has_reached_is_no_work(lib):
    h = _handle(lib, 32, 8, 128, 64, "bf16")
    rc, (items, group_items, tiles, *_) = _check(lib, h, 16, [0, 3], [8192], [100, 8191, 0], 9000)
    alone = _check(lib, h, 16, [0], [], [100, 8191, 0], 9000)
    assert rc == 0 and group_items == 0 and (items, tiles) == (alone[1][0], alone[1][2])
    for lens in ([100, 8192, 0], [8192, 0, 0], [0, 0, 9000]):
        rc, (_, group_items, *_) = _check(lib, h, 16, [0, 3], [8192], lens, 9000)
        assert rc == 0 and group_items > 0
    rc, (_, group_items, *_) = _check(lib, h, 16, [0, 1, 3], [8192, 50], [8191, 8192, 49], 9000)
    assert rc == 0 and group_items == 8                              # the second prefix's kv heads
    lib.dflash_destroy(h)


@pytest.mark.parametrize("shape", SHAPES)
def test_every_tile_is_taken_once_where_most_prefixes_are_not_read(lib, shape):
    h = _handle(lib, *shape)
    r = random.Random(repr(shape))
    for _ in range(60):
        S, rows, n = r.choice([1, 3, 17, 100, 700]), r.choice([1, 7, 32]), r.choice([1, 2, 40])
        starts = sorted(r.randint(0, S) for _ in range(n + 1))
        prefix = [r.randint(0, 20000) for _ in range(n)]
        lens = [r.choice([0, r.randint(0, 500), r.randint(0, 20000)]) for _ in range(S)]
        rc, info = _check(lib, h, rows, starts, prefix, lens, 20000)
        assert rc == 0, (rc, info)
        read = any(0 < prefix[g] <= lens[b] for g in range(n) for b in range(starts[g], starts[g + 1]))
        assert (info[1] > 0) == read
    lib.dflash_destroy(h)


@pytest.mark.parametrize("shape", [(1, 1, 128, 64, "bf16"), (1, 1, 128, 256, "bf16"), (4, 1, 128, 8, "bf16")])
def test_the_longest_contexts(lib, shape):
    h = _handle(lib, *shape)
    longest = 2 ** 31 - 1 - 512
    for starts, prefix, lens in (([0], [], [longest]), ([0, 1], [longest - 70], [longest]), ([0, 1], [longest], [longest])):
        rc, info = _check(lib, h, 1, starts, prefix, lens, longest)
        assert rc == 0 and info[2] >= longest // 128, (rc, info)
    for bound in (longest + 1, 2 ** 31 - 1):
        assert _check(lib, h, 1, [0], [], [bound], bound)[0] == -2
    lib.dflash_destroy(h)


def test_more_heads_a_group_than_the_call_takes_are_refused_by_the_check_too(lib):
    h = _handle(lib, 129, 1, 64, 64, "fp32")
    assert _check(lib, h, 1, [0], [], [5], 100)[0] == -2
    lib.dflash_destroy(h)
