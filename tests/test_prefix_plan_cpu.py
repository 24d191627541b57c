"""The work split of the shared-prefix attention, walked on the host with the kernels' own arithmetic: every key tile of
every item is taken by exactly one CTA, in chain order, and the partial results fit the workspace."""
import ctypes as C
import random

import pytest

from paper_2602_06036_b200 import binding, build, synth


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _handle(lib, hq, hkv, hd, page, dtype):
    c = synth.QWEN3_8B
    cfg = binding.Config(1, c.d_model, hq, hkv, hd, c.d_ffn, c.vocab, c.n_feat_layers, c.d_target, c.block_size, page,
                         binding.BF16 if dtype == "bf16" else binding.F32, c.vocab - 1, 1, 1e-6, hd ** -0.5, 0)
    h = C.c_void_p()
    assert lib.dflash_create(C.byref(cfg), C.byref(h)) == 0
    return h


def _check(lib, h, rows, starts, prefix, lens, bound):
    arr = lambda v: (C.c_int32 * max(len(v), 1))(*v)
    info = (C.c_int64 * 6)()
    rc = lib.dflash_prefix_plan_check(h, len(lens), rows, len(prefix), arr(starts), arr(prefix), arr(lens), bound, info)
    return rc, list(info)


SHAPES = [(32, 8, 128, 64, "bf16"), (8, 8, 128, 64, "bf16"), (28, 4, 128, 16, "bf16"), (128, 1, 128, 64, "bf16"), (6, 2, 64, 8, "bf16"),
          (4, 2, 64, 64, "fp32"), (32, 8, 128, 4, "bf16"), (66, 2, 64, 64, "fp32")]


@pytest.mark.parametrize("shape", SHAPES)
def test_every_tile_is_taken_once(lib, shape):
    h = _handle(lib, *shape)
    rng = random.Random(repr(shape))
    for _ in range(150):
        S = rng.choice([1, 1, 2, 3, 5, 17, 48, 100, 400])
        rows = rng.choice([1, 1, 2, 7, 16, 17, 32])
        n = rng.choice([0, 1, 1, 2, 3, S])
        cuts = sorted(rng.randint(0, S) for _ in range(n + 1))
        if n and rng.random() < 0.5:
            cuts[0], cuts[-1] = 0, S
        longest = rng.choice([0, 1, 63, 64, 65, 127, 128, 129, 1000, 5000, 70000])
        prefix = [rng.choice([0, 1, 63, 64, longest, rng.randint(0, longest), -3]) for _ in range(n)]
        lens = [rng.choice([0, longest, rng.randint(0, longest)]) for _ in range(S)]
        bound = max(0, longest - rng.choice([0, 0, 7]))             # some lengths above the caller's bound: clamped
        rc, info = _check(lib, h, rows, cuts, prefix, lens, bound)
        assert rc == 0, (rc, info, rows, cuts, prefix, lens, bound)
    lib.dflash_destroy(h)


def test_stretches_are_even_and_long_prefixes_come_in_blocks(lib):
    h = _handle(lib, 32, 8, 128, 64, "bf16")
    lens = [32768 + 31 * i for i in range(32)]
    rc, (items, group_items, tiles, segments, least, most) = _check(lib, h, 17, [0, 32], [32768], lens, 40000)
    assert rc == 0 and group_items >= 2 * 8 * 9 and most <= least + 32
    lib.dflash_destroy(h)


def test_bad_arguments_of_the_check_are_refused(lib):
    h = _handle(lib, 32, 8, 128, 64, "bf16")
    assert _check(lib, h, 33, [0, 1], [5], [9], 100)[0] == -1
    assert _check(lib, h, 1, [1, 0], [5], [9], 100)[0] == -1
    assert _check(lib, h, 1, [0, 2], [5], [9], 100)[0] == -1
    lib.dflash_destroy(h)
