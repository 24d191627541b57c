"""How a log probability call is cut up, on the host: every row has its CTAs, and each form that the kernels have is reached by some sizes."""
import ctypes as C

from tests.test_logprobs_adamw_abi_cpu import h, lib  # noqa: F401


def test_forms(lib, h):
    info = (C.c_int32 * 3)()
    seen = set()
    for dtype in (0, 1):
        for vocab in (1, 50, 5003, 16384, 16385, 32000, 57001, 100003, 151936, 400000, 2 ** 30):
            for rows in (1, 3, 12, 24, 48, 200, 591, 592, 1183, 1184, 2368, 4096, 2 ** 28):
                for tokens, top in ((0, 0), (1, 20), (64, 32), (65, 33), (128, 128)):
                    assert lib.dflash_token_logprobs_plan(h, dtype, rows, vocab, tokens, top, info) == 0
                    threads, cs, grid = info
                    assert threads in (64, 128, 256) and cs in (1, 2, 4, 8) and (threads == 256 or cs == 1)
                    assert tokens <= threads and 2 * top <= threads
                    assert 0 < grid <= rows * cs and (cs == 1 or grid == rows * cs) and grid < 2 ** 31
                    seen.add((threads, cs))
    assert seen == {(64, 1), (128, 1), (256, 1), (256, 2), (256, 4), (256, 8)}


def test_refusals(lib, h):
    info = (C.c_int32 * 3)()
    call = lib.dflash_token_logprobs_plan
    assert call(None, 0, 1, 1, 0, 0, info) == -1 and call(h, 0, 1, 1, 0, 0, None) == -1
    for args in ((2, 1, 1, 0, 0), (0, 0, 1, 0, 0), (0, 1, 0, 0, 0), (0, 1, 1, -1, 0), (0, 1, 1, 0, -1)):
        assert call(h, *args, info) == -1
    for args in ((0, 2 ** 28 + 1, 1, 0, 0), (0, 1, 2 ** 30 + 1, 0, 0), (0, 1, 1, 129, 0), (0, 1, 1, 0, 129)):
        assert call(h, *args, info) == -2
