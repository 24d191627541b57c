"""Every way in which a log probability call is cut up, asked of the library for the device at hand: clusters of 2, 4 and 8 CTAs a row, and CTAs of each size that go through
several rows, with rows where it can go wrong (tolerances: see tests/test_token_logprobs_gpu.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests.test_token_logprobs_gpu import BF16, F32, KINDS, check_forward, forward, given, lib, placed, row_of  # noqa: F401

pytestmark = pytest.mark.gpu

PARTS = ["first part", "last part", "middle part", "a value in each part"]


def rows_of(kinds, v, dtype, seed):
    """Rows of the kinds, those of PARTS with all that is not -inf in one CTA's part of the row (or with equal values far apart)."""
    rng = np.random.default_rng(seed)
    out = []
    for kind in kinds:
        if kind not in PARTS:
            out.append(row_of(kind, v, dtype, rng))
            continue
        z = np.full(v, -np.inf)
        if kind == "a value in each part":
            z[:: max(1, v // 40)] = 2.5
        else:
            at = {"first part": 0, "last part": v - v // 16, "middle part": v // 2}[kind]
            z[at:at + max(1, v // 16)] = rng.normal(size=max(1, v // 16))
        out.append(z)
    return torch.from_numpy(np.stack(out)).to(dtype)


def form(lib, dtype, n, v, k, top):
    info = (C.c_int32 * 3)()
    assert lib.lib.dflash_token_logprobs_plan(lib.h, binding.F32 if dtype is F32 else binding.BF16, n, v, k, top, info) == 0
    return tuple(info)


@pytest.mark.parametrize("top", [0, 3, 40, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cs,rows,v", [(8, 12, 200001), (4, 24, 100003), (2, 48, 100003)])
def test_clusters(lib, cs, rows, v, dtype, top):
    kinds = KINDS + PARTS                                       # 24
    z, tokens = rows_of(kinds, v, dtype, v + top), given(len(kinds), v, 3, 5)
    tokens[:, 0] = v // 2
    z, tokens = z.repeat(max(1, rows // 24), 1), tokens.repeat(max(1, rows // 24), 1)
    for at in range(0, len(z), rows):
        part, t = z[at:at + rows], tokens[at:at + rows]
        assert form(lib, dtype, rows, v, 3, top) == (256, cs, rows * cs)
        o = forward(lib, placed(part, 5, 3), t.cuda(), 1.0, top)
        torch.cuda.synchronize()
        for i in range(0, rows, 24):
            check_forward({k: None if x is None else x[i:i + 24] for k, x in o.items()}, part[i:i + 24], t[i:i + 24], 1.0, top)


@pytest.mark.parametrize("threads,v,dtype,top,k", [
    (64, 50, F32, 32, 3), (64, 1501, F32, 20, 1), (64, 5003, BF16, 20, 64), (64, 16001, BF16, 3, 0),
    (128, 5003, BF16, 20, 65), (128, 5003, F32, 33, 1), (128, 14300, F32, 32, 2), (128, 32000, BF16, 64, 128),
    (256, 5003, F32, 65, 1), (256, 33000, BF16, 40, 1), (256, 57001, F32, 128, 2)])
def test_ctas_that_go_through_several_rows(lib, threads, v, dtype, top, k):
    """Two and a half rows a CTA, other kinds of rows behind each other, whose starts differ: the next row's tiles are requested during a row's search, and
    everything in shared memory is used again."""
    kinds = KINDS + PARTS[:3]                                    # 23: no number of CTAs is a multiple of it
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    copies = int(2.5 * (1024 // threads) * sms) // len(kinds)
    n = copies * len(kinds)
    got = form(lib, dtype, n, v, k, top)
    assert got[:2] == (threads, 1) and 2 * got[2] < n
    z, tokens = rows_of(kinds, v, dtype, v + top), given(len(kinds), v, k, 5)
    zz = placed(z.cuda().repeat(copies, 1), 5 if v < 10000 else 1, 3)
    o = forward(lib, zz, tokens.cuda().repeat(copies, 1), 1.0, top)
    torch.cuda.synchronize()
    o = {key: x.reshape(copies, len(kinds), *x.shape[1:]).cpu() for key, x in o.items()}
    some = {}
    for i in range(copies):                                    # (copies differ in the last bits where they start elsewhere between two borders)
        part = {key: x[i] for key, x in o.items()}
        some.setdefault(tuple(x.numpy().tobytes() for x in part.values()), part)
    assert len(some) <= 8
    for part in some.values():
        check_forward(part, z, tokens, 1.0, top)


@pytest.mark.parametrize("n,v,dtype,top", [(50, 151936, BF16, 33), (444, 151936, BF16, 64), (444, 151936, F32, 80), (444, 151936, F32, 90), (1, 2000003, BF16, 40), (1, 2000003, F32, 64),
                                           (444, 65536, BF16, 64), (444, 65537, BF16, 64), (444, 65544, BF16, 64), (444, 73728, BF16, 64), (444, 131072, BF16, 64), (444, 147456, BF16, 64)])
def test_parts_of_more_than_eight_tiles(lib, n, v, dtype, top):
    """Where a thread's part of a row is kept in 16 cells, on either side of the rule (65536 bf16 entries are 8 tiles)."""
    kinds = (KINDS + PARTS)[:max(1, min(n, 24))] if n > 1 else ["a value in each part"]
    z, tokens = rows_of(kinds, v, dtype, v + top), given(len(kinds), v, 2, 5)
    copies = -(-n // len(kinds))
    zz = placed(z.cuda().repeat(copies, 1)[:n], 0, 0)
    o = forward(lib, zz, tokens.cuda().repeat(copies, 1)[:n], 1.0, top)
    torch.cuda.synchronize()
    for i in (0, (n // len(kinds) - 1) * len(kinds)):
        check_forward({k: x[i:i + len(kinds)] for k, x in o.items()}, z, tokens, 1.0, top)
