"""Rows in which one token is all but certain: its log probability -ln(1 + R), R = sum of the other terms, the row's ln S and its entropy keep their decimals however small R is.

Tolerances. u = 2^-24. A term of R is off by 4 |y| u (its exponent) and 8 u (the exponential and its rescaling), a thread adds at most V / 512 + 32 of them one behind the other (of
64 threads 8 times as many as of 512), the merges add 16: R by (V / 64 + 56 + 4 |y|) u of itself at most, |y| the largest that counts, 30 beyond the nearest. ln(1 + R) adds
2 u. The entropy's two parts, ln(1 + R) and sum of p |ln p|, have the same sign and the same relative errors, the second 4 u more."""
import numpy as np
import pytest
import torch

from tests.test_token_logprobs_gpu import BF16, F32, check_forward, forward, lib, placed  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def reference(z, T):
    """(place of the largest entry, ln S, entropy) of each row, without 1 + R."""
    z = z.double().numpy()
    at = z.argmax(1)
    y = (z - z.max(1, keepdims=True)) / T
    y[np.arange(len(z)), at] = -np.inf
    e = np.exp(y)
    log_sum = np.log1p(e.sum(1))
    return at, log_sum, log_sum - (e * np.where(np.isinf(y), 0.0, y)).sum(1) / (1 + e.sum(1)), -y.max(1)


def certain(n, v, dtype, gap, T, seed):
    """Rows of noise with one entry `gap` T above the rest, at every kind of place; some with others that were the largest before it."""
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(n, v))
    for r in range(n):
        at = [0, v - 1, v // 2, int(rng.integers(0, v))][r % 4]
        if r % 3 == 1:                                        # a rising row of some: each is set apart and taken back when the next one comes
            for k, p in enumerate(np.sort(rng.integers(0, v, 12))):
                z[r, p] = 5.0 * T * (k - 12)
            at = max(at, v - 2)
        z[r, at] = 0.0
        z[r, at] = z[r].max() + gap * T
    return torch.from_numpy(z).to(dtype)


@pytest.mark.parametrize("gap", [6.0, 12.0, 25.0, 60.0])
@pytest.mark.parametrize("n,v,dtype,T,pad,at", [
    (4, 50, F32, 1.0, 0, 0), (12, 1024, F32, 0.6, 0, 1), (12, 5003, BF16, 1.0, 3, 5), (12, 40000, F32, 1.5, 0, 0), (12, 200001, BF16, 1.0, 0, 0), (48, 100003, BF16, 0.8, 0, 0),
    (24, 100003, F32, 1.0, 0, 0), (1200, 900, BF16, 1.0, 0, 0), (1200, 1500, F32, 0.7, 1, 2), (700, 9000, BF16, 1.0, 0, 0), (12, 5003, F32, 1e-3, 0, 0), (12, 5003, F32, 1e22, 0, 0)])
@pytest.mark.parametrize("top", [0, 5])
def test_what_is_left_keeps_its_decimals(lib, n, v, dtype, T, pad, at, gap, top):
    z = certain(min(n, 24), v, dtype, gap, T, v).repeat(-(-n // 24), 1)[:n]
    place, log_sum, entropy, near = reference(z, T)
    tokens = torch.from_numpy(place.astype(np.int32))[:, None].contiguous()
    o = forward(lib, placed(z, pad, at), tokens.cuda(), T, top)
    torch.cuda.synchronize()
    got = {k: x.double().cpu().numpy() for k, x in o.items() if x is not None}
    rel = (v / 64 + 64 + 4 * (near + 30)) * U
    for what, value, want, extra in (("ln S", got["stats"][:, 1], log_sum, 1.0), ("log probability", got["logprob"][:, 0], -log_sum, 1.0), ("entropy", got["entropy"], entropy, 2.0)):
        off = np.abs(value - want)
        assert np.all(off <= extra * rel * np.abs(want) + 1e-38), f"{what}: {np.max(off / (extra * rel * np.abs(want) + 1e-38)):.2f} times the tolerance"
    if top:
        assert np.array_equal(got["top_ids"][:, 0], place) and np.array_equal(got["top_logprob"][:, 0], got["logprob"][:, 0])
    if gap < 20:
        check_forward(o, z, tokens, T, top)


@pytest.mark.parametrize("v,dtype", [(50, F32), (5003, BF16), (40000, F32), (200001, BF16)])
@pytest.mark.parametrize("apart", [1, 3, 8, 32, 256, 1024, 20000])
def test_several_equal_largest_entries(lib, v, dtype, apart):
    """Two, three and five of them, in one vector, one thread's vectors, one warp's and others': each counts once. +inf and NaN beside them as ever."""
    rng = np.random.default_rng(apart)
    z = rng.normal(size=(8, v))
    for r in range(8):
        for k in range((2, 3, 5)[r % 3]):
            z[r, (7 * r + k * apart) % v] = 30.0
    z[6, v // 2], z[7, v // 3] = np.inf, np.nan
    z = torch.from_numpy(z).to(dtype)
    tokens = torch.from_numpy(rng.integers(0, v, (8, 2)).astype(np.int32))
    tokens[:, 0] = torch.arange(8) * 7
    for copies in (1, 300):
        o = forward(lib, z.cuda().repeat(copies, 1), tokens.cuda().repeat(copies, 1), 1.0, 6)
        torch.cuda.synchronize()
        check_forward({k: x[-8:] for k, x in o.items()}, z, tokens, 1.0, 6)
