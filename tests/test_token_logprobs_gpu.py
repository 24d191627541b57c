"""Token log probabilities, entropy, alternatives and their gradient on the GPU against the oracle in 64 bits.

Tolerances. u = 2^-24. A term exp(y), y = (z - M) / T, is off by at most 4 |y| u (three roundings on the way to its exponent) and 8 u
(the exponential itself, 2 ulp, and its rescaling); a thread adds at most V / 512 + 32 terms one behind the other, the merges add 16.
So ln S is off by (V / 512 + 56 + 4 E|y|) u, with E|y| = entropy - ln S + 2 ln S at most. A log probability adds 4 u of its own two parts.
The entropy's sum has terms exp(y) y: the same relative error of each, so E|y| times it, and u of the whole. Gradients: p = exp(y - ln S) is off by
4 (|y| + ln S) u + 8 u, its factor by 8 u (|G| + |gH| (|ln p| + entropy)), and the result is rounded to its type. ln p and the entropy are themselves off by
the tolerances above whatever their size, which adds |gH| times those: a row of one entry has ln p = entropy = 0, and both come out as some u."""
import numpy as np
import pytest
import torch

from oracle import dflash_oracle as orc
from paper_2602_06036_b200 import binding, synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
HOLD = 4_000_000                 # clocks for which a stream is held: about 2 ms


@pytest.fixture(scope="module")
def lib():
    return binding.DFlash(synth.TINY)


def logits(n, v, dtype, seed, peaks=8):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(n, v)) * 2.5
    for r in range(n):
        at = rng.integers(0, v, min(peaks, v))
        z[r, at] = rng.normal(size=len(at)) * 3 + 10
    return torch.from_numpy(z).to(dtype)


def given(n, v, k, seed):
    t = np.random.default_rng(seed + 1).integers(0, v, (n, k))
    t[np.random.default_rng(seed + 2).random((n, k)) < 0.1] = -1
    return torch.from_numpy(t.astype(np.int32))


def placed(z, pad, at):
    """z on the GPU with `pad` entries between its rows, its first one `at` entries behind a 16-byte border; what is around it is NaN."""
    n, v = z.shape
    flat = torch.full((at + n * (v + pad) + 16,), float("nan"), dtype=z.dtype, device="cuda")
    d = flat[at:at + n * (v + pad)].view(n, v + pad)[:, :v]
    d.copy_(z)
    return d


def forward(lib, z, tokens, T=1.0, top=0, stream=None):
    n, k = tokens.shape
    e = lambda *s, dt=F32: torch.full(s, 7, dtype=dt, device="cuda")
    o = dict(logprob=e(n, k), stats=e(n, 2), entropy=e(n), top_ids=e(n, top, dt=torch.int32) if top else None, top_logprob=e(n, top) if top else None)
    lib.dflash_token_logprobs(z, tokens, temperature=T, stream=stream, **o)
    return o


def spread(ref, T):
    """What the tolerances need of each row: (ln S, E|y|), 0 where a row has no numbers."""
    log_sum = np.nan_to_num(ref["stats"][:, 1])
    return log_sum, np.nan_to_num(ref["entropy"]) + log_sum


def close(got, want, tol, what):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    tol = np.broadcast_to(tol, want.shape)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    off = np.abs(got[fine] - want[fine])
    assert np.all(off <= tol[fine]), f"{what}: {np.max(off / tol[fine]):.2f} times the tolerance"


def check_forward(o, z, tokens, T, top):
    ref = orc.token_logprobs(z.double().numpy(), tokens.numpy(), T, top)
    V = z.shape[1]
    log_sum, ey = spread(ref, T)
    tol = (V / 512 + 56 + 4 * ey + 4 * log_sum) * U
    close(o["stats"], ref["stats"], np.stack([np.zeros_like(tol), tol], 1), "stats")
    close(o["logprob"], ref["logprob"], tol[:, None] + 4 * U * np.abs(np.nan_to_num(ref["logprob"], neginf=0.0)), "logprob")
    close(o["entropy"], ref["entropy"], tol * (2 + ey), "entropy")
    if top:
        np.testing.assert_array_equal(o["top_ids"].cpu().numpy(), ref["top_ids"])
        close(o["top_logprob"], ref["top_logprob"], tol[:, None] + 4 * U * np.abs(np.nan_to_num(ref["top_logprob"], neginf=0.0)), "top_logprob")


@pytest.mark.parametrize("n,v,dtype,k,top,T,pad,at", [
    (1, 1, F32, 1, 3, 1.0, 0, 0),
    (2, 5, BF16, 2, 8, 0.5, 3, 1),
    (3, 17, F32, 1, 17, 2.0, 0, 3),
    (4, 1024, F32, 1, 5, 1.0, 0, 0),
    (7, 5003, BF16, 3, 20, 1.3, 0, 5),              # every row starts elsewhere between two 16-byte borders
    (5, 5003, F32, 128, 128, 0.7, 61, 1),
    (2, 16384, BF16, 1, 128, 1.0, 0, 0),            # one tile
    (2, 16385, BF16, 1, 1, 1.0, 7, 0),              # and one entry more
    (300, 4099, BF16, 2, 7, 1.0, 0, 0),             # more rows than CTAs at once
    (3, 151936, BF16, 1, 20, 1.0, 0, 0),            # eight CTAs a row
    (2, 151936, F32, 5, 64, 0.6, 0, 0),
    (1, 200001, BF16, 1, 128, 1.0, 0, 7),
    (100, 32000, F32, 1, 20, 1.0, 8, 0),            # four
    (200, 32000, BF16, 1, 5, 1.0, 0, 0),            # two
    (320, 32001, BF16, 0, 20, 1.0, 0, 0),           # one, several tiles, no given token
    (6, 32000, BF16, 4, 0, 1.0, 0, 0),
    (1300, 3001, BF16, 2, 9, 1.0, 3, 1),            # a CTA goes through several rows, which start differently
    (1200, 1500, F32, 1, 0, 1.0, 0, 2),
    (1, 3000001, BF16, 1, 30, 1.0, 0, 3),           # hundreds of tiles
])
def test_matches_the_oracle(lib, n, v, dtype, k, top, T, pad, at):
    z, tokens = logits(n, v, dtype, n + v), given(n, v, k, n + v)
    lib.status.zero_()
    o = forward(lib, placed(z, pad, at), tokens.cuda(), T, top)
    torch.cuda.synchronize()
    assert int(lib.status) == 0
    check_forward(o, z, tokens, T, top)


def row_of(kind, v, dtype, rng):
    low = torch.finfo(dtype).min
    inf = float("inf")
    z = rng.normal(size=v)
    if kind == "constant":
        z[:] = 1.5
    elif kind == "two values":
        z = np.where(rng.random(v) < 0.5, 1.0, 2.0)
    elif kind == "rising":
        z = np.arange(v) * (40.0 / v)
    elif kind == "falling":
        z = -np.arange(v) * (40.0 / v)
    elif kind == "masked":
        z[rng.random(v) < 0.999] = -inf
    elif kind == "all masked":
        z[:] = -inf
    elif kind == "lowest":
        z[rng.random(v) < 0.99] = low
    elif kind == "all lowest":
        z[:] = low
    elif kind == "lowest and -inf":
        z = np.where(rng.random(v) < 0.5, low, -inf)
    elif kind == "one":
        z[:] = -inf
        z[v // 2] = -300.0
    elif kind == "nan":
        z[v // 3] = np.nan
    elif kind == "nan and -inf":
        z[:] = -inf
        z[v // 3] = np.nan
    elif kind == "all nan":
        z[:] = np.nan
    elif kind == "inf":
        z[v // 3] = inf
    elif kind == "zeros of both signs":
        z = np.where(rng.random(v) < 0.5, 0.0, -0.0)
        z[rng.random(v) < 0.9] = -1.0
    elif kind == "huge":
        z *= 1e30
    elif kind == "one huge":
        z[v // 2] = 3e4
    elif kind.startswith("few threads"):                       # large entries where few threads look: many are above what bounds those threads' largest
        per = 16 // torch.empty(0, dtype=dtype).element_size()
        hot = (np.arange(v) // per * 37) % 256 < int(kind.split()[-1])
        z = np.where(hot, 20.0 + rng.random(v), z * 0.01)
    elif kind == "far ends":                                   # ties at the top of a range of values that passes 31 bits
        z = np.where(rng.random(v) < 0.5, 1.5e38, -1.5e38)
    return z


KINDS = ["constant", "two values", "rising", "falling", "masked", "all masked", "lowest", "all lowest", "lowest and -inf", "one", "nan", "nan and -inf", "all nan",
         "inf", "zeros of both signs", "huge", "one huge", "far ends", "few threads 6", "few threads 140"]


@pytest.mark.parametrize("v", [50, 5003, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [3, 128])
def test_rows_where_it_can_go_wrong(lib, v, dtype, top):
    rng = np.random.default_rng(v + top)
    z = torch.from_numpy(np.stack([row_of(k, v, dtype, rng) for k in KINDS])).to(dtype)
    tokens = given(len(KINDS), v, 3, 5)
    tokens[:, 0] = v // 2
    for copies in (1, 4):                                     # a row by several CTAs, and by one
        zz, tt = z.repeat(copies, 1), tokens.repeat(copies, 1)
        o = forward(lib, zz.cuda(), tt.cuda(), 1.0, top)
        torch.cuda.synchronize()
        for i in range(copies):                                # (rows that start elsewhere between the borders are added up in another order)
            check_forward({k: x[i * len(KINDS):(i + 1) * len(KINDS)] for k, x in o.items()}, z, tokens, 1.0, top)


@pytest.mark.parametrize("n,v,dtype,top,k", [
    (1200, 50, F32, 32, 3), (1200, 5003, BF16, 3, 64), (1200, 8001, F32, 32, 0), (1200, 16000, BF16, 20, 1),      # CTAs of 64 threads
    (1200, 5003, BF16, 20, 65), (1200, 5003, F32, 33, 1), (600, 14300, F32, 32, 2), (600, 32000, BF16, 64, 128),   # of 128
    (600, 57000, BF16, 8, 1),
    (600, 5003, F32, 65, 1), (600, 33000, BF16, 40, 1),                                                             # of 256
])
def test_such_rows_by_the_hundred(lib, n, v, dtype, top, k):
    """Short rows that are many go to smaller CTAs."""
    rng = np.random.default_rng(v + top)
    z = torch.from_numpy(np.stack([row_of(kind, v, dtype, rng) for kind in KINDS])).to(dtype)
    tokens = given(len(KINDS), v, k, 5)
    copies = n // len(KINDS)
    zz = placed(z.repeat(copies, 1), 5 if v < 10000 else 0, 3)
    o = forward(lib, zz, tokens.repeat(copies, 1).cuda(), 1.0, top)
    torch.cuda.synchronize()
    some = {}
    for i in range(copies):                                    # (copies differ in the last bits where they start elsewhere between two borders)
        part = {key: x[i * len(KINDS):(i + 1) * len(KINDS)] for key, x in o.items()}
        some.setdefault(tuple(x.cpu().numpy().tobytes() for x in part.values()), part)
    assert len(some) <= 8
    for part in some.values():
        check_forward(part, z, tokens, 1.0, top)


def test_tiny_and_large_temperatures(lib):
    z, tokens = logits(4, 3001, F32, 9), given(4, 3001, 4, 9)
    for T in (1e-30, 1e-3, 1e6):
        check_forward(forward(lib, z.cuda(), tokens.cuda(), T, 9), z, tokens, T, 9)


def test_a_token_outside_the_vocabulary_is_flagged(lib):
    z = logits(3, 100, F32, 2)
    tokens = torch.tensor([[1, 100], [2, 3], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32)
    lib.status.zero_()
    o = forward(lib, z.cuda(), tokens.cuda())
    torch.cuda.synchronize()
    assert int(lib.status) == binding.DEV_BAD_TOKEN and o["logprob"][0, 1] == 0 and o["logprob"][2].tolist() == [0, 0]
    check_forward(o, z, tokens, 1.0, 0)
    lib.status.zero_()
    d = torch.empty(3, 100, device="cuda")
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], torch.ones(3, 2, device="cuda"), d)
    torch.cuda.synchronize()
    assert int(lib.status) == binding.DEV_BAD_TOKEN and not d[2].any()
    lib.status.zero_()


def test_no_rows_and_outputs_that_are_not_wanted(lib):
    empty = torch.empty(0, 10, device="cuda")
    lib.dflash_token_logprobs(empty, torch.empty(0, 1, dtype=torch.int32, device="cuda"), torch.empty(0, 1, device="cuda"))
    z, tokens = logits(3, 1000, BF16, 4), given(3, 1000, 2, 4)
    full = forward(lib, z.cuda(), tokens.cuda(), 1.0, 4)
    lp, ids, top = (torch.empty_like(full[k]) for k in ("logprob", "top_ids", "top_logprob"))
    lib.dflash_token_logprobs(z.cuda(), tokens.cuda(), lp)
    lib.dflash_token_logprobs(z.cuda(), None, None, top_ids=ids, top_logprob=top)
    torch.cuda.synchronize()
    assert torch.equal(lp, full["logprob"]) and torch.equal(ids, full["top_ids"]) and torch.equal(top, full["top_logprob"])


def check_backward(d, z, tokens, g, gh, T, out, rows=slice(None)):
    zz, g64 = z.double().numpy(), g.double().numpy()
    h64 = None if gh is None else gh.double().numpy()
    want = orc.token_logprobs_backward(zz, tokens.numpy(), g64, h64, T)
    f = orc.token_logprobs(zz, tokens.numpy(), T)
    valid = (tokens.numpy() >= 0) & (tokens.numpy() < z.shape[1])
    lp = np.nan_to_num(np.where(np.isfinite(f["lp"]), f["lp"], 0.0))
    p = np.nan_to_num(np.exp(f["lp"]))
    log_sum = np.nan_to_num(f["stats"][:, 1:])
    G = np.abs(np.where(valid, g64, 0)).sum(1, keepdims=True)
    H = np.zeros_like(G) if h64 is None else np.abs(h64)[:, None]
    size = p * (G + H * (1 + np.abs(lp) + np.nan_to_num(f["entropy"])[:, None]))
    own = np.zeros_like(zz)
    for r in range(len(zz)):
        np.add.at(own[r], tokens.numpy()[r][valid[r]], np.abs(g64[r][valid[r]]))
    V = z.shape[1]
    stats = (V / 512 + 56 + 8 * (np.abs(lp).max(1, keepdims=True) * 0 + 12)) * U          # of the forward call's ln S and entropy
    tol = (size * (4 * (np.abs(lp) + 2 * log_sum) * U + 24 * U + 4 * stats) + (2 + tokens.shape[1]) * U * own) / T
    tol = tol + HALF_STEP[out] * 1.001 * np.abs(np.nan_to_num(want)) + 1e-37
    close(d, want, tol, "gradient")


@pytest.mark.parametrize("n,v,dtype,out,k,T,pad,at,pad_out,at_out,entropy", [
    (1, 1, F32, F32, 1, 1.0, 0, 0, 0, 0, True),
    (2, 7, BF16, BF16, 3, 0.5, 1, 1, 0, 0, True),
    (8, 1024, F32, F32, 1, 1.0, 0, 0, 0, 0, True),
    (3, 5003, BF16, BF16, 2, 1.3, 0, 5, 0, 5, True),           # both start alike between the borders
    (3, 5003, BF16, BF16, 2, 1.3, 61, 5, 0, 2, True),          # and not
    (5, 5003, F32, BF16, 64, 2.0, 0, 1, 3, 7, False),
    (4, 5001, BF16, F32, 128, 0.7, 0, 0, 0, 0, True),
    (3, 4096, F32, F32, 128, 1.0, 0, 2, 0, 3, False),
    (2, 151936, BF16, BF16, 1, 1.0, 0, 0, 0, 0, True),
    (1, 151936, F32, BF16, 32, 2.0, 0, 0, 0, 0, False),
    (700, 3001, BF16, BF16, 1, 1.0, 0, 0, 0, 0, True),
    (2, 8193, F32, F32, 0, 1.0, 0, 0, 0, 0, True),             # the entropy alone
])
def test_gradient_matches_the_oracle(lib, n, v, dtype, out, k, T, pad, at, pad_out, at_out, entropy):
    z, tokens = logits(n, v, dtype, n + v), given(n, v, k, n + v)
    if k > 2:
        tokens[:, 1] = tokens[:, 2]                             # the same token twice
    rng = np.random.default_rng(v)
    g = torch.from_numpy(rng.normal(size=(n, k))).float()
    g[n // 2] = 0.0
    gh = torch.from_numpy(rng.normal(size=n)).float() if entropy else None
    zd = placed(z, pad, at)
    o = forward(lib, zd, tokens.cuda(), T)
    around = torch.full((at_out + n * (v + pad_out) + 16,), 5.0, dtype=out, device="cuda")
    d = around[at_out:at_out + n * (v + pad_out)].view(n, v + pad_out)[:, :v]
    lib.dflash_token_logprobs_bwd(zd, tokens.cuda(), o["stats"], g.cuda(), d, temperature=T, entropy=o["entropy"] if entropy else None,
                                  d_entropy=gh.cuda() if entropy else None)
    torch.cuda.synchronize()
    check_backward(d, z, tokens, g, gh, T, out)
    d.fill_(5.0)
    assert bool((around == 5.0).all())                          # nothing outside of the rows is written


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [50, 9001])
def test_gradient_of_rows_where_it_can_go_wrong(lib, dtype, v):
    rng = np.random.default_rng(v)
    z = torch.from_numpy(np.stack([row_of(k, v, dtype, rng) for k in KINDS])).to(dtype)
    n = len(KINDS)
    tokens = given(n, v, 4, 6)
    tokens[:, :2] = v // 2
    g, gh = torch.from_numpy(rng.normal(size=(n, 4))).float(), torch.from_numpy(rng.normal(size=n)).float()
    o = forward(lib, z.cuda(), tokens.cuda())
    d = torch.empty(n, v, dtype=dtype, device="cuda")
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], g.cuda(), d, entropy=o["entropy"], d_entropy=gh.cuda())
    check_backward(d, z, tokens, g, gh, 1.0, dtype)
    # nothing comes in: zeros, whatever the logits hold
    d.fill_(3.0)
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], torch.zeros_like(g).cuda(), d, entropy=o["entropy"], d_entropy=torch.zeros(n, device="cuda"))
    assert not d.any()
    g[tokens >= 0] = 0.0                                        # only tokens that are none have a gradient
    d.fill_(3.0)
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], g.cuda(), d)
    assert not d.any()


@pytest.mark.parametrize("v,dtype,out,k,pad,at", [
    (1000, F32, F32, 64, 0, 0), (1000, BF16, BF16, 64, 3, 1), (5003, BF16, BF16, 3, 0, 0), (8192, F32, BF16, 1, 0, 1),      # CTAs of 64 and of 128 threads
    (5003, BF16, BF16, 65, 0, 2), (9001, BF16, BF16, 128, 0, 0), (4096, F32, F32, 128, 5, 0), (4099, F32, F32, 2, 0, 0),     # of 128 and 256
])
def test_gradients_of_rows_by_the_thousand(lib, v, dtype, out, k, pad, at):
    """Many rows go to smaller CTAs. An entry's gradient is worked out alike in all of them, so a few rows on their own (checked against the oracle) have the same."""
    n = 2400
    z = torch.from_numpy(np.random.default_rng(v).normal(size=(n, v)).astype(np.float32) * 3).to(dtype)
    tokens = given(n, v, k, v)
    tokens[:, k // 2] = tokens[:, 0]
    rng = np.random.default_rng(v)
    g, gh = torch.from_numpy(rng.normal(size=(n, k))).float(), torch.from_numpy(rng.normal(size=n)).float()
    zd, td, gd, ghd = placed(z, pad, at), tokens.cuda(), g.cuda(), gh.cuda()
    o = forward(lib, zd, td, 1.3)
    whole = torch.full((n, v), 5.0, dtype=out, device="cuda")
    lib.dflash_token_logprobs_bwd(zd, td, o["stats"], gd, whole, temperature=1.3, entropy=o["entropy"], d_entropy=ghd)
    for from_, to in ((0, 40), (1184, 1224), (2360, 2400)):
        part = torch.full((n, v), 5.0, dtype=out, device="cuda")[from_:to]
        lib.dflash_token_logprobs_bwd(zd[from_:to], td[from_:to], o["stats"][from_:to].contiguous(), gd[from_:to].contiguous(), part, temperature=1.3,
                                      entropy=o["entropy"][from_:to].contiguous(), d_entropy=ghd[from_:to].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(part, whole[from_:to])
        check_backward(part, z[from_:to], tokens[from_:to], g[from_:to], gh[from_:to], 1.3, out)
    some = torch.empty(1300, v, dtype=out, device="cuda")
    lib.dflash_token_logprobs_bwd(zd[:1300], td[:1300], o["stats"][:1300], gd[:1300], some, temperature=1.3, entropy=o["entropy"][:1300], d_entropy=ghd[:1300])
    torch.cuda.synchronize()
    assert torch.equal(some[:1184], whole[:1184]) and torch.equal(some, whole[:1300])


@pytest.mark.parametrize("dtype,v,pad", [(BF16, 20000, 0), (F32, 5003, 5)])
def test_gradient_in_the_logits_own_place(lib, dtype, v, pad):
    z, tokens = logits(9, v, dtype, 3), given(9, v, 40, 3)
    zd = placed(z, pad, 0)
    o = forward(lib, zd, tokens.cuda(), 0.8)
    g, gh = torch.randn(9, 40, device="cuda"), torch.randn(9, device="cuda")
    apart = torch.empty(9, v + pad, dtype=dtype, device="cuda")[:, :v]
    args = dict(temperature=0.8, entropy=o["entropy"], d_entropy=gh)
    lib.dflash_token_logprobs_bwd(zd, tokens.cuda(), o["stats"], g, apart, **args)
    lib.dflash_token_logprobs_bwd(zd, tokens.cuda(), o["stats"], g, zd, **args)
    torch.cuda.synchronize()
    assert torch.equal(zd, apart)


def test_gradient_through_the_alternatives(lib):
    """top_ids handed back as tokens: -1 entries take part in nothing."""
    z = logits(6, 400, F32, 8)
    z[2] = float("-inf")
    z[2, 7] = 1.0
    o = forward(lib, z.cuda(), given(6, 400, 1, 8).cuda(), 1.0, 16)
    again = forward(lib, z.cuda(), o["top_ids"])
    keep = o["top_ids"] >= 0
    assert torch.equal(again["logprob"][keep], o["top_logprob"][keep]) and int(keep[2].sum()) == 1
    g = torch.randn(6, 16)
    d = torch.empty(6, 400, device="cuda")
    lib.dflash_token_logprobs_bwd(z.cuda(), o["top_ids"], o["stats"], g.cuda(), d)
    check_backward(d, z, o["top_ids"].cpu(), g, None, 1.0, F32)


def test_rows_beyond_32_bits(lib):
    """The last row begins 2^31 entries behind the first one, in the logits and in the gradient."""
    n, v, apart = 9, 5000, 2 ** 28
    z, tokens = logits(n, v, BF16, 31), given(n, v, 2, 31)
    zd = torch.empty(8 * apart + v, dtype=BF16, device="cuda").as_strided((n, v), (apart, 1))
    zd.copy_(z)
    o = forward(lib, zd, tokens.cuda(), 1.0, 9)
    torch.cuda.synchronize()
    check_forward(o, z, tokens, 1.0, 9)
    g = torch.randn(n, 2)
    lib.dflash_token_logprobs_bwd(zd, tokens.cuda(), o["stats"], g.cuda(), zd)
    check_backward(zd, z, tokens, g, None, 1.0, BF16)


def test_runs_agree_bit_by_bit(lib):
    z, tokens = logits(64, 32000, BF16, 12).cuda(), given(64, 32000, 64, 12).cuda()
    tokens[:, 1::2] = tokens[:, ::2]
    g = torch.randn(64, 64, device="cuda")
    first = None
    for _ in range(5):
        o = forward(lib, z, tokens, 0.9, 100)
        d = torch.empty(64, 32000, device="cuda")
        lib.dflash_token_logprobs_bwd(z, tokens, o["stats"], g, d, temperature=0.9)
        now = list(o.values()) + [d]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(now, first))


def test_two_streams_at_once_and_a_replayed_graph(lib):
    n, v = 40, 50000
    zs = [logits(n, v, BF16, 20 + i).cuda() for i in range(3)]
    tokens = given(n, v, 2, 20).cuda()
    g = torch.randn(n, 2, device="cuda")

    def both(z, d, stream=None):
        o = forward(lib, z, tokens, 1.0, 20, stream=stream)
        lib.dflash_token_logprobs_bwd(z, tokens, o["stats"], g, d, stream=stream)
        return o

    want = []
    for z in zs:
        d = torch.empty(n, v, dtype=BF16, device="cuda")
        want.append(list(both(z, d).values()) + [d])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(HOLD)
    for z, s in zip(zs, streams):
        with torch.cuda.stream(s):
            d = torch.empty(n, v, dtype=BF16, device="cuda")
            got.append(list(both(z, d, s).values()) + [d])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    z, d = zs[0].clone(), torch.empty(n, v, dtype=BF16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = both(z, d)
    for i in (2, 1, 0):
        z.copy_(zs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(list(o.values()) + [d], want[i]))


def test_refusals_of_the_binding(lib):
    z, tokens = torch.zeros(4, 100, device="cuda"), torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    lp = torch.empty(4, 1, device="cuda")
    for bad in (lambda: lib.dflash_token_logprobs(z.half(), tokens, lp), lambda: lib.dflash_token_logprobs(z.t(), tokens, lp),
                lambda: lib.dflash_token_logprobs(z[:1].expand(4, 100), tokens, lp), lambda: lib.dflash_token_logprobs(z, tokens.long(), lp),
                lambda: lib.dflash_token_logprobs(z, tokens, lp[:3]), lambda: lib.dflash_token_logprobs(z.cpu(), tokens, lp),
                lambda: lib.dflash_token_logprobs(z, tokens[:, :0], None, top_ids=tokens, top_logprob=lp[:2]),
                lambda: lib.dflash_token_logprobs_bwd(z, tokens, lp.expand(4, 2), lp, torch.empty_like(z)),
                lambda: lib.dflash_token_logprobs_bwd(z, tokens, torch.empty(4, 2, device="cuda"), lp, torch.empty(4, 99, device="cuda"))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(binding.DFlashError):
        lib.dflash_token_logprobs(z, tokens, lp, temperature=0.0)
