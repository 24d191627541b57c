"""Shared-prefix attention of scores of tens and hundreds of thousands, against the definition in 64 bits.

Queries and keys are whole numbers, so that every q . k is exact in fp32 (all partial sums stay below 2^24): with m the number that a query
holds in its elements 1.., c that of a key, t the key's element 0 and 1 the query's, q . k = m c (hd - 1) + t. Keys of the same c differ by t
alone, up to 40 x scale x log2(e) = 7.3 log2 units; keys of another c by more than 900, which makes them 0 or 1 in 64 bits too.

Tolerances, with p the exact probabilities, A = sum_k p_k |v_k|, n keys:
  tensor cores: x = s * scale_log2 - m is rounded once, for keys that count (less than 32 below the maximum, which tops the reference by
      16 at most) by 2^-20 at most; scale_log2 is off by 3 roundings of 2^-24, of a difference of less than 8 for keys that share c; the exponential by
      2^-22. The reference m cancels in the quotient. Together below delta = 2^-18
  CUDA cores: s * scale_log2 is rounded by itself, 2^-24 |z| each for the key and the maximum: delta = 2^-18 + 2^-23 |z|
  P rounded to bf16: 2^-8 (tensor cores); sums: n 2^-23; out rounded once: 2^-8 (bf16), 2^-24 (fp32)
|out - ref| <= (2 delta + n 2^-23 + P) A + rounding |ref|;  |lse - ref| <= delta + n 2^-23 + 2^-21 (1 + |ref|)"""
import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding, synth
from tests.test_prefix_attention_gpu import Batch, config

pytestmark = pytest.mark.gpu
LOG2E = 1.4426950408889634


def whole_numbers(x, top, seed):
    """Puts whole numbers in place of queries and keys; `top`: about the largest |score| in log2 units. Sequences alternate in sign."""
    cfg, g = x.cfg, synth.substream(seed, "whole")
    hd = cfg.head_dim
    per = 96 * (hd - 1) * cfg.softmax_scale * LOG2E          # log2 units of c = 1 at m = 96
    c = max(2, min(256, round(top / per)))
    q = torch.ones(x.q.shape)
    q[..., 1:] = torch.randint(64, 128, x.q.shape[:3] + (1,), generator=g).float()
    q[1::2, ..., 1:] *= -1                                   # the maximum of these sequences is a large negative number
    k = torch.full(x.k.shape, float(c))
    k[..., 0] = torch.randint(-20, 21, x.k.shape[:3], generator=g).float()
    x.q, x.k = q.to(x.q.dtype), k.to(x.k.dtype)
    hole = torch.isnan(x.pool[:, :, 0])
    keys = torch.full(hole.shape, float(c))
    keys[:, ::3] = c - 1                                     # pages whose keys lie far below (or above) the others
    keys[..., 0] = torch.randint(-20, 21, hole.shape[:-1], generator=g).float()
    x.pool[:, :, 0] = torch.where(hole, float("nan"), keys).to(x.pool.dtype)
    assert 128 * 256 * hd < 2 ** 24


def check(x, out, lse, causal, simt):
    o, ls = out.double().cpu().numpy(), lse.double().cpu().numpy()
    bf16 = x.cfg.dtype == "bf16"
    assert np.isfinite(o).all() and np.isfinite(ls).all()
    for b in range(x.S):
        ref, rl, A, mag, n = x.reference(b, causal)
        delta = 2.0 ** -18 + (2.0 ** -23 * float(mag.max()) * LOG2E if simt else 0.0)
        tol = (2 * delta + n * 2.0 ** -23 + (0.0 if simt else 2.0 ** -8)) * A + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref)
        err = np.abs(o[b] - ref)
        assert (err <= tol).all(), (b, float((err / tol).max()), int((err > tol).sum()))
        tl = delta + n * 2.0 ** -23 + 2.0 ** -21 * (1 + np.abs(rl))
        assert (np.abs(ls[b] - rl) <= tl).all(), (b, float((np.abs(ls[b] - rl) / tl).max()))


SHAPES = [({}, False), (dict(hq=6, hkv=2, hd=64, page=16), False), (dict(hq=20, hkv=4), False), (dict(hq=8, hkv=2, page=4), True),
          (dict(hq=4, hkv=2, hd=64, dtype="fp32"), True)]
BATCHES = [("one_key", 1, [0], [], [0] * 8), ("one_cached_key", 1, [0], [], [1] * 8), ("a_few", 16, [0], [], [0, 1, 5, 63, 64, 65, 128, 200]),
           ("behind_a_prefix", 7, [0, 3, 6], [300, 131], [300, 301, 700, 131, 400, 140])]


@pytest.mark.parametrize("top", [2.0 ** e for e in range(14, 19)])
@pytest.mark.parametrize("batch", BATCHES, ids=[b[0] for b in BATCHES])
@pytest.mark.parametrize("shape,simt", SHAPES, ids=["hd128", "hd64", "five_heads", "page4", "fp32"])
def test_large_scores(shape, simt, batch, top):
    cfg = config(layers=1, **shape)
    lib = binding.DFlash(cfg)
    name, rows, starts, prefix, lens = batch
    x = Batch(cfg, rows, starts, prefix, lens, seed=len(name), layer=0)
    whole_numbers(x, top, seed=int(top))
    for mode in (0, 1):
        out, lse = x.run(lib, mode)
        torch.cuda.synchronize()
        assert int(lib.status.item()) == 0
        check(x, out, lse, mode == 1, simt)
