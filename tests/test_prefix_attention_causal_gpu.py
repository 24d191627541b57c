"""Shared-prefix attention in mode CAUSAL: the block rows that a row does not see have no say in it, whatever they hold."""
import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests.test_prefix_attention_gpu import Batch, config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,rows,starts,prefix,lens", [
    ({}, 16, [0, 3], [200], [200, 263, 391, 40]),
    (dict(hq=6, hkv=2, hd=64, page=16), 10, [0], [], [0, 64, 70, 130]),
    (dict(hq=28, hkv=4), 17, [0, 4], [64], [64, 65, 129, 500]),
    (dict(hq=16, hkv=2), 32, [0, 2], [100], [100, 170, 128, 0]),                 # two query tiles an item
    (dict(hq=8, hkv=2, page=4), 7, [0, 2], [30], [31, 100]),
    (dict(hq=4, hkv=2, hd=64, dtype="fp32"), 8, [0, 3], [131], [131, 140, 221])])
@pytest.mark.parametrize("kinds", [("nan",), ("inf",), ("inf", "-inf", "nan")], ids=["nan", "inf", "mixed"])
def test_later_block_rows_have_no_say_in_earlier_ones(shape, rows, starts, prefix, lens, kinds):
    """CAUSAL: a padded row of a block may hold NaN or infinities. Rows that see it get them in these elements, the others nothing."""
    cfg = config(layers=1, **shape)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, rows, starts, prefix, lens, seed=rows, layer=0)
    G = cfg.n_q_heads // cfg.n_kv_heads
    v = x.v.clone()
    for b in range(x.S):
        for i, kind in enumerate(kinds):
            key = rows - 1 - (b + 2 * i) % (rows - 1)                            # 1 .. rows-1
            v[b, key, i % cfg.n_kv_heads, 5 + 9 * i:40 + 7 * i:3] = float(kind)
        if b % 2:
            v[b, rows - 1] = float("nan")                                        # a whole row
            x.k[b, rows - 1] = float("nan")
    x.v = v
    out, lse = x.run(lib, 1)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    clean = torch.where(torch.isfinite(v.float()), v.float(), torch.zeros(())).to(v.dtype)
    seen = torch.tril(torch.ones(rows, rows, dtype=torch.bool))
    any_of = lambda what: torch.einsum("rk,bkhd->brhd", seen.float(), what.float()).repeat_interleave(G, dim=2) > 0
    nan, pos, neg = any_of(torch.isnan(v)), any_of(v == float("inf")), any_of(v == float("-inf"))
    dead = torch.zeros(x.S, rows, 1, 1, dtype=torch.bool)
    dead[1::2, rows - 1] = True                                                  # the row that sees its own NaN key
    want = torch.zeros(out.shape)
    want[pos] = float("inf")
    want[neg] = float("-inf")
    want[(nan | (pos & neg) | dead).expand(out.shape)] = float("nan")
    bad = ~torch.isfinite(want)
    got, lse = out.float().cpu(), lse.cpu()
    assert torch.equal(~torch.isfinite(got), bad)
    assert torch.equal(got[bad & ~torch.isnan(want)], want[bad & ~torch.isnan(want)]) and torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isnan(lse), dead[..., 0].expand(lse.shape)) and torch.isfinite(lse[~torch.isnan(lse)]).all()
    x.v = clean
    x.k = torch.where(torch.isfinite(x.k.float()), x.k.float(), torch.zeros(())).to(x.k.dtype)
    for b in range(x.S):                                                         # the last row of an odd sequence aside, everything finite is right
        ref, rl, A, mag, n = x.reference(b, True)
        delta = mag * (cfg.head_dim + 8) * 2.0 ** -23 + 2.0 ** -20               # tolerances: tests/test_prefix_attention_gpu.py
        bf16 = cfg.dtype == "bf16"
        tol = (2 * delta[..., None] + n * 2.0 ** -23 + (2.0 ** -8 if bf16 else 0)) * A + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref)
        ok = ~bad[b].numpy()
        assert (np.abs(got[b].double().numpy() - ref)[ok] <= tol[ok]).all()
        live = ~dead[b, :, 0].expand(lse.shape[1:]).numpy()
        assert (np.abs(lse[b].double().numpy() - rl)[live] <= (delta + n * 2.0 ** -23 + 2.0 ** -21 * (1 + np.abs(rl)))[live]).all()
