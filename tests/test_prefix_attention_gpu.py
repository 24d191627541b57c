"""GPU parity of the attention of a batch that shares long prefixes (dflash_prefix_attention) with its definition in 64 bits.

Tolerances, per output component, with p the exact probabilities, n the number of keys and A = sum_k p_k |v_k|:
  scores   fp32 sums of hd exact products: each off by at most (hd + 8) 2^-23 scale sum_d |q_d k_d| (tensor cores add with a
           truncated last place, hence 2^-23), so p is off by the relative delta below; exp2 adds 2 ulp of its own
  P        rounded to bf16 before P V: 2^-8 a term (not in fp32)
  sums     n additions in fp32, 2^-23 each
  out      rounded once: 2^-8 (bf16) or 2^-24 (fp32) of the value
so |out - ref| <= (2 delta + n 2^-23 + P) A + rounding |ref|, and |lse - ref| <= delta + n 2^-23 + 2^-21 (1 + |ref|)."""
import random

import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding, synth

pytestmark = pytest.mark.gpu


def config(hq=32, hkv=8, hd=128, page=64, dtype="bf16", layers=2):
    return synth.DFlashConfig(n_layers=layers, d_model=256, n_q_heads=hq, n_kv_heads=hkv, head_dim=hd, d_ffn=256, vocab=256, n_feat_layers=1,
                              d_target=256, block_size=16, dtype=dtype, page_size=page)


class Batch:
    """A batch over a shared cache: the pool is NaN wherever no sequence has a position, and table entries that must not be
    read name a page that does not exist."""

    def __init__(self, cfg, rows, starts, prefix, lens, seed=0, q_std=1.0, layer=1, extra_pages=3, bound=None):
        self.cfg, self.R, self.starts, self.prefix, self.lens, self.layer = cfg, rows, list(starts), list(prefix), list(lens), layer
        S, ps = len(lens), cfg.page_size
        self.S = S
        self.group = [next((g for g in range(len(prefix)) if starts[g] <= b < starts[g + 1]), -1) for b in range(S)]
        self.shared = [prefix[g] if g >= 0 and lens[b] >= prefix[g] > 0 else 0 for b, g in enumerate(self.group)]
        self.bound = bound if bound is not None else max(list(lens) + list(prefix) + [0])
        need = [0] * S                                   # positions that are read through the own row
        for b in range(S):
            need[b] = lens[b]
            if self.group[b] >= 0 and starts[self.group[b]] == b:
                need[b] = max(need[b], prefix[self.group[b]])
        width = max([1] + [-(-n // ps) for n in need])
        table = np.full((S, width), 10 ** 6, dtype=np.int64)
        used = 0
        for b in range(S):
            leader = self.group[b] >= 0 and starts[self.group[b]] == b
            first = 0 if leader else self.shared[b] // ps
            have = -(-need[b] // ps)
            table[b, first:have] = np.arange(used, used + max(0, have - first))
            used += max(0, have - first)
        self.pages = used + extra_pages
        g = synth.substream(seed, "perm")
        perm = torch.randperm(self.pages, generator=g).numpy()
        self.table = np.where(table < 10 ** 6, perm[np.minimum(table, used)], table).astype(np.int32)
        pool = torch.full(synth.kv_pool_shape(cfg, self.pages), float("nan"), dtype=torch.float32)
        for b in range(S):
            lo = 0 if (self.group[b] >= 0 and starts[self.group[b]] == b) else self.shared[b]
            for p0 in range(lo, need[b]):
                pool[:, int(self.table[b, p0 // ps]), :, :, p0 % ps] = 0.0
        vals = synth.normal(pool.shape, 1.0, seed, "pool", torch.float32)
        self.pool = torch.where(pool == 0, vals, pool).to(cfg.torch_dtype)
        self.q = synth.normal((S, rows, cfg.n_q_heads, cfg.head_dim), q_std, seed, "q", cfg.torch_dtype)
        self.k = synth.normal((S, rows, cfg.n_kv_heads, cfg.head_dim), 1.0, seed, "k", cfg.torch_dtype)
        self.v = synth.normal((S, rows, cfg.n_kv_heads, cfg.head_dim), 1.0, seed, "v", cfg.torch_dtype)

    def cuda(self, dev="cuda:0"):
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
        self.d = dict(q=self.q.to(dev), k=self.k.to(dev), v=self.v.to(dev), table=torch.from_numpy(self.table).to(dev), pool=self.pool.to(dev),
                      lens=i32(self.lens), starts=i32(self.starts), prefix=i32(self.prefix))
        return self.d

    def run(self, lib, mode, d=None, out=None, lse=None, stream=None, bound=None):
        d = d or self.cuda()
        out = torch.full_like(d["q"], float("nan")) if out is None else out
        lse = torch.full(d["q"].shape[:3], float("nan"), dtype=torch.float32, device=d["q"].device) if lse is None else lse
        lib.dflash_prefix_attention(mode, d["q"], d["k"], d["v"], d["starts"] if self.prefix else None, d["prefix"] if self.prefix else None,
                                    d["lens"], self.bound if bound is None else bound, d["table"], d["pool"], self.layer, out, stream=stream, lse_out=lse)
        return out, lse

    def keys(self, b):
        """K, V [L, Hkv, hd] of sequence b in 64 bits, by the definition."""
        ps, pool = self.cfg.page_size, self.pool
        pos = np.arange(self.lens[b])
        row = np.where(pos < self.shared[b], self.starts[self.group[b]] if self.group[b] >= 0 else b, b)
        page = self.table[row, pos // ps] if len(pos) else np.zeros(0, dtype=np.int64)
        kv = pool[self.layer][torch.from_numpy(page.astype(np.int64)), :, :, torch.from_numpy(pos % ps)]        # [L, 2, Hkv, hd]
        kv = kv.double().numpy()
        return kv[:, 0], kv[:, 1]

    def reference(self, b, causal, keep=None):
        cfg, R, S = self.cfg, self.R, self.S
        G = cfg.n_q_heads // cfg.n_kv_heads
        K, V = self.keys(b)
        if keep is not None:
            K, V = K[keep], V[keep]
        L = len(K)
        K = np.concatenate([K, self.k[b].double().numpy()])
        V = np.concatenate([V, self.v[b].double().numpy()])
        q = self.q[b].double().numpy()
        out, A = np.empty(q.shape), np.empty(q.shape)
        lse, mag = np.empty(q.shape[:2]), np.empty(q.shape[:2])
        hide = np.zeros((R, L + R), dtype=bool)
        if causal:
            hide[:, L:] = np.arange(R)[None, :] > np.arange(R)[:, None]
        for h in range(cfg.n_q_heads):
            k, v = K[:, h // G], V[:, h // G]
            z = q[:, h] @ k.T * cfg.softmax_scale
            m = np.abs(q[:, h]) @ np.abs(k).T * cfg.softmax_scale
            z[hide], m[hide] = -np.inf, 0
            top = z.max(-1, keepdims=True)
            e = np.exp(z - top)
            lse[:, h] = top[:, 0] + np.log(e.sum(-1))
            p = e / e.sum(-1, keepdims=True)
            out[:, h], A[:, h], mag[:, h] = p @ v, p @ np.abs(v), m.max(-1)
        return out, lse, A, mag, L + R

    def check(self, out, lse, causal, seqs=None, keep=None):
        bf16 = self.cfg.dtype == "bf16"
        o, ls = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.isfinite(o).all() and np.isfinite(ls).all()
        for b in (range(self.S) if seqs is None else seqs):
            ref, rl, A, mag, n = self.reference(b, causal, keep)
            delta = (mag * (self.cfg.head_dim + 8) * 2.0 ** -23 + 2.0 ** -20)
            tol = (2 * delta[..., None] + n * 2.0 ** -23 + (2.0 ** -8 if bf16 else 0)) * A + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref)
            err = np.abs(o[b] - ref)
            assert (err <= tol).all(), (b, float((err / tol).max()), np.argwhere(err > tol)[:3].tolist())
            tl = delta + n * 2.0 ** -23 + 2.0 ** -21 * (1 + np.abs(rl))
            assert (np.abs(ls[b] - rl) <= tl).all(), (b, float((np.abs(ls[b] - rl) / tl).max()))


MODES = {"full": binding.ATTN_FULL, "causal": binding.ATTN_CAUSAL}
# (config, rows, group starts, prefix lengths, lengths)
CASES = [
    ("one_token", {}, 1, [0, 2], [64], [64, 65]),
    ("block", {}, 16, [0, 3], [200], [200, 263, 391]),
    ("no_groups", {}, 16, [0], [], [0, 1, 63, 64, 65, 127, 128, 129, 300]),
    ("prefix_inside_a_page", {}, 17, [0, 4], [131], [131, 132, 192, 500]),
    ("short_and_outside", {}, 8, [1, 4], [100], [70, 100, 99, 130, 260]),
    ("two_groups_and_an_empty_one", {}, 4, [0, 2, 2, 5], [300, 50, 0], [300, 420, 0, 17, 129]),
    ("nothing_cached", {}, 16, [0, 2], [0], [0, 0]),
    ("rows_fill_several_tiles", {}, 32, [0, 6], [640], [640, 641, 700, 704, 900, 1300]),
    ("one_head_a_group", dict(hq=8, hkv=8), 5, [0, 3], [150], [151, 150, 279]),
    ("seven_heads_a_group", dict(hq=28, hkv=4), 17, [0, 5], [333], [333, 400, 334, 461, 600]),
    ("five_heads_and_many_rows", dict(hq=20, hkv=4), 31, [0, 2], [77], [100, 205]),
    ("all_heads_a_group", dict(hq=128, hkv=1), 3, [0, 2], [130], [140, 266]),
    ("hd64", dict(hq=6, hkv=2, hd=64), 16, [0, 3], [500], [500, 513, 777]),
    ("page8", dict(hq=8, hkv=2, page=8), 16, [0, 3], [77], [77, 80, 203]),
    ("page16_hd64", dict(hq=16, hkv=4, hd=64, page=16), 10, [0, 2, 4], [300, 41], [301, 300, 41, 170]),
    ("page32", dict(hq=8, hkv=2, page=32), 2, [0, 2], [95], [96, 300]),
    ("page128", dict(hq=8, hkv=2, page=128), 16, [0, 2], [200], [260, 391]),
    ("page256", dict(hq=8, hkv=2, page=256), 16, [0, 2], [700], [701, 1000]),
    ("page4_bf16", dict(hq=8, hkv=2, page=4), 7, [0, 2], [30], [31, 100]),
    ("fp32_tiny", dict(hq=4, hkv=2, hd=64, dtype="fp32"), 8, [0, 3], [131], [131, 140, 221]),
    ("fp32_hd128", dict(hq=6, hkv=2, dtype="fp32", page=16), 17, [0, 2, 3], [70, 10], [70, 150, 9]),
    ("fp32_no_groups", dict(hq=4, hkv=4, hd=64, dtype="fp32", page=1), 1, [0], [], [0, 1, 70]),
]


@pytest.mark.parametrize("mode", ["full", "causal"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_matches_the_definition(case, mode):
    name, shape, rows, starts, prefix, lens = case
    cfg = config(**shape)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, rows, starts, prefix, lens, seed=len(name))
    out, lse = x.run(lib, MODES[mode])
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    x.check(out, lse, mode == "causal")


@pytest.mark.parametrize("shape,rows", [({}, 17), (dict(hq=20, hkv=4), 8), (dict(hq=7, hkv=1), 5), (dict(hq=6, hkv=2, hd=64), 31)])
def test_long_prefix_and_many_sequences_again_and_again_bit_for_bit(shape, rows):
    # with 5 or 7 heads a group the 128 rows of a query tile are not all used: what the others hold must not matter
    cfg = config(layers=1, **shape)
    lib = binding.DFlash(cfg)
    S = 24
    x = Batch(cfg, rows, [0, S], [5000], [5000 + 37 * b % 600 for b in range(S)], seed=3, layer=0)
    d = x.cuda()
    out, lse = x.run(lib, MODES["causal"], d)
    for k in range(20):
        if k % 4 == 3:                       # other work in between leaves other things in shared memory
            (torch.randn(2048, 2048, device="cuda:0") @ torch.randn(2048, 2048, device="cuda:0")).sum()
        again, lse2 = x.run(lib, MODES["causal"], d)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert int(lib.status.item()) == 0
    x.check(out, lse, True, seqs=(0, 7, S - 1))


@pytest.mark.parametrize("hq,hkv,rows,S,prefix,own", [(5, 1, 7, 9, 20000, 40), (7, 1, 3, 50, 12345, 700), (10, 2, 31, 5, 9001, 3), (3, 3, 32, 11, 6000, 0)])
def test_many_key_blocks_and_rows_that_straddle_query_tiles(hq, hkv, rows, S, prefix, own):
    # a prefix cut into dozens of blocks; neighbouring rows belong to different items, with different numbers of parts
    cfg = config(hq=hq, hkv=hkv, layers=1)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, rows, [0, S], [prefix], [prefix + own * b // S for b in range(S)], seed=S, layer=0)
    for mode in ("full", "causal"):
        out, lse = x.run(lib, MODES[mode])
        torch.cuda.synchronize()
        assert int(lib.status.item()) == 0
        x.check(out, lse, mode == "causal", seqs=(0, S // 2, S - 1))


@pytest.mark.parametrize("seed", range(16))
def test_random_batches(seed):
    r = random.Random(seed)
    hq, hkv, hd, page, dtype = r.choice([(32, 8, 128, 64, "bf16"), (8, 2, 128, 16, "bf16"), (12, 4, 64, 32, "bf16"), (10, 2, 128, 128, "bf16"),
                                         (8, 2, 64, 8, "bf16"), (4, 2, 64, 64, "fp32"), (5, 1, 128, 16, "fp32")])
    cfg = config(hq=hq, hkv=hkv, hd=hd, page=page, dtype=dtype)
    lib = binding.DFlash(cfg)
    S, rows = r.randint(1, 7), r.choice([1, 2, 7, 16, 17, 32])
    n = r.randint(0, 3)
    starts = sorted(r.randint(0, S) for _ in range(n + 1))
    prefix = [r.choice([0, 1, 63, 64, 127, 128, r.randint(0, 900)]) for _ in range(n)]
    lens = []
    for b in range(S):
        g = next((g for g in range(n) if starts[g] <= b < starts[g + 1]), -1)
        base = prefix[g] if g >= 0 and r.random() < 0.8 else 0
        lens.append(base + r.choice([0, 1, 62, 63, 64, 65, r.randint(0, 600)]))
    x = Batch(cfg, rows, starts, prefix, lens, seed=seed, q_std=r.choice([0.3, 1.0, 4.0]))
    for mode in ("full", "causal"):
        out, lse = x.run(lib, MODES[mode])
        torch.cuda.synchronize()
        assert int(lib.status.item()) == 0
        x.check(out, lse, mode == "causal")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nan_and_infinity_reach_the_rows_that_see_them_and_no_others(dtype):
    cfg = config(hq=8, hkv=2, hd=64, dtype=dtype, layers=1)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 4, [0, 3], [200], [200, 260, 150, 70], seed=31, layer=0)
    x.pool[0, int(x.table[0, 3]), 1, 0, 5, 7] = float("nan")          # value of position 197 of the prefix: kv head 0, element 7
    x.pool[0, int(x.table[1, 3]), 0, 1, 20, :] = float("nan")         # key of position 212 of sequence 1: kv head 1
    x.pool[0, int(x.table[3, 0]), 1, 1, 9, 3] = float("inf")          # value of position 9 of sequence 3: kv head 1, element 3
    x.k[2, 2, 0] = float("-inf")                                      # block key 2 of sequence 2: scores of both infinities, or NaN
    out, lse = x.run(lib, 1)
    torch.cuda.synchronize()
    o, l = out.float().cpu(), lse.cpu()
    bad = ~torch.isfinite(o)
    want = torch.zeros_like(bad)
    want[0, :, :4, 7] = True                                          # sequence 2 is shorter than the prefix and has its own pages
    want[1, :, :4, 7] = True
    want[1, :, 4:, :] = True
    want[3, :, 4:, 3] = True
    seen = x.q[2, 2:, :4].double() @ torch.full((64, 1), float("-inf"), dtype=torch.float64)
    want[2, 2:, :4] = ~torch.isfinite(seen) & ~(seen == float("-inf"))
    assert torch.equal(bad, want)
    assert torch.isnan(l[1, :, 4:]).all() and torch.isfinite(l[0]).all() and torch.isfinite(l[3]).all()


def test_two_handles_side_by_side():
    a, b = config(hq=8, hkv=2), config(hq=4, hkv=2, hd=64, dtype="fp32")
    la, lb = binding.DFlash(a), binding.DFlash(b)
    x, y = Batch(a, 16, [0, 3], [300], [300, 400, 500], seed=41), Batch(b, 8, [0, 2], [131], [131, 200], seed=42)
    dx, dy = x.cuda(), y.cuda()
    for _ in range(3):
        ox, oy = x.run(la, 1, dx), y.run(lb, 0, dy)
    torch.cuda.synchronize()
    x.check(*ox, True)
    y.check(*oy, False)


def test_contiguous_views_and_what_lies_around_them():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 3], [300], [300, 400, 500], seed=43)
    d = x.cuda()
    big = torch.full((5,) + tuple(d["q"].shape[1:]), 7.0, dtype=d["q"].dtype, device="cuda:0")
    q = torch.cat([d["q"][:1], d["q"], d["q"][:1]])                  # rows before and behind the batch
    out, lse = x.run(lib, 1, dict(d, q=q[1:4]), out=big[1:4])
    torch.cuda.synchronize()
    x.check(big[1:4], lse, True)
    assert bool((big[0] == 7).all()) and bool((big[4] == 7).all())


def test_scores_that_keep_growing():
    # the running maximum rises by far more than the kernel's gap in most tiles: the accumulator is rescaled each time
    cfg = config(hq=8, hkv=2, layers=1)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 2], [900], [1100, 1000], seed=5, q_std=8.0, layer=0)
    ramp = torch.linspace(0.1, 2.0, x.pages)
    x.pool = (x.pool.float() * ramp[torch.randperm(x.pages, generator=synth.substream(1, "r"))].view(1, -1, 1, 1, 1, 1)).to(cfg.torch_dtype)
    out, lse = x.run(lib, MODES["full"])
    torch.cuda.synchronize()
    x.check(out, lse, False)


def test_agrees_with_the_block_attention_of_single_sequences():
    cfg = synth.MID
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0], [], [0, 70, 200, 64], seed=9)
    d = x.cuda()
    out, lse = x.run(lib, MODES["full"], d)
    ref, rl = torch.empty_like(out), torch.empty_like(lse)
    lib.dflash_block_attention(MODES["full"], d["q"], d["k"], d["v"], d["lens"], x.bound, torch.where(d["table"] < 10 ** 6, d["table"], 0), d["pool"],
                               x.layer, ref, lse_out=rl)
    torch.cuda.synchronize()
    x.check(out, lse, False)
    x.check(ref, rl, False)


def test_bad_groups_are_flagged_and_read_unshared():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 4, [0], [], [100, 130, 70], seed=11)
    d = x.cuda()
    for starts in ([0, 2, 1, 3], [0, 4, 4, 4], [-1, 1, 2, 3]):
        lib.status.zero_()
        out, lse = torch.empty_like(d["q"]), torch.empty(d["q"].shape[:3], device="cuda:0")
        lib.dflash_prefix_attention(0, d["q"], d["k"], d["v"], torch.tensor(starts, dtype=torch.int32, device="cuda:0"),
                                    torch.tensor([64, 64, 64], dtype=torch.int32, device="cuda:0"), d["lens"], x.bound, d["table"], d["pool"], x.layer, out, lse_out=lse)
        torch.cuda.synchronize()
        assert int(lib.status.item()) == binding.DEV_BAD_GROUP
        x.check(out, lse, False)


@pytest.mark.parametrize("dtype,page", [("bf16", 64), ("bf16", 16), ("fp32", 64)])
def test_pages_outside_the_pool_are_left_out(dtype, page):
    cfg = config(hq=8, hkv=2, hd=64, page=page, dtype=dtype)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 4, [0, 2], [4 * page + 5], [5 * page, 6 * page + 1], seed=13)
    x.table[0, 1] = x.pages                 # in the prefix, for both sequences
    d = x.cuda()
    out, lse = x.run(lib, 0, d)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == binding.DEV_BAD_PAGE
    x.table[0, 1] = 0                       # the reference's gather needs some page there: its keys are dropped below
    for b in range(2):
        keep = np.ones(x.lens[b], dtype=bool)
        keep[page:2 * page] = False
        x.check(out, lse, False, seqs=(b,), keep=keep)


def test_a_length_above_the_bound_is_clamped_and_flagged():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 4, [0, 2], [100], [170, 300], seed=15)
    out, lse = x.run(lib, 0, bound=200)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == binding.DEV_CTX_OVERFLOW
    x.check(out, lse, False, seqs=(0,))
    x.lens[1] = 200
    x.check(out, lse, False, seqs=(1,))


def test_a_captured_call_follows_the_lengths_it_finds_and_shares_its_workspace():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 3], [300], [300, 400, 500], seed=17)
    y = Batch(cfg, 5, [0, 2], [129], [200, 150], seed=18)
    dx, dy = x.cuda(), y.cuda()
    x.run(lib, 1, dx)
    y.run(lib, 0, dy)
    torch.cuda.synchronize()
    outs = []
    graphs = []
    for b, d, mode in ((x, dx, 1), (y, dy, 0)):
        out, lse = torch.zeros_like(d["q"]), torch.zeros(d["q"].shape[:3], device="cuda:0")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.run(lib, mode, d, out, lse)
        graphs.append(g)
        outs.append((out, lse))
    big = Batch(config(hq=8, hkv=2), 32, [0, 40], [10], [12] * 40, seed=19)         # the workspace grows: the graphs keep theirs
    big.run(lib, 0)
    for _ in range(2):
        graphs[0].replay()
        graphs[1].replay()
    torch.cuda.synchronize()
    x.check(*outs[0], True)
    y.check(*outs[1], False)
    # other lengths and another grouping under the same graph
    x.lens, x.prefix, x.starts = [300, 290, 256], [40], [1, 3]
    x.group, x.shared = [-1, 0, 0], [0, 40, 40]
    own = torch.from_numpy(x.table.copy())
    own[1, :5] = own[0, :5]
    own[2, :5] = own[0, :5]
    x.table = own.numpy()
    dx["table"].copy_(own)
    for name, v in (("lens", x.lens), ("prefix", x.prefix), ("starts", x.starts)):
        dx[name].copy_(torch.tensor(v, dtype=torch.int32))
    graphs[0].replay()
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    x.check(*outs[0], True)


def test_another_stream_and_no_lse():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 3], [300], [300, 400, 500], seed=21)
    d = x.cuda()
    ref, lse = x.run(lib, 1, d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(ref)
    lib.dflash_prefix_attention(1, d["q"], d["k"], d["v"], d["starts"], d["prefix"], d["lens"], x.bound, d["table"], d["pool"], x.layer, out, stream=s)
    s.synchronize()
    assert torch.equal(out, ref)
    x.check(out, lse, True)


def test_offsets_past_32_bits():
    # a pool of 70000 pages (9.2e9 elements), the used ones at its end
    cfg = config(layers=1)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 2], [150], [200, 161], seed=23, layer=0)
    d = x.cuda()
    pages, shift = 70000, 70000 - x.pages
    pool = torch.empty(synth.kv_pool_shape(cfg, pages), dtype=cfg.torch_dtype, device="cuda:0")
    pool[:, shift:] = d["pool"]
    d["pool"] = pool
    d["table"] = torch.where(d["table"] < 10 ** 6, d["table"] + shift, d["table"])
    out, lse = x.run(lib, 1, d)
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    x.check(out, lse, True)


def test_refusals_leave_the_output_alone():
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    x = Batch(cfg, 16, [0, 2], [100], [100, 120], seed=25)
    d = x.cuda()
    out = torch.full_like(d["q"], 7.0)
    for bad in (dict(mode=2), dict(layer=2), dict(bound=-1)):
        with pytest.raises(binding.DFlashError) as e:
            lib.dflash_prefix_attention(bad.get("mode", 0), d["q"], d["k"], d["v"], d["starts"], d["prefix"], d["lens"], bad.get("bound", 200), d["table"],
                                        d["pool"], bad.get("layer", 0), out)
        assert e.value.code == -1
    for wrong in (dict(lens=d["lens"].long()), dict(q=d["q"].transpose(0, 1)), dict(pool=d["pool"].float()), dict(starts=d["starts"][:2].repeat(2))):
        a = dict(d, **wrong)
        with pytest.raises(AssertionError):
            lib.dflash_prefix_attention(0, a["q"], a["k"], a["v"], a["starts"], a["prefix"], a["lens"], 200, a["table"], a["pool"], 0, out)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_calls_on_two_streams_and_graphs_of_two_streams_overlap():
    """Eager calls on two streams have a workspace each, as have captured calls: they may run at once, in any order."""
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    batches = [Batch(cfg, 16, [0, 6], [1500], [1600 + 10 * i for i in range(6)], seed=31), Batch(cfg, 7, [1, 5], [700], [900, 1400, 800, 701, 2500], seed=32)]
    data = [b.cuda() for b in batches]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = [b.run(lib, 1, d) for b, d in zip(batches, data)]
    outs = [(torch.zeros_like(o), torch.zeros_like(l)) for o, l in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, d, o, s in zip(batches, data, outs, streams):
            b.run(lib, 1, d, *o, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
    graphs = []
    for b, d, o in zip(batches, data, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(10):
                b.run(lib, 1, d, *o)
        graphs.append(g)
    for o in outs:
        o[0].zero_()
        o[1].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        batches[0].run(lib, 1, data[0], *[torch.empty_like(t) for t in outs[0]])
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    for b, o, w in zip(batches, outs, want):
        assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
        b.check(*o, True)


@pytest.mark.parametrize("S,groups,dtype", [(600, 300, "bf16"), (400, 200, "bf16"), (530, 0, "bf16"), (700, 650, "bf16"), (1100, 3, "fp32")])
def test_more_sequences_and_groups_than_the_plan_keeps_in_shared_memory(S, groups, dtype):
    cfg = config(hq=4, hkv=2, hd=64, page=16, dtype=dtype, layers=1)
    lib = binding.DFlash(cfg)
    r = random.Random(S)
    starts = sorted(r.randint(0, S) for _ in range(groups + 1))
    prefix = [r.choice([0, 5, 16, 40, 70]) for _ in range(groups)]
    lens = []
    for b in range(S):
        g = next((g for g in range(groups) if starts[g] <= b < starts[g + 1]), -1)
        lens.append((prefix[g] if g >= 0 and r.random() < 0.9 else 0) + r.choice([0, 1, 15, 60, 90]))
    lens[S // 2] += 3000
    x = Batch(cfg, 3, starts, prefix, lens, seed=S, layer=0)
    out, lse = x.run(lib, MODES["causal"])
    torch.cuda.synchronize()
    assert int(lib.status.item()) == 0
    x.check(out, lse, True, seqs=[0, 1, S // 2 - 1, S // 2, S - 1] + [r.randrange(S) for _ in range(25)])


FIRST_CALL = """
import torch
from paper_2602_06036_b200 import binding
from tests.test_prefix_attention_gpu import Batch, config
cfg = config(hq=8, hkv=2)
lib = binding.DFlash(cfg)
x = Batch(cfg, 5, [0, 2], [100], [130, 161], seed=3)
d = x.cuda()
out, lse = torch.zeros_like(d["q"]), torch.zeros(d["q"].shape[:3], device="cuda:0")
ref = torch.zeros(x.pages, dtype=torch.int32, device="cuda:0")
one = torch.ones(1, dtype=torch.int32, device="cuda:0")
table = torch.full((3, 2), -1, dtype=torch.int32, device="cuda:0")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    x.run(lib, 1, d, out, lse)
    lib.dflash_pages_resize(one, one, one + 69, table, ref, torch.zeros_like(d["pool"]))      # a kept position without a page: left out
    lib.dflash_pages_resize(one, one - 1, one + 69, table, ref, torch.zeros_like(d["pool"]))
g.replay()
torch.cuda.synchronize()
x.check(out, lse, True)
assert table.tolist() == [[-1, -1], [0, 1], [-1, -1]] and int(ref.sum()) == 2 and int(lib.status.item()) == binding.DEV_BAD_PAGE
"""


def test_a_process_may_begin_with_a_captured_call():
    import subprocess
    import sys
    from pathlib import Path
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=Path(__file__).resolve().parents[1], capture_output=True, text=True, timeout=180)
    assert r.returncode == 0, r.stderr[-2000:]


def test_two_threads_with_one_handle():
    import threading
    cfg = config(hq=8, hkv=2)
    lib = binding.DFlash(cfg)
    batches = [Batch(cfg, 16, [0, 6], [800], [900 + 10 * i for i in range(6)], seed=51), Batch(cfg, 7, [1, 5], [700], [900, 1400, 800, 701, 1500], seed=52)]
    data = [b.cuda() for b in batches]
    want = [b.run(lib, 1, d) for b, d in zip(batches, data)]
    torch.cuda.synchronize()
    same, go = [[], []], threading.Barrier(2)

    def work(i):
        go.wait()
        outs = [batches[i].run(lib, 1, data[i]) for _ in range(60)]
        torch.cuda.synchronize()
        same[i] += [torch.equal(o, want[i][0]) and torch.equal(l, want[i][1]) for o, l in outs]

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert same == [[True] * 60] * 2
    assert int(lib.status.item()) == 0
