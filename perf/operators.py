"""Cases of the operators on a shared paged KV cache: block attention of a batch that shares long prefixes, and the
page operations (copy, fork, resize, compact) that make and keep such a cache.

`run` computes a case in elementary torch operations, or, with `own` set, by the calls a serving program makes of
this library. The shapes are those of the framework's drafter (32 query heads on 8 kv heads of 128, 64-token pages, blocks
of 16 rows, 17 verify rows, contexts up to 32768) and of its tiny fp32 configuration, with odd relatives of both.
"""
import torch

own = False

KIND = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
NEG = float("-inf")


def listed():
    big = dict(layers=5, hkv=8, hd=128, page=64, dtype="bf16")
    return [
        # a handful of short chats behind one system prompt on the tiny fp32 drafter: latency only
        dict(name="attn_tiny_fp32", op="attn", dtype="fp32", hq=4, hkv=2, hd=64, page=64, seqs=4, rows=8, groups=1, prefix=131,
             own=90, causal=False, short=False, loose=False),
        # plain decoding (one token a sequence) of 32 sequences behind an 8k system prompt
        dict(name="attn_decode", op="attn", dtype="bf16", hq=32, hkv=8, hd=128, page=64, seqs=32, rows=1, groups=1, prefix=8192,
             own=1500, causal=True, short=False, loose=False),
        # draft blocks of a head_dim-64 model on 16-token pages, two prompts, prefixes that end inside a page
        dict(name="attn_draft_hd64", op="attn", dtype="bf16", hq=16, hkv=4, hd=64, page=16, seqs=10, rows=16, groups=2, prefix=4003,
             own=700, causal=False, short=False, loose=True),
        # verify rows (16 drafts and the anchor) of the serving batch behind one long document
        dict(name="attn_verify", op="attn", dtype="bf16", hq=32, hkv=8, hd=128, page=64, seqs=32, rows=17, groups=1, prefix=32768,
             own=1000, causal=True, short=False, loose=False),
        # a second pool follows three copied pages of the tiny drafter, the last of them partly filled
        dict(name="copy_small", op="copy", layers=1, hkv=2, hd=64, page=64, dtype="fp32", pages=40, n=3, part=True),
        # 512 pages of the drafter's pool moved for a defragmentation or a hand-over
        dict(name="copy_large", op="copy", n=512, pages=1100, part=False, **big),
        # one prompt answered by four samples
        dict(name="fork_small", op="fork", parents=1, fanout=4, len=700, **big),
        # sixteen 32k documents, four continuations each, in a pool of one layer
        dict(name="fork_large", op="fork", parents=16, fanout=4, len=32768, layers=1, hkv=8, hd=128, page=64, dtype="bf16"),
        # room for the next block of 17 rows of eight sequences, every fourth of them a fork that still shares its last page
        dict(name="resize_step", op="resize", rows=8, len=1000, grow=17, freed=0, shared=2, **big),
        # end of a burst: 256 sequences, a third of them released, the others extended by 1k tokens, 32 pairs sharing pages
        dict(name="resize_batch", op="resize", rows=256, len=4096, grow=1024, freed=80, shared=64, layers=1, hkv=8, hd=128, page=64,
             dtype="bf16"),
        # a small pool after a few sequences have left
        dict(name="compact_small", op="compact", pages=200, live=90, moves=37, rows=12, layers=1, hkv=2, hd=128, page=64, dtype="bf16"),
        # the drafter's pool at half load, half of what lives lies behind the border
        dict(name="compact_large", op="compact", pages=2048, live=1024, moves=500, rows=64, **big),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["attn"] * 6 + ["copy", "copy", "fork", "fork", "resize", "resize", "compact", "compact"])
    if op == "attn":
        dtype = "fp32" if rng.random() < 0.15 else "bf16"
        hq, hkv, hd = rng.choice([(32, 8, 128), (32, 8, 128), (8, 8, 128), (28, 4, 128), (20, 4, 128), (64, 8, 128), (16, 4, 64), (6, 2, 64)])
        c = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, hd=hd, page=rng.choice([64, 64, 64, 16, 32, 128, 8, 256]), seqs=_log(rng, 1, 48),
                 rows=rng.choice([1, 1, 2, 5, 8, 10, 16, 16, 17, 31, 32]), groups=1, prefix=_log(rng, 1, 32768), own=_log(rng, 1, 3000),
                 causal=rng.random() < 0.5, short=rng.random() < 0.15, loose=rng.random() < 0.2)
        c["groups"] = rng.randint(1, min(3, c["seqs"]))
        most = 2.0e11 if dtype == "bf16" else 4.0e9
        while work(c)["flops"] > most:
            c["prefix"], c["seqs"], c["own"] = max(1, c["prefix"] * 2 // 3), max(c["groups"], c["seqs"] * 3 // 4), max(1, c["own"] * 3 // 4)
        return c
    layers, hkv, hd, page = rng.choice([(1, 2, 64, 64), (2, 2, 128, 64), (5, 8, 128, 64), (3, 4, 64, 16), (1, 8, 128, 128), (4, 2, 128, 8)])
    c = dict(op=op, layers=layers, hkv=hkv, hd=hd, page=page, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if op == "copy":
        n = _log(rng, 1, 250)
        return dict(c, n=n, pages=2 * n + rng.randint(0, 100), part=rng.random() < 0.5)
    if op == "fork":
        return dict(c, parents=_log(rng, 1, 12), fanout=rng.randint(1, 5), len=_log(rng, 1, 1500) * page // 8 + rng.randint(0, page))
    if op == "resize":
        rows = _log(rng, 2, 100)
        return dict(c, rows=rows, len=_log(rng, 8, 2000) * page // 64 + rng.randint(1, page), grow=_log(rng, 1, 1500) * page // 64 + 1,
                    freed=rng.randint(0, rows // 2), shared=2 * rng.randint(0, rows // 4))
    pages = _log(rng, 8, 1500)
    live = rng.randint(1, pages - 1)
    return dict(c, pages=pages, live=live, moves=rng.randint(0, min(live, pages - live)), rows=_log(rng, 1, 64))


# ---- what a case's sizes say (nothing here depends on the seed) -----------------------------------------------

def _spread(i, most):
    """A length in 0..most for the i-th sequence, scattered over the range."""
    return (i * 2654435761 + 40503) % 65521 * (most + 1) // 65521


def _groups(c):
    """First sequence of each group, and the end of the last one: near-equal runs; `loose` leaves the last sequence out."""
    n = c["seqs"] - (1 if c["loose"] and c["seqs"] > c["groups"] else 0)
    return [n * g // c["groups"] for g in range(c["groups"] + 1)]


def _attn_lens(c):
    """(prefix length of each group, cached length of each sequence, group of each sequence or -1)."""
    start = _groups(c)
    prefix = [max(1, c["prefix"] - 17 * g) for g in range(c["groups"])]
    lens, of = [], []
    for b in range(c["seqs"]):
        g = next((g for g in range(c["groups"]) if start[g] <= b < start[g + 1]), -1)
        of.append(g)
        tail = _spread(b, c["own"])
        lens.append(tail if g < 0 else prefix[g] + tail)
    if c["short"] and of[-1] >= 0:
        lens[-1] = prefix[of[-1]] // 2        # a sequence that has not got as far as its group's prefix
    return prefix, lens, of


def _fork_lens(c):
    return [max(1, c["len"] - 37 * p % (c["len"] // 4 + 1)) for p in range(c["parents"])]


def _resize_lens(c):
    """(length, new capacity) of each row: the last `freed` rows are released, the others get room for `grow` more."""
    out = []
    for i in range(c["rows"]):
        n = max(1, c["len"] - _spread(i // 2 if i < c["shared"] else i, c["len"] // 2))
        out.append((0, 0) if i >= c["rows"] - c["freed"] else (n, n + c["grow"]))
    return out


def _page_bytes(c):
    return c["layers"] * 2 * c["hkv"] * c["page"] * c["hd"] * SIZE[c["dtype"]]


def work(c):
    if c["op"] == "attn":
        prefix, lens, of = _attn_lens(c)
        rows = c["seqs"] * c["rows"]
        own_keys = sum(L if g < 0 or L < prefix[g] else L - prefix[g] for L, g in zip(lens, of))
        keys = own_keys + sum(prefix[g] for g in set(of) if g >= 0)
        block = c["seqs"] * (c["rows"] * (c["rows"] + 1) // 2 if c["causal"] else c["rows"] * c["rows"])
        seen = c["rows"] * sum(lens) + block
        es = SIZE[c["dtype"]]
        return {"bytes": es * c["hd"] * (2 * rows * c["hq"] + 2 * (rows + keys) * c["hkv"]) + 4 * rows * c["hq"],
                "flops": 4 * c["hd"] * c["hq"] * seen}
    pb, ps = _page_bytes(c), c["page"]
    if c["op"] == "copy":
        return {"bytes": sum(2 * pb * s // ps for s in _copy_slots(c)) + 12 * c["n"], "flops": 0}
    if c["op"] == "fork":
        lens = _fork_lens(c)
        entries = sum(-(-n // ps) for n in lens)
        return {"bytes": c["fanout"] * sum(2 * pb * (n % ps) // ps for n in lens) + 4 * entries * (1 + c["fanout"]) + 8 * entries, "flops": 0}
    if c["op"] == "resize":
        lens = _resize_lens(c)
        cow = sum(2 * pb * (n % ps) // ps for i, (n, _) in enumerate(lens) if i < c["shared"] and n)
        return {"bytes": cow + 8 * c["rows"] * _resize_width(c) + 8 * _resize_pages(c), "flops": 0}
    return {"bytes": 2 * pb * c["moves"] + 8 * c["pages"] + 8 * c["rows"] * _compact_width(c), "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(c, g, layers, pages):
    return _normal(g, layers, pages, 2, c["hkv"], c["page"], c["hd"], dtype=KIND[c["dtype"]])


def prepare(case, seed):
    c, g = case, _gen(seed)
    return {"attn": _prepare_attn, "copy": _prepare_copy, "fork": _prepare_fork, "resize": _prepare_resize, "compact": _prepare_compact}[c["op"]](c, g)


def _prepare_attn(c, g):
    S, R, ps, hd = c["seqs"], c["rows"], c["page"], c["hd"]
    prefix, lens, of = _attn_lens(c)
    start = _groups(c)
    width = max(1, max(-(-max(L, prefix[x] if x >= 0 else 0) // ps) for L, x in zip(lens, of)))
    table = torch.full((S, width), -1, dtype=torch.int64)
    used, partial = 0, []
    for b in range(S):                       # whole pages of a prefix are shared, everything behind them is a sequence's own
        x = of[b]
        share = prefix[x] // ps if x >= 0 and b > start[x] else 0
        have = -(-max(lens[b], prefix[x] if x >= 0 and b == start[x] else 0) // ps)
        share = min(share, lens[b] // ps)
        if share:
            table[b, :share] = table[start[x], :share]
        table[b, share:have] = torch.arange(used, used + have - share)
        if x >= 0 and b > start[x] and prefix[x] % ps and lens[b] >= prefix[x]:
            partial.append((b, start[x], prefix[x] // ps, prefix[x] % ps))
        used += max(0, have - share)
    pages = used + 2
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(int(torch.randint(1 << 30, (1,), generator=g, device="cuda"))))
    table = torch.where(table >= 0, perm[table.clamp(min=0)], torch.full_like(table, -1))
    pool = _pool(c, g, 1, pages)
    for b, lead, j, n in partial:            # a fork's copy of a page that the prefix fills in part
        pool[:, int(table[b, j]), :, :, :n] = pool[:, int(table[lead, j]), :, :, :n]
    dt = KIND[c["dtype"]]
    q = _normal(g, S, R, c["hq"], hd, dtype=dt)
    k, v = (_normal(g, S, R, c["hkv"], hd, dtype=dt) for _ in range(2))
    return {"case": c, "pool": pool, "q": q, "k": k, "v": v, "table": table.to(torch.int32).cuda(), "len": _ints(lens), "max_len": max(lens + prefix),
            "group_start": _ints(start), "prefix": _ints(prefix), "out": torch.empty_like(q),
            "lse": torch.empty((S, R, c["hq"]), dtype=torch.float32, device="cuda")}


def _copy_slots(c):
    return [1 + _spread(i, c["page"] - 1) if c["part"] else c["page"] for i in range(c["n"])]


def _prepare_copy(c, g):
    ids = torch.randperm(c["pages"], generator=g, device="cuda").to(torch.int32)
    return {"case": c, "pool": _pool(c, g, c["layers"], c["pages"]), "src": ids[:c["n"]].contiguous(), "dst": ids[c["n"]:2 * c["n"]].contiguous(),
            "slots": _ints(_copy_slots(c))}


def _counted(table, pages):
    """How many table entries hold each page."""
    flat = table.reshape(-1).long()
    return torch.zeros(pages + 1, dtype=torch.int32).scatter_add_(0, torch.where(flat >= 0, flat, pages), torch.ones_like(flat, dtype=torch.int32))[:pages]


def _scattered(table, pages, g):
    """Physical pages in place of 0, 1, ..., and the reference counts that go with them, both on the GPU."""
    perm = torch.randperm(pages, generator=g, device="cuda").cpu()
    table = torch.where(table >= 0, perm[table.clamp(min=0)], torch.full_like(table, -1)).to(torch.int32)
    return table.cuda(), _counted(table, pages).cuda()


def _prepare_fork(c, g):
    ps, lens, f = c["page"], _fork_lens(c), c["fanout"]
    width = max(-(-n // ps) for n in lens) + 1
    table = torch.full((c["parents"] * (1 + f), width), -1, dtype=torch.int64)
    used = 0
    for p, n in enumerate(lens):
        have = -(-n // ps)
        table[p, :have] = torch.arange(used, used + have)
        used += have
    parent = [p for p in range(c["parents"]) for _ in range(f)]
    pages = used + len(parent) + 3
    table, ref = _scattered(table, pages, g)
    return {"case": c, "pool": _pool(c, g, c["layers"], pages), "table": table, "ref": ref, "parent": _ints(parent),
            "child": _ints([c["parents"] + i for i in range(len(parent))]), "len": _ints([lens[p] for p in parent])}


def _resize_width(c):
    return max(-(-cap // c["page"]) for _, cap in _resize_lens(c) + [(0, c["len"])]) + 1


def _resize_pages(c):
    ps, lens = c["page"], _resize_lens(c)
    return sum(-(-max(cap, c["len"] if cap == 0 else 0) // ps) + 1 for _, cap in lens) + c["shared"] + 3


def _prepare_resize(c, g):
    ps, lens = c["page"], _resize_lens(c)
    table = torch.full((c["rows"], _resize_width(c)), -1, dtype=torch.int64)
    used = 0
    for i, (n, cap) in enumerate(lens):
        have = -(-(n if cap else c["len"]) // ps)
        if i < c["shared"] and i % 2 and cap:           # rows 2k and 2k+1 hold the same pages, the partly filled one among them
            table[i, :have] = table[i - 1, :have]
            continue
        table[i, :have] = torch.arange(used, used + have)
        used += have
    pages = _resize_pages(c)
    table, ref = _scattered(table, pages, g)
    order = torch.randperm(c["rows"], generator=g, device="cuda")
    n, cap = (_ints([x[k] for x in lens])[order].contiguous() for k in (0, 1))
    return {"case": c, "pool": _pool(c, g, c["layers"], pages), "table": table, "ref": ref, "rows": order.to(torch.int32), "len": n, "cap": cap}


def _compact_width(c):
    return -(-c["live"] // c["rows"]) + 4


def _prepare_compact(c, g):
    pages, live, moves, S = c["pages"], c["live"], c["moves"], c["rows"]
    front = torch.randperm(live, generator=g, device="cuda").cpu()[:live - moves]
    behind = live + torch.randperm(pages - live, generator=g, device="cuda").cpu()[:moves]
    ids = torch.cat([front, behind])[torch.randperm(live, generator=g, device="cuda").cpu()]
    width = _compact_width(c)
    table = torch.full((S, width), -1, dtype=torch.int64)
    at = torch.arange(live)
    table[at % S, at // S + 1] = ids
    table[:, 0] = ids[0]                                  # one page that every row shares
    table = table.to(torch.int32)
    return {"case": c, "pool": _pool(c, g, c["layers"], pages), "table": table.cuda(), "ref": _counted(table, pages).cuda()}


# ---- one pass -------------------------------------------------------------------------------------------------

def run(state):
    return {"attn": _attn, "copy": _copy, "fork": _fork, "resize": _resize, "compact": _compact}[state["case"]["op"]](state)


_handles = {}


def _handle(c, layers):
    """The library handle of a shape: a program keeps one for its drafter."""
    from paper_2602_06036_b200 import binding, synth
    key = (layers, c.get("hq", c["hkv"]), c["hkv"], c["hd"], c["page"], c["dtype"])
    if key not in _handles:
        _handles[key] = binding.DFlash(synth.DFlashConfig(n_layers=layers, d_model=256, n_q_heads=key[1], n_kv_heads=key[2], head_dim=key[3],
                                                          d_ffn=256, vocab=256, n_feat_layers=1, d_target=256, block_size=16,
                                                          dtype=c["dtype"], page_size=key[4]))
    return _handles[key]


def _attn(s):
    c = s["case"]
    if own:
        _handle(c, 1).dflash_prefix_attention(1 if c["causal"] else 0, s["q"], s["k"], s["v"], s["group_start"], s["prefix"], s["len"], s["max_len"],
                                              s["table"], s["pool"], 0, s["out"], lse_out=s["lse"])
        return s["out"], s["lse"]
    S, R, hkv, hd, ps = c["seqs"], c["rows"], c["hkv"], c["hd"], c["page"]
    G, L = c["hq"] // hkv, s["max_len"]
    dev = s["q"].device
    b, pos = torch.arange(S, device=dev), torch.arange(L, device=dev)
    x = torch.searchsorted(s["group_start"], b.to(torch.int32), right=True) - 1          # group of a sequence
    inside = (x >= 0) & (x < c["groups"])
    x = x.clamp(0, c["groups"] - 1)
    n = torch.where(inside & (s["len"] >= s["prefix"][x]), s["prefix"][x], 0)
    lead = torch.where(inside, s["group_start"][x], 0).long()
    j = (pos // ps).clamp(max=s["table"].shape[1] - 1)
    page = torch.where(pos < n[:, None], s["table"][lead][:, j], s["table"][:, j]).long()          # [S, L]
    seen = pos < s["len"][:, None]
    page = torch.where(seen, page, 0)
    kv = s["pool"][0]
    slot = (pos % ps)[None, :].expand(S, L)
    keys = torch.cat([kv[page, 0, :, slot], s["k"]], 1).float().permute(0, 2, 3, 1)                # [S, Hkv, hd, L + R]
    q = s["q"].float().view(S, R, hkv, G, hd).permute(0, 2, 1, 3, 4).reshape(S, hkv, R * G, hd)
    z = torch.matmul(q, keys).view(S, hkv, R, G, L + R) * hd ** -0.5
    del keys
    r = torch.arange(R, device=dev)
    tail = (r[None, :] <= r[:, None]) if c["causal"] else torch.ones(R, R, dtype=torch.bool, device=dev)
    mask = torch.cat([seen[:, None].expand(S, R, L), tail[None].expand(S, R, R)], 2)[:, None, :, None]
    z = z.masked_fill_(~mask, NEG)
    m = z.amax(-1, keepdim=True)
    z = z.sub_(m).exp_()
    total = z.sum(-1, keepdim=True)
    values = torch.cat([kv[page, 1, :, slot], s["v"]], 1).float()
    values = torch.where(torch.cat([seen, torch.ones(S, R, dtype=torch.bool, device=dev)], 1)[:, :, None, None], values, 0.0)
    out = torch.matmul(z.view(S, hkv, R * G, L + R), values.permute(0, 2, 1, 3)).view(S, hkv, R, G, hd) / total
    lse = (m + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(S, R, c["hq"])
    return out.permute(0, 2, 1, 3, 4).reshape(S, R, c["hq"], hd).to(s["q"].dtype), lse


def _copy_pages(pool, src, dst, slots):
    """The first slots[i] slots of page src[i] over those of page dst[i], in every layer, K and V and every head."""
    first = (torch.arange(pool.shape[4], device=pool.device) < slots[:, None]).view(1, len(src), 1, 1, -1, 1)
    pool[:, dst] = torch.where(first, pool[:, src], pool[:, dst])


def _copy_where(pool, do, src, dst, slots):
    """_copy_pages of the entries that `do` marks: the others repeat the first of them, or copy nothing."""
    first = torch.argmax(do.int())
    src, dst, slots = (torch.where(do, a, a[first]) for a in (src, dst, slots))
    _copy_pages(pool, src, dst, torch.where(do.any(), slots, 0))


def _copy(s):
    if own:
        c = s["case"]
        _handle(c, c["layers"]).dflash_pages_copy(s["src"], s["dst"], s["pool"], n_slots=s["slots"])
    else:
        _copy_pages(s["pool"], s["src"].long(), s["dst"].long(), s["slots"])
    return s["pool"]


def _free_pages(ref):
    """Free pages by rising index, in a list as long as the pool (its end holds nothing of use)."""
    free = ref == 0
    rank = torch.where(free, torch.cumsum(free, 0) - 1, len(ref))
    return torch.zeros(len(ref) + 1, dtype=torch.int64, device=ref.device).scatter_(0, rank, torch.arange(len(ref), device=ref.device))[:len(ref)]


def _fork(s):
    table, ref, pool = s["table"].clone(), s["ref"].clone(), s["pool"]      # the pass starts from the same cache each time
    if own:
        c = s["case"]
        _handle(c, c["layers"]).dflash_pages_fork(s["parent"], s["child"], s["len"], table, ref, pool)
        return table, ref, pool
    ps = pool.shape[4]
    j = torch.arange(table.shape[1], device=table.device)
    whole, rest = s["len"][:, None] // ps, s["len"] % ps
    rows = table[s["parent"].long()]
    shared = j < whole
    need = rest > 0
    fresh = _free_pages(ref)[torch.cumsum(need, 0) - need.long()]
    last = rows.gather(1, whole.long().clamp(max=table.shape[1] - 1)).squeeze(1).long()
    table[s["child"].long()] = torch.where(shared, rows, torch.where((j == whole) & need[:, None], fresh[:, None].int(), -1))
    ref.scatter_add_(0, torch.where(shared, rows, 0).reshape(-1).long(), shared.reshape(-1).int())
    ref.scatter_add_(0, fresh, need.int())
    _copy_where(pool, need, last, fresh, rest)
    return table, ref, pool


def _resize(s):
    table, ref, pool = s["table"].clone(), s["ref"].clone(), s["pool"]
    if own:
        c = s["case"]
        _handle(c, c["layers"]).dflash_pages_resize(s["rows"], s["len"], s["cap"], table, ref, pool)
        return table, ref, pool
    ps = pool.shape[4]
    j = torch.arange(table.shape[1], device=table.device)
    rows = table[s["rows"].long()].long()
    held = rows >= 0
    want = -(-s["cap"][:, None] // ps)
    first = s["len"][:, None] // ps                                            # the page that the next position falls into
    shared = held & (ref[rows.clamp(min=0)] > 1) & (j >= first) & (s["len"] < s["cap"])[:, None]
    need = (j < want) & (~held | shared)
    rank = torch.cumsum(need.reshape(-1), 0).view_as(rows) - 1
    fresh = _free_pages(ref)[rank.clamp(min=0)]
    drop = held & ((j >= want) | need)
    edge = first.clamp(max=table.shape[1] - 1)
    kept = (need & held).gather(1, edge).squeeze(1) & (s["len"] % ps > 0)
    dst = fresh.gather(1, edge).squeeze(1)
    src = rows.gather(1, edge).squeeze(1)
    table[s["rows"].long()] = torch.where(need, fresh, torch.where(j < want, rows, -1)).int()
    ref.scatter_add_(0, torch.where(drop, rows, 0).reshape(-1), -drop.reshape(-1).int())
    ref.scatter_add_(0, torch.where(need, fresh, 0).reshape(-1), need.reshape(-1).int())
    _copy_where(pool, kept, src, dst, s["len"] % ps)
    return table, ref, pool


def _compact(s):
    table, ref, pool = s["table"].clone(), s["ref"].clone(), s["pool"]
    if own:
        c = s["case"]
        n_live = torch.empty(1, dtype=torch.int32, device=table.device)
        _handle(c, c["layers"]).dflash_pages_compact(table, ref, pool, n_live=n_live)
        return table, ref, pool, n_live
    n = len(ref)
    at = torch.arange(n, device=ref.device)
    live = ref > 0
    n_live = live.sum()
    hole, mover = ~live & (at < n_live), live & (at >= n_live)
    count = hole.sum()
    most = n // 2
    # the i-th hole takes the i-th page behind the border, both by rising index
    dst, src = (torch.argsort(torch.where(x, at, at + n))[:most] for x in (hole, mover))
    pair = at[:most] < count
    to = torch.cat([at, at[:1]]).scatter_(0, torch.where(pair, src, n), dst)
    _copy_where(pool, pair, src, dst, torch.full_like(src, pool.shape[4]))
    table = torch.where(table >= 0, to[table.clamp(min=0).long()], -1).int()
    new = torch.cat([ref, ref[:1]])
    new.scatter_(0, torch.where(pair, src, n), torch.zeros_like(ref)[:most])
    new = new.scatter_(0, torch.where(pair, dst, n), ref[src])[:n]
    return table, new, pool, n_live.int().reshape(1)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    """Attention one sequence at a time over the list of its keys; page operations compute no numbers."""
    c = case
    if c["op"] != "attn":
        return None
    s = prepare(c, seed)
    prefix, lens, of = _attn_lens(c)
    start, ps, R, G = _groups(c), c["page"], c["rows"], c["hq"] // c["hkv"]
    table = s["table"].cpu().tolist()
    outs, lses = [], []
    for b in range(c["seqs"]):
        own_from = prefix[of[b]] if of[b] >= 0 and lens[b] >= prefix[of[b]] else 0
        where = [table[start[of[b]] if p < own_from else b][p // ps] * ps + p % ps for p in range(lens[b])]
        where = torch.tensor(where, dtype=torch.int64, device="cuda")
        out, lse = [], []
        for h in range(c["hkv"]):
            k, v = (torch.cat([s["pool"][0, :, i, h].reshape(-1, c["hd"])[where].double(), new[b, :, h].double()]) for i, new in ((0, s["k"]), (1, s["v"])))
            for qh in range(h * G, (h + 1) * G):
                z = s["q"][b, :, qh].double() @ k.T / c["hd"] ** 0.5
                if c["causal"]:
                    z[:, lens[b]:] += torch.triu(torch.full((R, R), NEG, dtype=torch.float64, device="cuda"), 1)
                lse.append(torch.logsumexp(z, 1))
                out.append(torch.exp(z - lse[-1][:, None]) @ v)
        outs.append(torch.stack(out, 1))
        lses.append(torch.stack(lse, 1))
    return torch.stack(outs), torch.stack(lses)
