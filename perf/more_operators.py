"""Cases of the operators on logits and weights: log probabilities of given tokens with entropy and top alternatives,
their gradient, and the AdamW step over many tensors.

`run` computes a case in elementary torch operations, or, with `own` set, by the calls that a serving or training program
makes of this library. Sizes are those of the framework's configurations (vocabularies of 151936, 32000, 5003 and 1024, blocks of 16
rows and 17 verify rows, 512 anchor blocks a sequence, the weights of the five-layer drafter and of the tiny one), with
odd relatives of them.
"""
import torch

own = False

KIND = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}
NEG = float("-inf")
BLOCK = 128                       # elements of an 8-bit state that share a scale
E4M3 = torch.float8_e4m3fn
BETA1, BETA2, EPS, LR, MAX_NORM = 0.9, 0.95, 1e-8, 6e-4, 1.0


def listed():
    return [
        # one short chat on the tiny fp32 drafter: latency only
        dict(name="logprobs_tiny", op="logprobs", dtype="fp32", rows=4, vocab=1024, tokens=1, top=5, temp=1.0, pad=0, masked=0.0),
        # a decode step of 32 sequences that asked for the log probabilities of what they get
        dict(name="logprobs_decode", op="logprobs", dtype="bf16", rows=32, vocab=151936, tokens=1, top=20, temp=1.0, pad=0, masked=0.0),
        # the same for all 17 rows that a verify pass of 32 sequences leaves, in its fp32 logits
        dict(name="logprobs_verify", op="logprobs", dtype="fp32", rows=544, vocab=151936, tokens=1, top=20, temp=0.7, pad=0, masked=0.0),
        # a grammar leaves few tokens of an odd vocabulary, in some rows none
        dict(name="logprobs_masked", op="logprobs", dtype="bf16", rows=160, vocab=5003, tokens=3, top=8, temp=1.3, pad=5, masked=0.97),
        # a teacher's alternatives for a part of a training batch
        dict(name="logprobs_teacher", op="logprobs", dtype="bf16", rows=2048, vocab=151936, tokens=1, top=64, temp=1.0, pad=0, masked=0.0),
        # gradient of a few rows of the tiny drafter
        dict(name="grad_tiny", op="grad", dtype="fp32", out="fp32", rows=8, vocab=1024, tokens=1, temp=1.0, pad=0, masked=0.0, entropy=True),
        # blocks of the drafter trained on 64 alternatives of its teacher
        dict(name="grad_distil", op="grad", dtype="fp32", out="bf16", rows=1024, vocab=32000, tokens=64, temp=2.0, pad=0, masked=0.0, entropy=False),
        # policy gradient with an entropy bonus over 4096 positions
        dict(name="grad_policy", op="grad", dtype="bf16", out="bf16", rows=4096, vocab=151936, tokens=1, temp=1.0, pad=0, masked=0.0, entropy=True),
        # the tiny drafter in fp32 throughout
        dict(name="adamw_tiny", op="adamw", shape="drafter", layers=1, d=256, q=256, kv=128, ffn=768, feats=768, weights="fp32", grads="fp32", bits=32,
             clip=False, packed=False),
        # many odd tensors one behind the other, bf16 weights without a copy in fp32
        dict(name="adamw_odd", op="adamw", shape="odd", count=160, largest=400009, weights="bf16", grads="bf16", bits=32, clip=True, packed=True),
        # the five-layer drafter: fp32 weights beside their bf16 copy, states in 32 bits
        dict(name="adamw_drafter", op="adamw", shape="drafter", layers=5, d=4096, q=4096, kv=1024, ffn=12288, feats=12288, weights="mixed", grads="bf16",
             bits=32, clip=True, packed=False),
        # the same with states in 8 bits
        dict(name="adamw_drafter_8bit", op="adamw", shape="drafter", layers=5, d=4096, q=4096, kv=1024, ffn=12288, feats=12288, weights="mixed", grads="bf16",
             bits=8, clip=True, packed=False),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "grad", "adamw"])
    if op == "adamw":
        c = dict(op=op)
        if rng.random() < 0.4:
            d = 64 * _log(rng, 2, 40)
            c.update(shape="drafter", layers=rng.randint(1, 4), d=d, q=d, kv=max(64, d // 4), ffn=d * rng.choice([2, 3]), feats=3 * d)
        else:
            c.update(shape="odd", count=_log(rng, 1, 300), largest=_log(rng, 7, 3000000))
        return dict(c, weights=rng.choice(["fp32", "bf16", "mixed"]), grads=rng.choice(["bf16", "fp32"]), bits=rng.choice([32, 8]),
                    clip=rng.random() < 0.6, packed=rng.random() < 0.3)
    vocab = rng.choice([151936, 151936, 100003, 65536, 32000, 5003, 1024, _log(rng, 5, 250000)])
    most = 300000000 if op == "logprobs" else 500000000
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp32"]), rows=_log(rng, 1, max(1, min(8192, most // vocab))), vocab=vocab,
             tokens=rng.choice([1, 1, 1, 2, 5, 17, 64, 128]), temp=rng.choice([1.0, 1.0, 0.6, 0.85, 1.5, 3.0]), pad=rng.choice([0, 0, 0, 1, 8, 61]),
             masked=rng.choice([0.0, 0.0, 0.0, 0.5, 0.99]))
    if op == "grad":
        return dict(c, out=rng.choice(["bf16", "fp32"]), entropy=rng.random() < 0.5)
    return dict(c, top=rng.choice([0, 1, 1, 5, 8, 20, 20, 32, 64, 100, 128]))


# ---- what a case's sizes say (nothing here depends on the seed) -----------------------------------------------

def _spread(i, most):
    """A number in 0..most for the i-th tensor, scattered over the range."""
    return (i * 2654435761 + 40503) % 65521 * (most + 1) // 65521


def _sizes(c):
    """Elements of each tensor of a step, and whether its weights decay (norm gains do not)."""
    if c["shape"] == "odd":
        return [(max(1, int(c["largest"] ** (0.3 + 0.7 * _spread(i, 1000) / 1000))) if i else c["largest"], i % 3 > 0) for i in range(c["count"])]
    d = c["d"]
    layer = [(d, False), ((c["q"] + 2 * c["kv"]) * d, True), (d * c["q"], True), (d, False), (2 * c["ffn"] * d, True), (d * c["ffn"], True)]
    return [(d * c["feats"], True), (d, False)] + layer * c["layers"] + [(d, False)]


def _starts(c, unit=1):
    """First element of each tensor in one buffer, and the buffer's length: one behind the other, or each on a border of 128 elements.
    With unit 128: the same for the scales of an 8-bit state."""
    at, starts = 0, []
    for n, _ in _sizes(c):
        starts.append(at)
        n = -(-n // unit)
        at += n if c["packed"] or unit > 1 else -(-n // BLOCK) * BLOCK
    return starts, at


def work(case):
    c = case
    if c["op"] == "adamw":
        n = sum(k for k, _ in _sizes(c))
        weights = {"fp32": 8, "bf16": 4, "mixed": 10}[c["weights"]]
        states = 16 if c["bits"] == 32 else 4
        scales = 0 if c["bits"] == 32 else 16 * sum(-(-k // BLOCK) for k, _ in _sizes(c))
        return {"bytes": n * (SIZE[c["grads"]] + weights + states) + scales, "flops": 15 * n}
    n, v = c["rows"], c["vocab"]
    if c["op"] == "logprobs":
        return {"bytes": n * v * SIZE[c["dtype"]] + n * (8 * c["tokens"] + 8 * c["top"] + 12), "flops": 6 * n * v}
    return {"bytes": n * v * (SIZE[c["dtype"]] + SIZE[c["out"]]) + n * (8 * c["tokens"] + 8 + (8 if c["entropy"] else 0)), "flops": 6 * n * v}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    return _prepare_adamw(case, _gen(seed)) if case["op"] == "adamw" else _prepare_rows(case, _gen(seed))


def _prepare_rows(c, g):
    """Logits as a language model leaves them: a broad floor, and in every row some entries well above it."""
    n, v = c["rows"], c["vocab"]
    dt = KIND[c["dtype"]]
    z = torch.empty((n, v + c["pad"]), dtype=dt, device="cuda")
    z.normal_(0.0, 2.5, generator=g)
    peaks = min(v, 40)
    gap = v // peaks                                     # one in each of `peaks` stretches, shifted round the row
    at = torch.randint(0, gap, (n, peaks), generator=g, device="cuda") + gap * torch.arange(peaks, device="cuda")
    at = (at + torch.randint(0, v, (n, 1), generator=g, device="cuda")) % v
    z.scatter_(1, at, (torch.randn((n, peaks), generator=g, device="cuda") * 3.0 + 10.0).to(dt))
    if c["masked"]:
        z.masked_fill_(torch.rand((n, v + c["pad"]), generator=g, device="cuda") < c["masked"], NEG)
        z[::37] = NEG                                     # rows that nothing is left of
    tokens = torch.randint(0, v, (n, c["tokens"]), generator=g, device="cuda")
    tokens[:, 0] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.7, at[:, 0], tokens[:, 0])
    tokens[torch.rand(tokens.shape, generator=g, device="cuda") < 0.05] = -1          # padding
    z = z[:, :v]
    s = {"case": c, "z": z, "tokens": tokens.to(torch.int32)}
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["op"] == "logprobs":
        s.update(logprob=torch.empty((n, c["tokens"]), **f32), stats=torch.empty((n, 2), **f32), entropy=torch.empty(n, **f32))
        if c["top"]:
            s.update(top_ids=torch.empty((n, c["top"]), dtype=torch.int32, device="cuda"), top_logprob=torch.empty((n, c["top"]), **f32))
        return s
    _, s["stats"], s["entropy"] = _row_stats(z, c["temp"])          # what the forward pass left
    s["d_logprob"] = torch.randn((n, c["tokens"]), generator=g, device="cuda") / n
    s["d_logprob"][3::16] = 0.0                                      # positions without loss
    s["d_entropy"] = None
    if c["entropy"]:
        s["d_entropy"] = torch.full((n,), 0.01 / n, device="cuda")
        s["d_entropy"][3::16] = 0.0
    s["dz"] = torch.empty((n, v), dtype=KIND[c["out"]], device="cuda")
    return s


def _prepare_adamw(c, g):
    """Weights, gradients and states of a run that has taken 99 steps. The tensors are pieces of one buffer of each kind."""
    starts, total = _starts(c)
    sizes = _sizes(c)
    f32 = dict(dtype=torch.float32, device="cuda")
    flat = lambda dt: torch.zeros(total, dtype=dt, device="cuda")  # noqa: E731
    s = {"case": c, "param": flat(torch.float32 if c["weights"] == "fp32" else torch.bfloat16), "master": flat(torch.float32) if c["weights"] == "mixed" else None,
         "grad": flat(KIND[c["grads"]]), "m": flat(torch.float32 if c["bits"] == 32 else E4M3), "v": flat(torch.float32 if c["bits"] == 32 else E4M3),
         "m_scale": None, "v_scale": None, "norm": torch.zeros(1, **f32)}
    if c["bits"] == 8:
        scale_at, scales = _starts(c, BLOCK)
        s["m_scale"], s["v_scale"] = torch.zeros(scales, **f32), torch.zeros(scales, **f32)
    entries = []
    for i, ((n, decays), at) in enumerate(zip(sizes, starts)):
        piece = lambda k: None if s[k] is None else s[k][at:at + n]  # noqa: B023,E731
        e = {"param": piece("param"), "grad": piece("grad"), "exp_avg": piece("m"), "exp_avg_sq": piece("v"), "master": piece("master"),
             "weight_decay": 0.1 if decays else 0.0}
        w = torch.randn(n, generator=g, device="cuda") * 0.02 + (0.0 if decays else 1.0)
        e["param"].copy_(w)
        if e["master"] is not None:
            e["master"].copy_(w)
        size = 10.0 ** (-3.5 - 1.5 * _spread(i, 1000) / 1000)              # gradients of a tensor's own magnitude
        e["grad"].copy_(torch.randn(n, generator=g, device="cuda") * size)
        m, v = torch.randn(n, generator=g, device="cuda").mul_(0.3 * size), torch.randn(n, generator=g, device="cuda").square_().add_(0.1).mul_(size * size)
        if c["bits"] == 32:
            e["exp_avg"].copy_(m)
            e["exp_avg_sq"].copy_(v)
        else:
            k = slice(scale_at[i], scale_at[i] + -(-n // BLOCK))
            e["exp_avg_scale"], e["exp_avg_sq_scale"] = s["m_scale"][k], s["v_scale"][k]
            for x, codes, scale in ((m, e["exp_avg"], e["exp_avg_scale"]), (v.sqrt_(), e["exp_avg_sq"], e["exp_avg_sq_scale"])):
                top = _blocks(x).abs().amax(1) / 448.0
                scale.copy_(top)
                codes.copy_((x / top.repeat_interleave(BLOCK)[:n]).to(E4M3))
        entries.append(e)
    s["entries"] = entries
    return s


def _blocks(x):
    """x in rows of 128 elements, zeros behind its end."""
    n = -(-x.numel() // BLOCK) * BLOCK
    return x.view(-1, BLOCK) if n == x.numel() else torch.cat([x, x.new_zeros(n - x.numel())]).view(-1, BLOCK)


# ---- one pass -------------------------------------------------------------------------------------------------

_handles = {}


def _handle():
    """The library handle that a program keeps; these operators use none of its model's sizes."""
    from paper_2602_06036_b200 import binding, synth
    if "tiny" not in _handles:
        _handles["tiny"] = binding.DFlash(synth.TINY)
    return _handles["tiny"]


def run(state):
    return {"logprobs": _logprobs, "grad": _grad, "adamw": _adamw}[state["case"]["op"]](state)


def _row_stats(z, temp):
    """(z - M) / T in fp32, (M, ln sum exp of it) and the entropy; a row of -inf only: (-inf, 0) and 0."""
    z = z.float()
    top = z.amax(1, keepdim=True)
    empty = top == NEG
    y = (z - torch.where(empty, 0.0, top)) / temp
    e = y.exp()
    total = torch.where(empty, 1.0, e.sum(1, keepdim=True))
    e.mul_(y.clamp(min=-1e30))
    log_total = total.log()
    entropy = log_total - e.sum(1, keepdim=True) / total
    return y, torch.cat([top, log_total], 1), entropy.squeeze(1)


def _logprobs(s):
    c = s["case"]
    if own:
        _handle().dflash_token_logprobs(s["z"], s["tokens"], s["logprob"], temperature=c["temp"], stats=s["stats"], entropy=s["entropy"],
                                        top_ids=s.get("top_ids"), top_logprob=s.get("top_logprob"))
        return s["logprob"], s["stats"], s["entropy"], s.get("top_ids"), s.get("top_logprob")
    y, stats, entropy = _row_stats(s["z"], c["temp"])
    log_total = stats[:, 1:]
    logprob = torch.where(s["tokens"] < 0, 0.0, y.gather(1, s["tokens"].long().clamp(min=0)) - log_total)
    if not c["top"]:
        return logprob, stats, entropy, None, None
    k = min(c["top"], c["vocab"])
    bits = (s["z"].float() + 0.0).view(torch.int32)                  # + 0.0: -0 and 0 are equal
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    key += (1 << 32) - 1 - torch.arange(c["vocab"], device=key.device)   # of equal values the lowest index
    ids = key.topk(k, 1).indices
    top = y.gather(1, ids)
    ids, top = torch.where(top == NEG, -1, ids).int(), top - log_total
    if k < c["top"]:
        ids, top = (torch.cat([x, torch.full((len(x), c["top"] - k), f, dtype=x.dtype, device=x.device)], 1) for x, f in ((ids, -1), (top, NEG)))
    return logprob, stats, entropy, ids, top


def _grad(s):
    c = s["case"]
    if own:
        _handle().dflash_token_logprobs_bwd(s["z"], s["tokens"], s["stats"], s["d_logprob"], s["dz"], temperature=c["temp"],
                                            entropy=s["entropy"] if c["entropy"] else None, d_entropy=s["d_entropy"])
        return s["dz"]
    top, log_total = s["stats"][:, :1], s["stats"][:, 1:]
    g = torch.where(s["tokens"] < 0, 0.0, s["d_logprob"])
    empty = top == NEG
    y = (s["z"].float() - torch.where(empty, 0.0, top)) / c["temp"] - log_total
    p = y.exp()
    each = g.sum(1, keepdim=True)
    if c["entropy"]:
        p.mul_(y.clamp_(min=-1e30).add_(s["entropy"][:, None]).mul_(s["d_entropy"][:, None]).add_(each))
    else:
        p.mul_(each)
    dz = p.neg_().scatter_add_(1, s["tokens"].long().clamp(min=0), g)
    return (dz / c["temp"]).masked_fill_(empty, 0.0).to(KIND[c["out"]])


def _adamw(s):
    c = s["case"]
    if own:
        if "plan" not in s:                                              # a program makes it once for its tensors and keeps it
            s["plan"] = _handle().adamw_plan(s["entries"])
        _handle().dflash_adamw_step(s["plan"], step=100, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, max_grad_norm=MAX_NORM if c["clip"] else 0.0,
                                    grad_norm=s["norm"] if c["clip"] else None)
    else:
        _plain_adamw(s, c)
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale")} | {"norm": s["norm"] if c["clip"] else None}


def _plain_adamw(s, c):
    factor = 1.0
    if c["clip"]:
        s["norm"].copy_(torch.stack([e["grad"].float().square().sum(dtype=torch.float64) for e in s["entries"]]).sum().sqrt())
        factor = (MAX_NORM / (s["norm"] + 1e-6)).clamp(max=1.0)
    for e in s["entries"]:
        g = e["grad"].float() * factor
        n = g.numel()
        w = e["param"] if e["master"] is None else e["master"]
        if c["bits"] == 32:
            m, v = e["exp_avg"], e["exp_avg_sq"]
        else:
            m = e["exp_avg"].float() * e["exp_avg_scale"].repeat_interleave(BLOCK)[:n]
            v = (e["exp_avg_sq"].float() * e["exp_avg_sq_scale"].repeat_interleave(BLOCK)[:n]).square_()
        m.mul_(BETA1).add_(g * (1 - BETA1))
        v.mul_(BETA2).add_(g.square_().mul_(1 - BETA2))
        root = v.sqrt()
        old = w.float()
        step = m * (LR / (1 - BETA1 ** 100)) / (root / (1 - BETA2 ** 100) ** 0.5 + EPS)
        new = old - (LR * e["weight_decay"]) * old - step
        w.copy_(new)
        if e["master"] is not None:
            e["param"].copy_(new)
        if c["bits"] == 8:
            for x, codes, scale in ((m, e["exp_avg"], e["exp_avg_scale"]), (root, e["exp_avg_sq"], e["exp_avg_sq_scale"])):
                scale.copy_(_blocks(x).abs().amax(1) / 448.0)
                inv = (1.0 / scale).repeat_interleave(BLOCK)[:n]
                q = x * inv
                if codes is e["exp_avg_sq"]:
                    q = torch.where(x > 0, q.clamp(min=2.0 ** -9), q)      # no root that is not 0 becomes 0
                codes.copy_(q.clamp_(-448.0, 448.0).to(E4M3))


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    s = prepare(c, seed)
    return {"logprobs": _exact_logprobs, "grad": _exact_grad, "adamw": _exact_adamw}[c["op"]](s, c)


def _exact_logprobs(s, c):
    """A few rows at a time; the alternatives by a stable sort."""
    parts = []
    for z, tok in zip(s["z"].split(256), s["tokens"].long().split(256)):
        z = z.double()
        lp = torch.log_softmax(z / c["temp"], 1)
        empty = torch.isneginf(z).all(1)
        lp[empty] = NEG
        logprob = lp.gather(1, tok.clamp(min=0)).masked_fill(tok < 0, 0.0)
        entropy = -(lp.exp() * lp.clamp(min=-1e300)).sum(1)
        top = z.max(1).values
        stats = torch.stack([top, torch.where(empty, 0.0, torch.logsumexp(z / c["temp"], 1) - top / c["temp"])], 1)
        if c["top"]:
            ids = torch.argsort(z, dim=1, descending=True, stable=True)[:, :c["top"]]
            best = lp.gather(1, ids)
            best = torch.nn.functional.pad(best, (0, c["top"] - best.shape[1]), value=NEG)
        else:
            best = None
        parts.append((logprob, stats, entropy, best))
    cat = [None if p[0] is None else torch.cat(p) for p in zip(*parts)]
    return cat[0], cat[1], cat[2], None, cat[3]


def _exact_grad(s, c):
    out = []
    for i, z in enumerate(s["z"].split(256)):
        rows = slice(256 * i, 256 * i + len(z))
        tok = s["tokens"][rows].long()
        lp = torch.log_softmax(z.double() / c["temp"], 1)
        p = lp.exp()
        g = s["d_logprob"][rows].double() * (tok >= 0)
        d = -p * g.sum(1, keepdim=True)
        for k in range(c["tokens"]):
            d[torch.arange(len(z)), tok[:, k].clamp(min=0)] += g[:, k]
        if c["entropy"]:
            plp = torch.where(p > 0, p * lp, 0.0)
            d -= s["d_entropy"][rows, None].double() * (plp - p * plp.sum(1, keepdim=True))
        d /= c["temp"]
        d[torch.isneginf(z).all(1)] = 0.0
        out.append(d.float() if c["out"] == "bf16" else d)           # (float: room; 16 bits more than the output has)
    return torch.cat(out)


def _exact_adamw(s, c):
    """Codes of an 8-bit state stand here before their rounding."""
    out = {k: None if s[k] is None else s[k].double() for k in ("param", "master", "m_scale", "v_scale")}
    out["m"], out["v"] = (torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in ("m", "v"))
    norm = torch.stack([e["grad"].double().norm() for e in s["entries"]]).norm()
    factor = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0) if c["clip"] else 1.0
    starts, scale_at = _starts(c)[0], _starts(c, BLOCK)[0]
    for e, at, sat in zip(s["entries"], starts, scale_at):
        n = e["grad"].numel()
        to = slice(at, at + n)
        share = slice(sat, sat + -(-n // BLOCK))
        m, v = e["exp_avg"].double(), e["exp_avg_sq"].double()
        if c["bits"] == 8:
            m *= e["exp_avg_scale"].double().repeat_interleave(BLOCK)[:n]
            v = (v * e["exp_avg_sq_scale"].double().repeat_interleave(BLOCK)[:n]) ** 2
        g = e["grad"].double() * factor
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        w = (e["param"] if e["master"] is None else e["master"]).double()
        w = w * (1 - LR * e["weight_decay"]) - LR * (m / (1 - BETA1 ** 100)) / ((v / (1 - BETA2 ** 100)).sqrt() + EPS)
        out["param"][to] = w
        if e["master"] is not None:
            out["master"][to] = w
        if c["bits"] == 32:
            out["m"][to], out["v"][to] = m, v
        else:
            for x, key in ((m, "m"), (v.sqrt(), "v")):
                scale = _blocks(x).abs().amax(1) / 448.0
                out[key + "_scale"][share] = scale
                out[key][to] = x / scale.repeat_interleave(BLOCK)[:n]
    return {k: out[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale")} | {"norm": norm.reshape(1) if c["clip"] else None}
