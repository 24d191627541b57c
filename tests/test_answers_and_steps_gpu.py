"""The operators on logits and weights as they stand behind the framework's own calls: the log probabilities of what a verify pass answers, and steps of the weights that
a handle holds, with drafts in between."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2602_06036_b200 import binding, synth
from tests.harness import TOL, Case, assert_close
from tests.test_token_logprobs_gpu import check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,layers,rows,lens", [("tiny", 2, 5, (0, 61, 130)), ("mid", 2, 17, (70, 200))])
def test_log_probabilities_of_a_verify_pass(name, layers, rows, lens):
    """[anchor, drafts] -> target's logits -> accepted tokens -> their log probabilities, entropy and alternatives, one call behind the other, then replayed from a graph."""
    cfg = dataclasses.replace(synth.TINY if name == "tiny" else synth.MID, n_layers=layers, block_size=min(rows, 16))
    case = Case(cfg, lens, seed=61, headroom=rows + 4)
    case.fill_pool_synthetic()
    lib, dev, S, gamma, V, top = case.lib, case.device, len(lens), rows - 1, cfg.vocab, 9
    tokens = torch.randint(0, V - 1, (S, rows), generator=synth.substream(61, "verify.tokens"), dtype=torch.int32).to(dev)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
    f32 = lambda *s: torch.zeros(s, device=dev)
    ids, logits, acc, out, bonus, new_len = i32(S, rows), f32(S * rows, V), i32(S), i32(S, rows), i32(S), i32(S)
    o = dict(logprob=f32(S * rows, 1), stats=f32(S * rows, 2), entropy=f32(S * rows), top_ids=i32(S * rows, top), top_logprob=f32(S * rows, top))
    given = i32(S * rows, 1)

    def work():
        lib.dflash_target_verify(tokens, case.ctx_len, max(lens), case.page_table, case.pool, [], ids, logits_out=logits)
        lib.dflash_verify_accept(tokens, rows, gamma, case.ctx_len, acc, out, bonus, new_len, logits=logits.view(S, rows, V), draft_offset=1)
        # the answer's tokens: the drafts that were kept and the target's own behind them
        kept = torch.arange(rows, device=dev)[None] < acc[:, None]
        given.copy_(torch.where(kept, out, -1).view(-1, 1))
        lib.dflash_token_logprobs(logits, given, **o)

    lib.status.zero_()
    work()
    torch.cuda.synchronize()
    assert int(lib.status) == 0
    check_forward(o, logits.cpu(), given.cpu(), 1.0, top)
    assert torch.equal(o["top_ids"][:, 0], ids.view(-1))
    assert int((given >= 0).sum()) >= S
    first = {k: v.clone() for k, v in o.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for v in o.values():
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o["top_ids"], first["top_ids"])
    check_forward(o, logits.cpu(), given.cpu(), 1.0, top)


def on_device(x):
    return {k: [on_device(e) for e in v] if isinstance(v, list) else v.cuda().contiguous() for k, v in x.items()}


def matrices(w):
    return [v for k, v in w.items() if k != "layers"] + [v for layer in w["layers"] for v in layer.values()]


@pytest.mark.parametrize("name,bits", [("tiny", 32), ("mid", 32), ("mid", 8)])
def test_drafts_between_steps_of_the_weights_that_the_handle_holds(name, bits):
    cfg = synth.TINY if name == "tiny" else synth.MID
    case = Case(cfg, (5, 130), seed=62)
    case.project_prefill(oracle=False)
    case.lib.close()
    weights = on_device(synth.pack_device_weights(cfg, case.w_cpu))
    rope = synth.rope_tables(cfg, case.max_pos)
    lib = binding.DFlash(cfg)
    lib.set_weights(weights, *rope)                            # tensors of the device are held, not copied
    entries = []
    for i, w in enumerate(matrices(weights)):
        n = w.numel()
        g = torch.Generator(device="cuda")
        g.manual_seed(i)
        e = {"param": w.view(-1), "grad": torch.randn(n, generator=g, device="cuda").to(w.dtype), "weight_decay": 0.1}
        if w.dtype is torch.bfloat16:
            e["master"] = w.view(-1).float()
        for k in ("exp_avg", "exp_avg_sq"):
            e[k] = torch.zeros(n, device="cuda") if bits == 32 else torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            if bits == 8:
                e[k + "_scale"] = torch.zeros(-(-n // 128), device="cuda")
        entries.append(e)
    plan = lib.adamw_plan(entries)
    S, B = case.S, cfg.block_size
    anchors = synth.make_anchors(cfg, S, 62).cuda()

    def draft(on, pool, hidden):
        on.dflash_draft_block(anchors, case.ctx_len, max(case.ctx_lens), case.page_table, pool, torch.zeros(S, B, dtype=torch.int32, device="cuda"), hidden_out=hidden)

    feats, n_new, none = case.feats_cpu.cuda(), torch.tensor(case.ctx_lens, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    made = []
    lib.status.zero_()
    for step in range(1, 5):
        hidden, pool = torch.zeros(S * B, cfg.d_model, device="cuda"), torch.zeros_like(case.pool)
        lib.dflash_adamw_step(plan, step, 0.01, max_grad_norm=1e9)
        if step % 2:                                           # with the context made by the new weights, and with the cached one
            lib.dflash_ctx_project(feats, n_new, none, case.page_table, pool)
        else:
            pool.copy_(case.pool)
            lib.dflash_adamw_step(plan, step, 0.01, max_grad_norm=1e9)
        draft(lib, pool, hidden)
        made.append((hidden, pool, on_device({k: [{m: x.clone() for m, x in layer.items()} for layer in v] if k == "layers" else v.clone() for k, v in weights.items()})))
    torch.cuda.synchronize()
    assert int(lib.status) == 0
    last = None
    for step, (hidden, pool, held) in enumerate(made, 1):
        fresh = binding.DFlash(cfg)
        fresh.set_weights(held, *rope)
        want, again = torch.zeros_like(hidden), torch.zeros_like(pool)
        if step % 2:
            fresh.dflash_ctx_project(feats, n_new, none, case.page_table, again)
        else:
            again.copy_(case.pool)
        draft(fresh, again, want)
        torch.cuda.synchronize()
        h = hidden.cpu().numpy()
        assert_close(pool.float().cpu().numpy(), again.float().cpu().numpy(), cfg.dtype, f"context of step {step}")
        assert_close(h, want.cpu().numpy(), cfg.dtype, f"draft of step {step}")
        assert last is None or np.linalg.norm(h - last) > 10 * TOL[cfg.dtype]["rel_l2"] * np.linalg.norm(h)      # a draft of the weights before would be found out
        last = h
