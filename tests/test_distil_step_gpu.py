"""A training step as it is put together: a teacher's alternatives, the student's log probabilities at them, the gradient of their cross entropy, and the
AdamW step of the weights, against the same in 64 bits."""
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import dflash_oracle as orc
from paper_2602_06036_b200 import binding, synth
from tests.conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_distilling_a_head_from_a_teacher_s_alternatives(bits):
    lib = binding.DFlash(synth.TINY)
    n, d, v, top, T = 96, 64, synth.TINY.vocab, 16, 2.0
    rng = np.random.default_rng(11)
    x, teacher, w0 = rng.normal(size=(n, d)), rng.normal(size=(n, v)) * 3.0, rng.normal(size=(v, d)) * d ** -0.5
    x, teacher, w0 = (a.astype(np.float32) for a in (x, teacher, w0))
    cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).float().cuda()
    e4m3 = lambda: torch.zeros(v * d, dtype=torch.float8_e4m3fn, device="cuda")
    f32 = lambda k: torch.zeros(k, device="cuda")
    weight, grad, xd = cuda(w0), torch.zeros(v, d, device="cuda"), cuda(x)
    entry = {"param": weight.view(-1), "grad": grad.view(-1), "weight_decay": 0.01}
    if bits == 32:
        entry.update(exp_avg=f32(v * d), exp_avg_sq=f32(v * d))
    else:
        entry.update(exp_avg=e4m3(), exp_avg_sq=e4m3(), exp_avg_scale=f32(v * d // 128), exp_avg_sq_scale=f32(v * d // 128))
    plan = lib.adamw_plan([entry])
    ids, t_lp = torch.empty(n, top, dtype=torch.int32, device="cuda"), torch.empty(n, top, device="cuda")
    lp, stats, entropy, dz = torch.empty(n, top, device="cuda"), torch.empty(n, 2, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, v, device="cuda")
    norm = torch.empty(1, device="cuda")
    lib.dflash_token_logprobs(cuda(teacher), None, None, temperature=T, top_ids=ids, top_logprob=t_lp)
    ref = orc.token_logprobs(teacher, np.zeros((n, 0), int), T, top)
    np.testing.assert_array_equal(ids.cpu().numpy(), ref["top_ids"])
    w, m, root = w0.astype(np.float64), np.zeros(v * d), np.zeros(v * d)
    for t in (1, 2, 3):
        z = xd @ weight.t()
        lib.dflash_token_logprobs(z, ids, lp, temperature=T, stats=stats, entropy=entropy)
        g = -t_lp.exp() / n
        lib.dflash_token_logprobs_bwd(z, ids, stats, g, dz, temperature=T)
        grad.copy_(dz.t() @ xd)
        lib.dflash_adamw_step(plan, t, 1e-2, 0.9, 0.95, 1e-8, max_grad_norm=0.1, grad_norm=norm)
        # the same in 64 bits from the weights before the step
        gr = orc.token_logprobs_backward(x.astype(np.float64) @ w.T, ref["top_ids"], -np.exp(ref["top_logprob"]) / n, None, T).T @ x.astype(np.float64)
        total = orc.adamw_norm([gr])
        np.testing.assert_allclose(float(norm), total, rtol=1e-4)
        new, m, v2 = orc.adamw_step(w.reshape(-1), gr.reshape(-1), m, root ** 2, t, 1e-2, 0.9, 0.95, 1e-8, 0.01, min(1.0, 0.1 / (total + 1e-6)))
        # products of 64 and 96 terms in 32 bits: 1e-5 of a gradient, which the first steps' quotient of near-equal m and sqrt(v) passes on at most as it is
        scale = np.abs(gr).reshape(-1).max()
        loose = 1e-2 * np.minimum(2.0, 1e-4 * scale / np.maximum(np.abs(gr).reshape(-1), 1e-30)) + 1e-6
        assert np.all(np.abs(weight.view(-1).double().cpu().numpy() - new) <= loose)
        w = weight.double().cpu().numpy()                       # each step is judged from the state that it finds
        wide = lambda k: entry[k].double().cpu().numpy() * (np.repeat(entry[k + "_scale"].double().cpu().numpy(), 128) if bits == 8 else 1.0)
        m, root = wide("exp_avg"), wide("exp_avg_sq") if bits == 8 else np.sqrt(wide("exp_avg_sq"))


FIRST_CALLS = """
import torch
from paper_2602_06036_b200 import binding, synth
lib = binding.DFlash(synth.TINY)
f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
torch.manual_seed(0)
sets = []
for n, v in ((3, 50000), (700, 2000)):                        # by clusters, and CTAs that go through several rows
    z = torch.randn(n, v, device="cuda").bfloat16()
    t = torch.randint(0, v, (n, 2), device="cuda", dtype=torch.int32)
    sets.append((z, t, dict(logprob=f(n, 2), stats=f(n, 2), entropy=f(n), top_ids=f(n, 7, dt=torch.int32), top_logprob=f(n, 7)), f(n, 2) + 0.5, torch.zeros_like(z)))
entry = dict(param=f(5000) + 1, grad=f(5000) + 0.1, exp_avg=f(5000), exp_avg_sq=f(5000))
plan, norm = lib.adamw_plan([entry]), f(1)

def work():
    for z, t, out, g, dz in sets:
        lib.dflash_token_logprobs(z, t, **out)
        lib.dflash_token_logprobs_bwd(z, t, out["stats"], g, dz)
    lib.dflash_adamw_step(plan, 1, 0.01, max_grad_norm=1.0, grad_norm=norm)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):                                 # nothing of the library has run in this process
    work()
graph.replay()
torch.cuda.synchronize()
got = [x.clone() for s in sets for x in (*s[2].values(), s[4])] + [entry["param"].clone(), norm.clone()]
for k in ("exp_avg", "exp_avg_sq"):
    entry[k].zero_()
entry["param"].fill_(1)
work()
torch.cuda.synchronize()
want = [x for s in sets for x in (*s[2].values(), s[4])] + [entry["param"], norm]
assert all(torch.equal(a, b) for a, b in zip(got, want)) and int(lib.status) == 0 and float(norm) > 0
print("same")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    run = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "same" in run.stdout, run.stderr[-2000:]
