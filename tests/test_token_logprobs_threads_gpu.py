"""First calls of several handles at once, each on a thread and a stream of its own: what a launcher remembers of a device is one for the whole process."""
import subprocess
import sys

import pytest

from tests.conftest import ROOT

pytestmark = pytest.mark.gpu

PROGRAM = """
import threading
import torch
from paper_2602_06036_b200 import binding, synth

N = 6
libs = [binding.DFlash(synth.TINY) for _ in range(N)]
streams = [torch.cuda.Stream() for _ in range(N)]
torch.manual_seed(0)
f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
cases = []
for n, v in ((3, 50000), (40, 50000), (500, 2000), (1300, 900), (2500, 700)):      # clusters, and CTAs of each size
    z = torch.randn(n, v, device="cuda").bfloat16()
    t = torch.randint(0, v, (n, 2), device="cuda", dtype=torch.int32)
    cases.append((z, t, [dict(logprob=f(n, 2), stats=f(n, 2), entropy=f(n), top_ids=f(n, 7, dt=torch.int32), top_logprob=f(n, 7)) for _ in range(N + 1)]))
torch.cuda.synchronize()
gate, errors = threading.Barrier(N), []

def work(i):
    try:
        for z, t, out in cases:
            gate.wait()
            libs[i].dflash_token_logprobs(z, t, **out[i], stream=streams[i])
    except BaseException as e:
        errors.append(e)
        gate.abort()

threads = [threading.Thread(target=work, args=(i,)) for i in range(N)]
for x in threads: x.start()
for x in threads: x.join()
torch.cuda.synchronize()
assert not errors, errors
for z, t, out in cases:
    libs[0].dflash_token_logprobs(z, t, **out[N])
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], out[N][k]) for o in out[:N] for k in o)
print("same")
"""


def test_first_calls_of_several_threads():
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "same" in run.stdout, run.stderr[-2000:]
