"""Incoming gradients whose sum passes fp32's range, which the temperature brings back (tolerances: see tests/test_token_logprobs_gpu.py)."""
import numpy as np
import pytest
import torch

from tests.test_token_logprobs_gpu import BF16, F32, check_backward, forward, given, lib, logits  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,v,dtype,out,k", [(3, 50, F32, F32, 5), (4, 5003, BF16, F32, 128), (2, 20000, F32, BF16, 64), (2400, 900, BF16, BF16, 3)])
@pytest.mark.parametrize("T,size", [(100.0, 1e38), (1000.0, 3e38), (1e6, 3e38), (1e37, 3e38)])
def test_sums_of_gradients_beyond_fp32(lib, n, v, dtype, out, k, T, size):
    z, tokens = logits(n, v, dtype, v), given(n, v, k, v)
    z[0, ::3] = float("-inf")                                 # (what stands before a probability of 0 has to be finite)
    tokens[:, 0] = tokens[:, k // 2] = v // 2
    rng = np.random.default_rng(v)
    g = torch.from_numpy(rng.uniform(0.5, 1, (n, k)) * size).float()
    gh = torch.from_numpy(rng.uniform(-1, 1, n) * size * 0.3).float()
    g[1] = 1e-30                                               # and small ones beside them
    gh[1] = 0.0
    o = forward(lib, z.cuda(), tokens.cuda(), T)
    d = torch.empty(n, v, dtype=out, device="cuda")
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], g.cuda(), d, temperature=T, entropy=o["entropy"], d_entropy=gh.cuda())
    torch.cuda.synchronize()
    for rows in (slice(0, min(n, 40)), slice(max(0, n - 40), n)):
        check_backward(d[rows], z[rows], tokens[rows], g[rows], gh[rows], T, out)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_large_gradient_of_the_entropy_leaves_tokens_of_probability_0_alone(lib, dtype):
    n, v = 6, 3000
    z, tokens = logits(n, v, dtype, v), given(n, v, 2, v)
    z[:, ::2] = float("-inf")
    z[:, 1::4] -= 2000.0
    g, gh = torch.zeros(n, 2), torch.full((n,), 1e36)
    o = forward(lib, z.cuda(), tokens.cuda(), 1.0)
    d = torch.empty(n, v, device="cuda")
    lib.dflash_token_logprobs_bwd(z.cuda(), tokens.cuda(), o["stats"], g.cuda(), d, entropy=o["entropy"], d_entropy=gh.cuda())
    torch.cuda.synchronize()
    check_backward(d, z, tokens, g, gh, 1.0, F32)
    assert not d[:, ::2].any() and not d[:, 1::4].any()
