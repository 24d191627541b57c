"""Logits whose difference passes fp32's range (tolerances: see tests/test_token_logprobs_gpu.py). Their log probability, divided by the temperature, does not."""
import numpy as np
import pytest
import torch

from tests.test_token_logprobs_gpu import BF16, F32, check_backward, check_forward, forward, given, lib  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v,copies", [(50, 1), (5003, 1), (40000, 1), (3001, 400)])      # one CTA a row, clusters, small CTAs
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [4.0, 100.0, 1e30, 1e37, 1e38])
def test_differences_beyond_fp32(lib, v, copies, dtype, T):
    rng = np.random.default_rng(v)
    low, inf = torch.finfo(dtype).min, float("inf")
    z = np.stack([np.where(rng.random(v) < 0.5, 3e38, -3e38), rng.uniform(-1, 1, v) * 3.3e38, np.where(rng.random(v) < 0.9, low, -low),
                  np.where(rng.random(v) < 0.9, -inf, rng.uniform(-1, 1, v) * 3e38), np.where(rng.random(v) < 0.9, low, rng.normal(size=v))])
    z[:2, v // 2] = -3.2e38
    z = torch.from_numpy(z).to(dtype)
    n = len(z)
    tokens = given(n, v, 5, v)
    tokens[:, 0] = v // 2
    o = forward(lib, z.repeat(copies, 1).cuda(), tokens.repeat(copies, 1).cuda(), T, 30)
    torch.cuda.synchronize()
    for i in (0, copies - 1):
        check_forward({k: x[i * n:(i + 1) * n] for k, x in o.items()}, z, tokens, T, 30)
    # gradients of the size that the temperature takes off again
    g, gh = torch.from_numpy(rng.normal(size=(n, 5)) * T).float(), torch.from_numpy(rng.normal(size=n) * T).float()
    d = torch.empty(n * copies, v, device="cuda")
    lib.dflash_token_logprobs_bwd(z.repeat(copies, 1).cuda(), tokens.repeat(copies, 1).cuda(), o["stats"], g.repeat(copies, 1).cuda(), d, temperature=T,
                                  entropy=o["entropy"], d_entropy=gh.repeat(copies).cuda())
    torch.cuda.synchronize()
    for i in (0, copies - 1):
        check_backward(d[i * n:(i + 1) * n], z, tokens, g, gh, T, F32)
