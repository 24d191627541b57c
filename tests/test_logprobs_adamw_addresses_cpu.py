"""Addresses between two elements are refused on the host, whichever argument they stand in (a kernel that followed one would fault)."""
import ctypes as C

import pytest

from paper_2602_06036_b200 import binding
from tests.test_logprobs_adamw_abi_cpu import P, h, lib  # noqa: F401


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("field", ["logits", "tokens", "logprob", "stats", "entropy", "top_ids", "top_logprob", "dev_status"])
def test_token_logprobs(lib, h, field, off):
    a = binding.TokenLogprobsArgs(P, 0, 0, 4, 1000, 1.0, 2, P, P, P, P, 5, P, P, P)
    setattr(a, field, P + off)
    assert lib.dflash_token_logprobs(h, C.byref(a), None) == -1


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("field", ["logits", "tokens", "stats", "entropy", "d_logprob", "d_entropy", "dlogits", "dev_status"])
def test_token_logprobs_bwd(lib, h, field, off):
    a = binding.TokenLogprobsBwdArgs(P, 0, 0, 4, 1000, 1.0, 2, P, P, P, P, P, 2 * P, 0, 0, P)
    setattr(a, field, P + off)
    assert lib.dflash_token_logprobs_bwd(h, C.byref(a), None) == -1


@pytest.mark.parametrize("off", [1, 2, 3])
@pytest.mark.parametrize("field", ["step_dev", "lr_dev", "grad_norm", "dev_status"])
def test_adamw(lib, h, field, off):
    t = binding.AdamwTensor(P, P, None, P, P, P, P, 5, 1, 1, 8, 0.1, 1.0)
    a = binding.AdamwArgs(C.pointer(t), 1, 1, None, 1e-3, None, 0.9, 0.95, 1e-8, 1.0, 1.0, P, P, lib.dflash_adamw_workspace_bytes(h, 1), P)
    setattr(a, field, P + off)
    assert lib.dflash_adamw_step(h, C.byref(a), None) == -1
