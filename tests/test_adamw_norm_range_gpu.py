"""The norm of gradients whose squares are no middling numbers, against the oracle in 64 bits (tolerances: see tests/test_adamw_gpu.py)."""
import pytest
import torch

from paper_2602_06036_b200 import binding
from tests.test_adamw_gpu import BF16, F32, U, lib, run_and_check, tensor  # noqa: F401

pytestmark = pytest.mark.gpu


def of_size(n, size, grads, at=0, bits=32):
    e = tensor(n, "fp32", grads, bits, seed=n, at=at)
    e["grad"].fill_(size)
    e["grad"][::3] *= -0.75
    return e


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("size", [5e18, 1.7e19])
def test_squares_that_pass_fp32s_range_together(lib, grads, size, at):
    """A thread adds up 32 squares (bf16) or 16 (fp32): of 5e18 each they pass 3.4e38. The step is taken, clipped."""
    run_and_check(lib, [of_size(9001, size, grads, at), of_size(7, size, grads, at), of_size(300, 1e-3, grads)], t=3, max_norm=1.0)


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("size", [1e-25, 3e-22, 1e-18, 1e-16])
def test_squares_that_vanish_below_it(lib, grads, size, at):
    """Gradients scaled up by the step: their norm is that of the scaled ones, and clips."""
    run_and_check(lib, [of_size(9001, size, grads, at), of_size(7, size, grads, at)], t=3, grad_scale=0.1 / size, max_norm=0.5)


def test_gradients_of_zero_beside_tiny_ones(lib):
    e = of_size(20000, 2e-24, F32)
    e["grad"][5000:] = 0.0
    run_and_check(lib, [e, of_size(100, 0.0, BF16)], t=1, grad_scale=2.0 ** 70, max_norm=1e-3)


@pytest.mark.parametrize("grads", [F32, BF16])
def test_a_gradient_whose_own_square_is_infinite_still_leaves_the_step_out(lib, grads):
    e = of_size(5000, 1e-3, grads)
    e["grad"][4321] = 2e19
    old, norm = e["param"].clone(), torch.zeros(1, device="cuda")
    lib.status.zero_()
    lib.dflash_adamw_step(lib.adamw_plan([e]), 1, 1e-3, grad_norm=norm)
    torch.cuda.synchronize()
    assert int(lib.status) == binding.DEV_NOT_FINITE and torch.isinf(norm).all() and torch.equal(e["param"], old)
    lib.status.zero_()
