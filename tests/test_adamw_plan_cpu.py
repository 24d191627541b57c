"""What a plan of the optimiser step refuses, and what the step refuses of a plan (tensors on the host: device -1; nothing is launched)."""
import pytest
import torch

from paper_2602_06036_b200 import binding

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HOST = -1


def entry(n=300, **over):
    e = {"param": torch.zeros(n, dtype=BF16), "grad": torch.zeros(n, dtype=BF16), "master": torch.zeros(n), "exp_avg": torch.zeros(n), "exp_avg_sq": torch.zeros(n)}
    return {**e, **over}


class Recorder(binding.DFlash):
    """A handle of device `index` that keeps its calls to itself."""

    def __init__(self, index):
        self._index, self.status, self.calls = index, torch.zeros(1, dtype=torch.int32), []
        self.lib = type("Library", (), {"dflash_adamw_step": None})

    def close(self):
        pass

    def _scratch(self, name, query, key, stream):
        return None, 0, 0

    def _call(self, fn, args, stream):
        self.calls.append(args)


@pytest.mark.parametrize("clip", [0.0, 1.0])
def test_a_plan_of_another_device_is_refused(clip):
    plan, own, other = binding.AdamwPlan([entry()], HOST), Recorder(HOST), Recorder(1)
    with pytest.raises(AssertionError, match="device"):
        other.dflash_adamw_step(plan, 1, 1e-3, max_grad_norm=clip)
    assert not other.calls
    own.dflash_adamw_step(plan, 1, 1e-3, max_grad_norm=clip)
    assert len(own.calls) == 1 and own.calls[0].n_tensors == 1


def test_a_gradient_over_what_the_step_writes_is_refused():
    """Written buffers lie apart from all others; gradients may be shared."""
    flat = torch.zeros(1000)
    four = lambda k, n=300: flat[k:k + n]
    e = lambda param, grad, **over: {"param": param, "grad": grad, "exp_avg": torch.zeros(len(param)), "exp_avg_sq": torch.zeros(len(param)), **over}
    g = torch.zeros(300)
    for bad in ([e(four(0), four(0))],                                            # its own weights
                [e(four(0), four(299))], [e(four(299), four(0))],                 # one entry of them
                [e(four(0), g), e(torch.zeros(100), four(100, 100))],              # inside of another tensor's
                [e(four(100, 100), torch.zeros(100)), e(torch.zeros(1000), flat)],  # around them
                [e(torch.zeros(1000), flat), e(torch.zeros(10), four(0, 10)), e(four(500, 100), torch.zeros(100))],      # behind a shorter gradient
                [e(four(0), g, exp_avg=g)], [e(four(0), g, exp_avg_sq=g)],
                [entry(grad=flat.view(BF16)[:300], master=four(0))]):
        with pytest.raises(AssertionError, match="overlap"):
            binding.AdamwPlan(bad, HOST)
    for good in ([e(four(0), four(300)), e(four(600), four(300))],                # one gradient for two tensors, in between them
                 [e(torch.zeros(1000), flat), e(torch.zeros(10), four(3, 10)), e(torch.zeros(300), four(0))],
                 [entry(0, grad=torch.zeros(0)), entry(3)]):
        assert binding.AdamwPlan([{**x, "grad": x["grad"].to(BF16) if x["param"].dtype is BF16 else x["grad"]} for x in good], HOST).n == len(good)
