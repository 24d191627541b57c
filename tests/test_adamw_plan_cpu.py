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
