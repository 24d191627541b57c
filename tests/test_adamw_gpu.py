"""The AdamW step on the GPU against the oracle in 64 bits.

Tolerances. u = 2^-24. g' carries three roundings (grad_scale, the clipping factor, the product) and the norm's own; m and v two products and a sum,
each of 2 u of its parts. The step's quotient carries those, a root, a sum, the bias corrections and a division: below 24 u of itself where m's parts do not
cancel, else 24 u of lr times the parts' quotient. w adds 3 u of itself. A state in 8 bits is off by half a step of its code: 2^-4 of the value, or 2^-10
of its block's scale below 2^-6 scales (2^-9 for a root that is kept from 0), after a relative error of 16 u that can carry a value over a border.
Squares below 2^-149 do not exist in fp32, and v has a step of that size, so that a root is off by up to 2^-74; a block whose largest magnitude is below
2^-117 is stored as 0."""
import numpy as np
import pytest
import torch

from oracle import dflash_oracle as orc
from paper_2602_06036_b200 import binding, synth

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
HOLD = 4_000_000                 # clocks for which a stream is held: about 2 ms


@pytest.fixture(scope="module")
def lib():
    return binding.DFlash(synth.TINY)


def tensor(n, weights="fp32", grads=F32, bits=32, seed=0, at=0, wd=0.1, fresh=False, spread=1.0):
    """A tensor of a step with all that belongs to it, every buffer `at` entries behind its border."""
    rng = np.random.default_rng(seed)
    on = lambda x, dt: torch.zeros(n + at, dtype=dt, device="cuda")[at:].copy_(torch.from_numpy(x))
    size = 10.0 ** (rng.normal(size=n) * spread - 3)
    w, g, m, v = rng.normal(size=n), rng.normal(size=n) * size, rng.normal(size=n) * size * 0.3, (rng.normal(size=n) ** 2 + 0.1) * size * size
    if fresh:
        m[:], v[:] = 0, 0
    e = {"param": on(w, F32 if weights == "fp32" else BF16), "grad": on(g, grads), "weight_decay": wd}
    if weights == "mixed":
        e["master"] = on(w, F32)
    if bits == 32:
        e["exp_avg"], e["exp_avg_sq"] = on(m, F32), on(v, F32)
    else:
        for key, x, root in (("exp_avg", m, False), ("exp_avg_sq", np.sqrt(v), True)):
            codes, scale = orc.state_codes(x, root)
            e[key] = torch.zeros(n + at, dtype=E4M3, device="cuda")[at:]
            e[key].copy_(torch.from_numpy(codes).float().to(E4M3))
            e[key + "_scale"] = torch.from_numpy(scale).float().cuda()
    return e


def host(t):
    return t.detach().double().cpu().numpy()


def values(e):
    """(w, g, m, v) of a tensor in 64 bits."""
    n = e["param"].numel()
    w = host(e["param"] if e.get("master") is None else e["master"])
    if e["exp_avg"].dtype == F32:
        return w, host(e["grad"]), host(e["exp_avg"]), host(e["exp_avg_sq"])
    wide = lambda k: np.repeat(host(e[k + "_scale"]), 128)[:n]
    return w, host(e["grad"]), host(e["exp_avg"]) * wide("exp_avg"), (host(e["exp_avg_sq"]) * wide("exp_avg_sq")) ** 2


def run_and_check(lib, entries, t=1, lr=6e-4, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0, max_norm=0.0, want_norm=True, on_device=False):
    before = [values(e) for e in entries]
    norm = torch.full((1,), -1.0, device="cuda") if want_norm else None
    plan = lib.adamw_plan(entries)
    lib.status.zero_()
    lib.dflash_adamw_step(plan, torch.tensor([t], dtype=torch.int32, device="cuda") if on_device else t, torch.tensor([lr], device="cuda") if on_device else lr,
                          beta1, beta2, eps, grad_scale, max_norm, norm)
    torch.cuda.synchronize()
    assert int(lib.status) == 0
    total = orc.adamw_norm([b[1] for b in before], grad_scale)
    if want_norm:
        np.testing.assert_allclose(float(norm), total, rtol=16 * U)
    factor = grad_scale * (min(1.0, max_norm / (total + 1e-6)) if max_norm > 0 else 1.0)
    lr64 = float(np.float32(lr)) if on_device else lr
    for e, (w, g, m, v) in zip(entries, before):
        rate = lr64 * e.get("lr_scale", 1.0)
        w1, m1, v1 = orc.adamw_step(w, g, m, v, t, rate, beta1, beta2, eps, e.get("weight_decay", 0.0), factor)
        parts = beta1 * np.abs(m) + (1 - beta1) * np.abs(g) * factor
        got_w, _, got_m, got_v = values(e)
        quotient = rate * parts / (1 - beta1 ** t) / (np.sqrt(v1 / (1 - beta2 ** t)) + eps)
        tol = 3 * U * np.abs(w) + 24 * U * quotient + 1e-38
        if e.get("master") is not None:
            assert torch.equal(e["param"], e["master"].to(BF16))
        elif e["param"].dtype == BF16:
            tol = tol + 2.0 ** -8 * np.abs(w1) * 1.001
        off = np.abs(got_w - w1)
        assert np.all(off <= tol), f"weights: {np.max(off / tol):.2f} times the tolerance"
        if e["exp_avg"].dtype == F32:
            assert np.all(np.abs(got_m - m1) <= 12 * U * parts + 1e-44)
            assert np.all(np.abs(got_v - v1) <= 16 * U * v1 + 1e-44)
        else:
            n = len(w)
            for key, x, least, gone in (("exp_avg", m1, 2.0 ** -10, 2.0 ** -117), ("exp_avg_sq", np.sqrt(v1), 2.0 ** -9, 2.0 ** -74)):
                tops = np.array([np.abs(x[i:i + 128]).max() for i in range(0, n, 128)])
                big = np.array([(parts if key == "exp_avg" else x)[i:i + 128].max() for i in range(0, n, 128)])
                assert np.all(np.abs(host(e[key + "_scale"]) - tops / 448) <= (16 * U * big + gone) / 448)
                s = np.repeat(tops / 448, 128)[:n]
                got = host(e[key]) * np.repeat(host(e[key + "_scale"]), 128)[:n]
                slack = 16 * U * (parts if key == "exp_avg" else x) + 16 * U * np.repeat(big, 128)[:n]
                assert np.all(np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), least * s) * 1.0001 + 2 * slack + gone)
                if key == "exp_avg_sq":
                    assert np.all(((host(e[key]) > 0) == (x > 0)) | (x < gone) | (448 * s < gone))


@pytest.mark.parametrize("weights", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
def test_each_type_at_odd_sizes_and_places(lib, weights, grads, bits):
    sizes = [1, 3, 4, 127, 128, 129, 1000, 2047, 2048, 2049, 12345]
    for at in (0, 1):
        entries = [tensor(n, weights, grads, bits, seed=n, at=at, wd=0.1 * (n % 2)) for n in sizes]
        run_and_check(lib, entries, t=7, max_norm=0.05)


def test_mixed_types_in_one_call(lib):
    entries = [tensor(500 + 37 * i, w, g, b, seed=i, at=i % 3) for i, (w, g, b) in enumerate((w, g, b) for w in ("fp32", "bf16", "mixed") for g in (F32, BF16)
                                                                                         for b in (32, 8))]
    entries.insert(3, tensor(0))
    entries[5]["lr_scale"] = 0.25
    run_and_check(lib, entries, t=3, max_norm=1e9, grad_scale=1 / 64)


@pytest.mark.parametrize("count", [1, 319, 320, 321, 700])
def test_many_tensors(lib, count):
    entries = [tensor(1 + (i * 7919) % 300, "mixed", BF16, 8 if i % 2 else 32, seed=i) for i in range(count)]
    run_and_check(lib, entries, t=2, max_norm=0.01)


def test_a_large_tensor(lib):
    run_and_check(lib, [tensor(5_000_003, "mixed", BF16, 8, seed=1), tensor(3_000_001, "bf16", BF16, 32, seed=2)], t=1000, max_norm=1.0)


def test_a_tensor_of_more_than_32_bits_of_entries(lib):
    """Three pieces of it, the last one behind entry 2^31, against the same step of each piece alone."""
    n, piece = 2 ** 31 + 301, 1024
    big = {"param": torch.empty(n, dtype=BF16, device="cuda"), "grad": torch.zeros(n, dtype=BF16, device="cuda"), "weight_decay": 0.1}
    for k in ("exp_avg", "exp_avg_sq"):
        big[k] = torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3)
        big[k + "_scale"] = torch.zeros(-(-n // 128), device="cuda")
    big["param"].fill_(1.0)
    parts = []
    for i, at in enumerate((0, 2 ** 30, 2 ** 31 - 768)):
        e = tensor(min(piece, n - at), "bf16", BF16, 8, seed=i)
        for k in ("param", "grad", "exp_avg", "exp_avg_sq"):
            big[k].view(torch.uint8 if k[0] == "e" else BF16)[at:at + piece].copy_(e[k].view(torch.uint8 if k[0] == "e" else BF16))
        for k in ("exp_avg_scale", "exp_avg_sq_scale"):
            big[k][at // 128:at // 128 + len(e[k])].copy_(e[k])
        parts.append((at, e))
    norm, same = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    lib.dflash_adamw_step(lib.adamw_plan([big]), 3, 1e-2, max_grad_norm=0.01, grad_norm=norm)
    lib.dflash_adamw_step(lib.adamw_plan([e for _, e in parts]), 3, 1e-2, max_grad_norm=0.01, grad_norm=same)
    torch.cuda.synchronize()
    assert abs(float(norm) / float(same) - 1) <= 4 * U          # added up in another order
    for at, e in parts:
        m = len(e["param"])
        off = (big["param"][at:at + m].float() - e["param"].float()).abs()
        assert bool((off <= 2.0 ** -7 * e["param"].float().abs()).all()) and bool((e["param"] != 1).any())      # a rounding either way where the factor is an ulp off
        same_code = big["exp_avg"].view(torch.uint8)[at:at + m] == e["exp_avg"].view(torch.uint8)
        assert float(same_code.float().mean()) > 0.98


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("t,beta1,beta2", [(1, 0.9, 0.999), (1, 0.0, 0.0), (100000, 0.95, 0.9999), (2 ** 31 - 1, 0.9, 0.95)])
def test_first_and_late_steps(lib, bits, t, beta1, beta2):
    for on_device in (False, True):
        run_and_check(lib, [tensor(777, "fp32", F32, bits, seed=4, fresh=t == 1)], t=t, beta1=beta1, beta2=beta2, on_device=on_device)


@pytest.mark.parametrize("bits", [32, 8])
def test_blocks_of_zeros_and_of_tiny_values(lib, bits):
    e = tensor(1000, "fp32", F32, bits, seed=5, fresh=True)
    e["grad"][:300] = 0.0
    e["grad"][300:600] *= 1e-30
    run_and_check(lib, [e], t=1)
    assert torch.isfinite(e["param"]).all()


def test_an_eight_bit_state_of_wide_spread_keeps_its_small_entries(lib):
    """Ten steps of constant gradients over six decades: every entry moves by the rate at each, as with states in 32 bits."""
    n = 4096
    e = tensor(n, "fp32", F32, 8, seed=6, fresh=True, spread=0.0, wd=0.0)
    e["grad"].copy_(torch.from_numpy(np.where(np.arange(n) % 2, 1.0, -1.0) * 10.0 ** np.random.default_rng(1).uniform(-6, 0, n)))
    w0, plan = e["param"].clone(), lib.adamw_plan([e])
    for t in range(1, 11):
        lib.dflash_adamw_step(plan, t, 1e-2, eps=1e-30)
    moved = -(e["param"] - w0) * e["grad"].sign() / 0.1
    # a factor (1 + 2^-4) of error in m a step and as much in sqrt(v), half of them carried on, and entries below 2^-6 scales of their block
    # (a factor of 2^15 to its largest, 10^-4.5) only to a step
    wide = e["grad"].abs().view(-1, 128)
    sure = (wide > 2.0 ** -14 * wide.amax(1, keepdim=True)).view(-1)
    assert int(sure.sum()) > n // 2 and float(moved[sure].min()) > 0.5 and float(moved[sure].max()) < 2.0
    assert float(moved.min()) >= 0.0


def test_a_norm_that_is_not_finite_leaves_everything_as_it_was(lib):
    for bad in (float("nan"), float("inf"), 1e30):
        entries = [tensor(400, "mixed", F32, 8, seed=1), tensor(300, "fp32", F32, 32, seed=2)]
        entries[1]["grad"][77] = bad
        old = [{k: v.clone() for k, v in e.items() if isinstance(v, torch.Tensor)} for e in entries]
        norm = torch.zeros(1, device="cuda")
        lib.status.zero_()
        lib.dflash_adamw_step(lib.adamw_plan(entries), 1, 1e-3, max_grad_norm=1.0, grad_norm=norm)
        torch.cuda.synchronize()
        assert int(lib.status) == binding.DEV_NOT_FINITE and not torch.isfinite(norm).any()
        for e, o in zip(entries, old):
            assert all(torch.equal(e[k].view(torch.uint8), x.view(torch.uint8)) for k, x in o.items())
    lib.status.zero_()


def test_a_clipping_norm_below_fp32s_range_still_clips(lib):
    """Gradients times 1e-50 / norm are 0 in fp32: new states stay 0, and so do the weights' steps."""
    e = tensor(300, "fp32", F32, 32, seed=4, wd=0.0, fresh=True)
    old = e["param"].clone()
    lib.dflash_adamw_step(lib.adamw_plan([e]), 1, 1e-3, max_grad_norm=1e-50)
    torch.cuda.synchronize()
    assert torch.equal(e["param"], old) and not e["exp_avg"].any() and not e["exp_avg_sq"].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_without_the_norm_such_a_gradient_stays_in_its_place(lib, bits):
    e = tensor(400, "fp32", F32, bits, seed=3)
    e["grad"][200] = float("nan")
    lib.dflash_adamw_step(lib.adamw_plan([e]), 1, 1e-3)
    torch.cuda.synchronize()
    w, _, m, v = values(e)
    ok = np.arange(400) != 200
    assert np.isnan(w[200]) and np.isfinite(w[ok]).all()
    near = ok if bits == 32 else (np.arange(400) // 128) != 1
    assert np.isnan(m[200]) and np.isnan(v[200]) and np.isfinite(m[near]).all() and np.isfinite(v[near]).all()
    if bits == 8:
        assert np.isnan(m[128:256]).all() and np.isnan(v[128:256]).all()


def test_nothing_to_do(lib):
    norm = torch.full((1,), 5.0, device="cuda")
    lib.dflash_adamw_step(lib.adamw_plan([]), 1, 1e-3)
    lib.dflash_adamw_step(lib.adamw_plan([tensor(0), tensor(0, "mixed", BF16, 8)]), 1, 1e-3, max_grad_norm=1.0)
    lib.dflash_adamw_step(lib.adamw_plan([]), 1, 1e-3, grad_norm=norm)
    torch.cuda.synchronize()
    assert float(norm) == 0.0


def test_runs_agree_bit_by_bit(lib):
    runs = []
    for _ in range(3):
        entries = [tensor(100003, "mixed", BF16, b, seed=b) for b in (8, 32)]
        norm = torch.zeros(1, device="cuda")
        for t in (1, 2, 3):
            lib.dflash_adamw_step(lib.adamw_plan(entries), t, 1e-3, max_grad_norm=0.5, grad_norm=norm)
        runs.append([v for e in entries for v in e.values() if isinstance(v, torch.Tensor)] + [norm])
    for r in runs[1:]:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(r, runs[0]))


def test_a_replayed_graph_takes_the_rate_and_the_step_from_the_device(lib):
    make = lambda: [tensor(3000, "mixed", BF16, 8, seed=1), tensor(501, "fp32", F32, 32, seed=2, at=1)]
    rates = [1e-3, 5e-4, 2e-4]
    eager, captured = make(), make()
    one = lib.adamw_plan(eager)
    for t, lr in enumerate(rates, 1):
        lib.dflash_adamw_step(one, torch.tensor([t], dtype=torch.int32, device="cuda"), torch.tensor([lr], device="cuda"), max_grad_norm=0.1)
    step, lr = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    plan = lib.adamw_plan(captured)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        lib.dflash_adamw_step(plan, step, lr, max_grad_norm=0.1)
    for x in rates:
        lr.fill_(x)
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager, captured):
        assert all(torch.equal(v.view(torch.uint8), b[k].view(torch.uint8)) for k, v in a.items() if isinstance(v, torch.Tensor))


def test_two_streams_at_once(lib):
    make = lambda k: [tensor(200_000 + k, "mixed", BF16, 8, seed=k), tensor(50_001, "bf16", BF16, 32, seed=k + 9)]
    sets, alone = [make(0), make(1)], [make(0), make(1)]
    for e in alone:
        lib.dflash_adamw_step(lib.adamw_plan(e), 1, 1e-3, max_grad_norm=0.1)
    streams, plans = [torch.cuda.Stream(), torch.cuda.Stream()], [lib.adamw_plan(e) for e in sets]
    for s in streams:
        with torch.cuda.stream(s):                             # its workspace exists before it is held
            lib.dflash_adamw_step(lib.adamw_plan([]), 1, 1e-3, grad_norm=torch.zeros(1, device="cuda"), stream=s)
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            torch.cuda._sleep(HOLD)
    for p, s in zip(plans, streams):
        lib.dflash_adamw_step(p, 1, 1e-3, max_grad_norm=0.1, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(alone, sets):
        for x, y in zip(a, b):
            assert all(torch.equal(v.view(torch.uint8), y[k].view(torch.uint8)) for k, v in x.items() if isinstance(v, torch.Tensor))


def test_refusals_of_the_plan(lib):
    good = lambda **over: {**tensor(300, "bf16", BF16, 8, seed=1), **over}
    z = lambda n, dt=F32: torch.zeros(n, dtype=dt, device="cuda")
    for bad in (good(grad=z(299, BF16)), good(grad=z(300, torch.float16)), good(param=z(300), master=z(300)), good(exp_avg_scale=None), good(exp_avg_sq_scale=z(2)),
                good(exp_avg=z(600, E4M3)[::2]), good(master=torch.zeros(300)), good(exp_avg_sq=z(300)), good(momentum=1)):
        with pytest.raises(AssertionError):
            lib.adamw_plan([bad])
    a = good()
    with pytest.raises(AssertionError, match="overlap"):
        lib.adamw_plan([a, good(param=a["param"])])
    with pytest.raises(AssertionError, match="overlap"):
        lib.adamw_plan([a, a])
    with pytest.raises(binding.DFlashError):
        lib.dflash_adamw_step(lib.adamw_plan([a]), 0, 1e-3)
