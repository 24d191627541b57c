"""The AdamW step's wide accesses behind every start, in chunks one by one and four behind each other, and behind entry 2^31, entry by entry against the formula in 64 bits
(tolerances: see tests/test_adamw_gpu.py)."""
import pytest
import torch

from tests.test_adamw_gpu import BF16, E4M3, F32, U, lib, run_and_check, tensor  # noqa: F401

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS, WD, T = 6e-4, 0.9, 0.95, 1e-8, 0.1, 7


@pytest.mark.parametrize("weights", ["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("grads", [F32, BF16])
@pytest.mark.parametrize("at", [0, 1, 2, 3])
def test_starts_behind_a_border(lib, weights, grads, at):
    """Sizes of several chunks of 4096 entries, so that whole ones lie inside."""
    run_and_check(lib, [tensor(n, weights, grads, 32, seed=n, at=at) for n in (4096, 4097, 8195, 20001, 100003)], t=3, max_norm=0.05)


@pytest.mark.parametrize("behind", [{"param": 1}, {"grad": 1}, {"exp_avg": 2}, {"exp_avg_sq": 3}, {"master": 1}, {"param": 3, "grad": 3, "master": 3, "exp_avg": 3}])
def test_buffers_that_start_apart(lib, behind):
    """One buffer begins elsewhere than the others: all entries one by one."""
    e = tensor(20001, "mixed", BF16, 32, seed=5)
    for k, off in behind.items():
        e[k] = torch.cat([e[k].new_zeros(off), e[k]])[off:]
    run_and_check(lib, [e, tensor(5000, "fp32", F32, 32, seed=6)], t=3, max_norm=0.05)


@pytest.mark.parametrize("behind", [{"exp_avg": 1}, {"exp_avg_sq": 2}, {"param": 4, "grad": 4, "master": 4, "exp_avg": 4, "exp_avg_sq": 4}, {"grad": 2, "param": 2, "master": 2}])
def test_buffers_of_8_bit_states_that_start_apart(lib, behind):
    e = tensor(20001, "mixed", BF16, 8, seed=5)
    for k, off in behind.items():
        wide = e[k].view(torch.uint8) if e[k].dtype is E4M3 else e[k]
        e[k] = torch.cat([wide.new_zeros(off), wide])[off:].view(e[k].dtype)
    run_and_check(lib, [e], t=3, max_norm=0.05)


def large(n, weights, grads, bits, at, seed):
    """A tensor of the sizes of tensor(), made on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    on = lambda dt, x: torch.zeros(n + at, dtype=dt, device="cuda")[at:].copy_(x)
    normal = lambda: torch.randn(n, generator=g, device="cuda")
    size = 10.0 ** (normal() - 3)
    w = normal()
    e = {"param": on(F32 if weights == "fp32" else BF16, w), "grad": on(grads, normal() * size), "weight_decay": WD}
    if weights == "mixed":
        e["master"] = on(F32, w)
    m, v = normal() * size * 0.3, (normal() ** 2 + 0.1) * size * size
    if bits == 32:
        e["exp_avg"], e["exp_avg_sq"] = on(F32, m), on(F32, v)
    else:
        for k, x in (("exp_avg", m), ("exp_avg_sq", v.sqrt())):
            top = torch.nn.functional.pad(x.abs(), (0, -n % 128)).view(-1, 128).amax(1) / 448
            e[k], e[k + "_scale"] = on(E4M3, (x / top.repeat_interleave(128)[:n]).clamp(-448, 448).to(E4M3)), top
    return e


def state(e, k):
    x = e[k].double()
    return x if e[k].dtype is F32 else x * e[k + "_scale"].double().repeat_interleave(128)[:x.numel()]


def check_large(lib, e):
    """One step, all entries."""
    w, g = e["param" if e.get("master") is None else "master"].double(), e["grad"].double()
    m, v = state(e, "exp_avg"), state(e, "exp_avg_sq")
    eight = e["exp_avg"].dtype is E4M3
    v = v * v if eight else v
    lib.dflash_adamw_step(lib.adamw_plan([e]), T, LR, B1, B2, EPS)
    torch.cuda.synchronize()
    parts = B1 * m.abs() + (1 - B1) * g.abs()
    m, v = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    under = (v / (1 - B2 ** T)).sqrt() + EPS
    tol = 3 * U * w.abs() + 24 * U * LR * parts / (1 - B1 ** T) / under + 1e-38
    w = w - LR * WD * w - LR * (m / (1 - B1 ** T)) / under
    if e.get("master") is not None:
        assert torch.equal(e["param"], e["master"].to(BF16))
        assert bool(((e["master"].double() - w).abs() <= tol).all())
    else:
        tol = tol + 2.0 ** -8 * w.abs() * 1.001 if e["param"].dtype is BF16 else tol
        assert bool(((e["param"].double() - w).abs() <= tol).all())
    if not eight:
        assert bool(((e["exp_avg"].double() - m).abs() <= 12 * U * parts + 1e-44).all())
        assert bool(((e["exp_avg_sq"].double() - v).abs() <= 16 * U * v + 1e-44).all())
        return
    for k, x, least, size in (("exp_avg", m, 2.0 ** -10, parts), ("exp_avg_sq", v.sqrt(), 2.0 ** -9, v.sqrt())):
        blocks = lambda y: torch.nn.functional.pad(y.abs(), (0, -y.numel() % 128)).view(-1, 128).amax(1)
        top, big = blocks(x), blocks(size)
        assert bool(((e[k + "_scale"].double() - top / 448).abs() <= 16 * U * big / 448).all())
        wide = lambda y: y.repeat_interleave(128)[:x.numel()]
        slack = 32 * U * (size + wide(big))
        assert bool(((state(e, k) - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), least * wide(top) / 448) * 1.0001 + slack).all())


@pytest.mark.parametrize("weights,grads,bits,at", [("fp32", F32, 32, 2), ("bf16", BF16, 32, 3), ("mixed", BF16, 32, 1), ("mixed", F32, 32, 2), ("bf16", F32, 32, 0), ("fp32", F32, 8, 0),
                                                   ("mixed", BF16, 8, 0), ("bf16", BF16, 8, 0), ("bf16", BF16, 8, 1)])
def test_four_chunks_behind_each_other(lib, weights, grads, bits, at):
    """So many entries that a CTA takes four chunks at a look at the table (64 x 4096 entries for each of two CTAs an SM)."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    check_large(lib, large(64 * 4096 * 2 * sms + 54321, weights, grads, bits, at, 3))


def test_behind_entry_2_to_the_31(lib):
    """Pieces of a tensor of more than 2^31 entries, its other entries 0, against the same step of each piece alone: every buffer of theirs, which the step changes."""
    n, piece = 2 ** 31 + 128 * 9, 1024
    zeros = lambda k, dt: torch.zeros(k, dtype=dt, device="cuda")
    big = {"param": zeros(n, BF16), "grad": zeros(n, BF16), "weight_decay": WD}
    for k in ("exp_avg", "exp_avg_sq"):
        big[k], big[k + "_scale"] = zeros(n, torch.uint8).view(E4M3), zeros(n // 128, F32)
    raw = lambda x: x.view(torch.uint8)
    pieces = []
    for i, at in enumerate((0, 2 ** 30, 2 ** 31 - 512, n - 512)):
        e = tensor(min(piece, n - at), "bf16", BF16, 8, seed=i)
        e["grad"].mul_(30)                                     # of the size of m, and beyond
        for k, x in e.items():
            if k != "weight_decay":
                to = at // 128 if k.endswith("scale") else at
                raw(big[k][to:to + len(x)]).copy_(raw(x))
        pieces.append((at, e, {k: x.clone() for k, x in e.items() if k != "weight_decay"}))
    for plan in ([big], [e for _, e, _ in pieces]):
        lib.dflash_adamw_step(lib.adamw_plan(plan), 3, 0.1)
    torch.cuda.synchronize()
    for at, e, before in pieces:
        for k, old in before.items():
            to = at // 128 if k.endswith("scale") else at
            assert torch.equal(raw(big[k][to:to + len(old)]), raw(e[k])), (at, k)
            if k != "grad":                                    # (a piece that was not stepped would differ)
                assert float((raw(e[k]).view(-1, old.element_size()) != raw(old).view(-1, old.element_size())).any(1).float().mean()) > 0.5, (at, k)
    assert not big["param"][piece:2 ** 30].any() and not big["exp_avg_sq_scale"][8:2 ** 23].any()
