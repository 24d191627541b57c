"""Refusals of the log probability and optimiser calls that the host can see (no GPU needed: nothing is launched), and the layouts of their
argument structs."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

from paper_2602_06036_b200 import binding, build
from tests.test_abi_cpu import ROOT, _cfg

P = 4096                 # a stand-in for device addresses: never followed on the host
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


@pytest.fixture()
def h(lib):
    p = C.c_void_p()
    assert lib.dflash_create(C.byref(_cfg()), C.byref(p)) == 0
    yield p
    lib.dflash_destroy(p)


def test_struct_layouts(lib):
    structs = {"dflash_token_logprobs_args": binding.TokenLogprobsArgs, "dflash_token_logprobs_bwd_args": binding.TokenLogprobsBwdArgs,
               "dflash_adamw_tensor": binding.AdamwTensor, "dflash_adamw_args": binding.AdamwArgs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "dflash.h"', "int main(void){"]
    for name, st in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in st._fields_]
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(src, "w").write("\n".join(lines + ["return 0;}"]))
        subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), src, "-o", exe])
        got = dict(x.split() for x in subprocess.check_output([exe], text=True).strip().splitlines())
    for name, st in structs.items():
        assert int(got[name]) == C.sizeof(st)
        for f, _ in st._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(st, f).offset, (name, f)


def refusals(call, make, cases):
    for field, value, code in cases:
        a = make()
        setattr(a, field, value)
        assert call(a) == code, (field, value)


def test_token_logprobs(lib, h):
    make = lambda: binding.TokenLogprobsArgs(P, 0, 0, 4, 1000, 1.0, 2, P, P, P, P, 5, P, P, None)
    refusals(lambda a: lib.dflash_token_logprobs(h, C.byref(a), None), make, (
        ("n_rows", -1, -1), ("vocab", 0, -1), ("n_tokens", -1, -1), ("n_top", -1, -1), ("logits_dtype", 2, -1), ("temperature", 0.0, -1),
        ("temperature", -1.0, -1), ("temperature", NAN, -1), ("temperature", INF, -1), ("temperature", 1e-40, -1), ("n_tokens", 129, -2), ("n_top", 129, -2),
        ("vocab", 2 ** 30 + 1, -2), ("n_rows", 2 ** 28 + 1, -2), ("logits", None, -1), ("logits", P + 2, -1), ("row_stride", 999, -1), ("row_stride", -5, -1),
        ("tokens", None, -1), ("logprob", None, -1), ("top_ids", None, -1), ("top_logprob", None, -1), ("stats", P + 4, -1), ("n_rows", 0, 0)))
    assert lib.dflash_token_logprobs(None, C.byref(make()), None) == -1 and lib.dflash_token_logprobs(h, None, None) == -1


def test_token_logprobs_bwd(lib, h):
    make = lambda: binding.TokenLogprobsBwdArgs(P, 1, 0, 4, 1000, 1.0, 2, P, P, P, P, P, 2 * P, 1, 0, None)
    call = lambda a: lib.dflash_token_logprobs_bwd(h, C.byref(a), None)
    refusals(call, make, (
        ("n_rows", -1, -1), ("vocab", 0, -1), ("n_tokens", -1, -1), ("logits_dtype", 2, -1), ("dlogits_dtype", 2, -1), ("temperature", 0.0, -1),
        ("temperature", NAN, -1), ("n_tokens", 129, -2), ("vocab", 2 ** 30 + 1, -2), ("n_rows", 2 ** 28 + 1, -2), ("logits", None, -1), ("dlogits", None, -1),
        ("stats", None, -1), ("tokens", None, -1), ("d_logprob", None, -1), ("entropy", None, -1), ("row_stride", 999, -1), ("dlogits_row_stride", 999, -1),
        ("logits", P + 1, -1), ("dlogits", P + 1, -1), ("n_rows", 0, 0)))
    a = make()
    a.n_rows, a.vocab = 2 ** 20, 2 ** 25                        # 2^32 pieces
    assert call(a) == -2
    a = make()
    a.dlogits, a.dlogits_dtype = P, 0                           # over its own logits in another type
    assert call(a) == -1
    a = make()
    a.dlogits, a.dlogits_row_stride = P, 1008
    assert call(a) == -1


def test_adamw(lib, h):
    def make(**over):
        t = dict(param=P, grad=P, master=None, exp_avg=P, exp_avg_sq=P, exp_avg_scale=P, exp_avg_sq_scale=P, n=5, param_dtype=1, grad_dtype=1, state_bits=8,
                 weight_decay=0.1, lr_scale=1.0)
        t.update(over)
        table = (binding.AdamwTensor * 2)(binding.AdamwTensor(n=0, param_dtype=0, grad_dtype=0, state_bits=32, weight_decay=0, lr_scale=1),
                                          binding.AdamwTensor(**t))
        a = binding.AdamwArgs(table, 2, 1, None, 1e-3, None, 0.9, 0.95, 1e-8, 1.0, 1.0, None, P, lib.dflash_adamw_workspace_bytes(h, 2), None)
        a.keep = table
        return a

    call = lambda a: lib.dflash_adamw_step(h, C.byref(a), None)
    refusals(call, make, (
        ("n_tensors", -1, -1), ("tensors", None, -1), ("beta1", 1.0, -1), ("beta1", -0.1, -1), ("beta2", 1.0, -1), ("beta2", NAN, -1), ("eps", 0.0, -1),
        ("eps", 1e-60, -1), ("eps", NAN, -1), ("grad_scale", 0.0, -1), ("grad_scale", INF, -1), ("max_grad_norm", NAN, -1), ("step", 0, -1), ("lr", NAN, -1),
        ("workspace", None, -3), ("workspace", P + 16, -3), ("workspace_bytes", 8, -3)))
    for over in (dict(n=-1), dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(weight_decay=NAN), dict(lr_scale=INF), dict(param=None),
                 dict(grad=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(exp_avg_scale=None), dict(exp_avg_sq_scale=None), dict(param=P + 1),
                 dict(grad=P + 1), dict(master=P + 2), dict(master=P, param_dtype=0), dict(state_bits=32, exp_avg=P + 2), dict(exp_avg_scale=P + 2)):
        assert call(make(**over)) == -1, over
    a = make()
    a.n_tensors, a.max_grad_norm = 0, 0.0
    assert call(a) == 0                                          # nothing to do
    assert lib.dflash_adamw_step(None, C.byref(make()), None) == -1 and lib.dflash_adamw_step(h, None, None) == -1
    w = lib.dflash_adamw_workspace_bytes
    assert 0 < w(h, 0) == w(h, 320) < w(h, 321) and w(h, -1) == -1 and w(None, 1) == -1


@pytest.mark.parametrize("temperature", [1e-45, 2.9e-39, 3.5e-39, 4.2e-39])
def test_temperatures_whose_factors_are_infinite(lib, h, temperature):
    """log2(e) / T passes fp32's range below 4.24e-39, where 1 / T (from 2.94e-39 on) still fits: 0 times it would make NaN of a row's maximum."""
    a = binding.TokenLogprobsArgs(P, 0, 0, 4, 1000, temperature, 2, P, P, P, P, 5, P, P, None)
    assert lib.dflash_token_logprobs(h, C.byref(a), None) == -1
    b = binding.TokenLogprobsBwdArgs(P, 1, 0, 4, 1000, temperature, 2, P, P, P, P, P, 2 * P, 1, 0, None)
    assert lib.dflash_token_logprobs_bwd(h, C.byref(b), None) == -1
