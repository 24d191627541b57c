"""Refusals of the shared-cache calls that the host can see (no GPU needed: nothing is launched), and the layouts of their
argument structs."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

from paper_2602_06036_b200 import binding, build, synth
from tests.test_abi_cpu import ROOT, _cfg, _qwen_cfg

P = 4096                 # a stand-in for device addresses: never followed on the host


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


@pytest.fixture()
def h(lib):
    p = C.c_void_p()
    assert lib.dflash_create(C.byref(_qwen_cfg()), C.byref(p)) == 0
    yield p
    lib.dflash_destroy(p)


def test_struct_layouts(lib):
    structs = {"dflash_prefix_attn_args": binding.PrefixAttnArgs, "dflash_pages_copy_args": binding.PagesCopyArgs,
               "dflash_pages_fork_args": binding.PagesForkArgs, "dflash_pages_resize_args": binding.PagesResizeArgs,
               "dflash_pages_compact_args": binding.PagesCompactArgs}
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


def _attn(lib, h, batch=2, rows=4, groups=1):
    need = lib.dflash_prefix_attention_workspace_bytes(h, batch, rows, groups)
    assert need > 0
    return binding.PrefixAttnArgs(0, P, P, P, batch, rows, groups, P, P, P, 100, P, 2, P, 8, 0, P, None, P, need, None)


def test_prefix_attention(lib, h):
    call = lambda a: lib.dflash_prefix_attention(h, C.byref(a), None)
    for field, value, code in (("mode", 2, -1), ("batch", -1, -1), ("rows", 33, -1), ("rows", -1, -1), ("n_groups", -1, -1), ("max_ctx_len", -1, -1),
                               ("max_pages", 0, -1), ("n_pool_pages", 0, -1), ("layer", -1, -1), ("layer", 5, -1), ("q", None, -1), ("k_blk", None, -1),
                               ("v_blk", None, -1), ("group_start", None, -1), ("prefix_len", None, -1), ("ctx_len", None, -1), ("page_table", None, -1),
                               ("kv_pool", None, -1), ("out", None, -1), ("q", P + 8, -1), ("out", P + 2, -1), ("kv_pool", P + 4, -1), ("batch", 65536, -2),
                               ("n_groups", 65536, -2), ("max_ctx_len", 2 ** 31 - 1, -2), ("workspace", None, -3), ("workspace", P + 16, -3),
                               ("workspace_bytes", 0, -3), ("batch", 3, -3)):
        a = _attn(lib, h)
        setattr(a, field, value)
        assert call(a) == code, (field, value)
    for field in ("batch", "rows"):
        a = _attn(lib, h)
        setattr(a, field, 0)
        assert call(a) == 0
    assert lib.dflash_prefix_attention(None, C.byref(_attn(lib, h)), None) == -1 and lib.dflash_prefix_attention(h, None, None) == -1
    w = lib.dflash_prefix_attention_workspace_bytes
    assert w(h, 2, 4, 0) < w(h, 2, 4, 1) <= w(h, 40, 4, 1) <= w(h, 40, 32, 9)
    assert w(h, -1, 4, 1) == -1 and w(h, 1, 33, 1) == -1 and w(h, 70000, 1, 1) == -2 and w(None, 1, 1, 1) == -1


def test_more_than_128_heads_a_group_are_refused(lib):
    p = C.c_void_p()
    assert lib.dflash_create(C.byref(_cfg(n_q_heads=129, n_kv_heads=1)), C.byref(p)) == 0
    assert lib.dflash_prefix_attention_workspace_bytes(p, 1, 1, 1) == -2
    a = binding.PrefixAttnArgs(0, P, P, P, 1, 1, 1, P, P, P, 100, P, 2, P, 8, 0, P, None, P, 1 << 40, None)
    assert lib.dflash_prefix_attention(p, C.byref(a), None) == -2
    lib.dflash_destroy(p)


def test_pages(lib, h):
    ws = lib.dflash_pages_workspace_bytes(4, 6, 100)
    assert ws > 0 and lib.dflash_pages_workspace_bytes(-1, 6, 100) == -1 and lib.dflash_pages_workspace_bytes(65536, 6, 100) == -2
    copy = lambda: binding.PagesCopyArgs(4, None, P, P, None, P, 100, None)
    fork = lambda: binding.PagesForkArgs(4, P, P, P, P, 9, 6, P, P, 100, None, None, None, P, ws, None)
    resize = lambda: binding.PagesResizeArgs(4, P, P, P, P, 9, 6, P, P, 100, None, None, None, P, ws, None)
    compact = lambda: binding.PagesCompactArgs(P, 9, 6, P, P, 100, None, None, None, None, P, ws, None)
    common = [("kv_pool", None, -1), ("kv_pool", P + 8, -1), ("n_pool_pages", 0, -1)]
    table = [("page_table", None, -1), ("ref_count", None, -1), ("n_rows", 0, -1), ("max_pages", 0, -1), ("copy_src", P, -1), ("copy_dst", P, -1),
             ("workspace", None, -3), ("workspace", P + 64, -3), ("workspace_bytes", 128, -3)]
    listed = [("n", -1, -1), ("n", 65536, -2)]
    for fn, make, cases in ((lib.dflash_pages_copy, copy, common + listed + [("src", None, -1), ("dst", None, -1)]),
                            (lib.dflash_pages_fork, fork, common + table + listed + [("parent", None, -1), ("child", None, -1), ("fork_len", None, -1)]),
                            (lib.dflash_pages_resize, resize, common + table + listed + [("rows", None, -1), ("keep_len", None, -1), ("capacity", None, -1)]),
                            (lib.dflash_pages_compact, compact, common + table)):
        for field, value, code in cases:
            a = make()
            setattr(a, field, value)
            assert fn(h, C.byref(a), None) == code, (fn.__name__, field, value)
        assert fn(None, C.byref(make()), None) == -1 and fn(h, None, None) == -1
        if fn is not lib.dflash_pages_compact:
            a = make()
            a.n = 0
            assert fn(h, C.byref(a), None) == 0


def test_pools_too_large_to_count_are_refused(lib, h):
    most = 1 << 30
    assert lib.dflash_pages_workspace_bytes(1, 1, most) > 0
    for n, width, pages in ((1, 1, most + 1), (1, most + 1, 8), (1, 1, 2 ** 31 - 1), (0, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert lib.dflash_pages_workspace_bytes(n, width, pages) == -2
    P = 1 << 20                                          # never followed
    for pages, width in ((most + 1, 4), (2 ** 31 - 1, 4), (8, most + 1)):
        if pages > most:
            a = binding.PagesCopyArgs(n=1, src=P, dst=P, kv_pool=P, n_pool_pages=pages)
            assert lib.dflash_pages_copy(h, C.byref(a), None) == -2
        table = dict(page_table=P, n_rows=2, max_pages=width, ref_count=P, kv_pool=P, n_pool_pages=pages, workspace=P, workspace_bytes=1 << 62)
        a = binding.PagesForkArgs(n=1, parent=P, child=P, fork_len=P, **table)
        assert lib.dflash_pages_fork(h, C.byref(a), None) == -2
        a = binding.PagesResizeArgs(n=1, rows=P, keep_len=P, capacity=P, **table)
        assert lib.dflash_pages_resize(h, C.byref(a), None) == -2
        a = binding.PagesCompactArgs(**table)
        assert lib.dflash_pages_compact(h, C.byref(a), None) == -2
