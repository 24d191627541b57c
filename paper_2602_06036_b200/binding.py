"""ctypes binding of libdflash_b200.so: argument marshalling only.

Every step of the path runs in the library's CUDA kernels; this file turns torch tensors into the
plain pointers and sizes of `include/dflash.h`. There is no CPU fallback: if the library is missing
or fails to load, `load()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
from typing import Dict, Optional

import torch

from .synth import DFlashConfig

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdflash_b200.so")
_lib = None

F32, BF16 = 0, 1
ATTN_FULL, ATTN_CAUSAL = 0, 1
VERIFY_LOGITS, VERIFY_IDS = 0, 1
DEV_BAD_TOKEN, DEV_BAD_PAGE, DEV_CTX_OVERFLOW, DEV_TIMEOUT = 1, 2, 4, 8
DEV_BAD_ROW, DEV_POOL_FULL, DEV_BAD_GROUP, DEV_NOT_FINITE = 16, 32, 64, 128

EXPORTS = (
    "dflash_create", "dflash_destroy", "dflash_set_weights", "dflash_workspace_bytes",
    "dflash_ctx_project", "dflash_draft_block", "dflash_verify_accept", "dflash_block_attention",
    "dflash_lmhead_argmax", "dflash_status_string", "dflash_launch_count", "dflash_profile_enable",
    "dflash_profile_read", "dflash_family_name", "dflash_trace_enable", "dflash_trace_read",
    "dflash_verify_accept_static", "dflash_sample_rows", "dflash_verify_accept_sample",
    "dflash_sample_workspace_bytes", "dflash_target_verify", "dflash_block_loss", "dflash_attention_plan",
    "dflash_block_attention_bwd", "dflash_gemm_plan_check", "dflash_prefix_attention",
    "dflash_prefix_attention_workspace_bytes", "dflash_prefix_plan_check", "dflash_pages_copy", "dflash_pages_fork",
    "dflash_pages_resize", "dflash_pages_compact", "dflash_pages_workspace_bytes", "dflash_token_logprobs",
    "dflash_token_logprobs_bwd", "dflash_token_logprobs_plan", "dflash_adamw_step", "dflash_adamw_workspace_bytes",
)
N_FAMILIES = 15


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "n_feat_layers",
        "d_target", "block_size", "page_size", "dtype", "mask_token_id", "use_rope")] + [
        ("rms_eps", C.c_float), ("softmax_scale", C.c_float), ("qk_norm", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("g1", "W_qkv", "W_o", "g2", "W_gateup", "W_down", "g_q", "g_k")]


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("W_c", C.c_void_p), ("g_c", C.c_void_p),
                ("layers", C.POINTER(LayerWeights)), ("g_f", C.c_void_p), ("W_lm", C.c_void_p),
                ("rope_cos", C.c_void_p), ("rope_sin", C.c_void_p), ("rope_max_pos", C.c_int32)]


class CtxArgs(C.Structure):
    _fields_ = [("feats", C.c_void_p), ("batch", C.c_int32), ("max_new", C.c_int32), ("n_new", C.c_void_p),
                ("ctx_len", C.c_void_p), ("page_table", C.c_void_p), ("max_pages", C.c_int32),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class DraftArgs(C.Structure):
    _fields_ = [("anchor_ids", C.c_void_p), ("batch", C.c_int32), ("ctx_len", C.c_void_p),
                ("max_ctx_len", C.c_int32), ("page_table", C.c_void_p), ("max_pages", C.c_int32),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64), ("draft_ids", C.c_void_p), ("top1", C.c_void_p),
                ("margin", C.c_void_p), ("hidden_out", C.c_void_p), ("logits_out", C.c_void_p),
                ("dev_status", C.c_void_p), ("block_rows", C.c_int32), ("ctx", C.POINTER(CtxArgs))]


class VerifyArgs(C.Structure):
    _fields_ = [("mode", C.c_int32), ("logits", C.c_void_p), ("logits_dtype", C.c_int32),
                ("logits_row_stride", C.c_int64), ("target_ids", C.c_void_p), ("draft_ids", C.c_void_p),
                ("draft_stride", C.c_int32), ("batch", C.c_int32), ("gamma", C.c_int32), ("vocab", C.c_int32),
                ("ctx_len", C.c_void_p), ("accept_len", C.c_void_p), ("out_tokens", C.c_void_p),
                ("bonus", C.c_void_p), ("new_ctx_len", C.c_void_p), ("target_ids_out", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class TargetArgs(C.Structure):
    _fields_ = [("token_ids", C.c_void_p), ("batch", C.c_int32), ("rows", C.c_int32), ("ctx_len", C.c_void_p),
                ("max_ctx_len", C.c_int32), ("page_table", C.c_void_p), ("max_pages", C.c_int32),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("tap_layers", C.POINTER(C.c_int32)),
                ("n_taps", C.c_int32), ("feats_out", C.c_void_p), ("logits_out", C.c_void_p),
                ("ids_out", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("dev_status", C.c_void_p)]


class BlockLossArgs(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("logits_dtype", C.c_int32), ("row_stride", C.c_int64),
                ("n_blocks", C.c_int32), ("block_rows", C.c_int32), ("vocab", C.c_int32), ("targets", C.c_void_p),
                ("gamma", C.c_float), ("row_loss", C.c_void_p), ("loss_sum", C.c_void_p), ("dlogits", C.c_void_p),
                ("dlogits_dtype", C.c_int32), ("dlogits_row_stride", C.c_int64), ("grad_scale", C.c_float),
                ("dev_status", C.c_void_p)]


class SampleArgs(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("logits_dtype", C.c_int32), ("row_stride", C.c_int64),
                ("n_rows", C.c_int32), ("vocab", C.c_int32), ("temperature", C.c_float), ("u", C.c_void_p),
                ("ids", C.c_void_p), ("prob", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class VerifySampleArgs(C.Structure):
    _fields_ = [("target_logits", C.c_void_p), ("target_dtype", C.c_int32), ("target_row_stride", C.c_int64),
                ("draft_logits", C.c_void_p), ("draft_dtype", C.c_int32), ("draft_row_stride", C.c_int64),
                ("draft_rows_per_seq", C.c_int32), ("draft_ids", C.c_void_p), ("draft_stride", C.c_int32),
                ("batch", C.c_int32), ("gamma", C.c_int32), ("vocab", C.c_int32), ("temperature", C.c_float),
                ("u_accept", C.c_void_p), ("u_final", C.c_void_p), ("ctx_len", C.c_void_p),
                ("accept_len", C.c_void_p), ("out_tokens", C.c_void_p), ("bonus", C.c_void_p),
                ("new_ctx_len", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("dev_status", C.c_void_p)]


class AttnArgs(C.Structure):
    _fields_ = [("mode", C.c_int32), ("q", C.c_void_p), ("k_blk", C.c_void_p), ("v_blk", C.c_void_p),
                ("batch", C.c_int32), ("rows", C.c_int32), ("ctx_len", C.c_void_p), ("max_ctx_len", C.c_int32),
                ("page_table", C.c_void_p), ("max_pages", C.c_int32), ("kv_pool", C.c_void_p),
                ("n_pool_pages", C.c_int32), ("layer", C.c_int32), ("out", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p),
                ("lse_out", C.c_void_p)]


class AttnBwdArgs(C.Structure):
    _fields_ = [("mode", C.c_int32), ("q", C.c_void_p), ("k_blk", C.c_void_p), ("v_blk", C.c_void_p), ("out", C.c_void_p),
                ("lse", C.c_void_p), ("dout", C.c_void_p), ("batch", C.c_int32), ("rows", C.c_int32), ("ctx_len", C.c_void_p),
                ("max_ctx_len", C.c_int32), ("page_table", C.c_void_p), ("max_pages", C.c_int32), ("kv_pool", C.c_void_p),
                ("n_pool_pages", C.c_int32), ("layer", C.c_int32), ("shared_page_row", C.c_int32), ("dq", C.c_void_p),
                ("dk_blk", C.c_void_p), ("dv_blk", C.c_void_p), ("dkv_ctx", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class PrefixAttnArgs(C.Structure):
    _fields_ = [("mode", C.c_int32), ("q", C.c_void_p), ("k_blk", C.c_void_p), ("v_blk", C.c_void_p), ("batch", C.c_int32),
                ("rows", C.c_int32), ("n_groups", C.c_int32), ("group_start", C.c_void_p), ("prefix_len", C.c_void_p),
                ("ctx_len", C.c_void_p), ("max_ctx_len", C.c_int32), ("page_table", C.c_void_p), ("max_pages", C.c_int32),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("layer", C.c_int32), ("out", C.c_void_p),
                ("lse_out", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class PagesCopyArgs(C.Structure):
    _fields_ = [("n", C.c_int32), ("count", C.c_void_p), ("src", C.c_void_p), ("dst", C.c_void_p), ("n_slots", C.c_void_p),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("dev_status", C.c_void_p)]


class PagesForkArgs(C.Structure):
    _fields_ = [("n", C.c_int32), ("parent", C.c_void_p), ("child", C.c_void_p), ("fork_len", C.c_void_p),
                ("page_table", C.c_void_p), ("n_rows", C.c_int32), ("max_pages", C.c_int32), ("ref_count", C.c_void_p),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("copy_src", C.c_void_p), ("copy_dst", C.c_void_p),
                ("copy_slots", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class PagesResizeArgs(C.Structure):
    _fields_ = [("n", C.c_int32), ("rows", C.c_void_p), ("keep_len", C.c_void_p), ("capacity", C.c_void_p),
                ("page_table", C.c_void_p), ("n_rows", C.c_int32), ("max_pages", C.c_int32), ("ref_count", C.c_void_p),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("copy_src", C.c_void_p), ("copy_dst", C.c_void_p),
                ("copy_slots", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64), ("dev_status", C.c_void_p)]


class PagesCompactArgs(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("n_rows", C.c_int32), ("max_pages", C.c_int32), ("ref_count", C.c_void_p),
                ("kv_pool", C.c_void_p), ("n_pool_pages", C.c_int32), ("n_live", C.c_void_p), ("copy_src", C.c_void_p),
                ("copy_dst", C.c_void_p), ("n_copies", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("dev_status", C.c_void_p)]


class TokenLogprobsArgs(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("logits_dtype", C.c_int32), ("row_stride", C.c_int64), ("n_rows", C.c_int32), ("vocab", C.c_int32),
                ("temperature", C.c_float), ("n_tokens", C.c_int32), ("tokens", C.c_void_p), ("logprob", C.c_void_p), ("stats", C.c_void_p),
                ("entropy", C.c_void_p), ("n_top", C.c_int32), ("top_ids", C.c_void_p), ("top_logprob", C.c_void_p), ("dev_status", C.c_void_p)]


class TokenLogprobsBwdArgs(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("logits_dtype", C.c_int32), ("row_stride", C.c_int64), ("n_rows", C.c_int32), ("vocab", C.c_int32),
                ("temperature", C.c_float), ("n_tokens", C.c_int32), ("tokens", C.c_void_p), ("stats", C.c_void_p), ("entropy", C.c_void_p),
                ("d_logprob", C.c_void_p), ("d_entropy", C.c_void_p), ("dlogits", C.c_void_p), ("dlogits_dtype", C.c_int32),
                ("dlogits_row_stride", C.c_int64), ("dev_status", C.c_void_p)]


class AdamwTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("master", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
                ("exp_avg_scale", C.c_void_p), ("exp_avg_sq_scale", C.c_void_p), ("n", C.c_int64), ("param_dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("state_bits", C.c_int32), ("weight_decay", C.c_float), ("lr_scale", C.c_float)]


class AdamwArgs(C.Structure):
    _fields_ = [("tensors", C.POINTER(AdamwTensor)), ("n_tensors", C.c_int32), ("step", C.c_int32), ("step_dev", C.c_void_p), ("lr", C.c_double),
                ("lr_dev", C.c_void_p), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("grad_scale", C.c_double),
                ("max_grad_norm", C.c_double), ("grad_norm", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("dev_status", C.c_void_p)]


class LmHeadArgs(C.Structure):
    _fields_ = [("hidden", C.c_void_p), ("hidden_is_f32", C.c_int32), ("n_rows", C.c_int32),
                ("apply_norm", C.c_int32), ("ids", C.c_void_p), ("top1", C.c_void_p), ("margin", C.c_void_p),
                ("logits_out", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64),
                ("dev_status", C.c_void_p)]


def load():
    """Load the shared library (once). Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} not found: build it with `python -m paper_2602_06036_b200.build`")
    lib = C.CDLL(_LIB_PATH)
    lib.dflash_create.argtypes = [C.POINTER(Config), C.POINTER(C.c_void_p)]
    lib.dflash_create.restype = C.c_int32
    lib.dflash_destroy.argtypes = [C.c_void_p]
    lib.dflash_destroy.restype = None
    lib.dflash_set_weights.argtypes = [C.c_void_p, C.POINTER(Weights)]
    lib.dflash_set_weights.restype = C.c_int32
    lib.dflash_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
    lib.dflash_workspace_bytes.restype = C.c_int64
    for name, st in (("dflash_ctx_project", CtxArgs), ("dflash_draft_block", DraftArgs),
                     ("dflash_verify_accept", VerifyArgs), ("dflash_verify_accept_static", VerifyArgs), ("dflash_block_attention", AttnArgs),
                     ("dflash_lmhead_argmax", LmHeadArgs), ("dflash_sample_rows", SampleArgs),
                     ("dflash_verify_accept_sample", VerifySampleArgs), ("dflash_target_verify", TargetArgs),
                     ("dflash_block_loss", BlockLossArgs), ("dflash_block_attention_bwd", AttnBwdArgs),
                     ("dflash_prefix_attention", PrefixAttnArgs), ("dflash_pages_copy", PagesCopyArgs), ("dflash_pages_fork", PagesForkArgs),
                     ("dflash_pages_resize", PagesResizeArgs), ("dflash_pages_compact", PagesCompactArgs),
                     ("dflash_token_logprobs", TokenLogprobsArgs), ("dflash_token_logprobs_bwd", TokenLogprobsBwdArgs), ("dflash_adamw_step", AdamwArgs)):
        fn = getattr(lib, name)
        fn.argtypes = [C.c_void_p, C.POINTER(st), C.c_void_p]
        fn.restype = C.c_int32
    lib.dflash_sample_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.dflash_sample_workspace_bytes.restype = C.c_int64
    lib.dflash_attention_plan.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_int64)]
    lib.dflash_attention_plan.restype = C.c_int32
    lib.dflash_gemm_plan_check.argtypes = [C.c_int32] * 7 + [C.POINTER(C.c_int32)]
    lib.dflash_gemm_plan_check.restype = C.c_int32
    lib.dflash_prefix_attention_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32]
    lib.dflash_prefix_attention_workspace_bytes.restype = C.c_int64
    lib.dflash_pages_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
    lib.dflash_pages_workspace_bytes.restype = C.c_int64
    lib.dflash_adamw_workspace_bytes.argtypes = [C.c_void_p, C.c_int32]
    lib.dflash_adamw_workspace_bytes.restype = C.c_int64
    i32p = C.POINTER(C.c_int32)
    lib.dflash_prefix_plan_check.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, i32p, i32p, i32p, C.c_int32, C.POINTER(C.c_int64)]
    lib.dflash_prefix_plan_check.restype = C.c_int32
    lib.dflash_token_logprobs_plan.argtypes = [C.c_void_p] + [C.c_int32] * 5 + [i32p]
    lib.dflash_token_logprobs_plan.restype = C.c_int32
    lib.dflash_status_string.argtypes = [C.c_int32]
    lib.dflash_status_string.restype = C.c_char_p
    lib.dflash_launch_count.argtypes = []
    lib.dflash_launch_count.restype = C.c_int64
    lib.dflash_profile_enable.argtypes = [C.c_void_p, C.c_int32]
    lib.dflash_profile_enable.restype = C.c_int32
    lib.dflash_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.dflash_profile_read.restype = C.c_int32
    lib.dflash_trace_enable.argtypes = [C.c_void_p, C.c_void_p, C.c_int32]
    lib.dflash_trace_enable.restype = C.c_int32
    lib.dflash_trace_read.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    lib.dflash_trace_read.restype = C.c_int32
    lib.dflash_family_name.argtypes = [C.c_int32]
    lib.dflash_family_name.restype = C.c_char_p
    _lib = lib
    return lib


class DFlashError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"dflash error {code}: {load().dflash_status_string(code).decode()}")


def _check(rc: int):
    if rc != 0:
        raise DFlashError(rc)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device-contiguous tensor expected"
    return C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


# cudaStream_t of a device's current stream, without the Stream object around it where torch offers that (1 us less)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
# torch.cuda.current_device() without its look at whether CUDA is initialised, which a handle's tensors have seen to
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def launch_count() -> int:
    return int(load().dflash_launch_count())


class AdamwPlan:
    """The tensors of an optimiser step as the library takes them (see DFlash.adamw_plan). Keeps them alive; their addresses are those of the plan. So a
    gradient has to stay where it is: after `p.grad = None` (zero_grad's default) the next backward pass makes another tensor, of which the plan knows
    nothing. Clear gradients in place (zero_grad(set_to_none=False)), or make a new plan."""

    def __init__(self, entries, index: int):
        self.tensors = [dict(e) for e in entries]
        self.n = len(self.tensors)
        self.index = index
        self.table = (AdamwTensor * max(self.n, 1))()
        spans = []                                            # (start, end, tensor, name) of every buffer
        for i, e in enumerate(self.tensors):
            unknown = set(e) - {"param", "grad", "exp_avg", "exp_avg_sq", "master", "exp_avg_scale", "exp_avg_sq_scale", "weight_decay", "lr_scale"}
            assert not unknown, f"tensor {i}: unknown {sorted(unknown)}"
            param, n = e["param"], e["param"].numel()
            bits = 32 if e["exp_avg"].dtype is torch.float32 else 8
            state = (torch.float32,) if bits == 32 else (torch.float8_e4m3fn, torch.uint8)
            weights = (torch.float32, torch.bfloat16)

            def address(name, types, size, needed=True):
                t = e.get(name)
                if t is None:
                    assert not needed, f"tensor {i}: {name} missing"
                    return None
                assert t.dtype in types, f"tensor {i}: {name} has type {t.dtype}, expected {types}"
                assert t.get_device() == index and t.is_contiguous(), f"tensor {i}: {name} has to be contiguous and on device {index}"
                assert t.numel() == size, f"tensor {i}: {name} has {t.numel()} entries, expected {size}"
                if size:
                    spans.append((t.data_ptr(), t.data_ptr() + size * t.element_size(), i, name))
                return t.data_ptr()

            assert e.get("master") is None or param.dtype is torch.bfloat16, f"tensor {i}: a master copy goes with a bf16 param"
            scales = -(-n // 128)
            self.table[i] = AdamwTensor(
                address("param", weights, n), address("grad", weights, n), address("master", (torch.float32,), n, False), address("exp_avg", state, n),
                address("exp_avg_sq", state, n), *((address(k, (torch.float32,), scales) if bits == 8 else None) for k in ("exp_avg_scale", "exp_avg_sq_scale")),
                n, F32 if param.dtype is torch.float32 else BF16, F32 if e["grad"].dtype is torch.float32 else BF16, bits,
                float(e.get("weight_decay", 0.0)), float(e.get("lr_scale", 1.0)))
        # what is written lies apart from everything else; gradients are only read, so that tensors may share them
        last_read = last_written = (0, 0, 0, "")                # of the spans before, those that reach furthest
        for s in sorted(spans):
            reads = s[3] == "grad"
            for a in (last_written,) if reads else (last_written, last_read):
                assert a[1] <= s[0], f"{a[3]} of tensor {a[2]} and {s[3]} of tensor {s[2]} overlap"
            if reads:
                last_read = max(last_read, s, key=lambda x: x[1])
            else:
                last_written = s


class DFlash:
    """Owns a library handle plus the torch tensors whose pointers it lent to the library."""

    def __init__(self, cfg: DFlashConfig, device: str = "cuda:0"):
        self.lib = load()
        self.cfg = cfg
        self.device = torch.device(device)
        self.ccfg = Config(cfg.n_layers, cfg.d_model, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.d_ffn,
                           cfg.vocab, cfg.n_feat_layers, cfg.d_target, cfg.block_size, cfg.page_size,
                           F32 if cfg.dtype == "fp32" else BF16, cfg.mask_token_id, cfg.use_rope,
                           cfg.rms_eps, cfg.softmax_scale, int(getattr(cfg, "qk_norm", 0)))
        hp = C.c_void_p()
        _check(self.lib.dflash_create(C.byref(self.ccfg), C.byref(hp)))
        self.h = hp
        self._keep = {}
        self._ws = None
        self._scratches = {}
        self._needs = {}
        self._launching = threading.Lock()
        self._index = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)

    def close(self):
        if getattr(self, "h", None):
            self.lib.dflash_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- set-up -------------------------------------------------------------------------
    def set_weights(self, packed: Dict, rope_cos: torch.Tensor, rope_sin: torch.Tensor):
        """`packed` = synth.pack_device_weights(...) moved to the device (any mapping with the same keys). Contiguous tensors of the handle's device are
        held as they are, without a copy: what changes them in place (dflash_adamw_step) holds for the calls behind it on the stream."""
        dev = self.device
        keep = {k: packed[k].to(dev).contiguous() for k in ("embed", "W_c", "g_c", "g_f", "W_lm")}
        keep["layers"] = [{k: v.to(dev).contiguous() for k, v in lw.items()} for lw in packed["layers"]]
        keep["rope_cos"] = rope_cos.to(dev, torch.float32).contiguous()
        keep["rope_sin"] = rope_sin.to(dev, torch.float32).contiguous()
        arr = (LayerWeights * self.cfg.n_layers)()
        for i, lw in enumerate(keep["layers"]):
            arr[i] = LayerWeights(*(lw[k].data_ptr() for k in ("g1", "W_qkv", "W_o", "g2", "W_gateup", "W_down")),
                                  *((lw[k].data_ptr() if k in lw else None) for k in ("g_q", "g_k")))
        w = Weights(keep["embed"].data_ptr(), keep["W_c"].data_ptr(), keep["g_c"].data_ptr(), arr,
                    keep["g_f"].data_ptr(), keep["W_lm"].data_ptr(), keep["rope_cos"].data_ptr(),
                    keep["rope_sin"].data_ptr(), keep["rope_cos"].shape[0])
        _check(self.lib.dflash_set_weights(self.h, C.byref(w)))
        self._keep = keep

    def workspace_bytes(self, max_batch: int, max_rows: int) -> int:
        n = self.lib.dflash_workspace_bytes(self.h, max_batch, max_rows)
        if n < 0:
            raise DFlashError(int(n))
        return int(n)

    def workspace(self, max_batch: int, max_rows: int) -> torch.Tensor:
        need = self.workspace_bytes(max_batch, max_rows)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def profile(self, fn, steps: int):
        """Run `fn` `steps` times with an event pair around every launch of this handle.
        Returns {family: (microseconds per launch, launches per step)}."""
        _check(self.lib.dflash_profile_enable(self.h, 1))
        ms = (C.c_float * N_FAMILIES)()
        n = (C.c_int32 * N_FAMILIES)()
        try:
            for _ in range(steps):
                fn()
                _check(self.lib.dflash_profile_read(self.h, ms, n))
        finally:
            self.lib.dflash_profile_enable(self.h, 0)
        out = {}
        for f in range(N_FAMILIES):
            if n[f]:
                out[self.lib.dflash_family_name(f).decode()] = (1e3 * ms[f] / n[f], n[f] / steps)
        return out

    def trace(self, fn, capacity: int = 256):
        """Run `fn` once with the device-side timeline on. Returns a list of
        (family, start_ns, dependency_resolved_ns, main_loop_end_ns, end_ns) relative to the first start."""
        buf = torch.zeros(capacity * 4, dtype=torch.int64, device=self.device)
        _check(self.lib.dflash_trace_enable(self.h, C.c_void_p(buf.data_ptr()), capacity))
        try:
            fn()
            torch.cuda.synchronize()
            fam = (C.c_int32 * capacity)()
            n = C.c_int32()
            _check(self.lib.dflash_trace_read(self.h, fam, C.byref(n)))
        finally:
            self.lib.dflash_trace_enable(self.h, None, 0)
        rec = buf.cpu().view(capacity, 4).tolist()
        inv = lambda v: (~v) & 0xFFFFFFFFFFFFFFFF if v else 0
        fix = lambda v: v & 0xFFFFFFFFFFFFFFFF
        rows = []
        for i in range(n.value):
            r = rec[i]
            if r[3] == 0 and r[0] == 0:
                continue
            rows.append((self.lib.dflash_family_name(fam[i]).decode(), inv(fix(r[0])), inv(fix(r[1])), fix(r[2]), fix(r[3])))
        if not rows:
            return rows
        t0 = min(r[1] for r in rows if r[1])
        return [(f, a - t0 if a else None, b - t0 if b else None, c - t0 if c else None, d - t0 if d else None)
                for f, a, b, c, d in rows]

    # ---- the path -----------------------------------------------------------------------
    def dflash_ctx_project(self, feats, n_new, ctx_len, page_table, kv_pool, stream=None):
        """feats [S, max_new, k*D_t]; n_new (or None) and ctx_len int32 [S]; writes kv_pool in place."""
        S, max_new = feats.shape[0], feats.shape[1]
        ws = self.workspace(S, S * max_new)
        a = CtxArgs(_ptr(feats), S, max_new, _ptr(n_new), _ptr(ctx_len), _ptr(page_table), page_table.shape[1],
                    _ptr(kv_pool), kv_pool.shape[1], _ptr(ws), ws.numel(), _ptr(self.status))
        _check(self.lib.dflash_ctx_project(self.h, C.byref(a), _stream(stream)))

    def dflash_draft_block(self, anchor_ids, ctx_len, max_ctx_len, page_table, kv_pool, draft_ids,
                           top1=None, margin=None, hidden_out=None, logits_out=None, stream=None, block_rows=0, ctx=None):
        """block_rows: rows per sequence in this call (0 = the handle's block size).
        ctx = (feats [S, max_new, k*D_t], n_new or None, ctx_len_before): run that context projection inside
        this call, chained with the first layer's QKV contraction."""
        S = anchor_ids.shape[0]
        rows = S * self.cfg.block_size
        cptr = None
        if ctx is not None:
            feats, n_new, len_before = ctx
            rows = max(rows, S * feats.shape[1])
            self._ctx_keep = CtxArgs(_ptr(feats), S, feats.shape[1], _ptr(n_new), _ptr(len_before), _ptr(page_table),
                                     page_table.shape[1], _ptr(kv_pool), kv_pool.shape[1], None, 0, _ptr(self.status))
            cptr = C.pointer(self._ctx_keep)
        ws = self.workspace(S, rows)
        a = DraftArgs(_ptr(anchor_ids), S, _ptr(ctx_len), int(max_ctx_len), _ptr(page_table), page_table.shape[1],
                      _ptr(kv_pool), kv_pool.shape[1], _ptr(ws), ws.numel(), _ptr(draft_ids), _ptr(top1),
                      _ptr(margin), _ptr(hidden_out), _ptr(logits_out), _ptr(self.status), int(block_rows), cptr)
        _check(self.lib.dflash_draft_block(self.h, C.byref(a), _stream(stream)))

    def dflash_verify_accept(self, draft_ids, draft_stride, gamma, ctx_len, accept_len, out_tokens, bonus,
                             new_ctx_len, logits=None, target_ids=None, target_ids_out=None,
                             draft_offset=0, stream=None):
        """Mode LOGITS when `logits` [S, gamma+1, V] is given, else mode IDS with target_ids [S, gamma+1]."""
        S = ctx_len.shape[0]
        ws = self.workspace(S, S * (gamma + 1))
        dptr = C.c_void_p(draft_ids.data_ptr() + 4 * draft_offset)
        if logits is not None:
            mode, vocab = VERIFY_LOGITS, logits.shape[-1]
            ldt = F32 if logits.dtype == torch.float32 else BF16
        else:
            mode, vocab, ldt = VERIFY_IDS, self.cfg.vocab, F32
        a = VerifyArgs(mode, _ptr(logits), ldt, 0, _ptr(target_ids), dptr, draft_stride, S, gamma, vocab,
                       _ptr(ctx_len), _ptr(accept_len), _ptr(out_tokens), _ptr(bonus), _ptr(new_ctx_len),
                       _ptr(target_ids_out), _ptr(ws), ws.numel(), _ptr(self.status))
        _check(self.lib.dflash_verify_accept(self.h, C.byref(a), _stream(stream)))

    def dflash_verify_accept_static(self, draft_ids, draft_stride, gamma, ctx_len, accept_len, out_tokens, bonus,
                                    new_ctx_len, logits, target_ids_out=None, stream=None):
        """Logits-mode verify/accept on the library's built-in scratch: no workspace is passed, nothing is
        allocated. For callers that cannot allocate device memory; at most DFLASH_STATIC_MAX_ROWS rows, and
        calls must not overlap on the GPU (they share the scratch)."""
        S = ctx_len.shape[0]
        ldt = F32 if logits.dtype == torch.float32 else BF16
        a = VerifyArgs(VERIFY_LOGITS, _ptr(logits), ldt, 0, None, _ptr(draft_ids), draft_stride, S, gamma,
                       logits.shape[-1], _ptr(ctx_len), _ptr(accept_len), _ptr(out_tokens), _ptr(bonus),
                       _ptr(new_ctx_len), _ptr(target_ids_out), None, 0, _ptr(self.status))
        _check(self.lib.dflash_verify_accept_static(self.h, C.byref(a), _stream(stream)))

    def dflash_target_verify(self, token_ids, ctx_len, max_ctx_len, page_table, kv_pool, tap_layers, ids_out,
                             feats_out=None, logits_out=None, stream=None):
        """The target's verify pass: token_ids [S, rows]; writes the block's K/V into kv_pool at positions
        ctx_len .. ctx_len + rows - 1, the tapped hidden rows into feats_out [S, rows, len(tap_layers) * D]."""
        S, rows = token_ids.shape
        ws = self.workspace(S, S * rows)
        taps = (C.c_int32 * max(len(tap_layers), 1))(*tap_layers)
        a = TargetArgs(_ptr(token_ids), S, rows, _ptr(ctx_len), int(max_ctx_len), _ptr(page_table), page_table.shape[1],
                       _ptr(kv_pool), kv_pool.shape[1], taps, len(tap_layers), _ptr(feats_out), _ptr(logits_out),
                       _ptr(ids_out), _ptr(ws), ws.numel(), _ptr(self.status))
        _check(self.lib.dflash_target_verify(self.h, C.byref(a), _stream(stream)))

    def _sample_ws(self, n_rows, vocab):
        need = int(self.lib.dflash_sample_workspace_bytes(n_rows, vocab))
        if need < 0:
            raise DFlashError(-1)
        ws = getattr(self, "_samp_ws", None)
        if ws is None or ws.numel() < need:
            ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            self._samp_ws = ws
        return ws

    def dflash_block_loss(self, logits, targets, gamma, row_loss, loss_sum=None, dlogits=None, grad_scale=1.0, stream=None):
        """Position-weighted cross entropy of draft blocks. logits [n_blocks, B, V] (row 0 of a block = anchor, no
        loss), targets [n_blocks, B] int32 (< 0: ignored). row_loss [n_blocks * B] fp32; loss_sum [2] fp32;
        dlogits like logits (fp32 or bf16) = grad_scale * w_k * (softmax - onehot)."""
        nb, B, V = logits.shape
        a = BlockLossArgs(_ptr(logits), F32 if logits.dtype == torch.float32 else BF16, logits.stride(1), nb, B, V,
                          _ptr(targets), float(gamma), _ptr(row_loss), _ptr(loss_sum), _ptr(dlogits),
                          (F32 if dlogits.dtype == torch.float32 else BF16) if dlogits is not None else F32,
                          dlogits.stride(1) if dlogits is not None else 0, float(grad_scale), _ptr(self.status))
        _check(self.lib.dflash_block_loss(self.h, C.byref(a), _stream(stream)))

    def dflash_sample_rows(self, logits, temperature, u, ids, prob=None, stream=None):
        """ids[m] = inverse-CDF draw from softmax(logits[m] / T) with the uniform u[m]."""
        n, V = logits.shape[0], logits.shape[-1]
        ws = self._sample_ws(n, V)
        a = SampleArgs(_ptr(logits), F32 if logits.dtype == torch.float32 else BF16, logits.stride(0), n, V,
                       float(temperature), _ptr(u), _ptr(ids), _ptr(prob), _ptr(ws), ws.numel(), _ptr(self.status))
        _check(self.lib.dflash_sample_rows(self.h, C.byref(a), _stream(stream)))

    def dflash_verify_accept_sample(self, target_logits, draft_logits, draft_rows_per_seq, draft_ids, draft_stride,
                                    gamma, temperature, u_accept, u_final, ctx_len, accept_len, out_tokens, bonus,
                                    new_ctx_len, draft_row_offset=0, draft_offset=0, stream=None):
        """Speculative-sampling verification. target_logits [S, gamma+1, V]; draft_logits: 2-D [rows, V] with
        draft j of sequence b at row draft_row_offset + b * draft_rows_per_seq + j."""
        S, V = ctx_len.shape[0], target_logits.shape[-1]
        ws = self._sample_ws(S * (2 * gamma + 1), V)
        dl = draft_logits.reshape(-1, V) if draft_logits is not None else None
        dl_ptr = C.c_void_p(dl.data_ptr() + draft_row_offset * dl.stride(0) * dl.element_size()) if dl is not None else None
        a = VerifySampleArgs(_ptr(target_logits), F32 if target_logits.dtype == torch.float32 else BF16, 0, dl_ptr,
                             (F32 if dl.dtype == torch.float32 else BF16) if dl is not None else F32,
                             dl.stride(0) if dl is not None else 0, draft_rows_per_seq,
                             C.c_void_p(draft_ids.data_ptr() + 4 * draft_offset) if draft_ids is not None else None,
                             draft_stride, S, gamma, V, float(temperature), _ptr(u_accept), _ptr(u_final),
                             _ptr(ctx_len), _ptr(accept_len), _ptr(out_tokens), _ptr(bonus), _ptr(new_ctx_len),
                             _ptr(ws), ws.numel(), _ptr(self.status))
        _check(self.lib.dflash_verify_accept_sample(self.h, C.byref(a), _stream(stream)))

    def dflash_block_attention(self, mode, q, k_blk, v_blk, ctx_len, max_ctx_len, page_table, kv_pool, layer,
                               out, stream=None, lse_out=None):
        S, R = q.shape[0], q.shape[1]
        ws = self.workspace(S, S * R)
        a = AttnArgs(mode, _ptr(q), _ptr(k_blk), _ptr(v_blk), S, R, _ptr(ctx_len), int(max_ctx_len),
                     _ptr(page_table), page_table.shape[1], _ptr(kv_pool), kv_pool.shape[1], layer, _ptr(out),
                     _ptr(ws), ws.numel(), _ptr(self.status), _ptr(lse_out))
        _check(self.lib.dflash_block_attention(self.h, C.byref(a), _stream(stream)))

    def dflash_block_attention_bwd(self, mode, q, k_blk, v_blk, out, lse, dout, ctx_len, max_ctx_len, page_table, kv_pool, layer,
                                   dq, dk_blk, dv_blk, dkv_ctx=None, shared_page_row=False, stream=None):
        """Gradients of dflash_block_attention: dq / dk_blk / dv_blk like q / k_blk / v_blk; dkv_ctx fp32
        [n_pool_pages, 2, Hkv, page_size, hd] (one layer, the pool's layout) or None."""
        S, R = q.shape[0], q.shape[1]
        ws = self.workspace(S, S * R)
        a = AttnBwdArgs(mode, _ptr(q), _ptr(k_blk), _ptr(v_blk), _ptr(out), _ptr(lse), _ptr(dout), S, R, _ptr(ctx_len),
                        int(max_ctx_len), _ptr(page_table), page_table.shape[1], _ptr(kv_pool), kv_pool.shape[1], layer,
                        1 if shared_page_row else 0, _ptr(dq), _ptr(dk_blk), _ptr(dv_blk), _ptr(dkv_ctx), _ptr(ws), ws.numel(),
                        _ptr(self.status))
        _check(self.lib.dflash_block_attention_bwd(self.h, C.byref(a), _stream(stream)))

    # ---- a batch over a shared cache --------------------------------------------------------
    # (The argument checks of these calls are kept to a few attribute reads a tensor: a decode step makes several of the calls, and
    # their kernels take no longer than the host does for one.)
    def _dev(self, t, dtype, *shape):
        """Address of a contiguous tensor of this handle's device, of the given type and shape; None for None."""
        if t is None:
            return None
        if t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous():
            return t.data_ptr()
        assert t.dtype is dtype, f"{dtype} tensor expected, got {t.dtype}"
        assert t.get_device() == self._index and t.is_contiguous(), f"contiguous tensor on {self.device} expected"
        raise AssertionError(f"shape {shape} expected, got {tuple(t.shape)}")

    def _pool(self, kv_pool):
        c = self.cfg
        return self._dev(kv_pool, c.torch_dtype, c.n_layers, kv_pool.shape[1], 2, c.n_kv_heads, c.page_size, c.head_dim)

    def _scratch(self, name, query, key, stream):
        """Workspace of the calls below for the sizes in `key`: (tensor, address, bytes). Every stream has its own, grown on demand, so that calls
        on two streams may overlap. A captured call takes a fresh one from its graph's memory, where it stays the graph's: graphs share
        none with each other or with calls outside."""
        need = self._needs.get((name, key))
        if need is None:
            need = int(query(*key))
            if need < 0:
                raise DFlashError(need)
            need = self._needs[name, key] = max(need, 256)
        if stream is None and _current_device() == self._index:
            captured, raw = torch.cuda.is_current_stream_capturing(), _current_stream(self._index)
        else:
            with torch.cuda.device(self._index), torch.cuda.stream(stream):
                captured, raw = torch.cuda.is_current_stream_capturing(), _current_stream(self._index)
        kept = None if captured else self._scratches.get((name, raw))
        if kept is None or kept[2] < need:
            with torch.cuda.device(self._index), torch.cuda.stream(stream):
                t = torch.empty(need, dtype=torch.uint8, device=self.device)
            kept = (t, t.data_ptr(), need)
            if not captured:
                self._scratches[name, raw] = kept
        return kept

    def _call(self, fn, args, stream):
        """The library launches on the current device, which has to be the handle's. One thread at a time: the launches of a call share a workspace."""
        raw = stream.cuda_stream if stream is not None else _current_stream(self._index)
        with self._launching:
            if _current_device() == self._index:
                rc = fn(self.h, C.byref(args), raw)
            else:
                with torch.cuda.device(self._index):
                    rc = fn(self.h, C.byref(args), raw)
        if rc != 0:
            raise DFlashError(rc)

    def _prefix_ws(self, batch, rows, groups):
        return self.lib.dflash_prefix_attention_workspace_bytes(self.h, batch, rows, groups)

    def dflash_prefix_attention(self, mode, q, k_blk, v_blk, group_start, prefix_len, ctx_len, max_ctx_len, page_table, kv_pool, layer,
                                out, stream=None, lse_out=None):
        """dflash_block_attention of a batch in which sequences group_start[g] .. group_start[g+1]-1 share their first
        prefix_len[g] positions (read from the page-table row of the first of them, once for all). group_start int32 [n+1] and
        prefix_len int32 [n], or both None: nothing is shared."""
        c, dt, i32 = self.cfg, self.cfg.torch_dtype, torch.int32
        S, R = q.shape[0], q.shape[1]
        hq, hkv, hd = c.n_q_heads, c.n_kv_heads, c.head_dim
        n = 0 if prefix_len is None else prefix_len.shape[0]
        width = page_table.shape[1]
        held, ws, ws_bytes = self._scratch("prefix_attention", self._prefix_ws, (S, R, n), stream)
        a = PrefixAttnArgs(mode, self._dev(q, dt, S, R, hq, hd), self._dev(k_blk, dt, S, R, hkv, hd), self._dev(v_blk, dt, S, R, hkv, hd), S, R, n,
                           self._dev(group_start, i32, n + 1) if n else None, self._dev(prefix_len, i32, n) if n else None, self._dev(ctx_len, i32, S),
                           int(max_ctx_len), self._dev(page_table, i32, S, width), width, self._pool(kv_pool), kv_pool.shape[1], layer,
                           self._dev(out, dt, S, R, hq, hd), self._dev(lse_out, torch.float32, S, R, hq), ws, ws_bytes, self.status.data_ptr())
        self._call(self.lib.dflash_prefix_attention, a, stream)

    def dflash_pages_copy(self, src, dst, kv_pool, n_slots=None, count=None, stream=None):
        """Page src[i] -> dst[i] in every layer (its first n_slots[i] slots); entries with a negative source do nothing,
        nor do those from count[0] on."""
        n, i32 = src.shape[0], torch.int32
        a = PagesCopyArgs(n, self._dev(count, i32, 1), self._dev(src, i32, n), self._dev(dst, i32, n), self._dev(n_slots, i32, n), self._pool(kv_pool),
                          kv_pool.shape[1], self.status.data_ptr())
        self._call(self.lib.dflash_pages_copy, a, stream)

    def _pages_list(self, fn, st, lists, page_table, ref_count, kv_pool, copies, stream):
        n, i32 = lists[0].shape[0], torch.int32
        rows, width = page_table.shape
        pages = kv_pool.shape[1]
        cs, cd, cn = copies if copies is not None else (None, None, None)
        held, ws, ws_bytes = self._scratch("pages", self.lib.dflash_pages_workspace_bytes, (n, width, pages), stream)
        a = st(n, *[self._dev(t, i32, n) for t in lists], self._dev(page_table, i32, rows, width), rows, width, self._dev(ref_count, i32, pages),
               self._pool(kv_pool), pages, self._dev(cs, i32, n), self._dev(cd, i32, n), self._dev(cn, i32, n), ws, ws_bytes, self.status.data_ptr())
        self._call(fn, a, stream)

    def dflash_pages_fork(self, parent, child, fork_len, page_table, ref_count, kv_pool, copies=None, stream=None):
        """Row child[i] takes over the first fork_len[i] positions of row parent[i]: whole pages shared, a last partial one
        copied. copies = (src, dst, n_slots), int32 [n] each, receives the page copies made."""
        self._pages_list(self.lib.dflash_pages_fork, PagesForkArgs, (parent, child, fork_len), page_table, ref_count, kv_pool, copies, stream)

    def dflash_pages_resize(self, rows, keep_len, capacity, page_table, ref_count, kv_pool, copies=None, stream=None):
        """Row rows[i] gets pages for capacity[i] positions (0 releases it), its own ones from position keep_len[i] on."""
        self._pages_list(self.lib.dflash_pages_resize, PagesResizeArgs, (rows, keep_len, capacity), page_table, ref_count, kv_pool, copies, stream)

    def dflash_pages_compact(self, page_table, ref_count, kv_pool, n_live=None, copies=None, stream=None):
        """Moves the pages in use to the front of the pool. n_live int32 [1] receives their number; copies = (src, dst, count),
        int32 [n_pool_pages // 2], the same, and [1], the moves made."""
        i32 = torch.int32
        rows, width = page_table.shape
        pages = kv_pool.shape[1]
        cs, cd, cn = copies if copies is not None else (None, None, None)
        held, ws, ws_bytes = self._scratch("pages", self.lib.dflash_pages_workspace_bytes, (0, width, pages), stream)
        a = PagesCompactArgs(self._dev(page_table, i32, rows, width), rows, width, self._dev(ref_count, i32, pages), self._pool(kv_pool), pages,
                             self._dev(n_live, i32, 1), self._dev(cs, i32, pages // 2), self._dev(cd, i32, pages // 2), self._dev(cn, i32, 1), ws, ws_bytes,
                             self.status.data_ptr())
        self._call(self.lib.dflash_pages_compact, a, stream)

    # ---- scoring, distilling, stepping --------------------------------------------------------
    def _logit_rows(self, t, shape=None):
        """Address, type and row stride of logits [rows, vocab] whose rows may lie apart."""
        rows, v = size = t.shape
        apart, step = t.stride()
        dt = t.dtype
        assert dt is torch.bfloat16 or dt is torch.float32, "fp32 or bf16 logits [rows, vocab] expected"
        assert t.get_device() == self._index, f"tensor on {self.device} expected"
        assert shape is None or size == shape, f"shape {tuple(shape)} expected, got {tuple(size)}"
        assert (step == 1 or v <= 1) and (apart >= v or rows <= 1), "rows of neighbouring entries that do not overlap expected"
        return t.data_ptr(), F32 if dt is torch.float32 else BF16, apart if rows > 1 else v

    def dflash_token_logprobs(self, logits, tokens, logprob, temperature=1.0, stats=None, entropy=None, top_ids=None, top_logprob=None, stream=None):
        """logprob [n, k] of tokens int32 [n, k] (negative: none) under softmax(logits [n, V] / T). stats [n, 2] receives (M, ln sum exp((z - M) / T)),
        entropy [n] nats, top_ids / top_logprob [n, m] the m most likely tokens. tokens and logprob may both be None."""
        n, v = logits.shape
        k = 0 if tokens is None else tokens.shape[1]
        m = 0 if top_ids is None else top_ids.shape[1]
        z, dt, ld = self._logit_rows(logits)
        f32 = torch.float32
        a = TokenLogprobsArgs(z, dt, ld, n, v, float(temperature), k, self._dev(tokens, torch.int32, n, k), self._dev(logprob, f32, n, k),
                              self._dev(stats, f32, n, 2), self._dev(entropy, f32, n), m, self._dev(top_ids, torch.int32, n, m),
                              self._dev(top_logprob, f32, n, m), self.status.data_ptr())
        self._call(self.lib.dflash_token_logprobs, a, stream)

    def dflash_token_logprobs_bwd(self, logits, tokens, stats, d_logprob, dlogits, temperature=1.0, entropy=None, d_entropy=None, stream=None):
        """dlogits [n, V] from the gradients d_logprob [n, k] and d_entropy [n] (or None) of dflash_token_logprobs; stats and entropy are its outputs.
        dlogits may be logits."""
        n, v = logits.shape
        k = 0 if tokens is None else tokens.shape[1]
        z, dt, ld = self._logit_rows(logits)
        dz, ddt, dld = self._logit_rows(dlogits, logits.shape)
        f32 = torch.float32
        a = TokenLogprobsBwdArgs(z, dt, ld, n, v, float(temperature), k, self._dev(tokens, torch.int32, n, k), self._dev(stats, f32, n, 2),
                                 self._dev(entropy, f32, n), self._dev(d_logprob, f32, n, k), self._dev(d_entropy, f32, n), dz, ddt, dld,
                                 self.status.data_ptr())
        self._call(self.lib.dflash_token_logprobs_bwd, a, stream)

    def adamw_plan(self, entries) -> AdamwPlan:
        """entries: one dict a tensor with param (fp32 or bf16), grad (fp32 or bf16), exp_avg and exp_avg_sq (fp32; or float8_e4m3fn with fp32
        exp_avg_scale and exp_avg_sq_scale, one for 128 entries), and where wanted master (fp32, beside a bf16 param), weight_decay (0), lr_scale (1). All contiguous."""
        return AdamwPlan(entries, self._index)

    def _adamw_ws(self, n):
        return self.lib.dflash_adamw_workspace_bytes(self.h, n)

    def dflash_adamw_step(self, plan: AdamwPlan, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, max_grad_norm=0.0, grad_norm=None, stream=None):
        """One AdamW step of all tensors of the plan. step (from 1) and lr: numbers, or int32 / fp32 tensors of one entry on the device (for captured
        calls). max_grad_norm > 0 clips by the norm of all gradients; grad_norm fp32 [1] receives it."""
        assert plan.index == self._index, f"plan of tensors on device {plan.index} given to a handle on device {self._index}"
        on_device = lambda x: isinstance(x, torch.Tensor)  # noqa: E731
        ws, ws_bytes = None, 0
        if max_grad_norm > 0 or grad_norm is not None:
            held, ws, ws_bytes = self._scratch("adamw", self._adamw_ws, (plan.n,), stream)
        a = AdamwArgs(plan.table, plan.n, 0 if on_device(step) else int(step), self._dev(step, torch.int32, 1) if on_device(step) else None,
                      0.0 if on_device(lr) else float(lr), self._dev(lr, torch.float32, 1) if on_device(lr) else None, float(beta1), float(beta2), float(eps),
                      float(grad_scale), float(max_grad_norm), self._dev(grad_norm, torch.float32, 1), ws, ws_bytes, self.status.data_ptr())
        self._call(self.lib.dflash_adamw_step, a, stream)

    def dflash_lmhead_argmax(self, hidden, apply_norm, ids, top1=None, margin=None, logits_out=None, stream=None):
        M = hidden.shape[0]
        ws = self.workspace(1, M)
        a = LmHeadArgs(_ptr(hidden), 1 if hidden.dtype == torch.float32 else 0, M, 1 if apply_norm else 0,
                       _ptr(ids), _ptr(top1), _ptr(margin), _ptr(logits_out), _ptr(ws), ws.numel(),
                       _ptr(self.status))
        _check(self.lib.dflash_lmhead_argmax(self.h, C.byref(a), _stream(stream)))
