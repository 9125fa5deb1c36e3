"""Thin ctypes binding of the C ABI in include/td.h.

Argument marshalling only: every step of put and get runs in the CUDA library.  PyTorch
supplies device memory (`torch.empty(...).data_ptr()`) and streams; nothing here computes
on tensors.  There is no CPU fallback: if libtd.so cannot be loaded, or a call fails,
an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, List, Optional, Sequence, Tuple

from . import build as _build

I32, F32, BF16, F16 = 0, 1, 2, 3       # F16: operands of the operators, not columns
SCALAR, PROMPT, RESPONSE = 0, 1, 2
PACKED, PADDED = 0, 1
OUT_LEFT_PAD_PROMPT = 1            # td_get_out.flags
F_ADVANTAGE = 1
OK, EINVAL, EWORKSPACE, ECUDA, ETOOLARGE = 0, -1, -2, -3, -4
ERR_OOB_INDEX, ERR_DUP_PUT, ERR_LEN_MISMATCH, ERR_ARENA_FULL = 1, 2, 4, 8
ERR_OUT_TRUNCATED, ERR_LOOKBACK_TIMEOUT, ERR_BAD_LENGTH, ERR_COPY_TIMEOUT = 16, 32, 64, 128
(BAD_STORED_WITHOUT_ROW, BAD_ROW_PLACEMENT, BAD_ROW_OVERLAP, BAD_STATUS_BITS, BAD_SERVED_UNCLAIMED,
 BAD_SERVED_NOT_READY, BAD_COUNTERS) = 1, 2, 4, 8, 16, 32, 64          # td_debug_validate

ROWS_TOKEN, ROWS_STREAM = 0, 1                       # layout of logits rows
KL_K1, KL_K2, KL_K3 = 1, 2, 3
MEAN_TOKENS, MEAN_SAMPLES = 0, 1
(POLICY_LOSS, POLICY_PG, POLICY_KL, POLICY_ENTROPY, POLICY_CLIPPED, POLICY_OLD_KL, POLICY_RATIO, POLICY_TOKENS,
 POLICY_STATS) = range(9)
TOKENS_PROMPT, TOKENS_RESPONSE, TOKENS_SEQ = 1, 2, 3  # which tokens of a batch an id array holds

DTYPE_TAG = {"i32": I32, "f32": F32, "bf16": BF16}
CLASS_TAG = {"scalar": SCALAR, "prompt": PROMPT, "response": RESPONSE}
ELEM_SIZE = {I32: 4, F32: 4, BF16: 2}

# every symbol include/td.h declares
EXPORTS = ["td_query_workspace", "td_create", "td_destroy", "td_put", "td_get",
           "td_get_scratch_bytes", "td_reset", "td_status", "td_debug_table",
           "td_launch_count", "td_strerror", "td_kernel_timing", "td_kernel_timing_read",
           "td_put_host_stage_bytes", "td_put_host", "td_get_host", "td_put_many",
           "td_plan_bytes", "td_plan_create", "td_plan_destroy", "td_get_many", "td_get_static",
           "td_model_bytes", "td_put_back", "td_put_back_many", "td_put_many_host", "td_get_many_host", "td_get_many_host_stage_bytes", "td_debug_validate",
           "td_debug_lookback",
           "td_token_logprob", "td_token_logprob_grad", "td_policy_loss_workspace_bytes", "td_policy_loss",
           "td_embed", "td_embed_grad_workspace_bytes", "td_embed_grad",
           "td_cache_workspace_bytes", "td_cache_extend", "td_cache_fork", "td_cache_free", "td_cache_compact", "td_cache_write",
           "td_cache_attention_workspace_bytes", "td_cache_attention", "td_debug_cache_wait"]


class TdModel(C.Structure):
    _fields_ = [(k, C.c_uint64) for k in ("G", "N", "PL", "n", "SL", "M", "B", "C", "S")]


class TdColumn(C.Structure):
    _fields_ = [("name", C.c_char_p), ("dtype", C.c_int32), ("cls", C.c_int32), ("pad_bits", C.c_uint32)]


class TdConsumer(C.Structure):
    _fields_ = [("name", C.c_char_p), ("need_mask", C.c_uint32), ("out_mask", C.c_uint32),
                ("flags", C.c_uint32)]


class TdConfig(C.Structure):
    _fields_ = [("n_prompts", C.c_uint32), ("n_per_group", C.c_uint32), ("n_shards", C.c_uint32),
                ("n_columns", C.c_uint32), ("columns", C.POINTER(TdColumn)),
                ("n_consumers", C.c_uint32), ("consumers", C.POINTER(TdConsumer)),
                ("prompt_elems_per_shard", C.c_uint64), ("response_elems_per_shard", C.c_uint64),
                ("reward_column", C.c_uint32), ("adv_eps", C.c_float), ("device", C.c_int32)]


class TdResult(C.Structure):
    _fields_ = [("n_samples", C.c_uint32), ("n_groups", C.c_uint32),
                ("prompt_tokens", C.c_uint64), ("response_tokens", C.c_uint64),
                ("status", C.c_uint32), ("reserved", C.c_uint32)]


class TdGetOut(C.Structure):
    _fields_ = [("mode", C.c_int32), ("pad_prompt_to", C.c_uint32), ("pad_response_to", C.c_uint32),
                ("flags", C.c_uint32),
                ("indices", C.c_void_p), ("cu_prompt", C.c_void_p), ("cu_response", C.c_void_p),
                ("cu_seq", C.c_void_p), ("col", C.c_void_p * 32),
                ("col_capacity_elems", C.c_uint64 * 32), ("advantages", C.c_void_p),
                ("result", C.c_void_p), ("scratch", C.c_void_p), ("scratch_bytes", C.c_uint64),
                ("seq_prompt_col", C.c_uint32), ("seq_response_col", C.c_uint32), ("seq", C.c_void_p),
                ("seq_capacity_elems", C.c_uint64), ("seq_advantages", C.c_void_p)]


class TdPutItem(C.Structure):
    _fields_ = [("column", C.c_uint32), ("k", C.c_uint32), ("d_indices", C.c_void_p),
                ("d_cu", C.c_void_p), ("d_data", C.c_void_p), ("data_elems", C.c_uint64)]


class TdBackItem(C.Structure):
    _fields_ = [("column", C.c_uint32), ("reserved", C.c_uint32), ("d_data", C.c_void_p),
                ("data_elems", C.c_uint64)]


class TdBackReq(C.Structure):
    _fields_ = [("batch", C.c_void_p), ("max_samples", C.c_uint32), ("column", C.c_uint32),
                ("d_data", C.c_void_p), ("data_elems", C.c_uint64)]


class TdValidateReport(C.Structure):
    _fields_ = [("violations", C.c_uint32), ("reserved", C.c_uint32), ("first_sample", C.c_uint64),
                ("stored", C.c_uint64 * 32), ("served", C.c_uint64 * 32), ("arena_elems_used", C.c_uint64 * 3)]


class TdGetReq(C.Structure):
    _fields_ = [("consumer", C.c_uint32), ("max_samples", C.c_uint32), ("out", TdGetOut)]


class TdStats(C.Structure):
    _fields_ = [("put_accepted", C.c_uint64 * 32), ("got_samples", C.c_uint64 * 32),
                ("got_tokens", C.c_uint64 * 32), ("n_oob", C.c_uint64), ("n_dup", C.c_uint64),
                ("n_len_mismatch", C.c_uint64), ("n_arena_full", C.c_uint64),
                ("n_truncated", C.c_uint64), ("n_bad_length", C.c_uint64),
                ("n_claim_conflicts", C.c_uint64), ("n_lookback_timeouts", C.c_uint64),
                ("error_word", C.c_uint32), ("reserved", C.c_uint32)]


class TdBatch(C.Structure):
    _fields_ = [("max_samples", C.c_uint32), ("reserved", C.c_uint32), ("cu_prompt", C.c_void_p),
                ("cu_response", C.c_void_p), ("result", C.c_void_p)]


_LOGITS_FIELDS = [("logits", C.c_void_p), ("logits_stride", C.c_int64), ("dtype", C.c_int32), ("vocab", C.c_uint32),
                  ("n_rows", C.c_uint32), ("n_tokens", C.c_uint32), ("rows", C.c_int32), ("temperature", C.c_float),
                  ("device", C.c_int32), ("targets", C.c_void_p), ("batch", C.POINTER(TdBatch))]


class TdLogprobArgs(C.Structure):
    _fields_ = _LOGITS_FIELDS + [("logprob", C.c_void_p), ("norm", C.c_void_p), ("entropy", C.c_void_p),
                                 ("entropy_bf16", C.c_void_p), ("status", C.c_void_p)]


class TdLogprobGradArgs(C.Structure):
    _fields_ = _LOGITS_FIELDS + [("norm", C.c_void_p), ("entropy", C.c_void_p), ("grad_logprob", C.c_void_p),
                                 ("grad_entropy", C.c_void_p), ("grad_logits", C.c_void_p),
                                 ("grad_stride", C.c_int64), ("status", C.c_void_p)]


class TdPolicyArgs(C.Structure):
    _fields_ = [("batch", C.POINTER(TdBatch)), ("n_tokens", C.c_uint64), ("row_width", C.c_uint64),
                ("column_dtype", C.c_int32), ("kl_kind", C.c_int32), ("reduction", C.c_int32), ("device", C.c_int32),
                ("clip_low", C.c_float), ("clip_high", C.c_float), ("dual_clip", C.c_float), ("kl_coef", C.c_float),
                ("entropy_coef", C.c_float), ("norm", C.c_float), ("grad_scale", C.c_float), ("reserved", C.c_uint32),
                ("logprob", C.c_void_p), ("old_logprob", C.c_void_p), ("ref_logprob", C.c_void_p),
                ("entropy", C.c_void_p), ("mask", C.c_void_p), ("advantages", C.c_void_p),
                ("grad_logprob", C.c_void_p), ("grad_entropy", C.c_void_p), ("stats", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class TdEmbedArgs(C.Structure):
    _fields_ = [("ids", C.c_void_p), ("n_tokens", C.c_uint32), ("vocab", C.c_uint32), ("dim", C.c_uint32),
                ("dtype", C.c_int32), ("table", C.c_void_p), ("table_stride", C.c_int64), ("out", C.c_void_p),
                ("out_stride", C.c_int64), ("scale", C.c_float), ("tokens", C.c_int32), ("device", C.c_int32),
                ("reserved", C.c_uint32), ("batch", C.POINTER(TdBatch)), ("status", C.c_void_p)]


class TdEmbedGradArgs(C.Structure):
    _fields_ = [("ids", C.c_void_p), ("n_tokens", C.c_uint32), ("vocab", C.c_uint32), ("dim", C.c_uint32),
                ("dtype", C.c_int32), ("grad_out", C.c_void_p), ("out_stride", C.c_int64), ("grad_dtype", C.c_int32),
                ("accumulate", C.c_int32), ("grad_table", C.c_void_p), ("table_stride", C.c_int64),
                ("scale", C.c_float), ("tokens", C.c_int32), ("device", C.c_int32), ("reserved", C.c_uint32),
                ("batch", C.POINTER(TdBatch)), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
                ("status", C.c_void_p)]


class TdCache(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_pages", C.c_uint32), ("page_size", C.c_uint32), ("n_layers", C.c_uint32),
                ("n_heads", C.c_uint32), ("dim", C.c_uint32), ("layer_stride", C.c_int64), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("keys", C.c_void_p), ("values", C.c_void_p),
                ("max_seqs", C.c_uint32), ("max_pages", C.c_uint32), ("table", C.c_void_p), ("length", C.c_void_p),
                ("holders", C.c_void_p), ("status", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64),
                ("device", C.c_int32), ("reserved", C.c_uint32)]


class TdCacheWriteArgs(C.Structure):
    _fields_ = [("cache", C.POINTER(TdCache)), ("layer", C.c_uint32), ("n_rows", C.c_uint32), ("keys", C.c_void_p),
                ("values", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("cu", C.c_void_p)]


class TdCacheAttentionArgs(C.Structure):
    _fields_ = [("cache", C.POINTER(TdCache)), ("layer", C.c_uint32), ("n_rows", C.c_uint32), ("n_heads", C.c_uint32),
                ("group", C.c_uint32), ("window", C.c_uint32), ("reserved", C.c_uint32), ("scale", C.c_float),
                ("reserved2", C.c_uint32), ("seqs", C.c_void_p), ("q", C.c_void_p), ("q_row_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("out", C.c_void_p), ("out_row_stride", C.c_int64),
                ("out_head_stride", C.c_int64), ("lse", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class TdError(RuntimeError):
    def __init__(self, call: str, code: int):
        self.code = code
        msg = lib().td_strerror(code).decode() if _lib is not None else "?"
        super().__init__(f"{call} failed: {code} ({msg})")


_lib = None


def lib_path() -> str:
    """The library to load: libtd.so beside this file, or the build named by TD_LIB_PATH (a build
    of the same sources with other compiler flags: sanitizers, NVTX ranges)."""
    return os.environ.get("TD_LIB_PATH") or _build.LIB_PATH


def lib():
    """Loads libtd.so (raises if it is missing: there is no other implementation)."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with "
                               "`python -m paper_2507_19017_b200.build` (needs nvcc)")
        L = C.CDLL(path)
        vp, u32, u64 = C.c_void_p, C.c_uint32, C.c_uint64
        L.td_query_workspace.restype = C.c_int
        L.td_query_workspace.argtypes = [C.POINTER(TdConfig), C.POINTER(C.c_size_t)]
        L.td_create.restype = C.c_int
        L.td_create.argtypes = [C.POINTER(TdConfig), vp, C.c_size_t, C.POINTER(vp)]
        L.td_destroy.restype = C.c_int
        L.td_destroy.argtypes = [vp]
        L.td_put.restype = C.c_int
        L.td_put.argtypes = [vp, u32, vp, u32, vp, vp, u64, vp]
        L.td_get.restype = C.c_int
        L.td_get.argtypes = [vp, u32, u32, C.POINTER(TdGetOut), vp]
        L.td_get_scratch_bytes.restype = C.c_size_t
        L.td_get_scratch_bytes.argtypes = [vp]
        L.td_reset.restype = C.c_int
        L.td_reset.argtypes = [vp, vp]
        L.td_status.restype = C.c_int
        L.td_status.argtypes = [vp, C.POINTER(TdStats), vp]
        L.td_debug_table.restype = C.c_int
        L.td_debug_table.argtypes = [vp, C.c_int, u32, C.POINTER(vp), C.POINTER(C.c_size_t)]
        L.td_launch_count.restype = u64
        L.td_launch_count.argtypes = [vp]
        L.td_strerror.restype = C.c_char_p
        L.td_strerror.argtypes = [C.c_int]
        L.td_kernel_timing.restype = C.c_int
        L.td_kernel_timing.argtypes = [vp, C.c_int]
        L.td_kernel_timing_read.restype = C.c_int
        L.td_kernel_timing_read.argtypes = [vp, C.c_int, C.POINTER(u64), C.POINTER(C.c_double)]
        L.td_put_host_stage_bytes.restype = C.c_size_t
        L.td_put_host_stage_bytes.argtypes = [vp, u32, u32, u64]
        L.td_put_host.restype = C.c_int
        L.td_put_host.argtypes = [vp, u32, vp, u32, vp, vp, u64, vp, C.c_size_t, vp]
        L.td_get_host.restype = C.c_int
        L.td_get_host.argtypes = [vp, u32, u32, C.POINTER(TdGetOut), C.POINTER(TdGetOut), vp]
        L.td_put_many.restype = C.c_int
        L.td_put_many.argtypes = [vp, C.POINTER(TdPutItem), u32, vp]
        L.td_put_back.restype = C.c_int
        L.td_put_back.argtypes = [vp, C.POINTER(TdGetOut), u32, C.POINTER(TdBackItem), u32, vp]
        L.td_put_back_many.restype = C.c_int
        L.td_put_back_many.argtypes = [vp, C.POINTER(TdBackReq), u32, vp]
        L.td_put_many_host.restype = C.c_int
        L.td_put_many_host.argtypes = [vp, C.POINTER(TdPutItem), u32, vp, C.c_size_t, vp]
        L.td_get_many_host.restype = C.c_int
        L.td_get_many_host.argtypes = [vp, vp, C.POINTER(TdGetOut), u32, vp, C.c_size_t, vp]
        L.td_get_many_host_stage_bytes.restype = C.c_size_t
        L.td_get_many_host_stage_bytes.argtypes = [vp]
        L.td_debug_validate.restype = C.c_int
        L.td_debug_validate.argtypes = [vp, vp, C.POINTER(TdValidateReport)]
        L.td_debug_lookback.restype = C.c_int
        L.td_debug_lookback.argtypes = [vp, u32, u32]
        L.td_plan_bytes.restype = C.c_size_t
        L.td_plan_bytes.argtypes = [vp, u32]
        L.td_plan_create.restype = C.c_int
        L.td_plan_create.argtypes = [vp, C.POINTER(TdGetReq), u32, vp, C.c_size_t, vp, C.POINTER(vp)]
        L.td_plan_destroy.restype = C.c_int
        L.td_plan_destroy.argtypes = [vp]
        L.td_get_many.restype = C.c_int
        L.td_get_many.argtypes = [vp, vp, vp]
        L.td_get_static.restype = C.c_int
        L.td_get_static.argtypes = [vp, u32, u32, C.POINTER(TdGetOut), vp]
        L.td_model_bytes.restype = C.c_int
        L.td_model_bytes.argtypes = [C.POINTER(TdModel), C.POINTER(u64), C.POINTER(u64), C.POINTER(C.c_double)]
        for name, args in (("td_token_logprob", TdLogprobArgs), ("td_token_logprob_grad", TdLogprobGradArgs),
                           ("td_policy_loss", TdPolicyArgs), ("td_embed", TdEmbedArgs), ("td_embed_grad", TdEmbedGradArgs),
                           ("td_cache_write", TdCacheWriteArgs), ("td_cache_attention", TdCacheAttentionArgs)):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = [C.POINTER(args), vp]
        L.td_policy_loss_workspace_bytes.restype = C.c_size_t
        L.td_policy_loss_workspace_bytes.argtypes = [u32]
        L.td_embed_grad_workspace_bytes.restype = C.c_size_t
        L.td_embed_grad_workspace_bytes.argtypes = [u32, u32, u32]
        for name, extra in (("td_cache_extend", 2), ("td_cache_fork", 1), ("td_cache_free", 1), ("td_cache_compact", 2)):
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = [vp] * (extra + 2)
        L.td_debug_cache_wait.restype = C.c_int
        L.td_debug_cache_wait.argtypes = [u32, u32]
        L.td_cache_workspace_bytes.restype = C.c_size_t
        L.td_cache_workspace_bytes.argtypes = [u32, u32]
        L.td_cache_attention_workspace_bytes.restype = C.c_size_t
        L.td_cache_attention_workspace_bytes.argtypes = [u32, u32, u32]
        _lib = L
    return _lib


def model_bytes(G, N, PL, n, SL, M, B=4, C_=0, S=1):
    """Eq. 1, Eq. 2 and Eq. 4 of the paper's volume model, in bytes: (cv, tcv, tcv_dock)."""
    m = TdModel(G, N, PL, n, SL, M, B, C_, S)
    cv, tcv, dock = C.c_uint64(), C.c_uint64(), C.c_double()
    _check("td_model_bytes", lib().td_model_bytes(C.byref(m), C.byref(cv), C.byref(tcv), C.byref(dock)))
    return cv.value, tcv.value, dock.value


def _check(call: str, rc: int):
    if rc != 0:
        raise TdError(call, rc)


def make_config(G: int, N: int, S: int, columns: Sequence[Tuple[str, str, int]],
                consumers: Sequence[Tuple[int, int, bool]], prompt_cap: int, response_cap: int,
                reward_column: int, eps: float = 1e-6, device: int = 0):
    """columns: (dtype tag, class tag, pad_bits); consumers: (need_mask, out_mask, advantage).
    Returns (TdConfig, keepalive) - keep the second value alive as long as the first."""
    cols = (TdColumn * len(columns))(*[TdColumn(None, DTYPE_TAG[d], CLASS_TAG[c], int(p))
                                       for d, c, p in columns])
    cons = (TdConsumer * len(consumers))(*[TdConsumer(None, int(a), int(b), F_ADVANTAGE if f else 0)
                                           for a, b, f in consumers])
    cfg = TdConfig(G, N, S, len(columns), cols, len(consumers), cons, prompt_cap, response_cap,
                   reward_column, eps, device)
    return cfg, (cols, cons)


def query_workspace(cfg: TdConfig) -> int:
    out = C.c_size_t(0)
    _check("td_query_workspace", lib().td_query_workspace(C.byref(cfg), C.byref(out)))
    return out.value


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class GetBuffers:
    """Device buffers of one get, allocated once and reusable for any number of calls."""

    def __init__(self, dock: "Dock", consumer: int, max_samples: int, mode: int = PACKED,
                 pad_prompt_to: int = 0, pad_response_to: int = 0,
                 capacities: Optional[Dict[int, int]] = None, want: Optional[Sequence[int]] = None,
                 prompt_tokens_cap: Optional[int] = None, response_tokens_cap: Optional[int] = None,
                 seq: Optional[Tuple[int, int]] = None, seq_adv: bool = False, seq_cap: Optional[int] = None,
                 host_payload: bool = False, left_pad_prompts: bool = False):
        """seq = (prompt column, response column) adds the fused token stream, seq_adv its
        advantage twin; seq_cap is the room behind each (default: both token caps together).
        left_pad_prompts (PADDED mode): prompt rows end at their width, the pad in front.
        host_payload: the column buffers (and the stream) are pinned host memory that the device
        writes directly; indices, cu_seqlens, advantages and the result block stay on the device."""
        import torch
        dev = dock.device
        self.host_payload = host_payload

        def payload(n, dtype):
            if host_payload:
                return torch.empty(n, dtype=dtype, pin_memory=True)
            return torch.empty(n, dtype=dtype, device=dev)

        self.dock, self.consumer, self.max_samples, self.mode = dock, consumer, max_samples, mode
        self.pad_prompt_to, self.pad_response_to = pad_prompt_to, pad_response_to
        self.flags = OUT_LEFT_PAD_PROMPT if left_pad_prompts else 0
        i32 = torch.int32
        self.indices = torch.zeros(max_samples, dtype=i32, device=dev)
        self.cu_prompt = torch.zeros(max_samples + 1, dtype=i32, device=dev)
        self.cu_response = torch.zeros(max_samples + 1, dtype=i32, device=dev)
        self.cu_seq = torch.zeros(max_samples + 1, dtype=i32, device=dev)
        self.result = torch.zeros(C.sizeof(TdResult), dtype=torch.uint8, device=dev)
        self.scratch = torch.zeros(lib().td_get_scratch_bytes(dock.handle), dtype=torch.uint8, device=dev)
        need, outm, adv = dock.consumers[consumer]
        self.advantages = torch.zeros(max_samples, dtype=torch.float32, device=dev) if adv else None
        self.cols: Dict[int, "torch.Tensor"] = {}
        self.caps: Dict[int, int] = {}
        tdt = {I32: torch.int32, F32: torch.float32, BF16: torch.bfloat16}
        for c, (dt, cls, _pad) in enumerate(dock.columns):
            if not (outm >> c) & 1 or (want is not None and c not in want):
                continue
            if capacities is not None and c in capacities:
                cap = int(capacities[c])
            elif cls == SCALAR:
                cap = max_samples
            elif mode == PADDED:
                cap = max_samples * (pad_prompt_to if cls == PROMPT else pad_response_to)
            else:
                cap = prompt_tokens_cap if cls == PROMPT else response_tokens_cap
                if cap is None:
                    raise ValueError("packed ragged columns need prompt_tokens_cap / response_tokens_cap "
                                     "or explicit capacities")
            self.caps[c] = cap
            self.cols[c] = payload(max(cap, 1), tdt[dt])
        go = TdGetOut()
        go.mode, go.pad_prompt_to, go.pad_response_to = mode, pad_prompt_to, pad_response_to
        go.flags = self.flags
        go.indices, go.cu_prompt = self.indices.data_ptr(), self.cu_prompt.data_ptr()
        go.cu_response, go.cu_seq = self.cu_response.data_ptr(), self.cu_seq.data_ptr()
        for c, t in self.cols.items():
            go.col[c] = t.data_ptr()
            go.col_capacity_elems[c] = self.caps[c]
        go.advantages = self.advantages.data_ptr() if self.advantages is not None else None
        go.result = self.result.data_ptr()
        go.scratch, go.scratch_bytes = self.scratch.data_ptr(), self.scratch.numel()
        self.seq = self.seq_advantages = None
        if seq is not None or seq_adv:
            cap = int(seq_cap) if seq_cap is not None else int(prompt_tokens_cap) + int(response_tokens_cap)
            go.seq_capacity_elems = cap
            if seq is not None:
                go.seq_prompt_col, go.seq_response_col = seq
                self.seq = payload(max(cap, 1), tdt[dock.columns[seq[0]][0]])
                go.seq = self.seq.data_ptr()
            if seq_adv:
                self.seq_advantages = payload(max(cap, 1), torch.float32)
                go.seq_advantages = self.seq_advantages.data_ptr()
        self.struct = go

    def read_result(self) -> TdResult:
        """Copies the result block to the host (synchronises the current stream)."""
        host = self.result.cpu().numpy().tobytes()
        return TdResult.from_buffer_copy(host)


class HostGetBuffers:
    """Pinned host mirrors of a GetBuffers, the destination of td_get_host."""

    def __init__(self, bufs: GetBuffers):
        import torch
        self.indices = torch.zeros(bufs.indices.shape, dtype=bufs.indices.dtype).pin_memory()
        self.cu_prompt = torch.zeros(bufs.cu_prompt.shape, dtype=torch.int32).pin_memory()
        self.cu_response = torch.zeros(bufs.cu_response.shape, dtype=torch.int32).pin_memory()
        self.cu_seq = torch.zeros(bufs.cu_seq.shape, dtype=torch.int32).pin_memory()
        self.advantages = (torch.zeros(bufs.advantages.shape, dtype=torch.float32).pin_memory()
                           if bufs.advantages is not None else None)
        # payload that the device already writes into host memory needs no second buffer
        self.payload_in_place = bool(getattr(bufs, "host_payload", False))
        self.cols = ({c: t for c, t in bufs.cols.items()} if self.payload_in_place else
                     {c: torch.zeros(t.shape, dtype=t.dtype).pin_memory() for c, t in bufs.cols.items()})
        # the result block too lives in pinned memory: a copy into pageable memory stalls the caller
        self._result_mem = torch.zeros(C.sizeof(TdResult), dtype=torch.uint8).pin_memory()
        self.result = TdResult.from_address(self._result_mem.data_ptr())
        go = TdGetOut()
        go.mode, go.pad_prompt_to, go.pad_response_to = bufs.mode, bufs.pad_prompt_to, bufs.pad_response_to
        go.flags = getattr(bufs, "flags", 0)
        go.indices, go.cu_prompt = self.indices.data_ptr(), self.cu_prompt.data_ptr()
        go.cu_response, go.cu_seq = self.cu_response.data_ptr(), self.cu_seq.data_ptr()
        for c, t in self.cols.items():
            go.col[c] = None if self.payload_in_place else t.data_ptr()      # NULL: nothing to copy
            go.col_capacity_elems[c] = t.numel()
        go.advantages = self.advantages.data_ptr() if self.advantages is not None else None
        go.result = C.addressof(self.result)
        self.struct = go

    def bytes_valid(self, dock: "Dock") -> int:
        """Bytes td_get_host copied to the host for the last call."""
        r, n = self.result, self.result.n_samples
        total = C.sizeof(TdResult) + n * 4 + 3 * (n + 1) * 4 + (n * 4 if self.advantages is not None else 0)
        for c, t in self.cols.items():
            dt, cls, _ = dock.columns[c]
            if cls == SCALAR:
                e = n
            elif self.struct.mode == PACKED:
                e = r.prompt_tokens if cls == PROMPT else r.response_tokens
            else:
                e = n * (self.struct.pad_prompt_to if cls == PROMPT else self.struct.pad_response_to)
            total += e * ELEM_SIZE[dt]
        return total


class Plan:
    """A fixed list of gets (one GetBuffers each) that td_get_many serves in one call."""

    def __init__(self, dock: "Dock", bufs: Sequence[GetBuffers], stream=None):
        import torch
        self.dock, self.bufs = dock, list(bufs)
        n = len(self.bufs)
        reqs = (TdGetReq * n)()
        for j, b in enumerate(self.bufs):
            reqs[j].consumer, reqs[j].max_samples = b.consumer, b.max_samples
            reqs[j].out = b.struct
        self.nbytes = lib().td_plan_bytes(dock.handle, n)
        self.memory = torch.empty(self.nbytes, dtype=torch.uint8, device=dock.device)
        h = C.c_void_p()
        _check("td_plan_create", lib().td_plan_create(dock.handle, reqs, n, self.memory.data_ptr(),
                                                      self.nbytes, _stream_ptr(stream), C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().td_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Dock:
    """A transfer dock living in one torch-allocated workspace on `device`."""

    def __init__(self, G: int, N: int, S: int, columns: Sequence[Tuple[str, str, int]],
                 consumers: Sequence[Tuple[int, int, bool]], prompt_cap: int, response_cap: int,
                 reward_column: int, eps: float = 1e-6, device: int = 0):
        import torch
        self.G, self.N, self.S, self.n = G, N, S, G * N
        self.columns = [(DTYPE_TAG[d], CLASS_TAG[c], int(p)) for d, c, p in columns]
        self.consumers = [(int(a), int(b), bool(f)) for a, b, f in consumers]
        self.device = torch.device("cuda", device)
        self.cfg, self._keep = make_config(G, N, S, columns, consumers, prompt_cap, response_cap,
                                           reward_column, eps, device)
        self.workspace_bytes = query_workspace(self.cfg)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        _check("td_create", lib().td_create(C.byref(self.cfg), self.workspace.data_ptr(),
                                            self.workspace_bytes, C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            lib().td_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the four calls ---------------------------------------------------
    def put(self, column: int, indices, cu, data, stream=None):
        """indices int32 [k], cu int32 [k+1] or None, data: device tensors."""
        k = indices.numel()
        _check("td_put", lib().td_put(self.handle, column, indices.data_ptr(), k,
                                      cu.data_ptr() if cu is not None else None,
                                      data.data_ptr(), data.numel(), _stream_ptr(stream)))

    def put_many(self, items, stream=None):
        """items: (column, indices, cu or None, data) device tensors, stored in this order, or
        put_items() of them."""
        arr = items if isinstance(items, C.Array) else self.put_items(items)
        _check("td_put_many", lib().td_put_many(self.handle, arr, len(arr), _stream_ptr(stream)))

    def put_back(self, bufs: GetBuffers, items: Sequence[Tuple], stream=None):
        """items: (column, data) device tensors holding the rows of the batch last served into
        `bufs`, packed in batch order; the batch size is read on the device."""
        arr = (TdBackItem * len(items))()
        for j, (column, data) in enumerate(items):
            arr[j] = TdBackItem(column, 0, data.data_ptr(), data.numel())
        _check("td_put_back", lib().td_put_back(self.handle, C.byref(bufs.struct), bufs.max_samples,
                                                arr, len(items), _stream_ptr(stream)))

    def put_back_many(self, reqs: Sequence[Tuple], stream=None):
        """reqs: (bufs, column, data): column sent back for the batch last served into bufs."""
        arr = (TdBackReq * len(reqs))()
        for j, (bufs, column, data) in enumerate(reqs):
            arr[j] = TdBackReq(C.addressof(bufs.struct), bufs.max_samples, column, data.data_ptr(), data.numel())
        _check("td_put_back_many", lib().td_put_back_many(self.handle, arr, len(reqs), _stream_ptr(stream)))

    def plan(self, bufs: Sequence[GetBuffers], stream=None) -> "Plan":
        return Plan(self, bufs, stream)

    def get_many(self, plan: "Plan", stream=None):
        _check("td_get_many", lib().td_get_many(self.handle, plan.handle, _stream_ptr(stream)))

    def get(self, bufs: GetBuffers, stream=None, max_samples: Optional[int] = None):
        _check("td_get", lib().td_get(self.handle, bufs.consumer,
                                      bufs.max_samples if max_samples is None else max_samples,
                                      C.byref(bufs.struct), _stream_ptr(stream)))

    def get_static(self, bufs: GetBuffers, stream=None):
        """The same get with the scan scratch inside the library (no scratch buffer needed;
        docks of at most 16384 prompts; calls must not overlap on the GPU)."""
        _check("td_get_static", lib().td_get_static(self.handle, bufs.consumer, bufs.max_samples,
                                                    C.byref(bufs.struct), _stream_ptr(stream)))

    def reset(self, stream=None):
        _check("td_reset", lib().td_reset(self.handle, _stream_ptr(stream)))

    def status(self, stream=None) -> TdStats:
        st = TdStats()
        _check("td_status", lib().td_status(self.handle, C.byref(st), _stream_ptr(stream)))
        return st

    # -- host-buffer variants ----------------------------------------------
    def put_host(self, column: int, indices, cu, data, stage, stream=None):
        """indices / cu / data: host tensors (pinned for asynchronous copies); stage: a device
        uint8 tensor of at least put_host_stage_bytes()."""
        k = indices.numel()
        _check("td_put_host", lib().td_put_host(self.handle, column, indices.data_ptr(), k,
                                                cu.data_ptr() if cu is not None else None,
                                                data.data_ptr(), data.numel(), stage.data_ptr(),
                                                stage.numel(), _stream_ptr(stream)))

    def put_host_stage_bytes(self, column: int, k: int, data_elems: int) -> int:
        return lib().td_put_host_stage_bytes(self.handle, column, k, data_elems)

    @staticmethod
    def put_items(items: Sequence[Tuple]):
        """The td_put_item array of (column, indices, cu or None, data) tensors, reusable across calls."""
        arr = (TdPutItem * len(items))()
        for j, (column, indices, cu, data) in enumerate(items):
            arr[j] = TdPutItem(column, indices.numel(), indices.data_ptr(),
                               cu.data_ptr() if cu is not None else None, data.data_ptr(), data.numel())
        return arr

    @staticmethod
    def host_outs(hosts: Sequence["HostGetBuffers"]):
        """The td_get_out array of a list of host mirrors, reusable across calls."""
        return (TdGetOut * len(hosts))(*[h.struct for h in hosts])

    def put_many_host(self, items, stage, stream=None):
        """items: (column, indices, cu or None, data) HOST tensors, or put_items() of them; stage:
        device uint8 tensor."""
        arr = items if isinstance(items, C.Array) else self.put_items(items)
        _check("td_put_many_host", lib().td_put_many_host(self.handle, arr, len(arr), stage.data_ptr(),
                                                          stage.numel(), _stream_ptr(stream)))

    def get_many_host(self, plan: "Plan", hosts, stage=None, stream=None):
        """hosts: HostGetBuffers per request of the plan, or host_outs() of them; stage: device
        uint8 tensor of get_many_host_stage_bytes(plan) bytes, or None."""
        arr = hosts if isinstance(hosts, C.Array) else self.host_outs(hosts)
        _check("td_get_many_host", lib().td_get_many_host(self.handle, plan.handle, arr, len(arr),
                                                          stage.data_ptr() if stage is not None else None,
                                                          stage.numel() if stage is not None else 0,
                                                          _stream_ptr(stream)))

    def get_many_host_stage_bytes(self, plan: "Plan") -> int:
        return lib().td_get_many_host_stage_bytes(plan.handle)

    def get_host(self, bufs: GetBuffers, host: "HostGetBuffers", stream=None):
        _check("td_get_host", lib().td_get_host(self.handle, bufs.consumer, bufs.max_samples,
                                                C.byref(bufs.struct), C.byref(host.struct),
                                                _stream_ptr(stream)))

    # -- measurement ------------------------------------------------------
    def kernel_timing(self, enable: bool):
        _check("td_kernel_timing", lib().td_kernel_timing(self.handle, 1 if enable else 0))

    def kernel_timing_read(self, which: int) -> Tuple[int, float]:
        n, ms = C.c_uint64(0), C.c_double(0.0)
        _check("td_kernel_timing_read", lib().td_kernel_timing_read(self.handle, which, C.byref(n), C.byref(ms)))
        return n.value, ms.value

    # -- inspection -------------------------------------------------------
    def table(self, which: int, index: int = 0):
        """Device table as a uint8 torch tensor view (copy it before the dock changes)."""
        import torch
        ptr, nbytes = C.c_void_p(), C.c_size_t()
        _check("td_debug_table", lib().td_debug_table(self.handle, which, index, C.byref(ptr), C.byref(nbytes)))
        off = ptr.value - self.workspace.data_ptr()
        return self.workspace[off:off + nbytes.value]

    def validate(self, stream=None) -> TdValidateReport:
        """Self-check of the dock's tables (synchronises the stream); report.violations == 0 if sound."""
        rep = TdValidateReport()
        _check("td_debug_validate", lib().td_debug_validate(self.handle, _stream_ptr(stream), C.byref(rep)))
        return rep

    def debug_lookback(self, poll_limit: int = 0, skip_tile: int = 0xFFFFFFFF):
        """Test hook: poll limit of the scan's look-back wait (0 = default) and a tile that withholds
        its descriptor (0xFFFFFFFF = none)."""
        _check("td_debug_lookback", lib().td_debug_lookback(self.handle, poll_limit, skip_tile))

    def launch_count(self) -> int:
        return lib().td_launch_count(self.handle)


# -- operators a model runs on a served batch ------------------------------------
_TAG: Dict = {}               # torch dtype -> TD_* tag
_KINDS: Dict = {}             # element kind of a vector -> torch dtypes


def _torch_types():
    import torch
    _KINDS.update(i32=(torch.int32,), f32=(torch.float32,), bf16=(torch.bfloat16,), u8=(torch.uint8,),
                  mask=(torch.bool, torch.uint8))
    _TAG.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})


def _tag(t, what: str, allowed) -> int:
    if not _TAG:
        _torch_types()
    tag = _TAG.get(t.dtype)
    if tag not in allowed:
        raise ValueError(f"{what}: {t.dtype} is not supported here")
    return tag


def _vector(t, n: int, what: str, kind: str, device: int) -> int:
    """Address of a contiguous device tensor of at least n elements of the kind, 0 for None."""
    if t is None:
        return 0
    if not _KINDS:
        _torch_types()
    if t.dtype not in _KINDS[kind] or t.numel() < n or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{what}: needs a contiguous {kind} tensor of at least {n} elements on cuda:{device}, "
                         f"got {t.dtype} {tuple(t.shape)} strides {tuple(t.stride())} on {t.device}")
    return t.data_ptr()


def _matrix(t, what: str, device: int):
    """(address, row stride, dtype tag, rows, columns) of a device matrix of floats whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or t.get_device() != device or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what}: needs a matrix with contiguous rows on cuda:{device}, got {tuple(shape)} "
                         f"strides {stride} on {t.device}")
    rows, cols = shape
    # torch may give a matrix of one row, or of none, any row stride
    return t.data_ptr(), stride[0] if rows > 1 else cols, _tag(t, what, _FLOATS), rows, cols


def _device_of(t, what: str) -> int:
    d = t.get_device()
    if d < 0:
        raise ValueError(f"{what}: needs a CUDA tensor")
    return d


def _op_stream(stream, device: int) -> int:
    if stream is None:
        global _current_stream
        if _current_stream is None:
            import torch
            torch.cuda.init()
            # the handle alone; torch.cuda.current_stream() builds a Stream object around it, at 1.3 us a call
            _current_stream = torch._C._cuda_getCurrentRawStream
        return _current_stream(device)
    return _stream_ptr(stream)


class _Op:
    """A call (args struct, stream) whose struct is packed from the fields' values in order: packing takes
    0.1 us where filling a ctypes.Structure takes 0.6 to 1.5."""
    _CODES = {C.c_void_p: "P", C.c_int32: "i", C.c_uint32: "I", C.c_int64: "q", C.c_uint64: "Q", C.c_float: "f"}

    def __init__(self, name: str, args):
        self.name, self.func = name, None
        self.pack = struct.Struct("@" + "".join(self._CODES.get(t, "P") for _, t in args._fields_)).pack

    def __call__(self, stream: int, *values):
        if self.func is None:
            self.func = C.CFUNCTYPE(C.c_int, C.c_char_p, C.c_void_p)((self.name, lib()))
        rc = self.func(self.pack(*values), stream)
        if rc != 0:
            raise TdError(self.name, rc)


_TOKEN_LOGPROB, _TOKEN_LOGPROB_GRAD = _Op("td_token_logprob", TdLogprobArgs), _Op("td_token_logprob_grad", TdLogprobGradArgs)
_POLICY_LOSS, _EMBED, _EMBED_GRAD = _Op("td_policy_loss", TdPolicyArgs), _Op("td_embed", TdEmbedArgs), _Op("td_embed_grad", TdEmbedGradArgs)
_current_stream = None
_FLOATS = (F32, BF16, F16)


class Batch:
    """The row structure of a batch: cu_seqlens as a get writes them, and where its number of
    samples is decided on the device, the get's result block."""

    def __init__(self, cu_prompt=None, cu_response=None, result=None):
        some = cu_response if cu_response is not None else cu_prompt
        if some is None:
            raise ValueError("a batch needs cu_prompt or cu_response")
        self.device = _device_of(some, "cu_response")
        n = some.numel() - 1
        if n < 0:
            raise ValueError("cu arrays have one entry more than samples")
        self.cu_prompt, self.cu_response, self.result = cu_prompt, cu_response, result       # kept alive
        self.max_samples = n
        self.struct = TdBatch(n, 0, *(p or None for p in (_vector(cu_prompt, n + 1, "cu_prompt", "i32", self.device),
            _vector(cu_response, n + 1, "cu_response", "i32", self.device),
            _vector(result, C.sizeof(TdResult), "result", "u8", self.device))))
        self.address = C.addressof(self.struct)

    @classmethod
    def of(cls, bufs: GetBuffers) -> "Batch":
        """The batch last served into `bufs` when the stream gets there; its size stays on the device."""
        return cls(bufs.cu_prompt, bufs.cu_response, bufs.result)


def _batch_address(batch: Optional[Batch], device: int) -> int:
    if batch is None:
        return 0
    if batch.device != device:
        raise ValueError(f"batch: on cuda:{batch.device}, the operands are on cuda:{device}")
    return batch.address


class LogprobBuffers:
    """Outputs of token_logprob for up to n_tokens tokens, in token order: logprob, norm (row maximum
    and log-sum, what the gradient needs), entropy, entropy_bf16 (a column's type), status."""

    def __init__(self, n_tokens: int, device: int = 0, entropy: bool = False, entropy_bf16: bool = False):
        import torch
        dev = torch.device("cuda", device)
        f32 = torch.float32
        self.n_tokens, self.device = n_tokens, device
        self.logprob = torch.zeros(n_tokens, dtype=f32, device=dev)
        self.norm = torch.zeros(n_tokens, 2, dtype=f32, device=dev)
        self.entropy = torch.zeros(n_tokens, dtype=f32, device=dev) if entropy else None
        self.entropy_bf16 = torch.zeros(n_tokens, dtype=torch.bfloat16, device=dev) if entropy_bf16 else None
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self._addresses = (self.logprob.data_ptr(), self.norm.data_ptr(), self.entropy.data_ptr() if entropy else 0,
                           self.entropy_bf16.data_ptr() if entropy_bf16 else 0, self.status.data_ptr())


def token_logprob(out: LogprobBuffers, logits, targets, temperature: float = 1.0, batch: Optional[Batch] = None,
                  rows: int = ROWS_TOKEN, stream=None) -> LogprobBuffers:
    """Log-probability (and entropy) of `targets` (int32) under the rows of `logits` (float32, bfloat16
    or float16, rows contiguous, any row stride) at a temperature.  rows = ROWS_STREAM: logits
    follow the batch's fused token stream, targets its packed response column."""
    device, n = out.device, targets.numel()
    if n > out.n_tokens:
        raise ValueError(f"targets: {n} tokens, the buffers hold {out.n_tokens}")
    x, stride, tag, n_rows, vocab = _matrix(logits, "logits", device)
    _TOKEN_LOGPROB(_op_stream(stream, device), x, stride, tag, vocab, n_rows, n, rows, temperature, device,
                   _vector(targets, 0, "targets", "i32", device), _batch_address(batch, device), *out._addresses)
    return out


def token_logprob_grad(grad_logits, logits, targets, norm, grad_logprob=None, entropy=None, grad_entropy=None,
                       temperature: float = 1.0, batch: Optional[Batch] = None, rows: int = ROWS_TOKEN, status=None,
                       stream=None):
    """Gradient of token_logprob with respect to the logits, written to every row of grad_logits
    (which may be `logits`), from the gradients with respect to logprob and entropy and what the
    forward call left in norm and entropy."""
    device, n = _device_of(grad_logits, "grad_logits"), targets.numel()
    x, stride, tag, n_rows, vocab = _matrix(logits, "logits", device)
    g, gstride, gtag, grad_rows, grad_vocab = _matrix(grad_logits, "grad_logits", device)
    if tag != gtag or grad_rows != n_rows or grad_vocab != vocab:
        raise ValueError("grad_logits: needs the shape and type of logits")
    _TOKEN_LOGPROB_GRAD(_op_stream(stream, device), x, stride, tag, vocab, n_rows, n, rows, temperature, device,
                        _vector(targets, 0, "targets", "i32", device), _batch_address(batch, device),
                        _vector(norm, 2 * n, "norm", "f32", device), _vector(entropy, n, "entropy", "f32", device),
                        _vector(grad_logprob, n, "grad_logprob", "f32", device),
                        _vector(grad_entropy, n, "grad_entropy", "f32", device), g, gstride,
                        _vector(status, 1, "status", "i32", device))
    return grad_logits


class PolicyLossConfig:
    """Coefficients of policy_loss (td_policy_args has the formulas)."""

    def __init__(self, clip_low: float = 0.2, clip_high: float = 0.2, dual_clip: float = 0.0, kl_coef: float = 0.0,
                 kl_kind: int = KL_K3, entropy_coef: float = 0.0, reduction: int = MEAN_TOKENS, norm: float = 0.0,
                 grad_scale: float = 1.0):
        self.clip_low, self.clip_high, self.dual_clip = clip_low, clip_high, dual_clip
        self.kl_coef, self.kl_kind, self.entropy_coef = kl_coef, kl_kind, entropy_coef
        self.reduction, self.norm, self.grad_scale = reduction, norm, grad_scale


class PolicyLossBuffers:
    """Outputs and workspace of policy_loss for up to n_tokens positions and max_samples samples:
    grad_logprob, grad_entropy (entropy=True), stats with its views terms (loss, pg, kl, entropy),
    rates (clipped, old kl, ratio) and tokens."""

    def __init__(self, n_tokens: int, max_samples: int, device: int = 0, entropy: bool = False):
        import torch
        dev = torch.device("cuda", device)
        self.n_tokens, self.max_samples, self.device = n_tokens, max_samples, device
        self.grad_logprob = torch.zeros(n_tokens, dtype=torch.float32, device=dev)
        self.grad_entropy = torch.zeros(n_tokens, dtype=torch.float32, device=dev) if entropy else None
        self.stats = torch.zeros(POLICY_STATS, dtype=torch.float32, device=dev)
        self.terms, self.rates, self.tokens = self.stats[:4], self.stats[4:7], self.stats[7:]
        nbytes = lib().td_policy_loss_workspace_bytes(max_samples)
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
        self._addresses = (self.grad_logprob.data_ptr(), self.grad_entropy.data_ptr() if entropy else 0, self.stats.data_ptr(),
                           self.workspace.data_ptr(), nbytes)


def policy_loss(out: PolicyLossBuffers, batch: Batch, logprob, advantages, old_logprob=None, ref_logprob=None,
                entropy=None, mask=None, config: Optional[PolicyLossConfig] = None, row_width: int = 0,
                stream=None) -> PolicyLossBuffers:
    """Clipped policy loss with a KL term and its gradients over the response tokens of a batch.
    Per-token tensors are packed (row_width = 0: sample i at cu_response[i]) or padded (sample i at
    i * row_width); old_logprob and ref_logprob are float32 or bfloat16 columns; mask is bool or
    uint8; advantages are per sample."""
    device, n = out.device, logprob.numel()
    if n > out.n_tokens or batch.max_samples > out.max_samples:
        raise ValueError(f"{n} positions of {batch.max_samples} samples, the buffers hold {out.n_tokens} of {out.max_samples}")
    c = config if config is not None else PolicyLossConfig()
    some = old_logprob if old_logprob is not None else ref_logprob
    column, kind = F32, "f32"
    if some is not None and _tag(some, "old_logprob / ref_logprob", (F32, BF16)) == BF16:
        column, kind = BF16, "bf16"
    _POLICY_LOSS(_op_stream(stream, device), _batch_address(batch, device), n, row_width, column, c.kl_kind, c.reduction, device,
                 c.clip_low, c.clip_high, c.dual_clip, c.kl_coef, c.entropy_coef, c.norm, c.grad_scale, 0,
                 _vector(logprob, n, "logprob", "f32", device), _vector(old_logprob, n, "old_logprob", kind, device),
                 _vector(ref_logprob, n, "ref_logprob", kind, device), _vector(entropy, n, "entropy", "f32", device),
                 _vector(mask, n, "mask", "mask", device),
                 _vector(advantages, batch.max_samples, "advantages", "f32", device), *out._addresses)
    return out


def embed(out, ids, table, scale: float = 1.0, batch: Optional[Batch] = None, tokens: int = TOKENS_SEQ, status=None,
          stream=None):
    """out[t] = scale * table[ids[t]] (ids int32; out and table float32, bfloat16 or float16); zeros
    where ids[t] is no token and, with a batch, behind its tokens."""
    device, n = _device_of(out, "out"), ids.numel()
    o, ostride, otag, out_rows, out_dim = _matrix(out, "out", device)
    t, tstride, tag, vocab, dim = _matrix(table, "table", device)
    if tag != otag or out_rows != n or out_dim != dim:
        raise ValueError(f"out: needs shape ({n}, {dim}) and type {table.dtype}")
    _EMBED(_op_stream(stream, device), _vector(ids, 0, "ids", "i32", device), n, vocab, dim, tag, t, tstride, o, ostride, scale,
           tokens, device, 0, _batch_address(batch, device), _vector(status, 1, "status", "i32", device))
    return out


class EmbedGradWorkspace:
    """Workspace of embed_grad for up to n_tokens positions, vocab table rows and dim columns."""

    def __init__(self, n_tokens: int, vocab: int, dim: int, device: int = 0):
        import torch
        self.device = device
        self.nbytes = lib().td_embed_grad_workspace_bytes(n_tokens, vocab, dim)
        self.memory = torch.empty(self.nbytes, dtype=torch.uint8, device=torch.device("cuda", device))
        self.address = self.memory.data_ptr()


def embed_grad(grad_table, ids, grad_out, workspace: EmbedGradWorkspace, scale: float = 1.0, accumulate: bool = False,
               batch: Optional[Batch] = None, tokens: int = TOKENS_SEQ, status=None, stream=None):
    """Gradient of embed with respect to the table: row v gets scale * the sum of grad_out over the
    positions of id v.  accumulate: added to the rows that occur; otherwise every row is written.
    grad_table is float32 or of grad_out's type."""
    device, n = _device_of(grad_table, "grad_table"), ids.numel()
    g, gstride, gtag, vocab, dim = _matrix(grad_table, "grad_table", device)
    o, ostride, tag, out_rows, out_dim = _matrix(grad_out, "grad_out", device)
    if out_rows != n or out_dim != dim:
        raise ValueError(f"grad_out: needs shape ({n}, {dim})")
    if workspace.device != device:
        raise ValueError(f"workspace: on cuda:{workspace.device}, the operands are on cuda:{device}")
    _EMBED_GRAD(_op_stream(stream, device), _vector(ids, 0, "ids", "i32", device), n, vocab, dim, tag, o, ostride, gtag,
                1 if accumulate else 0, g, gstride, scale, tokens, device, 0, _batch_address(batch, device),
                workspace.address, workspace.nbytes, _vector(status, 1, "status", "i32", device))
    return grad_table


# -- a paged key-value cache for generation ---------------------------------------
_CACHE_WRITE, _CACHE_ATTENTION = _Op("td_cache_write", TdCacheWriteArgs), _Op("td_cache_attention", TdCacheAttentionArgs)


def _strides(t) -> Tuple:
    """Element strides; torch may give an axis of one entry, or of none, any."""
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape, t.stride()))


class Cache:
    """A paged key-value cache: keys and values [layers, pages, page_size, heads, dim] (float32, bfloat16 or
    float16; the same strides, dim contiguous; None, None with a page_size: tables only), table int32
    [max_seqs, max_pages], length int32 [max_seqs], holders int32 [pages].  All are the caller's tensors and are read and written
    in place; an empty cache has zero lengths and holders.  status collects ERR_* bits."""

    def __init__(self, keys, values, table, length, holders, page_size: Optional[int] = None):
        import torch
        device = self.device = _device_of(holders, "holders")
        self.keys, self.values, self.table, self.length, self.holders = keys, values, table, length, holders     # kept alive
        if len(table.shape) != 2:
            raise ValueError(f"table: needs a matrix, got {tuple(table.shape)}")
        (self.max_seqs, self.max_pages), self.n_pages = table.shape, holders.numel()
        shape, strides, addresses, tag = (0, self.n_pages, page_size, 0, 0), (0, 0, 0, 0, 0), (None, None), F32
        if (keys is None) != (values is None) or (keys is None and page_size is None):
            raise ValueError("a cache needs keys and values, or neither and a page_size")
        if keys is not None:
            shape, strides, tag = tuple(keys.shape), _strides(keys), _tag(keys, "keys", _FLOATS)
            if (len(shape) != 5 or tuple(values.shape) != shape or values.dtype != keys.dtype or _strides(values) != strides
                    or keys.get_device() != device or values.get_device() != device):
                raise ValueError(f"keys, values: need the same shape [layers, pages, page_size, heads, dim], strides and type on "
                                 f"cuda:{device}, got {shape} and {tuple(values.shape)}")
            if shape[1] != self.n_pages or (page_size is not None and page_size != shape[2]):
                raise ValueError(f"keys: {shape[1]} pages of {shape[2]} tokens, holders and page_size say {self.n_pages} of {page_size}")
            if strides[4] > 1 or (shape[4] > 1 and strides[4] != 1) or any(n > 1 and s == 0 for n, s in zip(shape, strides)):
                raise ValueError(f"keys: dim must be contiguous and no axis broadcast, got strides {strides}")
            addresses = keys.data_ptr(), values.data_ptr()
        self.n_layers, _, self.page_size, self.n_heads, self.dim = shape
        self.tag = tag
        self.status = torch.zeros(1, dtype=torch.int32, device=torch.device("cuda", device))
        nbytes = lib().td_cache_workspace_bytes(self.n_pages, self.max_seqs)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", device))
        self.struct = TdCache(tag, self.n_pages, self.page_size, self.n_layers, self.n_heads, self.dim, *strides[:4], *addresses,
                              self.max_seqs, self.max_pages, _vector(table, 0, "table", "i32", device),
                              _vector(length, self.max_seqs, "length", "i32", device), _vector(holders, 0, "holders", "i32", device),
                              self.status.data_ptr(), self.workspace.data_ptr(), nbytes, device, 0)
        self.address = C.addressof(self.struct)

    @classmethod
    def empty(cls, n_layers: int, n_pages: int, page_size: int, n_heads: int, dim: int, max_seqs: int, max_pages: int, dtype,
              device: int = 0, heads_first: bool = True) -> "Cache":
        """An empty cache of its own memory; heads_first: a token's heads lie side by side, otherwise a head's tokens of a page."""
        import torch
        dev = torch.device("cuda", device)
        shape = (n_layers, n_pages, page_size, n_heads, dim) if heads_first else (n_layers, n_pages, n_heads, page_size, dim)
        keys, values = (torch.zeros(shape, dtype=dtype, device=dev) for _ in range(2))
        if not heads_first:
            keys, values = keys.transpose(2, 3), values.transpose(2, 3)
        table, length, holders = (torch.zeros(n, dtype=torch.int32, device=dev) for n in ((max_seqs, max_pages), max_seqs, n_pages))
        return cls(keys, values, table, length, holders)


class _CacheCall:
    """A call (cache, addresses, stream), its function looked up once."""

    def __init__(self, name: str, extra: int):
        self.name, self.extra, self.func = name, extra, None

    def __call__(self, cache: Cache, stream, *addresses):
        if self.func is None:
            self.func = C.CFUNCTYPE(C.c_int, *[C.c_void_p] * (self.extra + 2))((self.name, lib()))
        rc = self.func(cache.address, *addresses, _op_stream(stream, cache.device))
        if rc != 0:
            raise TdError(self.name, rc)


_CACHE_EXTEND, _CACHE_FORK = _CacheCall("td_cache_extend", 2), _CacheCall("td_cache_fork", 1)
_CACHE_FREE, _CACHE_COMPACT = _CacheCall("td_cache_free", 1), _CacheCall("td_cache_compact", 2)


def cache_extend(cache: Cache, add=None, cu=None, stream=None):
    """Room for add[s] more tokens (int32 [max_seqs]; None: one for every sequence that has any): lengths grow, and the
    pages that takes are the lowest free ones, in order of sequence.  cu (int32 [max_seqs + 1]): written with the
    running sum of the tokens, as cache_write takes it."""
    _CACHE_EXTEND(cache, stream, _vector(add, cache.max_seqs, "add", "i32", cache.device) or None,
                  _vector(cu, cache.max_seqs + 1, "cu", "i32", cache.device) or None)


def cache_fork(cache: Cache, parent, stream=None):
    """Empty sequences s with parent[s] >= 0 (int32 [max_seqs]) become copies of parent[s]: full pages shared, a partly
    filled last page copied in every layer."""
    _CACHE_FORK(cache, stream, _vector(parent, cache.max_seqs, "parent", "i32", cache.device) or None)


def cache_free(cache: Cache, release=None, stream=None):
    """Sequences with release[s] (bool or uint8 [max_seqs]; None: all) give back their pages and become empty."""
    _CACHE_FREE(cache, stream, _vector(release, cache.max_seqs, "release", "mask", cache.device) or None)


def cache_compact(cache: Cache, used=None, moved=None, stream=None):
    """Held pages move to the lowest numbers, tables and holders follow.  used (int32 [1]): how many they are;
    moved (int32 [pages]): every page's new number, -1 for a free one."""
    _CACHE_COMPACT(cache, stream, _vector(used, 1, "used", "i32", cache.device) or None,
                   _vector(moved, cache.n_pages, "moved", "i32", cache.device) or None)


def _rows_of_heads(t, what: str, cache: Cache, heads: Optional[int] = None):
    """(address, row stride, head stride, rows, heads) of [rows, heads, dim] in the cache's type."""
    shape, strides = tuple(t.shape), _strides(t)
    if (len(shape) != 3 or shape[2] != cache.dim or (heads is not None and shape[1] != heads) or t.get_device() != cache.device
            or (shape[2] > 1 and strides[2] != 1)):
        raise ValueError(f"{what}: needs [rows, {heads or 'heads'}, {cache.dim}] with contiguous rows on cuda:{cache.device}, got {shape} "
                         f"strides {strides} on {t.device}")
    if _tag(t, what, _FLOATS) != cache.tag:
        raise ValueError(f"{what}: {t.dtype}, the cache has another type")
    return t.data_ptr(), strides[0], strides[1], shape[0], shape[1]


def cache_write(cache: Cache, keys, values, cu, layer: int = 0, stream=None):
    """Keys and values [rows, heads, dim] of new tokens into a layer: rows cu[s] .. cu[s + 1] - 1 are the newest tokens of
    sequence s, in order (cu int32 [max_seqs + 1], from cache_extend)."""
    k, row, head, n, _ = _rows_of_heads(keys, "keys", cache, cache.n_heads)
    v, row_v, head_v, n_v, _ = _rows_of_heads(values, "values", cache, cache.n_heads)
    if (row, head, n) != (row_v, head_v, n_v):
        raise ValueError("keys, values: need the same shape and strides")
    _CACHE_WRITE(_op_stream(stream, cache.device), cache.address, layer, n, k, v, row, head,
                 _vector(cu, cache.max_seqs + 1, "cu", "i32", cache.device))


class AttentionBuffers:
    """Outputs and workspace of cache_attention for up to n_rows rows of n_heads heads of dim elements, a multiple of 8 and 256 at
    most: out [n_rows, n_heads, dim] (a tensor of the caller's, with rows and heads on 16-byte boundaries, or allocated), lse
    (lse=True: float32 [n_rows, n_heads]).  The workspace has room for every form of the call, some 36 MB at 128 elements."""

    def __init__(self, n_rows: int, n_heads: int, dim: int, dtype, lse: bool = False, device: int = 0, out=None):
        import torch
        if dim % 8 or not 0 < dim <= 256:
            raise ValueError(f"dim: attention takes heads of a multiple of 8 elements, 256 at most, got {dim}")
        dev = torch.device("cuda", device)
        self.n_rows, self.n_heads, self.dim, self.device = n_rows, n_heads, dim, device
        self.out = out if out is not None else torch.zeros(n_rows, n_heads, dim, dtype=dtype, device=dev)
        strides = _strides(self.out)
        if (tuple(self.out.shape) != (n_rows, n_heads, dim) or self.out.dtype != dtype or self.out.get_device() != device
                or (dim > 1 and strides[2] != 1)):
            raise ValueError(f"out: needs {dtype} [{n_rows}, {n_heads}, {dim}] with contiguous rows on cuda:{device}")
        self.lse = torch.zeros(n_rows, n_heads, dtype=torch.float32, device=dev) if lse else None
        nbytes = lib().td_cache_attention_workspace_bytes(n_rows, n_heads, dim)
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
        self._addresses = (self.out.data_ptr(), strides[0], strides[1], self.lse.data_ptr() if lse else 0, self.workspace.data_ptr(), nbytes)


def cache_attention(out: AttentionBuffers, cache: Cache, q, seqs=None, layer: int = 0, window: int = 0, group: int = 1,
                    scale: Optional[float] = None, stream=None) -> AttentionBuffers:
    """Attention of one new token per row over a layer of the cache: q [rows, heads, dim] against the tokens of sequence
    seqs[row] (int32; None: the row's number; negative: none), the last `window` of them if it is not 0.  scale:
    1 / sqrt(dim) unless given.  group > 1: rows come in groups that share leading pages, which are read once where that spares
    enough; it pays for some hundred groups of 8 rows with 600 common tokens or of 4 with 2000 and more, and for groups of two rows, or
    a few groups of 4, group = 1 is faster.  The cache's and q's heads lie on 16-byte boundaries."""
    address, row, head, n, heads = _rows_of_heads(q, "q", cache)
    if n > out.n_rows or heads != out.n_heads or cache.dim != out.dim or out.device != cache.device or out.out.dtype != q.dtype:
        raise ValueError(f"q: {n} rows of {heads} x {cache.dim} {q.dtype}, the buffers hold {out.n_rows} of {out.n_heads} x {out.dim} "
                         f"{out.out.dtype} on cuda:{out.device}")
    try:
        _CACHE_ATTENTION(_op_stream(stream, cache.device), cache.address, layer, n, heads, group, window, 0,
                         cache.dim ** -0.5 if scale is None else scale, 0, _vector(seqs, n, "seqs", "i32", cache.device), address, row, head,
                         *out._addresses)
    except TdError as error:
        if error.code == EINVAL and (address | out._addresses[0] | (cache.struct.keys or 0) | (cache.struct.values or 0)) % 16 + sum(
                x * q.element_size() % 16 for x in (row, head, *out._addresses[1:3], cache.struct.layer_stride, cache.struct.page_stride,
                                                    cache.struct.token_stride, cache.struct.head_stride)):
            error.args = (f"{error}: keys, values, q and out, and all of their strides, have to be multiples of 16 bytes",)
        raise
    return out


def debug_cache_wait(block: int = 0xFFFFFFFF, tile: int = 0xFFFFFFFF):
    """Test hook: a block's wait for the products over a tile of common tokens counts as run out in later calls of
    cache_attention, whose heads that needed them are then NaN (ERR_COPY_TIMEOUT).  Without arguments: off again."""
    lib().td_debug_cache_wait(block, tile)
