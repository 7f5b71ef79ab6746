"""Binding of libhola_verify.so (ctypes, and native code for the calls of a serving loop, csrc/host_call.cpp): argument
marshalling only, every step runs in the CUDA kernels.

Function names mirror the C ABI (include/hola_verify.h).  Tensors are torch CUDA tensors; torch is used for
device memory and streams, nothing else.
"""
from __future__ import annotations

import ctypes
import os
import subprocess
import warnings
from array import array
from dataclasses import dataclass

import torch

from . import build as _build

HOLA_OK, HOLA_ERR_INVALID_ARG = 0, 1
HOLA_Q_BF16, HOLA_Q_F32 = 0, 1
HOLA_GATE_TARGET_ENTROPY, HOLA_GATE_DRAFT_ENTROPY = 0, 1
HOLA_FALLBACK_SAMPLE, HOLA_FALLBACK_GREEDY = 0, 1
HOLA_W_BF16, HOLA_W_INT8, HOLA_W8A8, HOLA_W8A16, HOLA_W_MIXED = 0, 1, 2, 3, 4
HOLA_HIDDEN_IN_PLACE, HOLA_HIDDEN_ON_LINES, HOLA_HIDDEN_8BIT = 0, 1, 2
HOLA_ARG_CLEAR_STATUS = 1
GROUP_ROWS, SUB_BLOCK, HOLA_PACE_WORDS = 256, 128, 256
FLAG_BAD_TOKEN, FLAG_BAD_UNIFORM, FLAG_TIMEOUT, FLAG_R_ZERO, FLAG_BAD_ADAPTER, FLAG_BAD_LOGIT, FLAG_BAD_BEAM = 1, 2, 4, 8, 16, 32, 64
HOLA_L_F32, HOLA_L_BF16, HOLA_L_F16 = 0, 1, 2
HOLA_T_F32, HOLA_T_BF16, HOLA_T_F16, HOLA_T_INT8, HOLA_T_MIXED = 0, 1, 2, 3, 4
HOLA_MAX_TOP, HOLA_MAX_RANK, HOLA_MAX_BEAMS = 32, 128, 32
HOLA_OPT_RING_SLOTS, HOLA_OPT_ROTATING_UNITS, HOLA_OPT_HOST_OVERLAP, HOLA_OPT_HOST_ROWS_ON_DEMAND, HOLA_OPT_PASSES, HOLA_OPT_PAIR_MMA, HOLA_OPT_HOST_IN_PLACE, HOLA_OPT_CONVERTER_GROUP, HOLA_OPT_FUSED_PASSES = 1, 2, 3, 4, 5, 6, 7, 8, 9

EXPORTS = ["hola_create", "hola_destroy", "hola_workspace_bytes", "hola_verify", "hola_verify_host",
           "hola_lm_head_entropy", "hola_accept_sample", "hola_host_traffic", "hola_shard_record_bytes", "hola_shard_lm_head",
           "hola_shard_accept", "hola_shard_sample", "hola_lm_head_entropy_static", "hola_lm_head_adapters", "hola_verify_adapters", "hola_token_logprobs", "hola_beam_select", "hola_beam_reorder", "hola_beam_states_check", "hola_embed", "hola_embed_grad", "hola_embed_grad_workspace_bytes", "hola_quantize_w8", "hola_quantize_w4", "hola_quantize_mixed", "hola_quantize_mixed_widths", "hola_plan", "hola_plan_ex", "hola_plan_for_shape", "hola_hidden_form_for_shape", "hola_sample_plan_for_shape", "hola_set_option", "hola_selftest_bounded_wait", "hola_selftest_staged_wait", "hola_selftest_mass_wait", "hola_selftest_pace", "hola_selftest_quotient", "hola_profile_begin", "hola_profile_end", "hola_strerror", "hola_last_cuda_error",
           "hola_version"]


class HolaError(RuntimeError):
    pass


class hola_verify_args(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("k", ctypes.c_int32), ("H", ctypes.c_int32), ("V", ctypes.c_int32),
                ("hidden", ctypes.c_void_p), ("W_lm", ctypes.c_void_p), ("draft_tok", ctypes.c_void_p),
                ("draft_q", ctypes.c_void_p), ("q_dtype", ctypes.c_int32), ("uniforms", ctypes.c_void_p),
                ("tau", ctypes.c_float), ("accept_len", ctypes.c_void_p), ("next_tok", ctypes.c_void_p),
                ("entropy", ctypes.c_void_p), ("logZ", ctypes.c_void_p), ("logits_out", ctypes.c_void_p),
                ("status_word", ctypes.c_void_p), ("gate_source", ctypes.c_int32), ("fallback", ctypes.c_int32),
                ("draft_entropy", ctypes.c_void_p), ("w_dtype", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("w_scale", ctypes.c_void_p), ("wmix", ctypes.c_void_p)]


class hola_wmix(ctypes.Structure):
    _fields_ = [("W16", ctypes.c_void_p), ("W8", ctypes.c_void_p), ("W4", ctypes.c_void_p), ("shift4", ctypes.c_void_p),
                ("group_width", ctypes.c_void_p), ("group_row", ctypes.c_void_p), ("rows16", ctypes.c_int32),
                ("rows8", ctypes.c_int32), ("rows4", ctypes.c_int32), ("reserved_", ctypes.c_int32)]


class hola_shard_args(ctypes.Structure):
    _fields_ = [("world", ctypes.c_int32), ("rank", ctypes.c_int32), ("v_offset", ctypes.c_int32),
                ("V_global", ctypes.c_int32), ("q_tok", ctypes.c_void_p), ("record_out", ctypes.c_void_p),
                ("records", ctypes.c_void_p), ("mass_out", ctypes.c_void_p), ("masses", ctypes.c_void_p)]


class hola_adapters(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("ids", ctypes.c_void_p),
                ("slots", ctypes.c_int32), ("rank", ctypes.c_int32)]


class hola_logprobs_args(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("V", ctypes.c_int32), ("T", ctypes.c_int32), ("n_top", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("l_dtype", ctypes.c_int32), ("k", ctypes.c_int32),
                ("tokens", ctypes.c_void_p), ("draft_tok", ctypes.c_void_p), ("accept_len", ctypes.c_void_p),
                ("next_tok", ctypes.c_void_p), ("logZ_in", ctypes.c_void_p), ("logprob", ctypes.c_void_p),
                ("rank", ctypes.c_void_p), ("entropy", ctypes.c_void_p), ("logZ", ctypes.c_void_p),
                ("top_ids", ctypes.c_void_p), ("top_logprobs", ctypes.c_void_p), ("status_word", ctypes.c_void_p)]


class hola_beam_args(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("W", ctypes.c_int32), ("V", ctypes.c_int32), ("n", ctypes.c_int32),
                ("logits", ctypes.c_void_p), ("seq_stride", ctypes.c_int64), ("beam_stride", ctypes.c_int64),
                ("l_dtype", ctypes.c_int32), ("end_token", ctypes.c_int32), ("logZ", ctypes.c_void_p), ("score", ctypes.c_void_p),
                ("finished", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("keep_slots", ctypes.c_int32),
                ("reserved_", ctypes.c_int32), ("score_out", ctypes.c_void_p), ("parent", ctypes.c_void_p),
                ("token", ctypes.c_void_p), ("finished_out", ctypes.c_void_p), ("status_word", ctypes.c_void_p)]


class hola_beam_state(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("seq_stride", ctypes.c_int64), ("beam_stride", ctypes.c_int64),
                ("outer_stride", ctypes.c_int64 * 2), ("dst_seq_stride", ctypes.c_int64), ("dst_beam_stride", ctypes.c_int64),
                ("dst_outer_stride", ctypes.c_int64 * 2), ("outer", ctypes.c_int64 * 2), ("run", ctypes.c_int64),
                ("position", ctypes.c_int64)]


class hola_reorder_args(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("W", ctypes.c_int32), ("n", ctypes.c_int32), ("count", ctypes.c_int32),
                ("states", ctypes.c_void_p), ("parent", ctypes.c_void_p), ("parent_stride", ctypes.c_int64),
                ("used", ctypes.c_void_p), ("status_word", ctypes.c_void_p)]


class hola_embed_args(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("V", ctypes.c_int32), ("H", ctypes.c_int32), ("v_offset", ctypes.c_int32),
                ("V_global", ctypes.c_int32), ("tokens", ctypes.c_void_p), ("wide_tokens", ctypes.c_int32), ("t_dtype", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("w_scale", ctypes.c_void_p), ("wmix", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("out_dtype", ctypes.c_int32), ("add", ctypes.c_void_p), ("add_stride", ctypes.c_int64),
                ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64), ("status_word", ctypes.c_void_p)]


class hola_embed_grad_args(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("V", ctypes.c_int32), ("H", ctypes.c_int32), ("v_offset", ctypes.c_int32),
                ("V_global", ctypes.c_int32), ("tokens", ctypes.c_void_p), ("wide_tokens", ctypes.c_int32), ("g_dtype", ctypes.c_int32),
                ("grad", ctypes.c_void_p), ("grad_stride", ctypes.c_int64), ("scale", ctypes.c_float), ("out_dtype", ctypes.c_int32),
                ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64), ("accumulate", ctypes.c_int32), ("reserved_", ctypes.c_int32),
                ("ids_out", ctypes.c_void_p), ("count_out", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_uint64), ("status_word", ctypes.c_void_p)]


class hola_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("tile_v", "grid", "stages", "rows_per_pass", "passes", "kernels_per_call")]


class hola_sample_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("ctas", "threads", "staged")]


_lib = None
_host = None            # the native helper (csrc/host_call.cpp), or None: arguments are then filled from Python
_entry = {}             # addresses of the entry points that it calls
_ADAPTER_ENTRIES = ("hola_lm_head_adapters", "hola_verify_adapters")     # those whose function takes a hola_adapters as well


def _load_host(lib: ctypes.CDLL):
    """The helper reads tensors through torch's C++ classes: it is built against the torch that runs."""
    global _host
    try:
        helper = _build.load_host()
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"host-side helper not available, calls cost a few microseconds more: {e}")
        return
    for name in ("hola_verify", "hola_verify_host", "hola_lm_head_entropy", "hola_quantize_mixed_widths", "hola_lm_head_adapters",
                 "hola_verify_adapters", "hola_token_logprobs", "hola_beam_select", "hola_beam_reorder", "hola_embed", "hola_embed_grad",
                 "hola_embed_grad_workspace_bytes"):
        _entry[name] = ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
    _host = helper


def load_library(path: str | None = None) -> ctypes.CDLL:
    """Loads the C-ABI library (building it first if the source is newer).  Raises if it cannot be had."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or (_build.LIB if os.path.exists(_build.LIB) and not _build.needs_build() else _build.build())
    lib = ctypes.CDLL(p)
    lib.hola_create.restype = ctypes.c_int
    lib.hola_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                ctypes.c_int, ctypes.c_int]
    lib.hola_destroy.restype = ctypes.c_int
    lib.hola_destroy.argtypes = [ctypes.c_void_p]
    lib.hola_workspace_bytes.restype = ctypes.c_size_t
    lib.hola_workspace_bytes.argtypes = [ctypes.c_int] * 4
    for name in ("hola_verify", "hola_verify_host", "hola_lm_head_entropy", "hola_accept_sample"):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [ctypes.c_void_p, ctypes.POINTER(hola_verify_args), ctypes.c_void_p]
    lib.hola_lm_head_entropy_static.restype = ctypes.c_int
    lib.hola_lm_head_entropy_static.argtypes = [ctypes.POINTER(hola_verify_args), ctypes.c_void_p]
    for name in ("hola_lm_head_adapters", "hola_verify_adapters"):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [ctypes.c_void_p, ctypes.POINTER(hola_verify_args), ctypes.POINTER(hola_adapters), ctypes.c_void_p]
    lib.hola_token_logprobs.restype = ctypes.c_int
    lib.hola_token_logprobs.argtypes = [ctypes.POINTER(hola_logprobs_args), ctypes.c_void_p]
    for name, args in (("hola_beam_select", hola_beam_args), ("hola_beam_reorder", hola_reorder_args), ("hola_embed", hola_embed_args),
                       ("hola_embed_grad", hola_embed_grad_args)):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [ctypes.POINTER(args), ctypes.c_void_p]
    lib.hola_beam_states_check.restype = ctypes.c_int
    lib.hola_beam_states_check.argtypes = [ctypes.POINTER(hola_reorder_args)]
    lib.hola_embed_grad_workspace_bytes.restype = ctypes.c_size_t
    lib.hola_embed_grad_workspace_bytes.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int]
    lib.hola_quantize_w8.restype = ctypes.c_int
    lib.hola_quantize_w8.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_void_p]
    lib.hola_quantize_w4.restype = ctypes.c_int
    lib.hola_quantize_w4.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                     ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]
    lib.hola_quantize_mixed.restype = ctypes.c_int
    lib.hola_quantize_mixed.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.POINTER(hola_wmix),
                                        ctypes.c_void_p, ctypes.c_void_p]
    lib.hola_quantize_mixed_widths.restype = ctypes.c_int
    lib.hola_quantize_mixed_widths.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                               ctypes.POINTER(hola_wmix), ctypes.c_void_p, ctypes.c_void_p]
    lib.hola_plan.restype = ctypes.c_int
    lib.hola_plan.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.POINTER(hola_plan_info)]
    lib.hola_plan_for_shape.restype = ctypes.c_int
    lib.hola_plan_for_shape.argtypes = [ctypes.c_int] * 5 + [ctypes.POINTER(hola_plan_info)]
    lib.hola_hidden_form_for_shape.restype = ctypes.c_int
    lib.hola_hidden_form_for_shape.argtypes = [ctypes.c_int] * 5 + [ctypes.POINTER(ctypes.c_int32)]
    lib.hola_sample_plan_for_shape.restype = ctypes.c_int
    lib.hola_sample_plan_for_shape.argtypes = [ctypes.c_int] * 6 + [ctypes.POINTER(hola_sample_info)]
    lib.hola_plan_ex.restype = ctypes.c_int
    lib.hola_plan_ex.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.POINTER(hola_plan_info)]
    lib.hola_profile_begin.restype = ctypes.c_int
    lib.hola_profile_begin.argtypes = [ctypes.c_void_p, ctypes.c_int]
    lib.hola_set_option.restype = ctypes.c_int
    lib.hola_set_option.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    for name in ("hola_selftest_bounded_wait", "hola_selftest_staged_wait", "hola_selftest_mass_wait"):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [ctypes.c_void_p, ctypes.c_longlong, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.hola_selftest_pace.restype = ctypes.c_int
    lib.hola_selftest_pace.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.hola_selftest_quotient.restype = ctypes.c_int
    lib.hola_selftest_quotient.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                           ctypes.c_void_p]
    lib.hola_shard_record_bytes.restype = ctypes.c_size_t
    lib.hola_shard_record_bytes.argtypes = [ctypes.c_int, ctypes.c_int]
    for name in ("hola_shard_lm_head", "hola_shard_accept", "hola_shard_sample"):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [ctypes.c_void_p, ctypes.POINTER(hola_verify_args), ctypes.POINTER(hola_shard_args),
                       ctypes.c_void_p]
    lib.hola_host_traffic.restype = ctypes.c_int
    lib.hola_host_traffic.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_ulonglong),
                                      ctypes.POINTER(ctypes.c_ulonglong)]
    lib.hola_profile_end.restype = ctypes.c_int
    lib.hola_profile_end.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_double),
                                     ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)]
    lib.hola_strerror.restype = ctypes.c_char_p
    lib.hola_strerror.argtypes = [ctypes.c_int]
    lib.hola_last_cuda_error.restype = ctypes.c_char_p
    lib.hola_last_cuda_error.argtypes = [ctypes.c_void_p]
    lib.hola_version.restype = ctypes.c_char_p
    if path is None:
        _lib = lib
        _load_host(lib)
    return lib


def _check(lib, ctx, status: int, what: str):
    if status != HOLA_OK:
        msg = lib.hola_strerror(status).decode()
        detail = lib.hola_last_cuda_error(ctx).decode() if ctx else ""
        raise HolaError(f"{what}: {msg}" + (f" [{detail}]" if detail else ""))


def _dptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream_ptr(stream) -> int:
    """cudaStream_t of a torch stream; None: the current stream of the current device, without making a Stream object
    for it (a quarter of what a call costs on the host)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream.cuda_stream


def _make_on(stream, dev, make):
    """make(), whose tensors a call fills that was given none: made on the stream that the call was given, since the allocator
    orders uses of a block on the stream it was made on only.  What the caller's current stream still has to read of them when they
    are dropped is waited for as well."""
    if stream is None:
        return make()
    if not isinstance(stream, torch.cuda.Stream):                # (whatever has a cuda_stream)
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=dev)
    here = torch.cuda.current_stream(dev)
    with torch.cuda.stream(stream):
        made = make()
    if here != stream:
        for t in (made.__dict__.values() if hasattr(made, "__dict__") else made):
            if isinstance(t, torch.Tensor):
                t.record_stream(here)
    return made


def hola_quantize_w8(W_lm: torch.Tensor, stream=None):
    """8-bit form of a bf16 W_lm [V, H] on the device: returns (q int8 [V, H], scale fp32 [V]).  The integers and the
    scales are computed by the library's kernel; torch only provides the two output buffers."""
    if W_lm.dtype != torch.bfloat16 or not W_lm.is_cuda or not W_lm.is_contiguous():
        raise HolaError("hola_quantize_w8 takes a contiguous bfloat16 device tensor")
    lib = load_library()
    V, H = W_lm.shape
    q, scale = _make_on(stream, W_lm.device, lambda: (torch.empty((V, H), dtype=torch.int8, device=W_lm.device),
                                                      torch.empty((V,), dtype=torch.float32, device=W_lm.device)))
    with torch.cuda.device(W_lm.device):
        _check(lib, None, lib.hola_quantize_w8(_dptr(W_lm), V, H, _dptr(q), _dptr(scale), _stream_ptr(stream)),
               "hola_quantize_w8")
    return q, scale


@dataclass
class MixedHead:
    """An LM head stored as groups of 256 vocabulary rows at 4, 8 or 16 bits (HOLA_W_MIXED): the device buffers and the
    hola_wmix struct that points at them.  Keep the object alive while calls that use it are in flight."""
    V: int
    H: int
    widths: list
    W16: torch.Tensor | None
    W8: torch.Tensor | None
    W4: torch.Tensor | None
    shift4: torch.Tensor | None
    w_scale: torch.Tensor
    group_width: torch.Tensor
    group_row: torch.Tensor
    struct: "hola_wmix" = None

    def weight_bytes(self) -> int:
        """Bytes of weights, scales and exponents one pass over the head streams."""
        n = self.w_scale.numel() * 4
        for t in (self.W16, self.W8, self.W4, self.shift4):
            n += 0 if t is None else t.numel() * t.element_size()
        return n


def hola_quantize_mixed(W_lm: torch.Tensor, widths, stream=None) -> MixedHead:
    """bf16 W_lm [V, H] -> the mixed-width form: widths[g] in {4, 8, 16} for group g of 256 vocabulary rows.  Codes,
    scales and exponents are made by one launch of the library's quantiser, to which the widths go as launch parameters (on
    another stream, for widths that are no plain list of integers and beyond 2048 groups: as two tables, in one copy);
    torch provides the buffers."""
    if W_lm.dtype != torch.bfloat16 or not W_lm.is_cuda or not W_lm.is_contiguous():
        raise HolaError("hola_quantize_mixed takes a contiguous bfloat16 device tensor")
    lib = load_library()
    if _host is not None and stream is None:
        st = hola_wmix()
        got = _host.quantize(_entry["hola_quantize_mixed_widths"], W_lm, widths, st, torch._C._cuda_getDevice(), _stream_ptr(None))
        if got is not None:
            _check(lib, None, got[0], "hola_quantize_mixed")
            return MixedHead(*got[1:], st)
    V, H = W_lm.shape
    ng = -(-V // GROUP_ROWS)
    widths = [int(x) for x in widths]
    if len(widths) != ng or not set(widths) <= {4, 8, 16} or H % SUB_BLOCK:
        raise HolaError(f"need {ng} widths out of 4, 8, 16 and H a multiple of {SUB_BLOCK}")
    dev = W_lm.device
    rows = [0] * 17                                              # rows of each width so far
    group_row = array("i")
    for wd in widths:
        group_row.append(rows[wd])
        rows[wd] += GROUP_ROWS
    if ng:
        rows[widths[-1]] -= ng * GROUP_ROWS - V                  # the last group may be ragged
        tables = torch.frombuffer(bytearray(group_row.tobytes() + bytes(widths)), dtype=torch.uint8)
    else:
        tables = torch.empty(0, dtype=torch.uint8)
    s = torch.cuda.current_stream(dev) if stream is None else stream
    if not isinstance(s, torch.cuda.Stream):                     # (as elsewhere, whatever has a cuda_stream)
        s = torch.cuda.ExternalStream(s.cuda_stream, device=dev)
    with torch.cuda.device(dev), torch.cuda.stream(s):
        W16 = torch.empty((rows[16], H), dtype=torch.bfloat16, device=dev) if rows[16] else None
        W8 = torch.empty((rows[8], H), dtype=torch.int8, device=dev) if rows[8] else None
        W4 = torch.empty((rows[4], H // 2), dtype=torch.uint8, device=dev) if rows[4] else None
        shift4 = torch.empty((H // SUB_BLOCK, rows[4]), dtype=torch.uint8, device=dev) if rows[4] else None
        w_scale = torch.empty((V,), dtype=torch.float32, device=dev)
        # (a copy from pageable memory has left that memory when the call returns)
        tables = tables.to(dev, non_blocking=True)
        head = MixedHead(V, H, widths, W16, W8, W4, shift4, w_scale, tables[4 * ng:], tables[:4 * ng].view(torch.int32))
        st = hola_wmix()
        st.W16, st.W8, st.W4, st.shift4 = (t.data_ptr() if t is not None else None for t in (W16, W8, W4, shift4))
        st.group_width, st.group_row = head.group_width.data_ptr(), head.group_row.data_ptr()
        st.rows16, st.rows8, st.rows4 = rows[16], rows[8], rows[4]
        head.struct = st
        if V:
            _check(lib, None, lib.hola_quantize_mixed(_dptr(W_lm), V, H, ctypes.byref(st), _dptr(w_scale), _stream_ptr(s)),
                   "hola_quantize_mixed")
    return head


def hola_lm_head_entropy_static(hidden, W_lm, logits, entropy, logZ, stream=None, status=None) -> None:
    """Steps 1-2 through the entry point that allocates no device memory (no context needed).

    For callers that cannot call cudaMalloc (all of HBM already handed to their own pool, a fixed memory budget,
    an allocator that is locked at this point): the library's only scratch for this call is a 1.25 MiB array
    built into it.  Every tensor is the caller's and lives on the current device: hidden bf16 [B, k+1, H],
    W_lm bf16 [V, H], and the outputs logits fp32 [B, k+1, V], entropy and logZ fp32 [B, k+1].
    At most 512 verify rows (B * (k+1)); larger calls raise HolaError and launch nothing.  Calls share the
    built-in array, so do not let two of them overlap on one GPU.  `status` (int32 [1] on the device, optional) gets
    HOLA_FLAG_TIMEOUT OR-ed in should an on-chip wait run out: it is the only way to learn of that here.
    """
    lib = load_library()
    B, k1, H = hidden.shape
    a = hola_verify_args()
    a.B, a.k, a.H, a.V = B, k1 - 1, H, W_lm.shape[0]
    a.hidden, a.W_lm = _dptr(hidden), _dptr(W_lm)
    a.logits_out, a.entropy, a.logZ = _dptr(logits), _dptr(entropy), _dptr(logZ)
    a.status_word = _dptr(status)
    _check(lib, None, lib.hola_lm_head_entropy_static(ctypes.byref(a), _stream_ptr(stream)),
           "hola_lm_head_entropy_static")


class AdapterBank:
    """Low-rank adapters resident on the device for hola_lm_head_adapters and hola_verify_adapters: slot s adds scale[s] * B[s] A[s] to
    the LM head of the sequences that name it.  Laid out once: A as [slots, rank, H], B as [slots, V, rank], the rank filled up with
    zeros to a multiple of 8."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None):
        """A: bf16 [slots, rank, H], B: bf16 [slots, V, rank], scale: fp32 [slots] (None: 1 for all)."""
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
            raise HolaError("AdapterBank takes A [slots, rank, H] and B [slots, V, rank]")
        if scale is not None and tuple(scale.shape) != (A.shape[0],):
            raise HolaError("AdapterBank: scale must have one value per slot")
        if A.dtype != torch.bfloat16 or B.dtype != torch.bfloat16 or A.device != B.device:
            raise HolaError("AdapterBank takes bfloat16 factors on one device")
        rank = A.shape[1]
        self._make(*A.shape, B.shape[1], A.device)
        self.A[:, :rank] = A
        self.B[:, :, :rank] = B
        if scale is not None:
            self.scale.copy_(scale)

    @classmethod
    def empty(cls, slots: int, rank: int, H: int, V: int, device=None) -> "AdapterBank":
        """Slots of zeros, to be filled by set() with adapters of up to this rank."""
        bank = cls.__new__(cls)
        device = torch.device("cuda" if device is None else device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        bank._make(slots, rank, H, V, device)
        return bank

    def _make(self, slots, rank, H, V, device):
        if slots < 1 or not 1 <= rank <= HOLA_MAX_RANK:
            raise HolaError(f"AdapterBank: at least one slot, ranks 1 .. {HOLA_MAX_RANK}")
        self.slots, self.rank, self.H, self.V, self.device = slots, -(-rank // 8) * 8, H, V, device
        self.A = torch.zeros((slots, self.rank, H), dtype=torch.bfloat16, device=device)
        self.B = torch.zeros((slots, V, self.rank), dtype=torch.bfloat16, device=device)
        self.scale = torch.ones((slots,), dtype=torch.float32, device=device)
        self.struct = st = hola_adapters()
        st.A, st.B, st.scale = self.A.data_ptr(), self.B.data_ptr(), self.scale.data_ptr()
        st.slots, st.rank = slots, self.rank
        self.address = ctypes.addressof(st)

    def set(self, slot: int, A: torch.Tensor, B: torch.Tensor, scale=None) -> None:
        """Puts an adapter into a slot, in order with the current stream's work: A bf16 [r, H], B bf16 [V, r], r at most the bank's
        rank; scale: a number or a tensor of one (None: 1)."""
        r = A.shape[0] if A.dim() == 2 else -1
        if not 0 <= slot < self.slots or not 1 <= r <= self.rank or tuple(A.shape) != (r, self.H) or tuple(B.shape) != (self.V, r):
            raise HolaError(f"AdapterBank.set: slot 0 .. {self.slots - 1}, A [r, {self.H}], B [{self.V}, r], r at most {self.rank}")
        if A.dtype != torch.bfloat16 or B.dtype != torch.bfloat16:
            raise HolaError("AdapterBank.set takes bfloat16 factors")
        self.A[slot, :r] = A
        self.A[slot, r:] = 0
        self.B[slot, :, :r] = B
        self.B[slot, :, r:] = 0
        self.scale[slot] = 1.0 if scale is None else scale


@dataclass
class TokenLogprobs:
    """What hola_token_logprobs fills; the fields that were not asked for are None.  `...` is the shape of the rows."""
    logprob: torch.Tensor | None        # fp32 [..., T], or [...] where the tokens came without that axis
    rank: torch.Tensor | None           # int32, like logprob
    entropy: torch.Tensor | None        # fp32 [...]
    logZ: torch.Tensor | None           # fp32 [...]
    top_ids: torch.Tensor | None        # int32 [..., n_top]
    top_logprobs: torch.Tensor | None   # fp32 [..., n_top]


_L_DTYPES = {torch.float32: HOLA_L_F32, torch.bfloat16: HOLA_L_BF16, torch.float16: HOLA_L_F16}


def _row_stride(t: torch.Tensor) -> int:
    """Entries from one row (last axis) of `t` to the next; the rows have to lie at one distance from each other."""
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise HolaError("hola_token_logprobs: the entries of a row must lie side by side")
    stride, rows = None, 1
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if stride is None:
            stride = s
        elif s != stride * rows:
            raise HolaError("hola_token_logprobs: the rows must lie at one distance from each other")
        rows *= n
    return t.shape[-1] if stride is None else stride


def hola_token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, n_top: int = 0, logZ: torch.Tensor | None = None,
                        emitted=None, want_rank: bool = True, out: TokenLogprobs | None = None, status: torch.Tensor | None = None,
                        stream=None) -> TokenLogprobs:
    """Log probabilities and ranks of given tokens, entropy, logZ and the `n_top` most probable entries of every row of `logits`
    (fp32, bf16 or fp16 [..., V]; the rows at any one distance from each other).

    tokens: int32 [..., T], or [...] for one per row; -1 is no token (logprob 0, rank -1).  emitted: (draft_tok [B, k], accept_len
    [B], next_tok [B]) of a verify call instead, for logits [B, k + 1, V]: position j holds draft_tok[b, j] up to accept_len[b],
    then next_tok[b], nothing behind.  logZ: fp32 [...] where it is known (a verify call's): entropy and logZ are not made then;
    the emitted form needs it.  Without ranks and alternatives nothing but the tokens' entries is read in that case.
    status: int32 [1] on the device, HOLA_FLAG_* bits are OR-ed in.  out: an earlier call's result of the same form, filled again.
    stream: where the call runs, and where its fresh outputs are made (see HolaVerify)."""
    lib = load_library()
    if _host is not None and stream is None and out is None:
        draft_tok, accept_len, next_tok = emitted if emitted is not None else (None, None, None)
        got = _host.score(_entry["hola_token_logprobs"], logits, tokens, n_top, logZ, draft_tok, accept_len, next_tok, emitted is not None,
                          want_rank, status, torch._C._cuda_getDevice(), _stream_ptr(None))
        if got is not None:
            if got[0]:
                _check(lib, None, got[0], "hola_token_logprobs")
            return TokenLogprobs(*got[1:])
    if logits.dtype not in _L_DTYPES or not logits.is_cuda or logits.dim() < 1:
        raise HolaError("hola_token_logprobs takes fp32, bf16 or fp16 logits on a device")
    shape, dev = logits.shape[:-1], logits.device
    a = hola_logprobs_args()
    if max(shape.numel(), logits.shape[-1], 0 if tokens is None or tokens.dim() == 0 else tokens.shape[-1]) > 2 ** 31 - 1:
        raise HolaError("hola_token_logprobs: more rows, entries or tokens per row than 32 bits count")       # (ctypes would cut them off)
    a.rows, a.V, a.n_top = shape.numel(), logits.shape[-1], n_top
    a.logits, a.row_stride, a.l_dtype = logits.data_ptr(), _row_stride(logits), _L_DTYPES[logits.dtype]

    def check(t, dtype, size, name):
        if t.dtype != dtype or t.device != dev or tuple(t.shape) != tuple(size) or not t.is_contiguous():
            raise HolaError(f"hola_token_logprobs: {name} must be a contiguous {dtype} tensor of shape {tuple(size)} on {dev}")
        return t.data_ptr()

    per_row = None                                               # shape of the tokens
    if emitted is not None:
        if tokens is not None or logits.dim() != 3 or logZ is None:
            raise HolaError("hola_token_logprobs: the emitted form takes logits [B, k + 1, V] and logZ, and no tokens")
        draft_tok, accept_len, next_tok = emitted
        B, k1 = shape
        a.k, a.T, per_row = k1 - 1, 1, shape
        if k1 > 1:
            a.draft_tok = check(draft_tok, torch.int32, (B, k1 - 1), "draft_tok")
        a.accept_len = check(accept_len, torch.int32, (B,), "accept_len")
        a.next_tok = check(next_tok, torch.int32, (B,), "next_tok")
    elif tokens is not None:
        per_row = tokens.shape
        if per_row[:len(shape)] != shape or len(per_row) > len(shape) + 1:
            raise HolaError("hola_token_logprobs: tokens must have the shape of the rows, and one more axis at most")
        a.T = per_row[-1] if len(per_row) > len(shape) else 1
        if a.T:
            a.tokens = check(tokens, torch.int32, per_row, "tokens")
    if logZ is not None:
        a.logZ_in = check(logZ, torch.float32, shape, "logZ")
    if n_top and not 0 < n_top <= min(a.V, HOLA_MAX_TOP):
        raise HolaError(f"hola_token_logprobs: n_top must be 0 .. min(V, {HOLA_MAX_TOP})")
    sums, some = logZ is None, per_row is not None and a.T > 0

    def field(name, dtype, size, wanted):
        if not wanted:
            return None
        t = torch.empty(size, dtype=dtype, device=dev) if out is None else getattr(out, name)
        if t is None:
            raise HolaError(f"hola_token_logprobs: out has no {name}")
        setattr(a, name, t.data_ptr() if out is None else check(t, dtype, size, name))
        return t

    def fields():
        return TokenLogprobs(field("logprob", torch.float32, per_row, some), field("rank", torch.int32, per_row, some and want_rank),
                             field("entropy", torch.float32, shape, sums), field("logZ", torch.float32, shape, sums),
                             field("top_ids", torch.int32, (*shape, n_top), n_top > 0),
                             field("top_logprobs", torch.float32, (*shape, n_top), n_top > 0))

    got = fields() if out is not None else _make_on(stream, dev, fields)
    if status is not None:
        a.status_word = check(status, torch.int32, (1,), "status")
    if a.rows == 0 or not (sums or some or n_top):
        return got
    with torch.cuda.device(dev):
        _check(lib, None, lib.hola_token_logprobs(ctypes.byref(a), _stream_ptr(stream)), "hola_token_logprobs")
    return got


# ------------------------------------------------------------------------------------------------ beams
@dataclass
class BeamSelection:
    """What hola_beam_select fills."""
    score: torch.Tensor                 # fp32 [B, n]
    parent: torch.Tensor                # int32 [B, n]
    token: torch.Tensor                 # int32 [B, n]
    finished: torch.Tensor | None       # bool [B, n], where beams can end (given all the same: filled with False)


def _same(what, t, dtype, size, dev, name):
    """Pointer of an operand that has to be a contiguous tensor of this type and shape on this device."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != dev or tuple(t.shape) != tuple(size) or not t.is_contiguous():
        raise HolaError(f"{what}: {name} must be a contiguous {dtype} tensor of shape {tuple(size)} on {dev}")
    return t.data_ptr()


def hola_beam_select(logits: torch.Tensor, logZ: torch.Tensor, score: torch.Tensor, n: int | None = None, finished: torch.Tensor | None = None,
                     end_token: int = -1, weight: torch.Tensor | None = None, keep_slots: bool = False, out: BeamSelection | None = None,
                     status: torch.Tensor | None = None, stream=None) -> BeamSelection:
    """The `n` best continuations (None: as many as there are beams) over the beams of each sequence and the vocabulary.

    logits: fp32, bf16 or fp16 [B, W, V], a row's entries side by side; logZ: fp32 [B, W], their log-sum-exp (hola_lm_head_entropy and
    hola_token_logprobs have it); score: fp32 [B, W], the beams' log probabilities so far, -inf for none.  Candidates are ordered by
    (score - logZ + logit) * weight in 64 bits, equal ones by beam, logit and id; out.score is score - logZ + logit.  finished: bool [B, W],
    beams that have ended: one candidate each, end_token at the score they have.  weight: fp32 [B, W], positive (length-normalised keys).
    keep_slots (n = W): the best child of a beam is put at the beam's own place instead of by rank, so that hola_beam_reorder has
    least to move.  Places without a candidate: score -inf, parent and token -1.
    status: int32 [1] on the device, HOLA_FLAG_* bits are OR-ed in.  out: an earlier call's result, filled again.  stream: see HolaVerify."""
    lib = load_library()
    what = "hola_beam_select"
    if _host is not None and stream is None and out is None and getattr(logits, "is_cuda", False):
        got = _host.beam_select(_entry[what], logits, logZ, score, n, finished, end_token, weight, keep_slots, status, torch._C._cuda_getDevice(),
                                _stream_ptr(None))
        if got is not None:
            if got[0]:
                _check(lib, None, got[0], what)
            return BeamSelection(*got[1:])
    if not isinstance(logits, torch.Tensor) or logits.dtype not in _L_DTYPES or not logits.is_cuda or logits.dim() != 3:
        raise HolaError(f"{what} takes fp32, bf16 or fp16 logits [B, W, V] on a device")
    B, W, V = logits.shape
    dev = logits.device
    n = W if n is None else n
    if not 1 <= W <= HOLA_MAX_BEAMS or not 1 <= n <= HOLA_MAX_BEAMS or not 1 <= V <= 1 << 27 or (keep_slots and n != W):
        raise HolaError(f"{what}: 1 .. {HOLA_MAX_BEAMS} beams and candidates, 1 .. 2^27 entries; keep_slots with as many candidates as beams")
    if V > 1 and logits.stride(2) != 1:
        raise HolaError(f"{what}: the entries of a row must lie side by side")
    if not -1 <= end_token < V or (finished is not None and end_token < 0):
        raise HolaError(f"{what}: end_token must be -1 .. V - 1, and a token where beams are finished")
    a = hola_beam_args()
    a.B, a.W, a.V, a.n, a.l_dtype, a.end_token, a.keep_slots = B, W, V, n, _L_DTYPES[logits.dtype], end_token, bool(keep_slots)
    a.logits, a.seq_stride, a.beam_stride = logits.data_ptr(), logits.stride(0), logits.stride(1)
    a.logZ, a.score = _same(what, logZ, torch.float32, (B, W), dev, "logZ"), _same(what, score, torch.float32, (B, W), dev, "score")
    if finished is not None:
        a.finished = _same(what, finished, torch.bool, (B, W), dev, "finished")
    if weight is not None:
        a.weight = _same(what, weight, torch.float32, (B, W), dev, "weight")
    if status is not None:
        a.status_word = _same(what, status, torch.int32, (1,), dev, "status")
    ends = end_token >= 0
    if out is None:
        out = _make_on(stream, dev, lambda: BeamSelection(
            torch.empty((B, n), dtype=torch.float32, device=dev), torch.empty((B, n), dtype=torch.int32, device=dev),
            torch.empty((B, n), dtype=torch.int32, device=dev), torch.empty((B, n), dtype=torch.bool, device=dev) if ends else None))
    a.score_out = _same(what, out.score, torch.float32, (B, n), dev, "out.score")
    a.parent, a.token = (_same(what, t, torch.int32, (B, n), dev, "out") for t in (out.parent, out.token))
    if ends or out.finished is not None:                         # (where no beam can end, none has)
        a.finished_out = _same(what, out.finished, torch.bool, (B, n), dev, "out.finished")
    with torch.cuda.device(dev):
        _check(lib, None, lib.hola_beam_select(ctypes.byref(a), _stream_ptr(stream)), what)
    return out


class BeamStates:
    """States of the beams for hola_beam_reorder, laid out once: tensors [..., B, W, ...] (token histories, keys and values, page tables).
    (Some 20 us of host time a tensor: for tensors that stay where they are, not for each step.)

    axes: the axis of the sequences in each tensor (one number: in all), the beams' is the next one.  positions: for each tensor the axis that counts
    positions, of which only the first used[b] are moved, or None.  into: tensors that take the reordered states (double buffers; perhaps with
    another number of beams), None: the tensors themselves.  Tensors that are written share no byte with one another nor with what is read;
    views side by side in one buffer do not.  Keep the object alive while calls that use it are in flight."""

    def __init__(self, tensors, axes=0, positions=None, into=None):
        tensors = list(tensors)
        axes = [axes] * len(tensors) if isinstance(axes, int) else list(axes)
        positions = [None] * len(tensors) if positions is None else list(positions)
        targets = tensors if into is None else list(into)
        if not len(tensors) == len(axes) == len(positions) == len(targets) or not tensors:
            raise HolaError("BeamStates takes tensors and one axis, one position axis or None, and one target for each")
        if not all(isinstance(t, torch.Tensor) and t.layout == torch.strided for t in (*tensors, *targets)):
            raise HolaError("BeamStates takes strided tensors")
        self.tensors, self.into, self.device = tensors, targets, tensors[0].device
        first = tensors[0].shape[axes[0]:axes[0] + 2] if 0 <= axes[0] <= tensors[0].dim() - 2 else (0, 0)
        self.B, self.W = first
        self.n = targets[0].shape[axes[0] + 1] if into is not None and targets[0].dim() == tensors[0].dim() else self.W
        self.in_place = into is None
        if not 1 <= self.W <= HOLA_MAX_BEAMS or not 1 <= self.n <= HOLA_MAX_BEAMS:
            raise HolaError(f"BeamStates: 1 .. {HOLA_MAX_BEAMS} beams")
        self.states = (hola_beam_state * len(tensors))()
        for st, x, y, axis, at in zip(self.states, tensors, targets, axes, positions):
            self._lay_out(st, x, y, axis, at)
        self.address, self.count = ctypes.addressof(self.states), len(tensors)
        a = hola_reorder_args()
        a.B, a.W, a.n, a.count, a.states = self.B, self.W, self.n, self.count, self.address
        if into is not None and any(x.data_ptr() == y.data_ptr() and x.numel() for x, y in zip(tensors, targets)):
            raise HolaError("BeamStates: a target overlaps its source")
        lib = load_library()
        status = lib.hola_beam_states_check(ctypes.byref(a))
        if status == HOLA_ERR_INVALID_ARG:
            raise HolaError("BeamStates: what is written shares memory with itself, with another state or with what is read")
        _check(lib, None, status, "BeamStates")

    def _lay_out(self, st, x, y, axis, at):
        if not 0 <= axis <= x.dim() - 2 or tuple(x.shape[axis:axis + 2]) != (self.B, self.W):
            raise HolaError(f"BeamStates: every tensor must have {self.B} sequences and {self.W} beams at its axis")
        if y.dtype != x.dtype or x.device != self.device or y.device != self.device or tuple(y.shape) != (*x.shape[:axis + 1], self.n, *x.shape[axis + 2:]):
            raise HolaError("BeamStates: a target must be like its tensor, but for the number of beams")
        rest = [d for d in range(x.dim()) if d not in (axis, axis + 1)]
        if at is not None and at not in rest:
            raise HolaError("BeamStates: the positions' axis must be one besides those of sequences and beams")
        for t in (x, y):                                         # (indices that share memory)
            if any(t.shape[d] > 1 and t.stride(d) == 0 for d in range(t.dim())):
                raise HolaError("BeamStates: expanded tensors hold no states of their own")
        size, outer, closed, position = 1, [], False, 0          # what lies side by side, from the last axis on
        for d in reversed(rest):
            if x.shape[d] == 1 and d != at:
                continue
            inside = not closed and all(t.stride(d) == size or t.shape[d] == 1 for t in (x, y))
            if d == at:
                if not inside:
                    raise HolaError("BeamStates: what belongs to a position must lie side by side, and the positions as well")
                position, closed = size, True                    # (axes outside the positions' are outer ones)
                size *= x.shape[d]
            elif inside:
                size *= x.shape[d]
            else:
                closed = True
                if outer and all(s == o * n for s, o, n in ((x.stride(d), outer[-1][1], outer[-1][0]), (y.stride(d), outer[-1][2], outer[-1][0]))):
                    outer[-1] = (outer[-1][0] * x.shape[d], *outer[-1][1:])
                else:
                    outer.append((x.shape[d], x.stride(d), y.stride(d)))
        if len(outer) > 2:
            raise HolaError("BeamStates: more than two axes beside the ones that lie side by side")
        e = x.element_size()
        beams = [(t.shape[axis + 1], t.stride(axis + 1)) for t in (x, y)]
        if any(count > 1 and stride < size for count, stride in beams):
            raise HolaError("BeamStates: beams must not share memory")
        outer += [(1, 0, 0)] * (2 - len(outer))
        st.src, st.dst, st.run, st.position = x.data_ptr(), y.data_ptr(), size * e, position * e
        st.seq_stride, st.beam_stride, st.dst_seq_stride, st.dst_beam_stride = (
            t.stride(d) * e for t, d in ((x, axis), (x, axis + 1), (y, axis), (y, axis + 1)))
        for i, (count, s, to) in enumerate(outer):
            st.outer[i], st.outer_stride[i], st.dst_outer_stride[i] = count, s * e, to * e


def hola_beam_reorder(states: BeamStates, parent: torch.Tensor, used: torch.Tensor | None = None, status: torch.Tensor | None = None,
                      stream=None) -> None:
    """new[b, i] = old[b, parent[b, i]] for all states.  parent: int32 [B, n], -1 .. W - 1, rows at any distance (n columns of a wider
    selection, say); -1 leaves a place as it was.  used: int32 [B], positions that hold something (states with a positions' axis)."""
    lib = load_library()
    what = "hola_beam_reorder"
    if not isinstance(states, BeamStates):
        raise HolaError(f"{what} takes BeamStates")
    dev = states.device
    if _host is not None and dev.type == "cuda" and dev.index == (device := torch._C._cuda_getDevice()):
        got = _host.beam_reorder(_entry[what], states.address, states.count, states.B, states.W, states.n, parent, used, status, device,
                                 _stream_ptr(stream))
        if got is not None:
            if got:
                _check(lib, None, got, what)
            return
    if (not isinstance(parent, torch.Tensor) or parent.dtype != torch.int32 or parent.device != dev or parent.dim() != 2 or parent.shape[0] != states.B
            or not 1 <= parent.shape[1] <= states.n or (parent.shape[1] > 1 and parent.stride(1) != 1) or dev.type != "cuda"):
        raise HolaError(f"{what}: parent must be an int32 tensor of {states.B} rows of up to {states.n} places side by side, on the states' device")
    a = hola_reorder_args()
    a.B, a.W, a.n, a.count, a.states = states.B, states.W, parent.shape[1], states.count, states.address
    a.parent, a.parent_stride = parent.data_ptr(), parent.stride(0)
    if used is not None:
        a.used = _same(what, used, torch.int32, (states.B,), dev, "used")
    if status is not None:
        a.status_word = _same(what, status, torch.int32, (1,), dev, "status")
    with torch.cuda.device(dev):
        _check(lib, None, lib.hola_beam_reorder(ctypes.byref(a), _stream_ptr(stream)), what)


# ------------------------------------------------------------------------------------------------ embeddings
_T_DTYPES = {torch.float32: HOLA_T_F32, torch.bfloat16: HOLA_T_BF16, torch.float16: HOLA_T_F16}
_TOKENS = {torch.int32: 0, torch.int64: 1}


def _rows_apart(what, t, shape, name):
    """(pointer, distance of the rows) of a tensor [*shape, H] whose rows lie at one distance."""
    if tuple(t.shape[:-1]) != tuple(shape) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise HolaError(f"{what}: {name} must have the tokens' shape and channels side by side")
    stride, rows = None, 1
    for size, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride = s
        elif s != stride * rows:
            raise HolaError(f"{what}: the rows of {name} must lie at one distance from each other")
        rows *= size
    return t.data_ptr(), t.shape[-1] if stride is None else stride


def _ids(what, tokens):
    if not isinstance(tokens, torch.Tensor) or tokens.dtype not in _TOKENS or not tokens.is_cuda or not tokens.is_contiguous():
        raise HolaError(f"{what} takes contiguous int32 or int64 tokens on a device")


def _part(what, a, v_offset, V_global):
    if v_offset < 0 or (V_global and v_offset + a.V > V_global) or (not V_global and v_offset) or not 0 <= V_global < 2 ** 31:
        raise HolaError(f"{what}: rows v_offset .. v_offset + V - 1 must be part of the V_global rows")
    a.v_offset, a.V_global = v_offset, V_global


def hola_embed(tokens: torch.Tensor, table, scale: float = 1.0, add: torch.Tensor | None = None, w_scale: torch.Tensor | None = None,
               out: torch.Tensor | None = None, dtype: torch.dtype | None = None, v_offset: int = 0, V_global: int = 0,
               status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """add + scale * table[tokens], [..., H] for tokens [...] (int32 or int64, -1: none).

    table: fp32, bf16, fp16 [V, H], int8 [V, H] with w_scale (hola_quantize_w8) or a MixedHead.  Evaluated in fp32; dtype: of the result
    (None: of out, of add, of the table, bf16 for the quantised ones).  add: the same type, [..., H]; it may be out.  v_offset, V_global: the table
    is rows v_offset .. of a vocabulary of V_global; tokens of other parts count as none.  Not recorded for autograd: the gradient of the
    table is hola_embed_grad's or hola_embed_grad_rows', by a call of one's own.
    status: int32 [1] on the device, HOLA_FLAG_* bits are OR-ed in.  stream: see HolaVerify."""
    lib = load_library()
    what = "hola_embed"
    if _host is not None and stream is None and out is None and getattr(tokens, "is_cuda", False) and (dtype is None or dtype in _T_DTYPES):
        mixed = type(table) is MixedHead and w_scale is None and table.w_scale is not None
        got = _host.embed(_entry[what], tokens, table, ctypes.addressof(table.struct) if mixed else 0, table.V if mixed else 0, table.H if mixed else 0,
                          scale, add, table.w_scale if mixed else w_scale, -1 if dtype is None else _T_DTYPES[dtype], v_offset, V_global, status,
                          torch._C._cuda_getDevice(), _stream_ptr(None))
        if got is not None:
            if got[0]:
                _check(lib, None, got[0], what)
            return got[1]
    _ids(what, tokens)
    dev, shape = tokens.device, tokens.shape
    a = hola_embed_args()
    if isinstance(table, MixedHead):
        if w_scale is not None or table.w_scale.device != dev:
            raise HolaError(f"{what}: a MixedHead carries its own scales, on the tokens' device")
        a.V, a.H, a.t_dtype, a.wmix, a.w_scale = table.V, table.H, HOLA_T_MIXED, ctypes.addressof(table.struct), table.w_scale.data_ptr()
        own = torch.bfloat16
    else:
        if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.device != dev or (table.dtype not in _T_DTYPES and table.dtype != torch.int8):
            raise HolaError(f"{what} takes a table [V, H] of fp32, bf16, fp16 or int8 on the tokens' device, or a MixedHead")
        if (table.dtype == torch.int8) != (w_scale is not None):
            raise HolaError(f"{what}: an int8 table goes with w_scale (fp32 per row), another one without")
        if max(table.shape) >= 2 ** 31:
            raise HolaError(f"{what}: more rows or channels than 32 bits count")
        a.V, a.H = table.shape
        a.table, a.row_stride = _rows_apart(what, table, (a.V,), "table")
        a.t_dtype = HOLA_T_INT8 if w_scale is not None else _T_DTYPES[table.dtype]
        if w_scale is not None:
            a.w_scale = _same(what, w_scale, torch.float32, (a.V,), dev, "w_scale")
        own = torch.bfloat16 if w_scale is not None else table.dtype
    _part(what, a, v_offset, V_global)
    for t in (out, add):
        dtype = t.dtype if dtype is None and t is not None else dtype
    dtype = own if dtype is None else dtype
    if dtype not in _T_DTYPES or any(t is not None and (t.dtype != dtype or t.device != dev or t.shape[-1:] != (a.H,)) for t in (out, add)):
        raise HolaError(f"{what}: fp32, bf16 or fp16 results; out and add of that type, with the table's channels, on the tokens' device")
    if tokens.numel() >= 2 ** 31:
        raise HolaError(f"{what}: more tokens than 32 bits count")
    a.N, a.tokens, a.wide_tokens, a.scale, a.out_dtype = tokens.numel(), tokens.data_ptr(), _TOKENS[tokens.dtype], scale, _T_DTYPES[dtype]
    if add is not None:
        a.add, a.add_stride = _rows_apart(what, add, shape, "add")
    if out is None:
        out, = _make_on(stream, dev, lambda: (torch.empty((*shape, a.H), dtype=dtype, device=dev),))
    a.out, a.out_stride = _rows_apart(what, out, shape, "out")
    if status is not None:
        a.status_word = _same(what, status, torch.int32, (1,), dev, "status")
    if a.N:
        with torch.cuda.device(dev):
            _check(lib, None, lib.hola_embed(ctypes.byref(a), _stream_ptr(stream)), what)
    return out


@dataclass
class TokenRows:
    """The gradient of a table by rows: what hola_embed_grad_rows fills.  The first count[0] entries hold something."""
    ids: torch.Tensor        # int32 [N], the distinct tokens, rising
    rows: torch.Tensor       # [N, H]
    count: torch.Tensor      # int32 [1]


def _embed_grad_native(what, tokens, grad, V, scale, dtype, v_offset, V_global, by_rows, out, status):
    """(result or rows, ids, count) through the native helper, None where the arguments have to be made from Python."""
    if _host is None or dtype not in _T_DTYPES or not getattr(tokens, "is_cuda", False):
        return None
    ids, rows, count = (out.ids, out.rows, out.count) if type(out) is TokenRows else (None, None, None)
    got = _host.embed_grad(_entry["hola_embed_grad"], _entry["hola_embed_grad_workspace_bytes"], tokens, grad, V, scale, _T_DTYPES[dtype], v_offset,
                           V_global, by_rows, ids, rows, count, status, torch._C._cuda_getDevice(), _stream_ptr(None))
    if got is not None and got[0]:
        _check(load_library(), None, got[0], what)
    return None if got is None else got[1:]


def _embed_grad(what, tokens, grad, V, scale, v_offset, V_global, status, stream, fill):
    lib = load_library()
    _ids(what, tokens)
    dev, N = tokens.device, tokens.numel()
    if not isinstance(grad, torch.Tensor) or grad.dtype not in _T_DTYPES or grad.device != dev or grad.dim() < 1:
        raise HolaError(f"{what} takes an fp32, bf16 or fp16 gradient on the tokens' device")
    H = grad.shape[-1]
    if not 1 <= V < 2 ** 31 - 2 or not 1 <= H < 2 ** 31 or N >= 2 ** 31 - 1:
        raise HolaError(f"{what}: sizes must be positive and fit 32 bits")
    a = hola_embed_grad_args()
    a.N, a.V, a.H, a.scale = N, V, H, scale
    _part(what, a, v_offset, V_global)
    a.tokens, a.wide_tokens, a.g_dtype = tokens.data_ptr(), _TOKENS[tokens.dtype], _T_DTYPES[grad.dtype]
    a.grad, a.grad_stride = _rows_apart(what, grad, tokens.shape, "grad")
    if status is not None:
        a.status_word = _same(what, status, torch.int32, (1,), dev, "status")
    a.workspace_bytes = lib.hola_embed_grad_workspace_bytes(N, V, H)
    if a.workspace_bytes == 0:
        raise HolaError(f"{what}: at most 2^25 tokens and 2^30 rows")
    out = _make_on(stream, dev, lambda: fill(a, dev, N, H))
    workspace, = _make_on(stream, dev, lambda: (torch.empty(a.workspace_bytes, dtype=torch.uint8, device=dev),))
    a.workspace = workspace.data_ptr()
    with torch.cuda.device(dev):
        _check(lib, None, lib.hola_embed_grad(ctypes.byref(a), _stream_ptr(stream)), what)
    return out


def hola_embed_grad(tokens: torch.Tensor, grad: torch.Tensor, V: int, scale: float = 1.0, out: torch.Tensor | None = None,
                    accumulate: bool = False, dtype: torch.dtype = torch.float32, v_offset: int = 0, V_global: int = 0,
                    status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient of a table [V, H] through hola_embed: row v is scale times the sum of grad[r] over the tokens r that are v (-1: none),
    in fp32, the same bits every time.  grad: fp32, bf16 or fp16 [..., H] for tokens [...].  out: fp32, bf16 or fp16 [V, H], filled (rows of
    tokens that do not occur: zeros), or with accumulate added to.  dtype: of a fresh result.  status, stream, v_offset, V_global: as
    for hola_embed."""
    what = "hola_embed_grad"
    if accumulate and out is None:
        raise HolaError(f"{what}: accumulate needs out")
    load_library()
    if stream is None and out is None:
        got = _embed_grad_native(what, tokens, grad, V, scale, dtype, v_offset, V_global, False, None, status)
        if got is not None:
            return got[0]

    def fill(a, dev, N, H):
        if (dtype if out is None else out.dtype) not in _T_DTYPES:
            raise HolaError(f"{what}: fp32, bf16 or fp16 results")
        t = torch.empty((V, H), dtype=dtype, device=dev) if out is None else out
        if tuple(t.shape) != (V, H) or t.device != dev:
            raise HolaError(f"{what}: out must be [V, H] on the tokens' device")
        a.out, a.out_stride = _rows_apart(what, t, (V,), "out")
        a.out_dtype, a.accumulate = _T_DTYPES[t.dtype], bool(accumulate)
        return (t,)

    return _embed_grad(what, tokens, grad, V, scale, v_offset, V_global, status, stream, fill)[0]


def hola_embed_grad_rows(tokens: torch.Tensor, grad: torch.Tensor, V: int, scale: float = 1.0, out: TokenRows | None = None,
                         dtype: torch.dtype = torch.float32, v_offset: int = 0, V_global: int = 0, status: torch.Tensor | None = None,
                         stream=None) -> TokenRows:
    """The same by rows: the distinct tokens in rising order, and the gradient's row of each.  out: an earlier call's result, or buffers
    with room for as many rows as there are tokens, apart from tokens and grad and from one another; what lies behind the distinct ones
    is left as it was."""
    what = "hola_embed_grad_rows"
    load_library()
    if stream is None and (out is None or type(out) is TokenRows):
        got = _embed_grad_native(what, tokens, grad, V, scale, dtype, v_offset, V_global, True, out, status)
        if got is not None:
            return out if out is not None else TokenRows(got[1], got[0], got[2])

    def fill(a, dev, N, H):
        got = out
        if got is None:
            if dtype not in _T_DTYPES:
                raise HolaError(f"{what}: fp32, bf16 or fp16 results")
            got = TokenRows(torch.empty((N,), dtype=torch.int32, device=dev), torch.empty((N, H), dtype=dtype, device=dev),
                            torch.empty((1,), dtype=torch.int32, device=dev))
        if got.rows.dtype not in _T_DTYPES or got.rows.device != dev or tuple(got.rows.shape) != (N, H):
            raise HolaError(f"{what}: out.rows must be fp32, bf16 or fp16, a row for each token, on the tokens' device")
        a.ids_out, a.count_out = _same(what, got.ids, torch.int32, (N,), dev, "out.ids"), _same(what, got.count, torch.int32, (1,), dev, "out.count")
        a.out, a.out_stride = _rows_apart(what, got.rows, (N,), "out.rows")
        a.out_dtype = _T_DTYPES[got.rows.dtype]
        return got

    return _embed_grad(what, tokens, grad, V, scale, v_offset, V_global, status, stream, fill)


@dataclass
class VerifyOutputs:
    accept_len: torch.Tensor   # int32 [B]
    next_tok: torch.Tensor     # int32 [B]
    entropy: torch.Tensor      # fp32 [B, k+1]
    logZ: torch.Tensor         # fp32 [B, k+1]
    logits: torch.Tensor | None
    status: torch.Tensor       # uint32 as int32 [1]
    draft_entropy: torch.Tensor | None = None   # fp32 [B, k], filled when the gate looks at the draft rows


class _FieldOnDemand:
    """What VerifyOutputs has of a field that an instance lacks: _fresh_outputs leaves out what the call does not fill, and it
    is made when somebody asks.  (Without __set__, so that an instance's own tensor comes first; a __getattr__ would make
    every attribute of every outputs object dearer.)"""

    def __init__(self, name: str):
        self.name = name

    def __get__(self, out, cls=None):
        lazy = None if out is None else out.__dict__.get("_lazy")
        if lazy is None:
            if out is None and self.name == "draft_entropy":
                return None                                      # (the field's default)
            raise AttributeError(f"{cls.__name__!r} object has no attribute {self.name!r}")
        B, k, dev = lazy
        t = (torch.zeros((B, k), dtype=torch.float32, device=dev) if self.name == "draft_entropy"
             else torch.empty(B, dtype=torch.int32, device=dev))
        setattr(out, self.name, t)
        return t


for _name in ("accept_len", "next_tok", "draft_entropy"):
    setattr(VerifyOutputs, _name, _FieldOnDemand(_name))


def _fresh_outputs(ctx: "HolaVerify", B: int, k1: int, want_logits: bool, draws: bool, draft_gate: bool, stream=None) -> VerifyOutputs:
    """Outputs a call makes for itself: only the tensors that it fills are allocated (one allocation costs the host as
    much as a fifth of a call), the others when somebody asks for them.  The status word is cleared by the call
    (HOLA_ARG_CLEAR_STATUS)."""
    if stream is not None:
        return _make_on(stream, ctx._dev, lambda: _fresh_outputs(ctx, B, k1, want_logits, draws, draft_gate))
    out = VerifyOutputs.__new__(VerifyOutputs)
    dev = ctx._dev
    out._lazy = (B, k1 - 1, dev)
    if _host is not None:
        _host.outputs(out, ctx.device, B, k1, ctx.V, want_logits, draws, draft_gate)
        return out
    # (sizes one by one and empty_like: the cheapest forms, 1.7 and 1.3 us against 2.4 with a tuple)
    out.entropy = e = torch.empty(B, k1, dtype=torch.float32, device=dev)
    out.logZ = torch.empty_like(e)
    out.logits = torch.empty(B, k1, ctx.V, dtype=torch.float32, device=dev) if want_logits else None
    out.status = torch.empty(1, dtype=torch.int32, device=dev)
    if draws:
        out.accept_len = a = torch.empty(B, dtype=torch.int32, device=dev)
        out.next_tok = torch.empty_like(a)
    if draft_gate:
        out.draft_entropy = torch.empty(B, k1 - 1, dtype=torch.float32, device=dev)
    return out


class HolaVerify:
    """Owns one hola_ctx.  Methods are named after the C entry points they call.

    stream=: the call runs there, in no order with the current stream, which is the caller's to make; outputs that the call makes for
    itself belong to that stream, and may be read on the current one (behind a wait for the other) and dropped at any time."""

    def __init__(self, maxB: int, maxK: int, H: int, V: int, device: int | None = None):
        if not torch.cuda.is_available():
            raise HolaError("hola_create: no CUDA device; this library has no CPU path")
        self.lib = load_library()
        self.device = torch.cuda.current_device() if device is None else int(device)
        self._dev = torch.device("cuda", self.device)
        self.maxB, self.maxK, self.H, self.V = maxB, maxK, H, V
        self._ctx = ctypes.c_void_p()
        st = self.lib.hola_create(ctypes.byref(self._ctx), self.device, maxB, maxK, H, V)
        _check(self.lib, None, st, "hola_create")

    def close(self):
        if getattr(self, "_ctx", None) and self._ctx.value:
            self.lib.hola_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -------------------------------------------------------------------------------------------------
    def hola_plan(self, B: int, k: int, w_dtype: int = HOLA_W_BF16) -> dict:
        info = hola_plan_info()
        _check(self.lib, self._ctx, self.lib.hola_plan_ex(self._ctx, B, k, w_dtype, ctypes.byref(info)), "hola_plan_ex")
        return {n: getattr(info, n) for n, _ in info._fields_}

    def hola_set_option(self, option: int, value: int):
        _check(self.lib, self._ctx, self.lib.hola_set_option(self._ctx, int(option), int(value)), "hola_set_option")

    def hola_selftest_bounded_wait(self, limit_cycles: int = 100000, stream=None) -> tuple[int, int, int]:
        """Runs the bounded-wait self-test; returns (status word, threads that reached the end, waits that gave up)
        after synchronising the stream."""
        dev = torch.device("cuda", self.device)
        status, counters = _make_on(stream, dev, lambda: [torch.zeros(n, dtype=torch.int32, device=dev) for n in (1, 2)])
        st = self.lib.hola_selftest_bounded_wait(self._ctx, int(limit_cycles), _dptr(status), _dptr(counters),
                                                 _stream_ptr(stream))
        _check(self.lib, self._ctx, st, "hola_selftest_bounded_wait")
        (torch.cuda.current_stream() if stream is None else stream).synchronize()
        return int(status.item()), int(counters[0].item()), int(counters[1].item())

    def hola_selftest_staged_wait(self, limit_cycles: int = 100000, stream=None) -> tuple[int, int, int, int]:
        """Runs the self-test of the wait on staged rows; returns (status word, threads that reached the end, waits that gave
        up, flags that the other CTA reported) after synchronising the stream."""
        status, counters = _make_on(stream, self._dev, lambda: [torch.zeros(n, dtype=torch.int32, device=self._dev) for n in (1, 3)])
        st = self.lib.hola_selftest_staged_wait(self._ctx, int(limit_cycles), _dptr(status), _dptr(counters),
                                                _stream_ptr(stream))
        _check(self.lib, self._ctx, st, "hola_selftest_staged_wait")
        (torch.cuda.current_stream() if stream is None else stream).synchronize()
        return (int(status.item()), *counters.tolist())

    def hola_selftest_mass_wait(self, limit_cycles: int = 100000, stream=None) -> tuple[int, int, int, int, int]:
        """Runs the self-test of the wait on the other CTAs' sums; returns (status word, threads that reached the end, waits
        that gave up, flags that the first CTA reported, CTAs that all sums had reached) after synchronising the stream."""
        status, counters = _make_on(stream, self._dev, lambda: [torch.zeros(n, dtype=torch.int32, device=self._dev) for n in (1, 4)])
        st = self.lib.hola_selftest_mass_wait(self._ctx, int(limit_cycles), _dptr(status), _dptr(counters), _stream_ptr(stream))
        _check(self.lib, self._ctx, st, "hola_selftest_mass_wait")
        (torch.cuda.current_stream() if stream is None else stream).synchronize()
        return (int(status.item()), *counters.tolist())

    def hola_selftest_pace(self, stream=None) -> torch.Tensor:
        """The pace counters of launches that hold several passes, behind what is queued on the stream: zeros between calls."""
        words, = _make_on(stream, self._dev, lambda: (torch.empty(HOLA_PACE_WORDS, dtype=torch.int32, device=self._dev),))
        _check(self.lib, self._ctx, self.lib.hola_selftest_pace(self._ctx, _dptr(words), _stream_ptr(stream)), "hola_selftest_pace")
        return words

    def hola_selftest_quotient(self, t: torch.Tensor, s: torch.Tensor, stream=None) -> torch.Tensor:
        """t / s (contiguous fp32 tensors on the context's device) as the kernels divide."""
        for x in (t, s):
            if x.dtype != torch.float32 or x.device != self._dev or not x.is_contiguous() or x.numel() != t.numel():
                raise HolaError("hola_selftest_quotient takes two contiguous fp32 tensors of one size on the context's device")
        out, = _make_on(stream, self._dev, lambda: (torch.empty_like(t),))
        st = self.lib.hola_selftest_quotient(self._ctx, _dptr(t), _dptr(s), t.numel(), _dptr(out), _stream_ptr(stream))
        _check(self.lib, self._ctx, st, "hola_selftest_quotient")
        return out

    def hola_profile_begin(self, max_calls: int):
        _check(self.lib, self._ctx, self.lib.hola_profile_begin(self._ctx, max_calls), "hola_profile_begin")

    def hola_shard_call(self, which: str, args, shard, stream=None):
        """hola_shard_lm_head / hola_shard_accept / hola_shard_sample on prepared argument structs."""
        if which not in ("hola_shard_lm_head", "hola_shard_accept", "hola_shard_sample"):
            raise HolaError(f"unknown entry point {which}")
        st = getattr(self.lib, which)(self._ctx, ctypes.byref(args), ctypes.byref(shard), _stream_ptr(stream))
        _check(self.lib, self._ctx, st, which)

    def hola_host_traffic(self) -> tuple[int, int]:
        """(host-to-device, device-to-host) bytes of the last hola_verify_host call."""
        up, down = ctypes.c_ulonglong(0), ctypes.c_ulonglong(0)
        _check(self.lib, self._ctx, self.lib.hola_host_traffic(self._ctx, ctypes.byref(up), ctypes.byref(down)),
               "hola_host_traffic")
        return int(up.value), int(down.value)

    def hola_profile_end(self, stream=None) -> dict:
        a, b, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int()
        st = self.lib.hola_profile_end(self._ctx, _stream_ptr(stream), ctypes.byref(a), ctypes.byref(b), ctypes.byref(n))
        _check(self.lib, self._ctx, st, "hola_profile_end")
        return {"lm_head_ms": a.value, "accept_sample_ms": b.value, "calls": n.value}

    def _args(self, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out: VerifyOutputs, B, k,
              gate_source: int = HOLA_GATE_TARGET_ENTROPY, fallback: int = HOLA_FALLBACK_SAMPLE, w_scale=None,
              a8: bool = False, draws: bool = True):
        mixed = W_lm if isinstance(W_lm, MixedHead) else None
        if mixed is not None:
            if mixed.V != self.V or mixed.H != self.H or w_scale is not None or a8:
                raise HolaError("a MixedHead carries its own scales and takes bf16 activations; its shape must be the context's")
            W_lm, w_scale = (mixed.W8 if mixed.W8 is not None else (mixed.W4 if mixed.W4 is not None else mixed.W16)), mixed.w_scale
        if hidden.dtype != torch.bfloat16 or (mixed is None and W_lm.dtype not in (torch.bfloat16, torch.int8)):
            raise HolaError("hidden must be bfloat16, W_lm bfloat16 or int8")
        if mixed is None and (W_lm.dtype == torch.int8) != (w_scale is not None):
            raise HolaError("an int8 W_lm goes with w_scale (fp32 per vocabulary row), a bfloat16 one without")
        if draft_q is not None and draft_q.dtype not in (torch.bfloat16, torch.float32):
            raise HolaError("draft_q must be bfloat16 or float32")
        for t in (hidden, W_lm, draft_tok, draft_q, uniforms):
            if t is not None and not t.is_contiguous():
                raise HolaError("all inputs must be contiguous")
        # (plain integers into the pointer fields: a c_void_p object for each would cost as much as the call itself)
        a = hola_verify_args()
        a.B, a.k, a.H, a.V = B, k, self.H, self.V
        a.hidden = hidden.data_ptr()
        if k > 0:
            if draft_tok is not None:
                a.draft_tok = draft_tok.data_ptr()
            if draft_q is not None:
                a.draft_q = draft_q.data_ptr()
        if draft_q is not None and draft_q.dtype == torch.float32:
            a.q_dtype = HOLA_Q_F32
        if uniforms is not None:
            a.uniforms = uniforms.data_ptr()
        a.tau = float(tau)
        # (an output that is missing stays a null pointer, which the library refuses where it needs it)
        if draws:
            if (t := out.accept_len) is not None:
                a.accept_len = t.data_ptr()
            if (t := out.next_tok) is not None:
                a.next_tok = t.data_ptr()
        if (t := out.entropy) is not None:
            a.entropy = t.data_ptr()
        if (t := out.logZ) is not None:
            a.logZ = t.data_ptr()
        if out.logits is not None:
            a.logits_out = out.logits.data_ptr()
        if out.status is not None:
            a.status_word = out.status.data_ptr()
        a.gate_source, a.fallback = int(gate_source), int(fallback)
        if a.gate_source == HOLA_GATE_DRAFT_ENTROPY and out.draft_entropy is not None:
            a.draft_entropy = out.draft_entropy.data_ptr()
        # a8: True = one 8-bit plane per hidden row (W8A8); "a16" = two planes (16-bit-class activations, W8A16)
        if a8 and w_scale is None:
            raise HolaError("8-bit activation planes (a8) go with an int8 W_lm and its scales")
        if w_scale is not None:
            a.w_scale = w_scale.data_ptr()
        if mixed is not None:
            a.w_dtype, a.wmix = HOLA_W_MIXED, ctypes.addressof(mixed.struct)
        else:
            a.W_lm = W_lm.data_ptr()
            if w_scale is not None:
                a.w_dtype = HOLA_W8A16 if a8 == "a16" else (HOLA_W8A8 if a8 else HOLA_W_INT8)
        return a

    def _native(self, entry, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, draws, flags, gate_source, fallback, w_scale,
                a8, stream, bank=None, ids=None):
        """The call through the native helper: its status, or None where the arguments have to be made from Python."""
        if _host is None or self.lib is not _lib:
            return None
        wmix = 0
        if type(W_lm) is MixedHead:
            if w_scale is not None or a8 or W_lm.V != self.V or W_lm.H != self.H:
                return None
            wmix, w_scale = ctypes.addressof(W_lm.struct), W_lm.w_scale
            W_lm = W_lm.W8 if W_lm.W8 is not None else (W_lm.W4 if W_lm.W4 is not None else W_lm.W16)
        if entry in _ADAPTER_ENTRIES:                            # (the form of the call is the entry point's, whatever it is given)
            if type(bank) is not AdapterBank or bank.H != self.H or bank.V != self.V or bank.device != self._dev:
                return None
            return _host.call(_entry[entry], self._ctx.value, self.H, self.V, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out,
                              draws, flags, gate_source, fallback, w_scale, a8, wmix, _stream_ptr(stream), bank.address, ids, self.device)
        return _host.call(_entry[entry], self._ctx.value, self.H, self.V, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out,
                          draws, flags, gate_source, fallback, w_scale, a8, wmix, _stream_ptr(stream))

    def alloc_outputs(self, B: int, k: int, want_logits: bool = False, device=None) -> VerifyOutputs:
        dev = torch.device("cuda", self.device) if device is None else device
        return VerifyOutputs(
            accept_len=torch.empty(B, dtype=torch.int32, device=dev),
            next_tok=torch.empty(B, dtype=torch.int32, device=dev),
            entropy=torch.empty((B, k + 1), dtype=torch.float32, device=dev),
            logZ=torch.empty((B, k + 1), dtype=torch.float32, device=dev),
            logits=torch.empty((B, k + 1, self.V), dtype=torch.float32, device=dev) if want_logits else None,
            status=torch.zeros(1, dtype=torch.int32, device=dev),
            draft_entropy=torch.zeros((B, k), dtype=torch.float32, device=dev))

    def hola_verify(self, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out: VerifyOutputs | None = None,
                    want_logits: bool = False, stream=None, gate_source: int = HOLA_GATE_TARGET_ENTROPY,
                    fallback: int = HOLA_FALLBACK_SAMPLE, w_scale=None, a8: bool = False) -> VerifyOutputs:
        """The whole verify step on device tensors, asynchronous on the stream.  With w_scale, W_lm is the int8 form
        made by hola_quantize_w8; with a8 as well, the hidden rows are quantised on the fly and the products run on
        the 8-bit tensor-core kind."""
        fresh = not out
        if fresh:
            B, k1 = hidden.shape[:2]
            out = _fresh_outputs(self, B, k1, want_logits, True, gate_source == HOLA_GATE_DRAFT_ENTROPY, stream)
        st = self._native("hola_verify", hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, 1,
                          HOLA_ARG_CLEAR_STATUS if fresh else 0, gate_source, fallback, w_scale, a8, stream)
        if st is None:
            B, k1 = hidden.shape[:2]
            a = self._args(hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, B, k1 - 1, gate_source, fallback, w_scale, a8)
            if fresh:
                a.flags = HOLA_ARG_CLEAR_STATUS
            st = self.lib.hola_verify(self._ctx, ctypes.byref(a), _stream_ptr(stream))
        if st:
            _check(self.lib, self._ctx, st, "hola_verify")
        return out

    def hola_lm_head_entropy(self, hidden, W_lm, out: VerifyOutputs | None = None, want_logits: bool = True,
                             stream=None, w_scale=None, a8: bool = False) -> VerifyOutputs:
        fresh = not out
        if fresh:
            B, k1 = hidden.shape[:2]
            out = _fresh_outputs(self, B, k1, want_logits, False, False, stream)
        st = self._native("hola_lm_head_entropy", hidden, W_lm, None, None, None, 0.0, out, 0,
                          HOLA_ARG_CLEAR_STATUS if fresh else 0, 0, 0, w_scale, a8, stream)
        if st is None:
            B, k1 = hidden.shape[:2]
            a = self._args(hidden, W_lm, None, None, None, 0.0, out, B, k1 - 1, w_scale=w_scale, a8=a8, draws=False)
            if fresh:
                a.flags = HOLA_ARG_CLEAR_STATUS
            st = self.lib.hola_lm_head_entropy(self._ctx, ctypes.byref(a), _stream_ptr(stream))
        if st:
            _check(self.lib, self._ctx, st, "hola_lm_head_entropy")
        return out

    @staticmethod
    def _check_adapters(bank, ids):
        if not isinstance(bank, AdapterBank) or not isinstance(ids, torch.Tensor):
            raise HolaError("adapters must be an AdapterBank and adapter_ids a tensor; hola_lm_head_entropy and hola_verify take the bare head")

    def _with_adapters(self, bank: AdapterBank, ids: torch.Tensor, hidden) -> hola_adapters:
        if bank.H != self.H or bank.V != self.V or bank.device != self._dev:
            raise HolaError("the adapter bank must be made for the context's H and V, on its device")
        if ids.dtype != torch.int32 or ids.device != self._dev or tuple(ids.shape) != (hidden.shape[0],) or not ids.is_contiguous():
            raise HolaError("adapter_ids must be a contiguous int32 tensor on the context's device, one per sequence")
        st = hola_adapters.from_buffer_copy(bank.struct)
        st.ids = ids.data_ptr()
        return st

    def hola_lm_head_adapters(self, hidden, W_lm, adapters: AdapterBank, adapter_ids, out: VerifyOutputs | None = None,
                              want_logits: bool = True, stream=None, w_scale=None, a8: bool = False) -> VerifyOutputs:
        """hola_lm_head_entropy with low-rank adapters beside the head: adapter_ids int32 [B] names each sequence's slot of the
        bank, -1 the bare head."""
        self._check_adapters(adapters, adapter_ids)
        fresh = not out
        if fresh:
            B, k1 = hidden.shape[:2]
            out = _fresh_outputs(self, B, k1, want_logits, False, False, stream)
        st = self._native("hola_lm_head_adapters", hidden, W_lm, None, None, None, 0.0, out, 0, HOLA_ARG_CLEAR_STATUS if fresh else 0, 0,
                          0, w_scale, a8, stream, adapters, adapter_ids)
        if st is None:
            B, k1 = hidden.shape[:2]
            ad = self._with_adapters(adapters, adapter_ids, hidden)
            a = self._args(hidden, W_lm, None, None, None, 0.0, out, B, k1 - 1, w_scale=w_scale, a8=a8, draws=False)
            if fresh:
                a.flags = HOLA_ARG_CLEAR_STATUS
            st = self.lib.hola_lm_head_adapters(self._ctx, ctypes.byref(a), ctypes.byref(ad), _stream_ptr(stream))
        if st:
            _check(self.lib, self._ctx, st, "hola_lm_head_adapters")
        return out

    def hola_verify_adapters(self, hidden, W_lm, draft_tok, draft_q, uniforms, tau, adapters: AdapterBank, adapter_ids,
                             out: VerifyOutputs | None = None, want_logits: bool = False, stream=None,
                             gate_source: int = HOLA_GATE_TARGET_ENTROPY, fallback: int = HOLA_FALLBACK_SAMPLE, w_scale=None,
                             a8: bool = False) -> VerifyOutputs:
        """hola_verify with low-rank adapters beside the head (see hola_lm_head_adapters)."""
        self._check_adapters(adapters, adapter_ids)
        fresh = not out
        if fresh:
            B, k1 = hidden.shape[:2]
            out = _fresh_outputs(self, B, k1, want_logits, True, gate_source == HOLA_GATE_DRAFT_ENTROPY, stream)
        st = self._native("hola_verify_adapters", hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, 1,
                          HOLA_ARG_CLEAR_STATUS if fresh else 0, gate_source, fallback, w_scale, a8, stream, adapters, adapter_ids)
        if st is None:
            B, k1 = hidden.shape[:2]
            ad = self._with_adapters(adapters, adapter_ids, hidden)
            a = self._args(hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, B, k1 - 1, gate_source, fallback, w_scale, a8)
            if fresh:
                a.flags = HOLA_ARG_CLEAR_STATUS
            st = self.lib.hola_verify_adapters(self._ctx, ctypes.byref(a), ctypes.byref(ad), _stream_ptr(stream))
        if st:
            _check(self.lib, self._ctx, st, "hola_verify_adapters")
        return out

    def hola_accept_sample(self, logits, entropy, logZ, draft_tok, draft_q, uniforms, tau, stream=None) -> VerifyOutputs:
        """Steps 3-5 from given fp32 logits [B, k+1, V] and their entropy / logZ."""
        B, k = logits.shape[0], logits.shape[1] - 1

        def made():
            out = self.alloc_outputs(B, k, False)
            out.entropy.copy_(entropy)
            out.logZ.copy_(logZ)
            return out

        out = _make_on(stream, self._dev, made)
        out.logits = logits
        a = hola_verify_args()
        a.B, a.k, a.H, a.V = B, k, self.H, self.V
        a.draft_tok = _dptr(draft_tok) if k > 0 else None
        a.draft_q = _dptr(draft_q) if k > 0 else None
        a.q_dtype = HOLA_Q_F32 if (draft_q is not None and draft_q.dtype == torch.float32) else HOLA_Q_BF16
        a.uniforms, a.tau = _dptr(uniforms), float(tau)
        a.accept_len, a.next_tok = _dptr(out.accept_len), _dptr(out.next_tok)
        a.entropy, a.logZ, a.logits_out, a.status_word = _dptr(out.entropy), _dptr(out.logZ), _dptr(logits), _dptr(out.status)
        _check(self.lib, self._ctx, self.lib.hola_accept_sample(self._ctx, ctypes.byref(a), _stream_ptr(stream)),
               "hola_accept_sample")
        return out

    def hola_verify_host(self, hidden, W_lm, draft_tok, draft_q, uniforms, tau, out: VerifyOutputs | None = None,
                         stream=None, gate_source: int = HOLA_GATE_TARGET_ENTROPY,
                         fallback: int = HOLA_FALLBACK_SAMPLE, w_scale=None, a8: bool = False) -> VerifyOutputs:
        """End-to-end form: per-step inputs and all outputs are HOST tensors (pinned for async copies);
        W_lm is the resident device weight.  Returns after the stream has been synchronised."""
        B, k = hidden.shape[0], hidden.shape[1] - 1
        if not isinstance(W_lm, MixedHead) and not W_lm.is_cuda:
            raise HolaError("W_lm must be resident on the device")
        for t in (hidden, draft_tok, draft_q, uniforms):
            if t is not None and not t.is_cpu:
                raise HolaError("hola_verify_host takes host tensors for the per-step inputs")
        out = out or self.alloc_outputs(B, k, False, device=torch.device("cpu"))
        st = None
        if out.logits is None:
            st = self._native("hola_verify_host", hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, 1, 0, gate_source,
                              fallback, w_scale, a8, stream)
        if st is None:
            a = self._args(hidden, W_lm, draft_tok, draft_q, uniforms, tau, out, B, k, gate_source, fallback, w_scale, a8)
            a.logits_out = None
            st = self.lib.hola_verify_host(self._ctx, ctypes.byref(a), _stream_ptr(stream))
        _check(self.lib, self._ctx, st, "hola_verify_host")
        return out


def hola_plan_for_shape(num_sms: int, H: int, V: int, rows: int, w_dtype: int = 0) -> dict:
    """Launch geometry for a shape alone (host arithmetic; needs the library, not a device)."""
    lib = load_library()
    info = hola_plan_info()
    st = lib.hola_plan_for_shape(int(num_sms), int(H), int(V), int(rows), int(w_dtype), ctypes.byref(info))
    if st != 0:
        raise HolaError(f"hola_plan_for_shape: status {st}")
    return {n: getattr(info, n) for n, _ in hola_plan_info._fields_}


def hola_hidden_form_for_shape(num_sms: int, H: int, V: int, rows: int, w_dtype: int = 0) -> int:
    """HOLA_HIDDEN_IN_PLACE, HOLA_HIDDEN_ON_LINES or HOLA_HIDDEN_8BIT: what becomes of the hidden rows ahead of the LM-head
    launch (the last two: by a kernel of its own)."""
    form = ctypes.c_int32()
    st = load_library().hola_hidden_form_for_shape(int(num_sms), int(H), int(V), int(rows), int(w_dtype), ctypes.byref(form))
    if st != 0:
        raise HolaError(f"hola_hidden_form_for_shape: status {st}")
    return form.value


def hola_sample_plan_for_shape(num_sms: int, B: int, k: int, V: int, q_dtype: int = HOLA_Q_BF16,
                               fallback: int = HOLA_FALLBACK_SAMPLE) -> dict:
    """Form of the accept/sample kernel for a shape (host arithmetic; needs the library, not a device)."""
    lib = load_library()
    info = hola_sample_info()
    st = lib.hola_sample_plan_for_shape(int(num_sms), int(B), int(k), int(V), int(q_dtype), int(fallback), ctypes.byref(info))
    if st != 0:
        raise HolaError(f"hola_sample_plan_for_shape: status {st}")
    return {n: getattr(info, n) for n, _ in hola_sample_info._fields_}
