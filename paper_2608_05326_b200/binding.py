"""ctypes binding of libqevict.so: the same entry points as include/qevict.h, plus a small convenience
class that owns the device workspace.  Argument marshalling only -- every step of the path runs in the
CUDA kernels of the library; there is no fallback of any kind."""

import ctypes as C
import operator
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqevict.so")
# QEVICT_TRACE_LIB=1 loads the tracing variant (build.build(trace=True)): the same kernels plus %globaltimer
# stamps, which qevict_kernel_timeline reads.  It is a measuring aid; numbers reported as throughput come from
# the normal library.
if os.environ.get("QEVICT_TRACE_LIB", "0") not in ("", "0"):
    LIB_PATH = os.path.join(_HERE, "libqevict_trace.so")
# QEVICT_CHECK_LIB=1 loads the checking variant (build.build(variant="check")): the same kernels with every table
# index range-checked before use and the pools poisoned with NaN at creation.
if os.environ.get("QEVICT_CHECK_LIB", "0") not in ("", "0"):
    LIB_PATH = os.path.join(_HERE, "libqevict_check.so")

QEVICT_OK = 0
QEVICT_ERR_INVALID_ARG = 1
DTYPE_FP16, DTYPE_BF16 = 0, 1
LAYOUT_PACKED, LAYOUT_PADDED = 0, 1
CODE_INT8, CODE_E4M3 = 0, 1
(QEVICT_TIER_NONE, QEVICT_TIER_OPEN, QEVICT_TIER_AGED, QEVICT_TIER_FULL, QEVICT_TIER_QUANT, QEVICT_TIER_EVICTED,
 QEVICT_TIER_SINK) = range(7)
QEVICT_RANK_CUMULATIVE, QEVICT_RANK_DECAYED, QEVICT_RANK_PNORM, QEVICT_RANK_KEYNORM = range(4)
TIER_NONE, TIER_OPEN, TIER_AGED, TIER_FULL, TIER_QUANT, TIER_EVICTED = range(6)
LEDGER_NONE, LEDGER_ACTIVE, LEDGER_DORMANT = range(3)
STATUS_NAMES = ["OK", "INVALID_ARG", "BAD_STATE", "NO_MEMORY", "UNSUPPORTED", "CUDA", "DEVICE_CHECK"]


class QEvictError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("qevict: %s (%s)" % (message, STATUS_NAMES[status] if 0 <= status < 7 else status))
        self.status = status


class qevict_config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("batch", C.c_int32), ("n_layers", C.c_int32), ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32), ("window", C.c_int32),
        ("quant_bits", C.c_int32), ("group_size", C.c_int32), ("fp_budget_windows", C.c_int32),
        ("q_budget_windows", C.c_int32), ("max_context", C.c_int32), ("rebalance_interval_hint", C.c_int32),
        ("softmax_scale", C.c_float), ("device", C.c_int32), ("sink_windows", C.c_int32), ("recent_windows", C.c_int32),
        ("rank_mode", C.c_int32), ("rank_param", C.c_float), ("one_way", C.c_int32), ("rope_base", C.c_float),
    ]


class qevict_stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in (
        "promotions", "quantizations", "reactivations", "deletions", "n_full", "n_quant", "n_aged", "n_open",
        "n_evicted", "decode_steps", "n_sink")]


class qevict_state_layout(C.Structure):
    _fields_ = [("n_window_slots", C.c_int32), ("n_fp_pages", C.c_int32), ("n_q_pages", C.c_int32), ("n_entries", C.c_int32),
                ("fp_pool_bytes", C.c_uint64), ("q_pool_bytes", C.c_uint64)]


_STATE_SCALARS = ("n_windows", "open_window", "open_fill", "n_live", "layer_prefilled", "layer_has_open", "layer_open_fill",
                  "layer_n_windows", "layer_aged")
_STATE_ARRAYS = ("tier", "ledger", "fp_page", "q_page", "importance", "event_mass", "fp_owner", "q_owner", "entries",
                 "last_mass", "fp_pool", "q_pool")


class qevict_state_view(C.Structure):
    _fields_ = ([("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in _STATE_SCALARS] +
                [("knorm_acc", C.c_float), ("counters", C.c_uint64 * 4), ("decode_steps", C.c_uint64)] +
                [(n, C.c_void_p) for n in _STATE_ARRAYS])


class qevict_prompt_args(C.Structure):
    _fields_ = ([("struct_size", C.c_uint32)] +
                [(n, C.c_int32) for n in ("device", "dtype", "layout", "n_seqs", "n_q_heads", "n_kv_heads", "head_dim",
                                          "max_q", "max_k", "causal")] + [("softmax_scale", C.c_float)] +
                [(n, C.c_int64) for n in ("total_q", "total_k")] +
                [(n, C.c_void_p) for n in ("q", "k", "v", "out", "lse", "q_bounds", "k_bounds")] +
                [(n, C.c_int64 * 3) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] + [("status", C.c_void_p)])


class qevict_kv8_cache(C.Structure):
    _fields_ = ([("struct_size", C.c_uint32)] +
                [(n, C.c_int32) for n in ("device", "dtype", "code", "n_seqs", "n_kv_heads", "head_dim", "block", "max_blocks",
                                          "n_pages")] +
                [(n, C.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "block_table",
                                           "status")])


class qevict_kv8_evict_args(C.Structure):
    _fields_ = ([("struct_size", C.c_uint32)] +
                [(n, C.c_int32) for n in ("device", "n_seqs", "max_blocks", "block", "n_pages", "budget", "sink", "recent")] +
                [(n, C.c_void_p) for n in ("table", "lens", "scores", "table_out", "lens_out", "scores_out", "kept", "freed",
                                           "n_freed")])


_lib = None

_SIGNATURES = {
    "qevict_version": (C.c_char_p, []),
    "qevict_build_flavour": (C.c_int32, []),
    "qevict_status_string": (C.c_char_p, [C.c_int]),
    "qevict_last_error": (C.c_char_p, [C.c_void_p]),
    "qevict_launch_count": (C.c_uint64, [C.c_void_p]),
    "qevict_budget_from_bytes": (C.c_int, [C.POINTER(qevict_config), C.c_uint64, C.c_double, C.POINTER(C.c_int32),
                                           C.POINTER(C.c_int32), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)]),
    "qevict_workspace_bytes": (C.c_int, [C.POINTER(qevict_config), C.POINTER(C.c_uint64)]),
    "qevict_create": (C.c_int, [C.POINTER(qevict_config), C.c_void_p, C.c_uint64, C.POINTER(C.c_void_p)]),
    "qevict_destroy": (C.c_int, [C.c_void_p]),
    "qevict_set_splits": (C.c_int, [C.c_void_p, C.c_int32]),
    "qevict_prefill_score_scratch_bytes": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(C.c_uint64)]),
    "qevict_prefill_score": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                      C.c_uint64, C.c_void_p]),
    "qevict_export_event_mass": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
    "qevict_set_kernel_timing": (C.c_int, [C.c_void_p, C.c_int32]),
    "qevict_kernel_time": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_uint64)]),
    "qevict_kernel_times": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_uint64)]),
    "qevict_kernel_timeline": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_double),
                                        C.POINTER(C.c_double), C.POINTER(C.c_int32)]),
    "qevict_prefill_assign": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
    "qevict_decode_attn": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qevict_decode_attn_host": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qevict_decode_attn_host_async": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qevict_decode_attn_noalloc": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qevict_wait_result": (C.c_int, [C.c_void_p]),
    "qevict_rebalance": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p]),
    "qevict_state_layout_of": (C.c_int, [C.c_void_p, C.POINTER(qevict_state_layout)]),
    "qevict_export_state": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(qevict_state_view)]),
    "qevict_import_state": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(qevict_state_view)]),
    "qevict_get_stats": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(qevict_stats)]),
    "qevict_check_device": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "qevict_export_tables": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32] + [C.c_void_p] * 7),
    "qevict_export_last_mass": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]),
    "qevict_export_fp_page": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]),
    "qevict_prompt_attn_scratch_bytes": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint64)]),
    "qevict_prompt_attn": (C.c_int, [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]),
    "qevict_kv8_append": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int64,
                                    C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "qevict_kv8_attn_scratch_bytes": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                                C.POINTER(C.c_uint64)]),
    "qevict_kv8_attn": (C.c_int, [C.c_void_p, C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_int32,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]),
    "qevict_kv8_evict": (C.c_int, [C.c_void_p, C.c_void_p]),
    "qevict_export_q_page": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32] + [C.c_void_p] * 5),
}


def lib():
    """The loaded shared library.  Raises if it has not been built (there is no other code path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(os.path.basename(LIB_PATH) + " is missing: run `python -m paper_2608_05326_b200.build` "
                               "(or __graft_entry__.build()) first; there is no fallback path")
        handle = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(status, handle=None):
    if status != QEVICT_OK:
        # without a handle: the calling thread's last failure of qevict_create / qevict_workspace_bytes
        msg = lib().qevict_last_error(handle).decode()
        raise QEvictError(status, msg or lib().qevict_status_string(status).decode())


def make_config(batch, n_layers, n_q_heads, n_kv_heads, head_dim, dtype, window, quant_bits, group_size,
                fp_budget_windows, q_budget_windows, max_context, rebalance_interval_hint=0, softmax_scale=0.0,
                device=0, sink_windows=0, recent_windows=0, rank_mode=0, rank_param=0.0, one_way=0, rope_base=0.0):
    dt = {"fp16": DTYPE_FP16, "bf16": DTYPE_BF16, torch.float16: DTYPE_FP16, torch.bfloat16: DTYPE_BF16}[dtype]
    return qevict_config(C.sizeof(qevict_config), batch, n_layers, n_q_heads, n_kv_heads, head_dim, dt, window,
                         quant_bits, group_size, fp_budget_windows, q_budget_windows, max_context,
                         rebalance_interval_hint, softmax_scale, device, sink_windows, recent_windows, rank_mode,
                         rank_param, int(one_way), float(rope_base))


# --- plain function wrappers, same names as the C entry points -----------------------------------------
def qevict_version():
    return lib().qevict_version().decode()


def qevict_budget_from_bytes(cfg, hist_bytes, q_frac):
    kf, kq, mf, mq = C.c_int32(), C.c_int32(), C.c_uint64(), C.c_uint64()
    _check(lib().qevict_budget_from_bytes(C.byref(cfg), int(hist_bytes), float(q_frac), C.byref(kf), C.byref(kq),
                                          C.byref(mf), C.byref(mq)))
    return kf.value, kq.value, mf.value, mq.value


def qevict_workspace_bytes(cfg):
    n = C.c_uint64()
    _check(lib().qevict_workspace_bytes(C.byref(cfg), C.byref(n)))
    return n.value


def qevict_create(cfg, device_mem_ptr, n_bytes):
    h = C.c_void_p()
    _check(lib().qevict_create(C.byref(cfg), device_mem_ptr, n_bytes, C.byref(h)))
    return h


def qevict_destroy(h):
    _check(lib().qevict_destroy(h))


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def qevict_prefill_assign(h, layer, k, v, ctx_tokens, window_scores, stream=None):
    _check(lib().qevict_prefill_assign(h, layer, _ptr(k), _ptr(v), ctx_tokens, _ptr(window_scores), _stream(stream)), h)


def qevict_decode_attn(h, layer, q, k_new, v_new, out, stream=None):
    _check(lib().qevict_decode_attn(h, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream(stream)), h)


def qevict_decode_attn_host(h, layer, q, k_new, v_new, out, stream=None):
    """q, k_new, v_new, out: HOST tensors (pinned or pageable)."""
    _check(lib().qevict_decode_attn_host(h, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream(stream)), h)


def qevict_decode_attn_host_async(h, layer, q, k_new, v_new, out, stream=None):
    """Host tensors (pinned); the caller synchronises the stream before reading `out`."""
    _check(lib().qevict_decode_attn_host_async(h, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream(stream)), h)


def qevict_decode_attn_noalloc(h, layer, q, k_new, v_new, out, stream=None):
    """qevict_decode_attn with the attention scratch in the library's built-in device array: for callers
    that must not allocate device memory.  Raises QEvictError(NO_MEMORY) if the call's scratch does not fit."""
    _check(lib().qevict_decode_attn_noalloc(h, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _stream(stream)), h)


def qevict_wait_result(h):
    """Blocks until the result of the last qevict_decode_attn_host_async call is in host memory."""
    _check(lib().qevict_wait_result(h), h)


def qevict_rebalance(h, layer, stream=None):
    _check(lib().qevict_rebalance(h, layer, _stream(stream)), h)


def qevict_state_layout_of(h):
    lay = qevict_state_layout()
    _check(lib().qevict_state_layout_of(h, C.byref(lay)), h)
    return lay


def _state_buffers(lay):
    """Host tensors of a snapshot, sized by the layout."""
    nw, i32, f32, u8 = lay.n_window_slots, torch.int32, torch.float32, torch.uint8
    return {
        "tier": torch.zeros(nw, dtype=u8), "ledger": torch.zeros(nw, dtype=u8),
        "fp_page": torch.zeros(nw, dtype=i32), "q_page": torch.zeros(nw, dtype=i32),
        "importance": torch.zeros(nw, dtype=f32), "event_mass": torch.zeros(nw, dtype=f32),
        "fp_owner": torch.zeros(lay.n_fp_pages, dtype=i32), "q_owner": torch.zeros(lay.n_q_pages, dtype=i32),
        "entries": torch.zeros((lay.n_entries, 2), dtype=i32), "last_mass": torch.zeros(lay.n_entries, dtype=f32),
        "fp_pool": torch.zeros(lay.fp_pool_bytes, dtype=u8), "q_pool": torch.zeros(lay.q_pool_bytes, dtype=u8),
    }


def _state_view(arrays):
    view = qevict_state_view()
    view.struct_size = C.sizeof(qevict_state_view)
    for n in _STATE_ARRAYS:
        t = arrays[n]
        assert not t.is_cuda and t.is_contiguous()
        setattr(view, n, t.data_ptr())
    return view


def qevict_export_state(h, layer, seq):
    """Snapshot of one unit: a dict of host tensors (tables, owner tables, work list, the unit's pages of both pools
    in the library's page layout) and scalars.  Synchronises."""
    arrays = _state_buffers(qevict_state_layout_of(h))
    view = _state_view(arrays)
    _check(lib().qevict_export_state(h, layer, seq, C.byref(view)), h)
    state = dict(arrays)
    for n in _STATE_SCALARS:
        state[n] = int(getattr(view, n))
    state["knorm_acc"] = float(view.knorm_acc)
    state["counters"] = [int(x) for x in view.counters]
    state["decode_steps"] = int(view.decode_steps)
    return state


def qevict_import_state(h, layer, seq, state):
    """Restores a unit from a snapshot made by qevict_export_state on a cache of the same configuration."""
    view = _state_view(state)
    for n in _STATE_SCALARS:
        setattr(view, n, int(state[n]))
    view.knorm_acc = float(state["knorm_acc"])
    for i in range(4):
        view.counters[i] = int(state["counters"][i])
    view.decode_steps = int(state["decode_steps"])
    _check(lib().qevict_import_state(h, layer, seq, C.byref(view)), h)


def qevict_set_splits(h, splits):
    _check(lib().qevict_set_splits(h, splits), h)


def qevict_set_kernel_timing(h, enable):
    _check(lib().qevict_set_kernel_timing(h, int(enable)), h)


def qevict_kernel_time(h):
    ms, n = C.c_double(), C.c_uint64()
    _check(lib().qevict_kernel_time(h, C.byref(ms), C.byref(n)), h)
    return ms.value, n.value


# --- calls without a cache handle: prompt attention, the 8-bit block-scaled cache ---------------------------------
# These are made once per layer and token, so what they cost on the host counts: argument structures are packed in one go
# (struct.Struct in place of a ctypes structure filled field by field), a check that passes is one expression, and the
# stream is read as a raw handle.
_DTYPES = {torch.float16: DTYPE_FP16, torch.bfloat16: DTYPE_BF16}
_CODES = {torch.int8: CODE_INT8, torch.float8_e4m3fn: CODE_E4M3}
_PROMPT_PACK = struct.Struct("@I10if2q7P12qP")
_KV8_PACK = struct.Struct("@I9i8P")
_EVICT_PACK = struct.Struct("@I8i9P")
for _pack, _cls in ((_PROMPT_PACK, qevict_prompt_args), (_KV8_PACK, qevict_kv8_cache), (_EVICT_PACK, qevict_kv8_evict_args)):
    assert _pack.size == C.sizeof(_cls), _cls

_i32, _f32, _u8 = torch.int32, torch.float32, torch.uint8


def _refuse(msg):
    raise QEvictError(QEVICT_ERR_INVALID_ARG, msg)


def _bound(x, name):
    """A size as the C side takes it: ctypes would cut one of more than 32 bits to its low ones."""
    try:
        n = operator.index(x)
    except TypeError:
        _refuse("%s must be an integer, got %r" % (name, x))
    if not -0x80000000 <= n <= 0x7fffffff:
        _refuse("%s does not fit 32 bits: %d" % (name, n))
    return n


def _want(t, name, device, dtype, shape=None):
    """Address of a tensor argument after checking what the C side cannot see: type, device, shape, contiguity."""
    try:
        if t.dtype is dtype and t.device == device and (shape is None or t.shape == shape) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor):
        _refuse("%s must be a tensor" % name)
    if t.dtype != dtype:
        _refuse("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        _refuse("%s must be on %s, got %s" % (name, device, t.device))
    if shape is not None and t.shape != torch.Size(shape):
        _refuse("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    _refuse("%s must be contiguous" % name)


def _current_stream(device):
    """Raw handle of the current stream of a device."""
    try:
        return torch._C._cuda_getCurrentRawStream(device.index)
    except AttributeError:  # a torch without that shortcut
        return torch.cuda.current_stream(device).cuda_stream


def _cuda(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse("%s must be a tensor on a CUDA device" % name)
    return t.device


def _check_stream(stream, device):
    """A stream of another device would leave the call on the current stream of the tensors' own, unordered with it."""
    if stream.device != device:
        _refuse("stream belongs to %s, the tensors to %s" % (stream.device, device))


def qevict_prompt_attn(q, k, v, cu_q=None, cu_k=None, max_q=None, max_k=None, causal=True, softmax_scale=0.0, out=None, lse=None,
                       return_lse=False, status=None, stream=None):
    """Softmax attention over whole prompts (full precision, grouped heads, causal against the end of the keys).

    Packed: q [total_q, H_q, d], k, v [total_k, H_kv, d], cu_q, cu_k int32 [n_seqs + 1] row bounds (cu_k defaults to cu_q),
    max_q, max_k bounds of the lengths (default: total_q, total_k); lse is [H_q, total_q].
    Padded: q [n_seqs, H_q, n, d], k, v [n_seqs, H_kv, m, d]; cu_q, cu_k int32 [n_seqs] lengths or None; lse is
    [n_seqs, H_q, n].
    Any strides that keep d contiguous and are multiples of 16 bytes.  Returns out, or (out, lse) with return_lse; rows
    of no sequence are not written.  No gradient is recorded.  status: int32 tensor of one element that the kernel sets to a
    nonzero code where a sequence was cut or it gave up.
    """
    if stream is not None:  # its buffers come from the allocator in that stream's order
        _check_stream(stream, _cuda(q, "q"))
        with torch.cuda.stream(stream):
            return qevict_prompt_attn(q, k, v, cu_q, cu_k, max_q, max_k, causal, softmax_scale, out, lse, return_lse, status)
    dev = _cuda(q, "q")
    dtype, shape, kshape = q.dtype, q.shape, k.shape
    if dtype not in _DTYPES:
        _refuse("q must be float16 or bfloat16")
    padded = len(shape) == 4
    sq, sk, sv = q.stride(), k.stride(), v.stride()
    if len(shape) != (4 if padded else 3) or len(kshape) != len(shape) or k.dtype is not dtype or v.dtype is not dtype or \
            k.device != dev or v.device != dev or kshape[-1] != shape[-1] or sq[-1] != 1 or sk[-1] != 1 or sv[-1] != 1:
        _refuse("q, k, v must be [tokens, heads, d] or [n_seqs, heads, tokens, d] of one type on one device, d contiguous")
    if kshape != v.shape:
        _refuse("k and v must have the same shape")
    if padded:
        n, hq, mq, d = shape
        _, hkv, mk, _ = kshape
        if kshape[0] != n:
            _refuse("q and k must have the same number of sequences")
        if (max_q is not None and max_q != mq) or (max_k is not None and max_k != mk):
            _refuse("the padded layout has its bounds in the shapes: max_q and max_k must be None")
        p_cq = 0 if cu_q is None else _want(cu_q, "cu_q", dev, _i32, (n,))
        p_ck = 0 if cu_k is None else _want(cu_k, "cu_k", dev, _i32, (n,))
        total_q = total_k = 0
        lse_shape = (n, hq, mq)
        sq, sk, sv = sq[:3], sk[:3], sv[:3]
    else:
        total_q, hq, d = shape
        total_k, hkv, _ = kshape
        if cu_q is None:
            _refuse("the packed layout needs cu_q")
        n = cu_q.numel() - 1
        if n < 0:
            _refuse("cu_q must hold n_seqs + 1 bounds")
        p_cq = _want(cu_q, "cu_q", dev, _i32, (n + 1,))
        p_ck = p_cq if cu_k is None else _want(cu_k, "cu_k", dev, _i32, (n + 1,))
        mq, mk = total_q if max_q is None else max_q, total_k if max_k is None else max_k
        lse_shape = (hq, total_q)
        sq, sk, sv = (0, sq[1], sq[0]), (0, sk[1], sk[0]), (0, sv[1], sv[0])
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != shape or out.dtype is not dtype or out.device != dev or out.stride(-1) != 1:
        _refuse("out must be like q")
    if lse is None:
        if return_lse:
            lse = q.new_empty(lse_shape, dtype=_f32)
    so = out.stride()
    so = so[:3] if padded else (0, so[1], so[0])
    try:
        args = _PROMPT_PACK.pack(
            C.sizeof(qevict_prompt_args), dev.index, _DTYPES[dtype], padded, n, hq, hkv, d, mq, mk, bool(causal), softmax_scale, total_q,
            total_k, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
            0 if lse is None else _want(lse, "lse", dev, _f32, lse_shape), p_cq, p_ck, *sq, *sk, *sv, *so,
            0 if status is None else _want(status, "status", dev, _i32, (1,)))
    except (struct.error, OverflowError) as e:
        _refuse("an argument does not fit its field (%s)" % e)
    need = C.c_uint64()
    library = lib()
    _check(library.qevict_prompt_attn_scratch_bytes(args, C.byref(need)))
    scratch = None if need.value == 0 else q.new_empty(need.value, dtype=_u8)
    _check(library.qevict_prompt_attn(args, None if scratch is None else scratch.data_ptr(), need.value, _current_stream(dev)))
    return (out, lse) if return_lse else out


def qevict_kv8_evict(block_table, lens, scores, block, n_pages, budget, sink=0, recent=0, in_place=False, stream=None):
    """Keeps the `budget` best full blocks of every sequence (the first `sink` and last `recent` always).  Returns a dict:
    block_table, lens, scores (new tensors, or the given ones with in_place), kept, freed, n_freed."""
    if stream is not None:
        _check_stream(stream, _cuda(block_table, "block_table"))
        with torch.cuda.stream(stream):
            return qevict_kv8_evict(block_table, lens, scores, block, n_pages, budget, sink, recent, in_place)
    dev = _cuda(block_table, "block_table")
    shape = block_table.shape
    if len(shape) != 2:
        _refuse("block_table must be [n_seqs, max_blocks]")
    n, mb = shape
    p_table = _want(block_table, "block_table", dev, _i32)
    p_lens = _want(lens, "lens", dev, _i32, (n,))
    p_scores = _want(scores, "scores", dev, _f32, shape)
    if in_place:
        table_out, scores_out, lens_out = block_table, scores, lens
        kept, freed = block_table.new_empty((2, n, mb)).unbind(0)
        n_freed = torch.empty_like(lens)
    else:
        table_out, kept, freed = block_table.new_empty((3, n, mb)).unbind(0)
        scores_out = torch.empty_like(scores)
        lens_out, n_freed = lens.new_empty((2, n)).unbind(0)
    try:
        args = _EVICT_PACK.pack(C.sizeof(qevict_kv8_evict_args), dev.index, n, mb, block, n_pages, budget, sink, recent, p_table, p_lens, p_scores,
                                table_out.data_ptr(), lens_out.data_ptr(), scores_out.data_ptr(), kept.data_ptr(), freed.data_ptr(),
                                n_freed.data_ptr())
    except (struct.error, OverflowError) as e:
        _refuse("an argument does not fit its field (%s)" % e)
    _check(lib().qevict_kv8_evict(args, _current_stream(dev)))
    return {"block_table": table_out, "lens": lens_out, "scores": scores_out, "kept": kept, "freed": freed, "n_freed": n_freed}


class Kv8Cache:
    """View of a cache in 8 bits with a scale for each block of tokens and KV head; the tensors stay the caller's.

    k_codes, v_codes [n_pages, H_kv, block, d] int8 or float8_e4m3fn; k_scale, v_scale [n_pages, H_kv] float32; k_tail,
    v_tail [n_seqs, H_kv, block, d] float16 or bfloat16; block_table [n_seqs, max_blocks] int32; status: optional int32
    tensor of one element that kernels set to a nonzero code when a table or length is unusable, rows were dropped or a block to
    be quantised is not finite.
    """

    def __init__(self, k_codes, v_codes, k_scale, v_scale, k_tail, v_tail, block_table, status=None):
        dev = _cuda(k_codes, "k_codes")
        code, dtype, shape, grid = k_codes.dtype, k_tail.dtype, k_codes.shape, block_table.shape
        if code not in _CODES or dtype not in _DTYPES:
            _refuse("codes must be int8 or float8_e4m3fn and tails float16 or bfloat16")
        if len(shape) != 4 or len(grid) != 2:
            _refuse("k_codes must be [n_pages, H_kv, block, d] and block_table [n_seqs, max_blocks]")
        n_pages, h_kv, block, d = shape
        n, mb = grid
        tail, scale = (n, h_kv, block, d), (n_pages, h_kv)
        self.device, self.dtype, self.n_seqs, self.max_blocks, self.block = dev, dtype, n, mb, block
        self.n_pages, self.n_kv_heads, self.head_dim = n_pages, h_kv, d
        self._view = _KV8_PACK.pack(
            C.sizeof(qevict_kv8_cache), dev.index, _DTYPES[dtype], _CODES[code], n, h_kv, d, block, mb, n_pages,
            _want(k_codes, "k_codes", dev, code), _want(v_codes, "v_codes", dev, code, shape),
            _want(k_scale, "k_scale", dev, _f32, scale), _want(v_scale, "v_scale", dev, _f32, scale),
            _want(k_tail, "k_tail", dev, dtype, tail), _want(v_tail, "v_tail", dev, dtype, tail),
            _want(block_table, "block_table", dev, _i32), 0 if status is None else _want(status, "status", dev, _i32, (1,)))
        self._tensors = (k_codes, v_codes, k_scale, v_scale, k_tail, v_tail, block_table, status)

    @classmethod
    def allocate(cls, n_pages, n_seqs, max_blocks, n_kv_heads, head_dim, block, dtype=torch.bfloat16, code=torch.int8, device="cuda"):
        """A cache with buffers of its own (an empty table; status word included): attributes k_codes, v_codes, k_scale,
        v_scale, k_tail, v_tail, block_table, status."""
        dev = torch.device(device)
        if dev.index is None:
            dev = torch.device(dev.type, torch.cuda.current_device())
        pool, tail = (n_pages, n_kv_heads, block, head_dim), (n_seqs, n_kv_heads, block, head_dim)
        t = {"k_codes": torch.zeros(pool, dtype=_u8, device=dev).view(code), "v_codes": torch.zeros(pool, dtype=_u8, device=dev).view(code),
             "k_scale": torch.ones((n_pages, n_kv_heads), device=dev), "v_scale": torch.ones((n_pages, n_kv_heads), device=dev),
             "k_tail": torch.zeros(tail, dtype=dtype, device=dev), "v_tail": torch.zeros(tail, dtype=dtype, device=dev),
             "block_table": torch.full((n_seqs, max_blocks), -1, dtype=_i32, device=dev),
             "status": torch.zeros(1, dtype=_i32, device=dev)}
        cache = cls(**t)
        for name, x in t.items():
            setattr(cache, name, x)
        return cache

    def append(self, k, v, start, cu_new=None, max_new=None, stream=None):
        """k, v [total, H_kv, d] (any strides that keep d contiguous): token i of sequence s is row cu_new[s] + i (without
        cu_new: one token each, row s) and becomes token start[s] + i.  start < 0: the sequence is left as it is.  max_new: bound
        of a sequence's tokens, which sizes the launch and beyond which tokens are dropped (default: all rows, or 1 without
        cu_new)."""
        n, dev, dtype, shape, st = self.n_seqs, self.device, self.dtype, k.shape, k.stride()
        if k.dtype is not dtype or v.dtype is not dtype or k.device != dev or v.device != dev or len(shape) != 3 or \
                shape[1] != self.n_kv_heads or shape[2] != self.head_dim:
            _refuse("k and v must be [tokens, %d, %d] %s on %s" % (self.n_kv_heads, self.head_dim, dtype, dev))
        if shape != v.shape or st != v.stride() or st[2] != 1:
            _refuse("k and v must have the same shape and strides, the last dimension contiguous")
        if stream is not None:
            _check_stream(stream, dev)
        if max_new is None:
            max_new = 1 if cu_new is None else shape[0]
        p_start = _want(start, "start", dev, _i32, (n,))
        p_cu = None if cu_new is None else _want(cu_new, "cu_new", dev, _i32, (n + 1,))
        _check(lib().qevict_kv8_append(self._view, k.data_ptr(), v.data_ptr(), st[0], st[1], shape[0], p_start, p_cu, _bound(max_new, "max_new"),
                                       _current_stream(dev) if stream is None else stream.cuda_stream))

    def attn(self, q, lens, max_len=None, scores=None, scores_out=None, softmax_scale=0.0, out=None, return_lse=False, stream=None):
        """Attention of one token per sequence, q [n_seqs, H_q, d], over the first lens[s] tokens of each.  Returns out, or
        (out[, lse][, scores_out]): scores [n_seqs, max_blocks] plus the probability mass of every block, in a new tensor
        or in scores_out (which may be scores).  max_len: bound of lens (default: what the table can hold).  No gradient
        is recorded."""
        if stream is not None:
            _check_stream(stream, self.device)
            with torch.cuda.stream(stream):
                return self.attn(q, lens, max_len, scores, scores_out, softmax_scale, out, return_lse)
        n, dev, dtype, shape = self.n_seqs, self.device, self.dtype, q.shape
        if len(shape) != 3 or shape[0] != n or shape[2] != self.head_dim:
            _refuse("q must be [%d, H_q, %d]" % (n, self.head_dim))
        p_q, hq = _want(q, "q", dev, dtype), shape[1]
        p_lens = _want(lens, "lens", dev, _i32, (n,))
        max_len = self.max_blocks * self.block if max_len is None else _bound(max_len, "max_len")
        grid = (n, self.max_blocks)
        p_in = p_so = None
        if scores is not None:
            p_in = _want(scores, "scores", dev, _f32, grid)
            if scores_out is None:
                scores_out = torch.empty_like(scores)
        if scores_out is not None:
            p_so = _want(scores_out, "scores_out", dev, _f32, grid)
        if out is None:
            out = torch.empty_like(q)
            p_out = out.data_ptr()
        else:
            p_out = _want(out, "out", dev, dtype, shape)
        lse = q.new_empty((n, hq), dtype=_f32) if return_lse else None
        need, view, library = C.c_uint64(), self._view, lib()
        _check(library.qevict_kv8_attn_scratch_bytes(view, hq, max_len, p_so is not None, C.byref(need)))
        scratch = q.new_empty(need.value, dtype=_u8)
        _check(library.qevict_kv8_attn(view, hq, softmax_scale, p_q, p_lens, max_len, p_out, None if lse is None else lse.data_ptr(),
                                       p_in, p_so, scratch.data_ptr(), need.value, _current_stream(dev)))
        if lse is None:
            return out if scores_out is None else (out, scores_out)
        return (out, lse) if scores_out is None else (out, lse, scores_out)


KERNEL_NAMES = ("append", "decode_attn", "combine", "route", "migrate")


def qevict_kernel_times(h):
    ms = (C.c_double * len(KERNEL_NAMES))()
    n = (C.c_uint64 * len(KERNEL_NAMES))()
    _check(lib().qevict_kernel_times(h, ms, n), h)
    return {name: (ms[i], n[i]) for i, name in enumerate(KERNEL_NAMES)}


def qevict_kernel_timeline(h, max_records=2560):
    kid = (C.c_int32 * max_records)()
    t0 = (C.c_double * max_records)()
    t1 = (C.c_double * max_records)()
    n = C.c_int32(0)
    _check(lib().qevict_kernel_timeline(h, max_records, kid, t0, t1, C.byref(n)), h)
    return [(KERNEL_NAMES[kid[i]] if 0 <= kid[i] < len(KERNEL_NAMES) else "k%d" % kid[i], t0[i], t1[i]) for i in range(n.value)]


def qevict_get_stats(h, layer=-1):
    st = qevict_stats()
    _check(lib().qevict_get_stats(h, layer, C.byref(st)), h)
    return {n: getattr(st, n) for n, _ in qevict_stats._fields_}


def qevict_check_device(h):
    """Synchronises; raises QEvictError(DEVICE_CHECK) if a kernel recorded a failed check, else returns 0."""
    code = C.c_int32(0)
    _check(lib().qevict_check_device(h, C.byref(code)), h)
    return code.value


def qevict_launch_count(h):
    return lib().qevict_launch_count(h)


class QEvictCache:
    """A cache handle together with the torch-allocated device workspace it lives in."""

    def __init__(self, cfg):
        self.cfg = cfg
        self.device = torch.device("cuda", cfg.device)
        self.torch_dtype = torch.float16 if cfg.dtype == DTYPE_FP16 else torch.bfloat16
        self.n_bytes = qevict_workspace_bytes(cfg)
        self.workspace = torch.empty(self.n_bytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        self.handle = qevict_create(cfg, C.c_void_p(base), self.n_bytes)
        self.max_windows = cfg.max_context // cfg.window

    def close(self):
        if self.handle is not None:
            torch.cuda.synchronize(self.device)
            qevict_destroy(self.handle)
            self.handle = None
            self.workspace = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the hot path -----------------------------------------------------------------------------
    def prefill_assign(self, layer, k, v, window_scores, stream=None):
        assert k.is_cuda and k.is_contiguous() and v.is_contiguous() and k.dtype == self.torch_dtype
        assert window_scores.dtype == torch.float32 and window_scores.is_contiguous()
        qevict_prefill_assign(self.handle, layer, k, v, k.shape[-2], window_scores, stream)

    def prefill_score(self, k, q_obs, stream=None):
        """k [batch, H_kv, ctx, d], q_obs [batch, n_obs, H_q, d] (device) -> window scores [batch, ctx / W] float32."""
        n_obs, ctx = q_obs.shape[1], k.shape[-2]
        need = C.c_uint64()
        _check(lib().qevict_prefill_score_scratch_bytes(self.handle, n_obs, ctx, C.byref(need)), self.handle)
        scratch = torch.empty(need.value, dtype=torch.uint8, device=self.device)
        scores = torch.empty((k.shape[0], ctx // self.cfg.window), dtype=torch.float32, device=self.device)
        _check(lib().qevict_prefill_score(self.handle, _ptr(k), _ptr(q_obs), n_obs, ctx, _ptr(scores), _ptr(scratch),
                                          need.value, _stream(stream)), self.handle)
        return scores

    def decode_attn(self, layer, q, k_new=None, v_new=None, out=None, stream=None):
        assert q.is_cuda and q.is_contiguous() and q.dtype == self.torch_dtype
        if out is None:
            out = torch.empty_like(q)
        qevict_decode_attn(self.handle, layer, q, k_new, v_new, out, stream)
        return out

    def decode_attn_host(self, layer, q, k_new, v_new, out, stream=None):
        qevict_decode_attn_host(self.handle, layer, q, k_new, v_new, out, stream)
        return out

    def decode_attn_host_async(self, layer, q, k_new, v_new, out, stream=None):
        qevict_decode_attn_host_async(self.handle, layer, q, k_new, v_new, out, stream)

    def wait_result(self):
        qevict_wait_result(self.handle)

    def rebalance(self, layer, stream=None):
        qevict_rebalance(self.handle, layer, stream)

    def set_splits(self, splits):
        qevict_set_splits(self.handle, splits)

    def set_kernel_timing(self, enable):
        qevict_set_kernel_timing(self.handle, enable)

    def kernel_time(self):
        """(summed milliseconds, launches) of the attention kernel since the last call."""
        return qevict_kernel_time(self.handle)

    def kernel_times(self):
        """{kernel name: (summed milliseconds, launches)} since the last call."""
        return qevict_kernel_times(self.handle)

    def kernel_timeline(self, max_records=2560):
        """[(kernel name, start, end)] of the launches since the last call (first 512 API calls), oldest first, in
        microseconds from the first start; tracing library only (QEVICT_TRACE_LIB=1)."""
        return qevict_kernel_timeline(self.handle, max_records)

    def stats(self, layer=-1):
        return qevict_get_stats(self.handle, layer)

    def launch_count(self):
        return qevict_launch_count(self.handle)

    def check_device(self):
        return qevict_check_device(self.handle)

    # -- exports (parity checks, snapshots) -------------------------------------------------------
    def export_state(self, layer, seq):
        return qevict_export_state(self.handle, layer, seq)

    def import_state(self, layer, seq, state):
        qevict_import_state(self.handle, layer, seq, state)

    def export_tables(self, layer, seq):
        n = self.max_windows
        dev = self.device
        out = {
            "n_windows": torch.zeros(1, dtype=torch.int32, device=dev),
            "tier": torch.zeros(n, dtype=torch.uint8, device=dev),
            "ledger": torch.zeros(n, dtype=torch.uint8, device=dev),
            "fp_page": torch.zeros(n, dtype=torch.int32, device=dev),
            "q_page": torch.zeros(n, dtype=torch.int32, device=dev),
            "importance": torch.zeros(n, dtype=torch.float32, device=dev),
        }
        _check(lib().qevict_export_tables(self.handle, layer, seq, _ptr(out["n_windows"]), _ptr(out["tier"]),
                                          _ptr(out["ledger"]), _ptr(out["fp_page"]), _ptr(out["q_page"]),
                                          _ptr(out["importance"]), _stream(None)), self.handle)
        return {k: v.cpu() for k, v in out.items()}

    def export_last_mass(self, layer, seq):
        m = torch.zeros(self.max_windows, dtype=torch.float32, device=self.device)
        _check(lib().qevict_export_last_mass(self.handle, layer, seq, _ptr(m), _stream(None)), self.handle)
        return m.cpu()

    def export_event_mass(self, layer, seq):
        m = torch.zeros(self.max_windows, dtype=torch.float32, device=self.device)
        _check(lib().qevict_export_event_mass(self.handle, layer, seq, _ptr(m), _stream(None)), self.handle)
        return m.cpu()

    def export_fp_page(self, layer, seq, page):
        c = self.cfg
        k = torch.empty((c.n_kv_heads, c.window, c.head_dim), dtype=self.torch_dtype, device=self.device)
        v = torch.empty_like(k)
        _check(lib().qevict_export_fp_page(self.handle, layer, seq, page, _ptr(k), _ptr(v), _stream(None)), self.handle)
        return k.cpu(), v.cpu()

    def export_q_page(self, layer, seq, page):
        c = self.cfg
        g = c.group_size
        kc = torch.empty((c.n_kv_heads, c.window, c.head_dim), dtype=torch.uint8, device=self.device)
        vc = torch.empty_like(kc)
        kp = torch.empty((c.n_kv_heads, c.window // g, c.head_dim, 2), dtype=self.torch_dtype, device=self.device)
        vp = torch.empty((c.n_kv_heads, c.window, c.head_dim // g, 2), dtype=self.torch_dtype, device=self.device)
        _check(lib().qevict_export_q_page(self.handle, layer, seq, page, _ptr(kc), _ptr(kp), _ptr(vc), _ptr(vp),
                                          _stream(None)), self.handle)
        return kc.cpu(), kp.cpu(), vc.cpu(), vp.cpu()
