"""ctypes binding of libsats.so: the C ABI of include/sats.h, one Python
function per entry point with the same name.

Marshalling only: tensors are passed as device pointers, the stream defaults
to torch's current stream, and a nonzero return code raises SatsError with the
library's own message.  Every step of the computation runs in the library's
HIP kernels; there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsats.so")

SATS_OK, SATS_ERR_NULL, SATS_ERR_SHAPE, SATS_ERR_HIP, SATS_ERR_WORKSPACE, SATS_ERR_ARG = 0, -1, -2, -3, -4, -5
SATS_ERR_DEVICE = -6
SATS_K_GATE, SATS_K_UP, SATS_K_DOWN, SATS_K_INSPECT, SATS_K_DENSE = 0, 1, 2, 3, 4
SATS_K_DEC_LAYER, SATS_K_DEC_LORA_V, SATS_K_CAL_ERR, SATS_K_CAL_GATEUP, SATS_K_ROUTE_ACCUM = 5, 6, 7, 8, 9
SATS_K_LORA_V = 10
SATS_K_DEC_REDUCE = 11
SATS_K_DENSE_DOWN = 12
SATS_K_DEC_REDUCE_LORA = 13
SATS_K_ROUTE_MERGE = 14
SATS_BATCH_AUTO, SATS_BATCH_MFMA, SATS_BATCH_SPLIT, SATS_BATCH_COMPACT = 0, 1, 2, 3
SATS_SINGLE_AUTO, SATS_SINGLE_OFF = 0, 1
SATS_PATH_SINGLE_TOKEN, SATS_PATH_BATCH_MFMA, SATS_PATH_BATCH_SPLIT, SATS_PATH_BATCH_COMPACT = 1, 2, 3, 4
SATS_KV_E4M3, SATS_KV_INT8 = 17, 18


class SatsOptions(ctypes.Structure):
    """sats_options of include/sats.h."""
    _fields_ = [("batch_path", ctypes.c_int), ("single_token", ctypes.c_int), ("dec_block_cols", ctypes.c_int),
                ("lora_per_token", ctypes.c_int)]


class SatsKvCache(ctypes.Structure):
    """sats_kv_cache of include/sats.h."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_layers", ctypes.c_int64),
                ("n_pages", ctypes.c_int64), ("n_kv_heads", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("head_dim", ctypes.c_int64), ("elem_bytes", ctypes.c_int32)]


class SatsKvCache8(ctypes.Structure):
    """sats_kv_cache8 of include/sats.h."""
    _anonymous_ = ("kv",)
    _fields_ = [("kv", SatsKvCache), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("q_elem_bytes", ctypes.c_int32)]


class SatsKvBatch(ctypes.Structure):
    """sats_kv_batch of include/sats.h."""
    _fields_ = [("table", ctypes.c_void_p), ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("n_tokens", ctypes.c_int64),
                ("max_q_len", ctypes.c_int64), ("max_kv_len", ctypes.c_int64)]


class SatsKvPages(ctypes.Structure):
    """sats_kv_pages of include/sats.h."""
    _fields_ = [("table", ctypes.c_void_p), ("len", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64)]


class SatsKvPrefix(ctypes.Structure):
    """sats_kv_prefix of include/sats.h."""
    _fields_ = [("seq_start", ctypes.c_void_p), ("len", ctypes.c_void_p), ("n_groups", ctypes.c_int64),
                ("max_tokens", ctypes.c_int64), ("max_len", ctypes.c_int64), ("max_own", ctypes.c_int64)]


class SatsLogitRules(ctypes.Structure):
    """sats_logit_rules of include/sats.h."""
    _fields_ = [("seqs", ctypes.c_void_p), ("history", ctypes.c_void_p), ("history_len", ctypes.c_void_p),
                ("prompt_len", ctypes.c_void_p), ("n_seqs", ctypes.c_int64), ("history_stride", ctypes.c_int64),
                ("max_history", ctypes.c_int64), ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("bias_start", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("n_bias", ctypes.c_int64), ("masks", ctypes.c_void_p),
                ("mask_of", ctypes.c_void_p), ("n_masks", ctypes.c_int64), ("mask_stride", ctypes.c_int64)]


# exported symbols and their argument types (p = pointer, i = int64, s = stream, n = int32)
_P, _I, _S, _N, _F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
_FWD = [_P] * 8 + [_I] * 4 + [_S]
_DENSE = [_P] * 5 + [_I] * 4 + [_S]
_INSPECT = _FWD + [_P] * 4
SIGNATURES = {
    "sats_mlp_forward": (_FWD, _N),
    "sats_mlp_dense": (_DENSE, _N),
    "sats_mlp_forward_noalloc": (_FWD, _N),
    "sats_mlp_forward_f32": (_FWD, _N),
    "sats_mlp_dense_f32": (_DENSE, _N),
    "sats_mlp_forward_inspect": (_INSPECT, _N),
    "sats_mlp_forward_inspect_f32": (_INSPECT, _N),
    "sats_reserve": ([_I, _I, _I, _I, _N, _S], _N),
    "sats_device_status": ([_S], _N),
    "sats_release": ([], _N),
    "sats_last_error": ([], ctypes.c_char_p),
    "sats_timing_begin": ([_N, _N], _N),
    "sats_timing_end": ([_N, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)], _N),
    "sats_kernel_name": ([_N], ctypes.c_char_p),
    "sats_mlp_forward_lora": ([_P] * 11 + [_I, _F] + [_P] * 3 + [_I] * 4 + [_S] + [_P] * 4, _N),
    "sats_mlp_forward_lora_f32": ([_P] * 11 + [_I, _F] + [_P] * 3 + [_I] * 4 + [_S] + [_P] * 4, _N),
    "sats_route_table": ([_P] * 3 + [_I, _P, _I, _I, ctypes.c_double] + [_P] * 4 + [_S], _N),
    "sats_set_options": ([ctypes.POINTER(SatsOptions)], _N),
    "sats_query_path": ([_I, _I, _I, _N, _N, _N, ctypes.POINTER(ctypes.c_int)], _N),
    "sats_calibration_curves": ([_P] * 4 + [_I] * 3 + [_P, _I] + [_P] * 4 + [_S], _N),
    "sats_qk_norm_rope": ([_P, _I, _P, _I, _P, _P, _F, _P, _I, _P, _P, _I, _P] + [_I] * 6 + [_N, _N, _S], _N),
    "sats_qkv_append": ([_P, _I, _P, _I, _P, _I, _P, _P, _F, _P, _I, _P, _P, _I, _P, _I, _P, _I, _I, _N, _S], _N),
    "sats_paged_attention": ([_P, _I, _P, _I, _P, _I, _F, _I, _I, _P, _P, _S], _N),
    "sats_cache_extend": ([_P] * 4 + [_I, _P, _S], _N),
    "sats_cache_fork": ([_P] * 4 + [_I, _P, _S], _N),
    "sats_cache_free": ([_P] * 5 + [_I, _S], _N),
    "sats_cache_compact": ([_P] * 3 + [_S], _N),
    "sats_cache_copy": ([_P] * 3 + [_I, _S], _N),
    "sats_sample": ([_P, _N, _I, _I, _I] + [_P] * 8 + [_S], _N),
    "sats_reserve_serving": ([_I] * 5 + [_S], _N),
    "sats_prefix_attention": ([_P, _I, _P, _I, _P, _P, _I, _F, _I, _I, _P, _P, _S], _N),
    "sats_cache_read": ([_P, _I, _P, _P, _I, _P, _I, _N, _S], _N),
    "sats_adjust_logits": ([_P, _N, _I, _P, _P, _N, _I, _I, _I, _S], _N),
    "sats_reserve_prefix": ([_P, _P, _P, _I, _S], _N),
    "sats_calibrate_sats": ([_P, _I] + [_P] * 3 + [_I] * 3 + [ctypes.c_double] * 3 + [_N] + [_P] * 3 + [_S], _N),
}


class SatsError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"sats error {code}: {msg}")
        self.code = code


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libsats.so (built by paper_2607_08991_amd.build); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2607_08991_amd.build` "
                          "(the HIP library is required: there is no other implementation)")
    # Load torch's HIP runtime first so that the library binds to the same one;
    # a second copy of the runtime in the process would not see the device.
    try:
        import torch  # noqa: F401
    except ImportError:  # pragma: no cover - the library also works without torch
        pass
    lib = ctypes.CDLL(path)
    for name, (args, res) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("device tensors are required")
    if not t.is_contiguous():
        raise ValueError("contiguous tensors are required")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(rc: int):
    if rc != SATS_OK:
        raise SatsError(rc, load().sats_last_error().decode())


def _call(name, *args):
    _check(getattr(load(), name)(*args))


def sats_mlp_forward(x, token_ids, W_gate_T, W_up_T, W_down, thresholds, route_lut, out,
                     n_tokens, d, d_ff, n_layers, stream=None):
    name = "sats_mlp_forward_f32" if _is_f32(x) else "sats_mlp_forward"
    _call(name, _ptr(x), _ptr(token_ids), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down),
          _ptr(thresholds), _ptr(route_lut), _ptr(out), n_tokens, d, d_ff, n_layers, _stream(stream))


def sats_mlp_forward_noalloc(x, token_ids, W_gate_T, W_up_T, W_down, thresholds, route_lut, out,
                             n_tokens, d, d_ff, n_layers, stream=None):
    """sats_mlp_forward on the library's fixed scratch array (bf16; allocates nothing)."""
    _call("sats_mlp_forward_noalloc", _ptr(x), _ptr(token_ids), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down),
          _ptr(thresholds), _ptr(route_lut), _ptr(out), n_tokens, d, d_ff, n_layers, _stream(stream))


def sats_mlp_dense(x, W_gate_T, W_up_T, W_down, out, n_tokens, d, d_ff, n_layers, stream=None):
    name = "sats_mlp_dense_f32" if _is_f32(x) else "sats_mlp_dense"
    _call(name, _ptr(x), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down), _ptr(out), n_tokens, d, d_ff,
          n_layers, _stream(stream))


def sats_mlp_forward_inspect(x, token_ids, W_gate_T, W_up_T, W_down, thresholds, route_lut, out,
                             n_tokens, d, d_ff, n_layers, stream=None, route_out=None,
                             active_count=None, active_idx=None, layer_in=None):
    name = "sats_mlp_forward_inspect_f32" if _is_f32(x) else "sats_mlp_forward_inspect"
    _call(name, _ptr(x), _ptr(token_ids), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down),
          _ptr(thresholds), _ptr(route_lut), _ptr(out), n_tokens, d, d_ff, n_layers,
          _stream(stream), _ptr(route_out), _ptr(active_count), _ptr(active_idx), _ptr(layer_in))


def sats_mlp_forward_lora(x, token_ids, W_gate_T, W_up_T, W_down, adapters, rank, scale, thresholds, route_lut,
                          out, n_tokens, d, d_ff, n_layers, stream=None, route_out=None, active_count=None,
                          active_idx=None, layer_in=None):
    """LoRA-aware routed sparse forward; adapters = (A_gate, B_gate, A_up, B_up_T, A_down, B_down)."""
    name = "sats_mlp_forward_lora_f32" if _is_f32(x) else "sats_mlp_forward_lora"
    if len(adapters) != 6:
        raise ValueError("adapters = (A_gate, B_gate, A_up, B_up_T, A_down, B_down)")
    _call(name, _ptr(x), _ptr(token_ids), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down),
          *(_ptr(m) for m in adapters), int(rank), float(scale), _ptr(thresholds), _ptr(route_lut), _ptr(out),
          n_tokens, d, d_ff, n_layers, _stream(stream), _ptr(route_out), _ptr(active_count), _ptr(active_idx),
          _ptr(layer_in))


def sats_reserve(max_tokens, d, d_ff, n_layers, elem_bytes, stream=None):
    _call("sats_reserve", max_tokens, d, d_ff, n_layers, elem_bytes, _stream(stream))


def sats_device_status(stream=None):
    """Synchronise the stream; raise SatsError if a device-side bounded wait gave up."""
    _call("sats_device_status", _stream(stream))


def sats_release():
    _call("sats_release")


def sats_set_options(batch_path=0, single_token=0, dec_block_cols=0, lora_per_token=0):
    """Execution options of the calling thread's later forward calls (all 0: the defaults)."""
    o = SatsOptions(batch_path, single_token, dec_block_cols, lora_per_token)
    _call("sats_set_options", ctypes.byref(o))


class options:
    """Context manager: sats_set_options(**kw) inside, the defaults after."""

    def __init__(self, **kw):
        self.kw = kw

    def __enter__(self):
        sats_set_options(**self.kw)
        return self

    def __exit__(self, *exc):
        _call("sats_set_options", None)
        return False


def sats_query_path(n_tokens, d, d_ff, elem_bytes, aligned16=True, n_cus=0) -> int:
    """The SATS_PATH_* a forward call of this shape takes under the current options (host only)."""
    path = ctypes.c_int(-1)
    _call("sats_query_path", n_tokens, d, d_ff, elem_bytes, int(bool(aligned16)), n_cus, ctypes.byref(path))
    return path.value


def sats_last_error() -> str:
    return load().sats_last_error().decode()


def sats_timing_begin(kind: int, capacity: int):
    _call("sats_timing_begin", kind, capacity)


def sats_timing_end(kind: int):
    """Returns (total_ms, count) of the launches timed since sats_timing_begin."""
    ms = ctypes.c_double(0.0)
    cnt = ctypes.c_int64(0)
    _check(load().sats_timing_end(kind, ctypes.byref(ms), ctypes.byref(cnt)))
    return ms.value, cnt.value


def sats_kernel_name(kind: int) -> str:
    return load().sats_kernel_name(kind).decode()


def _is_f32(x) -> bool:
    if isinstance(x, int) or x is None:
        raise ValueError("pass a tensor for x so the element type is known, or call load() directly")
    import torch
    if x.dtype == torch.float32:
        return True
    if x.dtype == torch.bfloat16:
        return False
    raise ValueError(f"x must be bfloat16 or float32, got {x.dtype}")


def _host(a, dtype):
    import numpy as np
    return np.ascontiguousarray(a, dtype=dtype)


def sats_calibration_curves(h, W_gate_T, W_up_T, W_down, n, d, d_ff, levels, err_rows=None, stream=None):
    """SATS curves of one layer (Eq. 3 candidates at `levels`, Eq. 6 errors, sparsities).

    h and the weights are device tensors (bf16); levels is a host sequence.
    Returns host arrays (t float32, err float64, sp float64); synchronises.
    """
    import numpy as np
    lv = _host(levels, np.float64)
    t = np.zeros(len(lv), np.float32)
    err = np.zeros(len(lv), np.float64)
    sp = np.zeros(len(lv), np.float64)
    _call("sats_calibration_curves", _ptr(h), _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down), n, d, d_ff,
          lv.ctypes.data, len(lv), t.ctypes.data, err.ctypes.data, sp.ctypes.data, _ptr(err_rows),
          _stream(stream))
    return t, err, sp


def sats_calibrate_sats(x_cal, n_cal, W_gate_T, W_up_T, W_down, d, d_ff, n_layers, s_tar,
                        coarse_step=0.05, fine_step=0.005, guardrail=True, stream=None):
    """SATS thresholds of a stack (Eq. 7-10, coarse to fine, final-layer guardrail).

    Returns (thresholds float32 [n_layers], budget b*, realized sparsity S(b*)); synchronises.
    """
    import numpy as np
    ts = np.zeros(n_layers, np.float32)
    b = ctypes.c_double(0.0)
    s = ctypes.c_double(0.0)
    _call("sats_calibrate_sats", _ptr(x_cal), n_cal, _ptr(W_gate_T), _ptr(W_up_T), _ptr(W_down), d, d_ff,
          n_layers, float(s_tar), float(coarse_step), float(fine_step), int(bool(guardrail)),
          ts.ctypes.data, ctypes.addressof(b), ctypes.addressof(s), _stream(stream))
    return ts, b.value, s.value


def sats_route_table(loss_base, loss_sparse, token_ids, heldout_ids, vocab, r_tar, route_lut, scores=None,
                     stream=None):
    """Routing table of Eq. 11-14 into route_lut (device uint8 [vocab]); returns (tau*, R(tau*)).

    Synchronises.  Empty splits may be passed as None.
    """
    tau = ctypes.c_double(0.0)
    r = ctypes.c_double(0.0)
    n = 0 if token_ids is None else token_ids.numel()
    nh = 0 if heldout_ids is None else heldout_ids.numel()
    _call("sats_route_table", _ptr(loss_base), _ptr(loss_sparse), _ptr(token_ids), n, _ptr(heldout_ids), nh,
          int(vocab), float(r_tar), _ptr(route_lut), _ptr(scores), ctypes.addressof(tau), ctypes.addressof(r),
          _stream(stream))
    return tau.value, r.value


# ------------------------------------------------------------------ serving

# These calls are short enough for the binding to show, so it looks at each tensor once.

_torch = None
_raw_stream = None


def _setup():
    global _torch, _raw_stream
    import torch
    of_device = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    current = getattr(torch._C, "_cuda_getDevice", None)
    _raw_stream = ((lambda: of_device(current())) if of_device and current
                   else lambda: torch.cuda.current_stream().cuda_stream)
    _torch = torch
    return torch


def _cur_stream(stream):
    if stream is None:
        return _raw_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _elem_bytes(t) -> int:
    torch = _torch or _setup()
    dt = t.dtype
    if dt is torch.bfloat16:
        return 2
    if dt is torch.float32:
        return 4
    raise ValueError(f"bfloat16 or float32 is required, got {dt}")


def _array(t, dtype, n, name):
    """Pointer of a contiguous device tensor of this type (and of n elements in one dimension)."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise ValueError(f"{name}: {dtype} is required, got {t.dtype}")
    if n is not None and t.shape != (n,):
        raise ValueError(f"{name}: shape ({n},) is required, got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensors are required")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensors are required")
    return t.data_ptr()


def _i32(t, n, name):
    return _array(t, (_torch or _setup()).int32, n, name)


def _f32(t, n, name):
    return _array(t, (_torch or _setup()).float32, n, name)


def _heads(t, dtype, name, shape):
    """(pointer, token stride) of [tokens][heads][head_dim] rows whose heads are dense."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {dtype} {shape} is required, got {t.dtype} {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensors are required")
    n, h, d = shape
    s0, s1, s2 = t.stride()
    if (s2 != 1 and d > 1) or (s1 != d and h > 1):
        raise ValueError(f"{name}: the heads of a token must be dense")
    return t.data_ptr(), (s0 if n > 1 else h * d)


class KVCache:
    """Keys and values of every layer in pages: k, v [n_layers][n_pages][n_kv_heads][page_size][head_dim].

    In bfloat16 or float32; or in 8 bits, k and v being float8_e4m3fn or int8 codes with a scale byte a
    row (k_scale, v_scale uint8 [n_layers][n_pages][n_kv_heads][page_size]), and dtype (bfloat16 or float32)
    the type of what is appended and of queries and results.
    """

    __slots__ = ("k", "v", "k_scale", "v_scale", "dtype", "c", "ref")

    def __init__(self, k, v, k_scale=None, v_scale=None, dtype=None):
        shape = k.shape
        if len(shape) != 5 or shape != v.shape or k.dtype is not v.dtype:
            raise ValueError("k and v must be alike: [n_layers][n_pages][n_kv_heads][page_size][head_dim]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        if k_scale is None and v_scale is None:
            esz = _elem_bytes(k)
            if dtype is not None and dtype is not k.dtype:
                raise ValueError("dtype is that of k and v, or of an 8-bit cache's queries")
            self.dtype = k.dtype
            self.c = SatsKvCache(_ptr(k), _ptr(v), *shape, esz)
        else:
            torch = _torch or _setup()
            form = SATS_KV_E4M3 if k.dtype is torch.float8_e4m3fn else SATS_KV_INT8 if k.dtype is torch.int8 else None
            if form is None or k_scale is None or v_scale is None:
                raise ValueError("k and v of float8_e4m3fn or int8 have scales, k_scale and v_scale")
            if k_scale.shape != shape[:4] or v_scale.shape != shape[:4]:
                raise ValueError("k_scale and v_scale must be [n_layers][n_pages][n_kv_heads][page_size]")
            self.dtype = dtype or torch.bfloat16
            if self.dtype is not torch.bfloat16 and self.dtype is not torch.float32:
                raise ValueError(f"bfloat16 or float32 is required, got {dtype}")
            self.c = SatsKvCache8(SatsKvCache(_ptr(k), _ptr(v), *shape, form), _array(k_scale, torch.uint8, None, "k_scale"),
                                  _array(v_scale, torch.uint8, None, "v_scale"), 2 if self.dtype is torch.bfloat16 else 4)
        self.ref = ctypes.byref(self.c)


class KVBatch:
    """The new tokens of a batch of sequences (sats_kv_batch).

    table [n_seqs][max_pages], q_start [n_seqs + 1] and kv_len [n_seqs] are device
    int32; max_q_len (default: n_tokens) and max_kv_len are upper bounds.
    """

    __slots__ = ("keep", "n_tokens", "c", "ref")

    def __init__(self, table, q_start, kv_len, n_tokens, max_q_len=None, max_kv_len=None):
        n, width = _table(table)
        if max_kv_len is None:
            raise ValueError("max_kv_len is required: an upper bound of kv_len")
        self.keep = (table, q_start, kv_len)
        self.n_tokens = n_tokens
        self.c = SatsKvBatch(_i32(table, None, "table"), _i32(q_start, n + 1, "q_start"), _i32(kv_len, n, "kv_len"),
                             n, width, n_tokens, n_tokens if max_q_len is None else max_q_len, max_kv_len)
        self.ref = ctypes.byref(self.c)


class KVPages:
    """The pages' state: table [n_seqs][max_pages], len [n_seqs], refs [n_pages], device int32."""

    __slots__ = ("table", "len", "refs", "n_pages", "c", "ref")

    def __init__(self, table, len, refs):
        n, width = _table(table)
        self.table, self.len, self.refs = table, len, refs
        self.n_pages = refs.numel()
        self.c = SatsKvPages(_i32(table, None, "table"), _i32(len, n, "len"), _i32(refs, self.n_pages, "refs"), n, width)
        self.ref = ctypes.byref(self.c)


class KVPrefix:
    """Groups of a batch's sequences that share a prefix (sats_kv_prefix).

    Sequences seq_start[g] .. seq_start[g + 1] - 1 have their first len[g] tokens in common; both are device
    int32, [n_groups + 1] and [n_groups].  max_tokens (new tokens of a group), max_len (of a prefix) and max_own
    (a sequence's tokens behind its prefix) are upper bounds.
    """

    __slots__ = ("keep", "c", "ref")

    def __init__(self, seq_start, len, max_tokens, max_len, max_own):
        n = len.numel()
        self.keep = (seq_start, len)
        self.c = SatsKvPrefix(_i32(seq_start, n + 1, "seq_start"), _i32(len, n, "len"), n, max_tokens, max_len, max_own)
        self.ref = ctypes.byref(self.c)


class LogitRules:
    """Rules on n rows of logits (sats_logit_rules); every array is on the device, None where a rule is not wanted.

    history int32 [n_seqs][width] ids so far (rows may be strided), the first history_len[s] of row s = seqs[i] (i)
    for row i, from prompt_len[s] on the answer's; repetition, frequency, presence float32 [n]; bias_start int32
    [n + 1], bias_ids int32 and bias float32 [n_bias]; masks int32 [n_masks][words] (rows may be strided), a bit
    an id, mask_of int32 [n] (no mask where it is none's number).
    """

    __slots__ = ("keep", "n", "vocab_words", "c", "ref")

    def __init__(self, history=None, history_len=None, prompt_len=None, seqs=None, repetition=None, frequency=None,
                 presence=None, bias_start=None, bias_ids=None, bias=None, masks=None, mask_of=None):
        self.keep = (history, history_len, prompt_len, seqs, repetition, frequency, presence, bias_start, bias_ids, bias,
                     masks, mask_of)
        n = None  # rows, as far as the arrays say
        for t, more in ((seqs, 0), (repetition, 0), (frequency, 0), (presence, 0), (mask_of, 0), (bias_start, 1)):
            if t is not None:
                if n is not None and t.numel() - more != n:
                    raise ValueError("the rules' arrays of a number a row must have the same rows")
                n = t.numel() - more
        if history is None and any(t is not None for t in (history_len, prompt_len, repetition, frequency, presence)):
            raise ValueError("penalties need history")
        if (bias is None) != (bias_ids is None) or (bias is None) != (bias_start is None):
            raise ValueError("biases need bias_start, bias_ids and bias")
        if masks is None and mask_of is not None:
            raise ValueError("mask_of needs masks")
        hp, n_seqs, h_stride, width = _rows(history, "history")
        mp, n_masks, m_stride, words = _rows(masks, "masks")
        self.n, self.vocab_words = n, (words if masks is not None else None)
        m = 0 if bias is None else bias.numel()
        f = lambda t, name: _f32(t, n, name)  # noqa: E731
        self.c = SatsLogitRules(
            _i32(seqs, n, "seqs"), hp, _i32(history_len, n_seqs if history is not None else None, "history_len"),
            _i32(prompt_len, n_seqs if history is not None else None, "prompt_len"), n_seqs, h_stride, width,
            f(repetition, "repetition"), f(frequency, "frequency"), f(presence, "presence"),
            _i32(bias_start, None, "bias_start"), _i32(bias_ids, m if bias is not None else None, "bias_ids"),
            _f32(bias, None, "bias"), m, mp, _i32(mask_of, n, "mask_of"), n_masks, m_stride)
        self.ref = ctypes.byref(self.c)


def _rows(t, name):
    """(pointer, rows, row stride, row length) of device int32 [rows][length] with dense rows."""
    if t is None:
        return None, 0, 0, 0
    if t.dtype is not (_torch or _setup()).int32 or len(t.shape) != 2 or not t.is_cuda:
        raise ValueError(f"{name}: a device int32 tensor of two dimensions is required")
    n, m = t.shape
    s0, s1 = t.stride()
    if (m > 1 and s1 != 1) or (n > 1 and s0 < m):
        raise ValueError(f"{name}: dense rows apart from each other are required")
    return t.data_ptr(), n, (s0 if n > 1 else m), m


def _table(table):
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("table must be [n_seqs][max_pages]")
    return shape


def _of_pool(cache, pages):
    if pages.n_pages != cache.c.n_pages:
        raise ValueError("refs must have an entry for every page of the cache")


def _rope(rope):
    if rope is None:
        return None, 0, 0
    n_pos, rot = rope.shape
    return _f32(rope, None, "rope"), n_pos, rot


def sats_qk_norm_rope(q, k, rope, positions, q_out, k_out, q_norm=None, k_norm=None, eps=1e-6, interleaved=False,
                      stream=None):
    """Head norms (where weights are given) and position rotation of q and k [tokens][heads][head_dim].

    rope [n_pos][rot_dim] float32: cosines, then sines, of a position's angles (None: no rotation).
    """
    shape, dt, esz = q.shape, q.dtype, _elem_bytes(q)
    n, hq, d = shape
    hk = k.shape[1]
    qp, qs = _heads(q, dt, "q", shape)
    kp, ks = _heads(k, dt, "k", (n, hk, d))
    op, os_ = _heads(q_out, dt, "q_out", shape)
    tp, ts = _heads(k_out, dt, "k_out", (n, hk, d))
    rp, n_pos, rot = _rope(rope)
    _call("sats_qk_norm_rope", qp, qs, kp, ks, _array(q_norm, dt, d, "q_norm"), _array(k_norm, dt, d, "k_norm"), eps,
          rp, n_pos, _i32(positions, n, "positions"), op, os_, tp, ts, n, hq, hk, d, rot, int(interleaved), esz,
          _cur_stream(stream))


def sats_qkv_append(q, k, v, rope, q_out, cache, layer, batch, q_norm=None, k_norm=None, eps=1e-6, positions=None,
                    interleaved=False, stream=None):
    """sats_qk_norm_rope of a batch's tokens, with k and v appended to a layer of the cache."""
    shape, dt, c = q.shape, cache.dtype, cache.c
    n, hq, d = shape
    if n != batch.n_tokens or d != c.head_dim:
        raise ValueError("q must have the batch's tokens and the cache's head_dim")
    rows = (n, c.n_kv_heads, d)
    qp, qs = _heads(q, dt, "q", shape)
    kp, ks = _heads(k, dt, "k", rows)
    vp, vs = _heads(v, dt, "v", rows)
    op, os_ = _heads(q_out, dt, "q_out", shape)
    rp, n_pos, rot = _rope(rope)
    _call("sats_qkv_append", qp, qs, kp, ks, vp, vs, _array(q_norm, dt, d, "q_norm"), _array(k_norm, dt, d, "k_norm"),
          eps, rp, n_pos, _i32(positions, n, "positions"), op, os_, cache.ref, layer, batch.ref, hq, rot,
          int(interleaved), _cur_stream(stream))


def _attend(q, cache, batch, out, lse):
    """(pointer, token stride, heads) of q, with out and lse looked at."""
    shape, dt = q.shape, cache.dtype
    n, hq, d = shape
    if n != batch.n_tokens or d != cache.c.head_dim:
        raise ValueError("q must have the batch's tokens and the cache's head_dim")
    if out.shape != shape or out.dtype is not dt:
        raise ValueError("out must be like q")
    if lse is not None and lse.shape != (n, hq):
        raise ValueError("lse must be [n_tokens][n_q_heads]")
    qp, qs = _heads(q, dt, "q", shape)
    return qp, qs, hq


def sats_paged_attention(q, cache, layer, batch, out, scale, window=0, n_sinks=0, lse=None, stream=None):
    """Attention of a batch's new tokens over a layer of the cache (window 0: every earlier key)."""
    qp, qs, hq = _attend(q, cache, batch, out, lse)
    _call("sats_paged_attention", qp, qs, cache.ref, layer, batch.ref, hq, scale, window, n_sinks, _ptr(out),
          _f32(lse, None, "lse"), _cur_stream(stream))


def sats_prefix_attention(q, cache, layer, batch, prefix, out, scale, window=0, n_sinks=0, lse=None, stream=None):
    """sats_paged_attention for a batch whose sequences share prefixes (KVPrefix), read once for 128 rows of a group (float32: 16)."""
    qp, qs, hq = _attend(q, cache, batch, out, lse)
    _call("sats_prefix_attention", qp, qs, cache.ref, layer, batch.ref, prefix.ref, hq, scale, window, n_sinks, _ptr(out),
          _f32(lse, None, "lse"), _cur_stream(stream))


def sats_cache_read(cache, layer, batch, k_out, v_out, stream=None):
    """Keys and values of a batch's tokens, as a layer of the cache holds them, in bfloat16 or float32.

    k_out, v_out [n_tokens][n_kv_heads][head_dim] of one type (one of them may be None).
    """
    c = cache.c
    shape = (batch.n_tokens, c.n_kv_heads, c.head_dim)
    like = k_out if k_out is not None else v_out
    if like is None:
        raise ValueError("k_out or v_out is required")
    kp, ks = (None, 0) if k_out is None else _heads(k_out, like.dtype, "k_out", shape)
    vp, vs = (None, 0) if v_out is None else _heads(v_out, like.dtype, "v_out", shape)
    _call("sats_cache_read", cache.ref, layer, batch.ref, kp, ks, vp, vs, _elem_bytes(like), _cur_stream(stream))


def sats_cache_extend(cache, pages, seqs, add, status=None, stream=None):
    """Room for add[i] more tokens in sequence seqs[i] (None: i); status int32 [2]: pages missing, items left out."""
    _of_pool(cache, pages)
    n = add.numel()
    _call("sats_cache_extend", cache.ref, pages.ref, _i32(seqs, n, "seqs"), _i32(add, n, "add"), n,
          _i32(status, 2, "status"), _cur_stream(stream))


def sats_cache_fork(cache, pages, src, dst, status=None, stream=None):
    """Sequence dst[i] (empty) becomes a copy of src[i]; status as in sats_cache_extend."""
    _of_pool(cache, pages)
    n = src.numel()
    _call("sats_cache_fork", cache.ref, pages.ref, _i32(src, n, "src"), _i32(dst, n, "dst"), n,
          _i32(status, 2, "status"), _cur_stream(stream))


def sats_cache_free(cache, pages, seqs, begin=None, end=None, stream=None):
    """Gives back the pages wholly in tokens begin[i] .. end[i] - 1 (None: from 0, to the length) of seqs[i]."""
    _of_pool(cache, pages)
    n = seqs.numel()
    _call("sats_cache_free", cache.ref, pages.ref, _i32(seqs, n, "seqs"), _i32(begin, n, "begin"),
          _i32(end, n, "end"), n, _cur_stream(stream))


def sats_cache_compact(cache, pages, n_used=None, stream=None):
    """Moves the pages in use to the front of the pool; n_used (device int32 [1]): how many they are."""
    _of_pool(cache, pages)
    _call("sats_cache_compact", cache.ref, pages.ref, _i32(n_used, 1, "n_used"), _cur_stream(stream))


def sats_cache_copy(cache, src_pages, dst_pages, stream=None):
    """Contents of pages src_pages[i] to dst_pages[i], in every layer."""
    n = src_pages.numel()
    _call("sats_cache_copy", cache.ref, _i32(src_pages, n, "src_pages"), _i32(dst_pages, n, "dst_pages"), n,
          _cur_stream(stream))


def sats_sample(logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, prob=None, n_kept=None,
                stream=None):
    """The next id of each row of logits [n][vocab] (rows may be strided) from u [n]."""
    n, vocab = logits.shape
    esz = _elem_bytes(logits)
    s0, s1 = logits.stride()
    if not logits.is_cuda or (vocab > 1 and s1 != 1):
        raise ValueError("logits must be a device tensor [n][vocab] with dense rows")
    _call("sats_sample", logits.data_ptr(), esz, s0 if n > 1 else vocab, n, vocab,
          _f32(temperature, n, "temperature"), _i32(top_k, n, "top_k"), _f32(top_p, n, "top_p"),
          _f32(min_p, n, "min_p"), _f32(u, n, "u"), _i32(tokens, n, "tokens"), _f32(prob, n, "prob"),
          _i32(n_kept, n, "n_kept"), _cur_stream(stream))


def sats_adjust_logits(logits, rules, out, stream=None):
    """out = logits [n][vocab] under the rules (LogitRules); rows may be strided, out may be logits."""
    n, vocab = logits.shape
    if out.shape != logits.shape or not logits.is_cuda or not out.is_cuda:
        raise ValueError("logits and out must be device tensors [n][vocab]")
    if rules.n is not None and rules.n != n:
        raise ValueError(f"the rules are for {rules.n} rows, the logits have {n}")
    if rules.vocab_words is not None and rules.vocab_words * 32 < vocab:
        raise ValueError("masks need a bit for every id")
    (s0, s1), (o0, o1) = logits.stride(), out.stride()
    if vocab > 1 and (s1 != 1 or o1 != 1):
        raise ValueError("logits and out must have dense rows")
    _call("sats_adjust_logits", logits.data_ptr(), _elem_bytes(logits), s0 if n > 1 else vocab, rules.ref, out.data_ptr(),
          _elem_bytes(out), o0 if n > 1 else vocab, n, vocab, _cur_stream(stream))


def sats_reserve_prefix(cache, batch, prefix, n_q_heads, stream=None):
    """Scratch memory of sats_prefix_attention calls up to these sizes, ahead of stream capture."""
    _call("sats_reserve_prefix", cache.ref, batch.ref, prefix.ref, n_q_heads, _stream(stream))


def sats_reserve_serving(max_items=0, n_pages=0, max_rows=0, vocab=0, head_dim=0, stream=None):
    """Scratch memory of the serving calls, ahead of stream capture."""
    _call("sats_reserve_serving", max_items, n_pages, max_rows, vocab, head_dim, _stream(stream))
