"""ctypes binding of libdynts.so: argument marshalling only.

Every function has the name and the argument order of its C counterpart in include/dynts.h.
Tensor arguments may be torch tensors (their data_ptr() is passed), integers (raw addresses) or
None.  Nothing here computes: every step of the path runs in the library's CUDA kernels.  If
the library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdynts.so")

DYNTS_OK = 0
DYNTS_ERR_INVALID_ARG = 1
DYNTS_ERR_OOM = 2
DYNTS_ERR_CAPACITY = 3
DYNTS_ERR_BUDGET = 4
DYNTS_ERR_STATE = 5
DYNTS_ERR_CUDA = 6
DYNTS_ERR_DEVICE = 7
DYNTS_BF16 = 0
DYNTS_FP32 = 1
DYNTS_BF16_KV8 = 2
DYNTS_SCORE_ATTENTION = 0
DYNTS_SCORE_EXTERNAL = 1
DYNTS_ROPE_ADJACENT = 1
DYNTS_ROPE_ROUND_ROBIN = 2

_STATUS_NAMES = {
    0: "DYNTS_OK", 1: "DYNTS_ERR_INVALID_ARG", 2: "DYNTS_ERR_OOM", 3: "DYNTS_ERR_CAPACITY",
    4: "DYNTS_ERR_BUDGET", 5: "DYNTS_ERR_STATE", 6: "DYNTS_ERR_CUDA", 7: "DYNTS_ERR_DEVICE",
}


class DyntsError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class dynts_config_t(C.Structure):
    _fields_ = [
        ("layers", C.c_int), ("batch", C.c_int), ("q_heads", C.c_int), ("kv_heads", C.c_int),
        ("head_dim", C.c_int), ("budget", C.c_int), ("window", C.c_int), ("evict_interval", C.c_int),
        ("capacity", C.c_int), ("dtype", C.c_int),
        ("seq_budgets", C.POINTER(C.c_int)),
        ("storage", C.c_void_p), ("storage_bytes", C.c_size_t), ("stream", C.c_void_p),
    ]


class dynts_extend_opts_t(C.Structure):
    _fields_ = [
        ("softcap", C.c_float), ("slopes", C.c_void_p), ("window", C.c_int), ("prefix", C.c_void_p), ("s_new", C.c_void_p),
        ("mass", C.c_void_p), ("stage", C.c_int), ("q_stride", C.c_longlong), ("k_stride", C.c_longlong), ("v_stride", C.c_longlong),
    ]


if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python paper_2601_18383_b200/build.py` "
        "(there is no CPU fallback)")

lib = C.CDLL(LIB_PATH)

_P = C.c_void_p
_sigs = {
    "dynts_cache_create": (_P, [C.c_int] * 5),
    "dynts_cache_set_shape": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, C.c_int]),
    "dynts_cache_bytes": (C.c_size_t, [C.POINTER(dynts_config_t)]),
    "dynts_cache_create_ex": (C.c_int, [C.POINTER(dynts_config_t), C.POINTER(_P)]),
    "dynts_cache_destroy": (None, [_P]),
    "dynts_cache_set_stream": (C.c_int, [_P, _P]),
    "dynts_prefill": (C.c_int, [_P, _P, _P, C.c_int, C.c_int]),
    "dynts_prefill_attn": (C.c_int, [_P, _P, _P, _P, _P, C.c_int, C.c_int]),
    "dynts_prompt_attn": (C.c_int, [_P, _P, _P, _P, _P, C.c_int]),
    "dynts_prefill_attn_layer": (C.c_int, [_P, C.c_int, _P, _P, _P, _P, C.c_int, C.c_int]),
    "dynts_cache_refresh_lengths": (C.c_int, [_P]),
    "dynts_prefill_seq": (C.c_int, [_P, C.c_int, _P, _P, C.c_int, C.c_int]),
    "dynts_decode_attn": (C.c_int, [_P, _P, _P, _P, _P, _P]),
    "dynts_decode_attn_layer": (C.c_int, [_P, C.c_int, _P, _P, _P, _P, _P]),
    "dynts_decode_attn_host": (C.c_int, [_P, _P, _P, _P, _P]),
    "dynts_evict": (C.c_int, [_P, C.c_int]),
    "dynts_evict_global": (C.c_int, [_P, C.c_int]),
    "dynts_aggregate_scores": (C.c_int, [_P, _P]),
    "dynts_evict_ex": (C.c_int, [_P, C.POINTER(C.c_int)]),
    "dynts_evict_noalloc": (C.c_int, [_P, _P, _P, _P] + [C.c_int] * 8 + [_P]),
    "dynts_evict_noalloc_status": (C.c_int, [_P]),
    "dynts_seq_reset": (C.c_int, [_P, C.c_int]),
    "dynts_cache_len": (C.c_int, [_P, C.c_int]),
    "dynts_cache_capacity": (C.c_int, [_P]),
    "dynts_cache_scores": (_P, [_P]),
    "dynts_cache_export": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, _P, _P, _P, _P, C.POINTER(C.c_int)]),
    "dynts_cache_import": (C.c_int, [_P, C.c_int, C.c_int, C.c_int, _P, _P, _P, _P, C.c_int, C.c_int]),
    "dynts_poll_error": (C.c_int, [_P]),
    "dynts_synchronize": (C.c_int, [_P]),
    "dynts_cache_set_launch": (C.c_int, [_P, C.c_int, C.c_int]),
    "dynts_cache_set_evict_launch": (C.c_int, [_P, C.c_int]),
    "dynts_cache_set_wait_limit": (C.c_int, [_P, C.c_uint]),
    "dynts_debug_drop_tile_load": (C.c_int, [_P, C.c_int]),
    "dynts_cache_launch_count": (C.c_longlong, [_P]),
    "dynts_cache_set_score_source": (C.c_int, [_P, C.c_int]),
    "dynts_cache_set_kv_scale": (C.c_int, [_P, C.c_float, C.c_float]),
    "dynts_append_scores": (C.c_int, [_P, _P]),
    "dynts_evict_at_budget": (C.c_int, [_P, C.c_int, C.c_double]),
    "dynts_predictor_mlp_scratch_bytes": (C.c_size_t, [C.c_int, C.c_int]),
    "dynts_predictor_mlp": (C.c_int, [_P] * 7 + [C.c_int, C.c_int, C.c_int, _P, C.c_size_t, _P, _P]),
    "dynts_extend_scratch_bytes": (C.c_size_t, [_P, _P, C.c_int]),
    "dynts_extend_attn": (C.c_int, [_P] * 6 + [C.POINTER(dynts_extend_opts_t), _P, C.c_size_t]),
    "dynts_extend_attn_layer": (C.c_int, [_P, C.c_int] + [_P] * 5 + [C.POINTER(dynts_extend_opts_t), _P, C.c_size_t]),
    "dynts_extend_commit": (C.c_int, [_P, _P]),
    "dynts_rope": (C.c_int, [_P] * 5 + [C.c_int] * 6 + [_P, C.c_int, C.c_double, C.c_int, _P, _P]),
    "dynts_evict_stats": (C.c_int, [_P, C.POINTER(C.c_longlong), C.POINTER(C.c_longlong)]),
    "dynts_last_error": (C.c_char_p, []),
    "dynts_version": (C.c_char_p, []),
}
for _name, (_res, _args) in _sigs.items():
    _fn = getattr(lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):          # numpy array (host buffers)
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)}")


def dynts_last_error() -> str:
    return lib.dynts_last_error().decode()


def dynts_version() -> str:
    return lib.dynts_version().decode()


def _check(status: int) -> int:
    if status != DYNTS_OK:
        raise DyntsError(status, dynts_last_error())
    return status


def dynts_cache_create(layers, kv_heads, head_dim, budget, window):
    h = lib.dynts_cache_create(layers, kv_heads, head_dim, budget, window)
    if not h:
        raise DyntsError(DYNTS_ERR_INVALID_ARG, dynts_last_error())
    return h


def dynts_cache_set_shape(c, batch, q_heads, dtype, evict_interval):
    return _check(lib.dynts_cache_set_shape(c, batch, q_heads, dtype, evict_interval))


def make_config(layers, batch, q_heads, kv_heads, head_dim, budget, window, evict_interval, dtype=DYNTS_BF16,
                capacity=0, seq_budgets: Optional[Sequence[int]] = None, storage=None, storage_bytes=0, stream=None):
    cfg = dynts_config_t()
    cfg.layers, cfg.batch, cfg.q_heads, cfg.kv_heads, cfg.head_dim = layers, batch, q_heads, kv_heads, head_dim
    cfg.budget, cfg.window, cfg.evict_interval, cfg.capacity, cfg.dtype = budget, window, evict_interval, capacity, dtype
    if seq_budgets is not None:
        arr = (C.c_int * len(seq_budgets))(*[int(x) for x in seq_budgets])
        cfg._keep = arr
        cfg.seq_budgets = C.cast(arr, C.POINTER(C.c_int))
    cfg.storage = _ptr(storage)
    cfg.storage_bytes = storage_bytes
    cfg.stream = stream
    return cfg


def dynts_cache_bytes(cfg: dynts_config_t) -> int:
    return lib.dynts_cache_bytes(C.byref(cfg))


def dynts_cache_create_ex(cfg: dynts_config_t):
    out = _P()
    _check(lib.dynts_cache_create_ex(C.byref(cfg), C.byref(out)))
    return out.value


def dynts_cache_destroy(c):
    lib.dynts_cache_destroy(c)


def dynts_cache_set_stream(c, stream):
    return _check(lib.dynts_cache_set_stream(c, stream))


def dynts_prefill(c, k, v, n_tokens, n_pinned):
    return _check(lib.dynts_prefill(c, _ptr(k), _ptr(v), n_tokens, n_pinned))


def dynts_prefill_attn(c, q, k, v, out, n_tokens, n_pinned):
    return _check(lib.dynts_prefill_attn(c, _ptr(q), _ptr(k), _ptr(v), _ptr(out), n_tokens, n_pinned))


def dynts_prefill_attn_layer(c, layer, q, k, v, out, n_tokens, n_pinned):
    return _check(lib.dynts_prefill_attn_layer(c, layer, _ptr(q), _ptr(k), _ptr(v), _ptr(out), n_tokens, n_pinned))


def dynts_cache_refresh_lengths(c):
    return _check(lib.dynts_cache_refresh_lengths(c))


def dynts_prompt_attn(c, q, k, v, out, n_tokens):
    return _check(lib.dynts_prompt_attn(c, _ptr(q), _ptr(k), _ptr(v), _ptr(out), n_tokens))


def dynts_prefill_seq(c, seq, k, v, n_tokens, n_pinned):
    return _check(lib.dynts_prefill_seq(c, seq, _ptr(k), _ptr(v), n_tokens, n_pinned))


def dynts_decode_attn(c, q, k_new, v_new, out, scores=None):
    return _check(lib.dynts_decode_attn(c, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(scores)))


def dynts_decode_attn_layer(c, layer, q, k_new, v_new, out, scores=None):
    return _check(lib.dynts_decode_attn_layer(c, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(scores)))


def dynts_decode_attn_host(c, q, k_new, v_new, out):
    return _check(lib.dynts_decode_attn_host(c, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out)))


def dynts_evict(c, budget=0):
    return _check(lib.dynts_evict(c, budget))


def dynts_evict_global(c, budget=0):
    return _check(lib.dynts_evict_global(c, budget))


def dynts_aggregate_scores(c, agg):
    return _check(lib.dynts_aggregate_scores(c, _ptr(agg)))


def dynts_evict_ex(c, seq_targets: Sequence[int]):
    arr = (C.c_int * len(seq_targets))(*[int(x) for x in seq_targets])
    return _check(lib.dynts_evict_ex(c, arr))


def dynts_evict_noalloc(K, V, pos, score, n_slabs, head_dim, dtype, capacity, n_rows, n_pinned, window, target,
                        stream=None):
    """In-place eviction of caller-owned slabs without any allocation (see include/dynts.h)."""
    return _check(lib.dynts_evict_noalloc(_ptr(K), _ptr(V), _ptr(pos), _ptr(score), n_slabs, head_dim, dtype,
                                          capacity, n_rows, n_pinned, window, target, stream))


def dynts_evict_noalloc_status(stream=None):
    """Waits for the stream; raises if the last allocation-free eviction recorded a device-side check."""
    return _check(lib.dynts_evict_noalloc_status(stream))


def dynts_seq_reset(c, seq):
    return _check(lib.dynts_seq_reset(c, seq))


def dynts_cache_len(c, seq=0) -> int:
    return lib.dynts_cache_len(c, seq)


def dynts_cache_capacity(c) -> int:
    return lib.dynts_cache_capacity(c)


def dynts_cache_scores(c) -> Optional[int]:
    return lib.dynts_cache_scores(c)


def dynts_cache_export(c, layer, seq, head, K, V, pos, score) -> int:
    n = C.c_int(0)
    _check(lib.dynts_cache_export(c, layer, seq, head, _ptr(K), _ptr(V), _ptr(pos), _ptr(score), C.byref(n)))
    return n.value


def dynts_cache_import(c, layer, seq, head, K, V, pos, score, n, n_pinned):
    return _check(lib.dynts_cache_import(c, layer, seq, head, _ptr(K), _ptr(V), _ptr(pos), _ptr(score), n, n_pinned))


def dynts_poll_error(c):
    return _check(lib.dynts_poll_error(c))


def dynts_synchronize(c):
    return _check(lib.dynts_synchronize(c))


def dynts_cache_set_launch(c, cluster=0, variant=0):
    return _check(lib.dynts_cache_set_launch(c, cluster, variant))


def dynts_cache_set_wait_limit(c, polls):
    return _check(lib.dynts_cache_set_wait_limit(c, polls))


def dynts_debug_drop_tile_load(c, item):
    return _check(lib.dynts_debug_drop_tile_load(c, item))


def dynts_cache_set_evict_launch(c, split=0):
    return _check(lib.dynts_cache_set_evict_launch(c, split))


def dynts_cache_set_score_source(c, source):
    return _check(lib.dynts_cache_set_score_source(c, source))


def dynts_cache_set_kv_scale(c, k_scale, v_scale):
    return _check(lib.dynts_cache_set_kv_scale(c, float(k_scale), float(v_scale)))


def dynts_append_scores(c, s_new):
    return _check(lib.dynts_append_scores(c, _ptr(s_new)))


def dynts_evict_at_budget(c, budget_B, ratio):
    return _check(lib.dynts_evict_at_budget(c, budget_B, ratio))


def dynts_predictor_mlp_scratch_bytes(d, batch) -> int:
    return lib.dynts_predictor_mlp_scratch_bytes(d, batch)


def dynts_predictor_mlp(h, W1, b1, W2, b2, W3, b3, d, batch, activation, scratch, scratch_bytes, scores, stream=None):
    return _check(lib.dynts_predictor_mlp(_ptr(h), _ptr(W1), _ptr(b1), _ptr(W2), _ptr(b2), _ptr(W3), _ptr(b3), d, batch,
                                          activation, _ptr(scratch), scratch_bytes, _ptr(scores), stream))


def _host_ints(x):
    """(address, keep-alive) of host int32 values: a CPU int32 tensor or array as it is, else a copy of a sequence."""
    if hasattr(x, "data_ptr"):
        if x.dtype is not _torch().torch.int32 or x.is_cuda or x.dim() != 1 or not x.is_contiguous():
            _invalid("host counts must be a contiguous int32 tensor on the CPU, or a sequence of ints")
        return x.data_ptr(), x
    if hasattr(x, "ctypes") and str(x.dtype) == "int32" and x.ndim == 1 and x.flags["C_CONTIGUOUS"]:
        return x.ctypes.data, x
    values = [int(v) for v in x]
    if values and not (-2 ** 31 <= min(values) and max(values) < 2 ** 31):  # (ctypes would cut them)
        _invalid("host counts must fit 32 bits")
    arr = (C.c_int * len(values))(*values)
    return C.addressof(arr), arr


class _Torch:
    """torch, and its current device and stream as plain integers (without a Python object for each call, where torch has that:
    the operators below take a few microseconds on the GPU)."""

    def __init__(self):
        import torch
        self.torch = torch
        self.int32, self.float32 = torch.int32, torch.float32
        self.dtypes = {torch.bfloat16: DYNTS_BF16, torch.float32: DYNTS_FP32}
        self.device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)


_torch_state = None


def _torch():
    global _torch_state
    if _torch_state is None:
        _torch_state = _Torch()
    return _torch_state


def dynts_extend_scratch_bytes(c, n_new, n_layers) -> int:
    p, keep = _host_ints(n_new)
    return lib.dynts_extend_scratch_bytes(c, p, n_layers)


def dynts_extend_attn(c, q, k_new, v_new, out, n_new, opts, scratch, scratch_bytes):
    p, keep = _host_ints(n_new)
    return _check(lib.dynts_extend_attn(c, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), p, C.byref(opts) if opts is not None else None,
                                        _ptr(scratch), scratch_bytes))


def dynts_extend_attn_layer(c, layer, q, k_new, v_new, out, n_new, opts, scratch, scratch_bytes):
    p, keep = _host_ints(n_new)
    return _check(lib.dynts_extend_attn_layer(c, layer, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(out), p,
                                              C.byref(opts) if opts is not None else None, _ptr(scratch), scratch_bytes))


def dynts_extend_commit(c, n_accept):
    p, keep = _host_ints(n_accept)
    return _check(lib.dynts_extend_commit(c, p))


def dynts_rope(q, k, pos, q_out, k_out, n_tokens, q_heads, kv_heads, head_dim, rot_dim, n_axes, sections, flags, theta, dtype, strides=None,
               stream=None):
    sec = (C.c_int * n_axes)(*sections) if sections is not None else None
    st = (C.c_longlong * 4)(*strides) if strides is not None else None
    return _check(lib.dynts_rope(_ptr(q), _ptr(k), _ptr(pos), _ptr(q_out), _ptr(k_out), n_tokens, q_heads, kv_heads, head_dim, rot_dim,
                                 n_axes, sec, flags, theta, dtype, st, stream))


def _invalid(message):
    raise DyntsError(DYNTS_ERR_INVALID_ARG, message)


def rope(q, k, positions, q_out=None, k_out=None, theta=10000.0, sections=None, rot_dim=None, adjacent=False, round_robin=False):
    """dynts_rope on torch tensors: q [n, Hq, d], k [n, Hkv, d] or None, positions int32 [n] or [axes, n].  The outputs are new
    tensors unless given (q_out=q, k_out=k: in place).  Rows of a token are contiguous, tokens may be strided.  Runs on torch's
    current stream of q's device.  rot_dim: by default what the sections hold, all of d without them.  Returns (q_out, k_out)."""
    t = _torch()
    if q_out is None:
        q_out = t.torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = t.torch.empty(k.shape, dtype=k.dtype, device=k.device)
    dt, dev, shape = q.dtype, q.get_device(), q.shape
    dtype = t.dtypes.get(dt)
    if dtype is None:
        _invalid("q must be bf16 or fp32")
    fits = len(shape) == 3 and dev >= 0 and q_out.dtype is dt and q_out.get_device() == dev and q_out.shape == shape
    strided = not (q.is_contiguous() and q_out.is_contiguous())
    hkv, k_ptr, k_out_ptr = 0, None, None
    if k is not None:
        k_shape = k.shape
        fits = (fits and len(k_shape) == 3 and k.dtype is dt and k.get_device() == dev and k_out.dtype is dt and k_out.get_device() == dev and
                k_out.shape == k_shape and k_shape[0] == shape[0] and k_shape[2] == shape[2])
        strided = strided or not (k.is_contiguous() and k_out.is_contiguous())
        k_ptr, k_out_ptr = k.data_ptr(), k_out.data_ptr()
    if not fits:
        _invalid("q, k and the outputs must be CUDA tensors [n, heads, d] of one type on one device")
    n, hq, d = shape
    if k is not None:
        hkv = k_shape[1]
    st = sec = None
    if strided:
        for z in (q, q_out) if k is None else (q, q_out, k, k_out):
            if z.stride(2) != 1 or (z.shape[1] > 1 and z.stride(1) != d) or (n > 1 and z.stride(0) < z.shape[1] * d):
                _invalid("the heads of a token must be contiguous and the tokens in order")
        if n > 1:
            st = (C.c_longlong * 4)(q.stride(0), 0 if k is None else k.stride(0), q_out.stride(0), 0 if k is None else k_out.stride(0))
    shape = positions.shape
    axes = 1 if len(shape) == 1 else shape[0]
    if positions.get_device() != dev or positions.dtype is not t.int32 or not positions.is_contiguous():
        _invalid("positions must be a contiguous int32 tensor on q's device")
    if len(shape) not in (1, 2) or shape[-1] != n or (sections is not None and len(sections) != axes):
        _invalid("positions are [n] or [axes, n], with a section for each axis")
    if sections is not None:
        if axes > 1:
            sec = (C.c_int * axes)(*sections)
        elif rot_dim is not None and 2 * sections[0] != rot_dim:
            _invalid("the section of one axis holds all pairs")
    if rot_dim is None:
        rot_dim = d if sections is None else 2 * sum(sections)
    if rot_dim > d or (sections is not None and any(not 0 <= x <= d for x in sections)):  # (also what ctypes would cut)
        _invalid("the sections and rot_dim must lie within d")
    flags = (DYNTS_ROPE_ADJACENT if adjacent else 0) | (DYNTS_ROPE_ROUND_ROBIN if round_robin else 0)
    args = (q.data_ptr(), k_ptr, positions.data_ptr(), q_out.data_ptr(), k_out_ptr, n, hq, hkv, d, rot_dim, axes, sec, flags, theta, dtype, st,
            t.stream(dev))
    if t.device() == dev:
        _check(lib.dynts_rope(*args))
    else:
        with t.torch.cuda.device(dev):
            _check(lib.dynts_rope(*args))
    return q_out, k_out


def dynts_evict_stats(c):
    """(rows scanned, rows moved) of the most recent eviction."""
    a, b = C.c_longlong(0), C.c_longlong(0)
    _check(lib.dynts_evict_stats(c, C.byref(a), C.byref(b)))
    return a.value, b.value


def dynts_cache_launch_count(c) -> int:
    return lib.dynts_cache_launch_count(c)


class Cache:
    """Convenience holder: takes the cache's device storage from PyTorch and keeps it alive.

    It only forwards to the functions above."""

    def __init__(self, layers, batch, q_heads, kv_heads, head_dim, budget, window, evict_interval,
                 dtype="bf16", seq_budgets=None, capacity=0, device="cuda:0"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.dtype_name = dtype
        self.torch_dtype = {"bf16": torch.bfloat16, "fp32": torch.float32, "bf16_kv8": torch.bfloat16}[dtype]   # q, k, v, out
        self.slab_dtype = torch.uint8 if dtype == "bf16_kv8" else self.torch_dtype   # rows as exported (E4M3 codes)
        self.layers, self.batch, self.q_heads, self.kv_heads, self.head_dim = layers, batch, q_heads, kv_heads, head_dim
        cfg = make_config(layers, batch, q_heads, kv_heads, head_dim, budget, window, evict_interval,
                          {"bf16": DYNTS_BF16, "fp32": DYNTS_FP32, "bf16_kv8": DYNTS_BF16_KV8}[dtype], capacity, seq_budgets)
        nbytes = dynts_cache_bytes(cfg)
        if nbytes == 0:
            raise DyntsError(DYNTS_ERR_INVALID_ARG, "invalid cache configuration")
        with torch.cuda.device(self.device):
            self.storage = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.storage.data_ptr()
            cfg.storage = (base + 255) // 256 * 256
            cfg.storage_bytes = nbytes
            cfg.stream = self._stream = torch.cuda.current_stream(self.device).cuda_stream
            self.handle = dynts_cache_create_ex(cfg)
        self.nbytes = nbytes
        self.capacity = dynts_cache_capacity(self.handle)
        self.device_index = self.storage.get_device()
        self.mass_shape = (layers, batch, kv_heads, self.capacity)
        self._scratch = []        # scratch of the chunk calls; outgrown pieces are kept for the work and graphs that still use them
        self._scratch_ptr, self._scratch_bytes = None, 0

    def close(self):
        if getattr(self, "handle", None):
            dynts_cache_destroy(self.handle)
            self.handle = None
            self.storage = None
            self._scratch = []
            self._scratch_ptr, self._scratch_bytes = None, 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, k, v, n_pinned=None):
        T = k.shape[-2]
        return dynts_prefill(self.handle, k, v, T, T if n_pinned is None else n_pinned)

    def prefill_attn(self, q, k, v, out, n_pinned=None):
        T = k.shape[-2]
        return dynts_prefill_attn(self.handle, q, k, v, out, T, T if n_pinned is None else n_pinned)

    def prefill_attn_layer(self, layer, q, k, v, out, n_pinned=None):
        T = k.shape[-2]
        return dynts_prefill_attn_layer(self.handle, layer, q, k, v, out, T, T if n_pinned is None else n_pinned)

    def refresh_lengths(self):
        return dynts_cache_refresh_lengths(self.handle)

    def prompt_attn(self, q, k, v, out):
        return dynts_prompt_attn(self.handle, q, k, v, out, k.shape[-2])

    def prefill_seq(self, seq, k, v, n_pinned=None):
        T = k.shape[-2]
        return dynts_prefill_seq(self.handle, seq, k, v, T, T if n_pinned is None else n_pinned)

    def decode_attn(self, q, k_new, v_new, out, scores=None):
        return dynts_decode_attn(self.handle, q, k_new, v_new, out, scores)

    def decode_attn_layer(self, layer, q, k_new, v_new, out, scores=None):
        return dynts_decode_attn_layer(self.handle, layer, q, k_new, v_new, out, scores)

    def decode_attn_host(self, q, k_new, v_new, out):
        return dynts_decode_attn_host(self.handle, q, k_new, v_new, out)

    def _extend(self, layer, q, k, v, out, n_new, s_new, mass, softcap, slopes, window, prefix, stage):
        t = _torch()
        counts, keep_n = _host_ints(n_new)
        listed = n_new.tolist() if hasattr(n_new, "tolist") else n_new
        if len(listed) != self.batch:
            _invalid("n_new needs a count for each sequence")
        total = sum(listed)
        dt, dev = self.torch_dtype, self.device_index
        if layer is None:
            wide, narrow = (self.layers, total, self.q_heads, self.head_dim), (self.layers, total, self.kv_heads, self.head_dim)
        else:
            wide, narrow = (total, self.q_heads, self.head_dim), (total, self.kv_heads, self.head_dim)
        if not (q.dtype is dt and k.dtype is dt and v.dtype is dt and out.dtype is dt and q.get_device() == dev and k.get_device() == dev and
                v.get_device() == dev and out.get_device() == dev and q.shape == wide and k.shape == narrow and v.shape == narrow and out.shape == wide):
            _invalid(f"q, k, v and out must be {dt} tensors on cuda:{dev}, here {wide} and {narrow} by n_new")
        if not out.is_contiguous():
            _invalid("out must be contiguous")
        strides = (0, 0, 0) if q.is_contiguous() and k.is_contiguous() and v.is_contiguous() else tuple(self._token_stride(x, total) for x in (q, k, v))
        for x, shape in ((s_new, (total,)), (mass, self.mass_shape), (slopes, (self.q_heads,))):
            if x is not None and (x.dtype is not t.float32 or x.get_device() != dev or x.shape != shape or not x.is_contiguous()):
                _invalid(f"s_new, mass and slopes must be contiguous fp32 tensors on cuda:{dev} (here: {shape})")
        prefixes = None
        if prefix is not None:
            if len(prefix) != self.batch:
                _invalid("prefix needs a count for each sequence")
            prefixes, keep_p = _host_ints(prefix)
        if not 0 <= window < 2 ** 31:
            _invalid("window must be an int of 32 bits, not negative")
        opts = dynts_extend_opts_t(softcap, None if slopes is None else slopes.data_ptr(), window, prefixes, None if s_new is None else s_new.data_ptr(),
                                   None if mass is None else mass.data_ptr(), 1 if stage else 0, *strides)
        need = lib.dynts_extend_scratch_bytes(self.handle, counts, self.layers if layer is None else 1)
        if need > self._scratch_bytes:
            # (a piece is never given back before the cache: the stream and captured graphs may still use it.  It comes from the
            # allocator's memory of the stream that will use it: another stream's may still be busy with what lay there.)
            with t.torch.cuda.stream(self.torch_stream()):
                self._scratch.append(t.torch.empty(max(need, 2 * self._scratch_bytes), dtype=t.torch.uint8, device=self.device))
            self._scratch_ptr, self._scratch_bytes = self._scratch[-1].data_ptr(), self._scratch[-1].numel()
        args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), counts, C.byref(opts), self._scratch_ptr, self._scratch_bytes)
        if t.device() != dev:
            with t.torch.cuda.device(dev):
                return self._extend_call(layer, args)
        return self._extend_call(layer, args)

    def torch_stream(self):
        """The stream the cache works on, as a torch stream."""
        cuda = self.torch.cuda
        return cuda.ExternalStream(self._stream, device=self.device) if self._stream else cuda.default_stream(self.device)

    def _token_stride(self, x, total):
        """Elements from one token of a strided q, k or v to the next."""
        heads, d = x.shape[-2], self.head_dim
        step = x.stride(-3) if total > 1 else heads * d
        if x.numel() and (x.stride(-1) != 1 or (heads > 1 and x.stride(-2) != d) or step < heads * d or
                          (x.dim() == 4 and self.layers > 1 and x.stride(0) != total * step)):
            _invalid("the heads of a token must be contiguous, the tokens in order and the layers adjoining")
        return step

    def _extend_call(self, layer, args):
        if layer is None:
            return _check(lib.dynts_extend_attn(self.handle, *args))
        return _check(lib.dynts_extend_attn_layer(self.handle, layer, *args))

    def extend_attn(self, q, k, v, out, n_new, s_new=None, mass=None, softcap=0.0, slopes=None, window=0, prefix=None, stage=False):
        """A chunk of n_new[b] tokens per sequence for all layers: q, out [L, n_total, Hq, d], k, v [L, n_total, Hkv, d]."""
        return self._extend(None, q, k, v, out, n_new, s_new, mass, softcap, slopes, window, prefix, stage)

    def extend_attn_layer(self, layer, q, k, v, out, n_new, s_new=None, mass=None, softcap=0.0, slopes=None, window=0, prefix=None,
                          stage=False):
        return self._extend(int(layer), q, k, v, out, n_new, s_new, mass, softcap, slopes, window, prefix, stage)

    def extend_commit(self, n_accept):
        if len(n_accept) != self.batch:
            _invalid("n_accept needs a count for each sequence")
        return dynts_extend_commit(self.handle, n_accept)

    def evict(self, budget=0):
        return dynts_evict(self.handle, budget)

    def evict_global(self, budget=0):
        return dynts_evict_global(self.handle, budget)

    def aggregate_scores(self, agg):
        return dynts_aggregate_scores(self.handle, agg)

    def evict_ex(self, targets):
        return dynts_evict_ex(self.handle, targets)

    def seq_reset(self, seq):
        return dynts_seq_reset(self.handle, seq)

    def len(self, seq=0):
        return dynts_cache_len(self.handle, seq)

    def set_launch(self, cluster=0, variant=0):
        return dynts_cache_set_launch(self.handle, cluster, variant)

    def set_wait_limit(self, polls):
        return dynts_cache_set_wait_limit(self.handle, polls)

    def debug_drop_tile_load(self, item):
        return dynts_debug_drop_tile_load(self.handle, item)

    def set_evict_launch(self, split=0):
        return dynts_cache_set_evict_launch(self.handle, split)

    def set_stream(self, stream):
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
        dynts_cache_set_stream(self.handle, handle)
        self._stream = handle or 0
        return DYNTS_OK

    def synchronize(self):
        return dynts_synchronize(self.handle)

    def poll_error(self):
        return dynts_poll_error(self.handle)

    def set_score_source(self, source):
        return dynts_cache_set_score_source(self.handle, source)

    def set_kv_scale(self, k_scale, v_scale):
        return dynts_cache_set_kv_scale(self.handle, k_scale, v_scale)

    def append_scores(self, s_new):
        return dynts_append_scores(self.handle, s_new)

    def evict_at_budget(self, budget_B, ratio):
        r = dynts_evict_at_budget(self.handle, budget_B, ratio)
        return r

    def evict_stats(self):
        return dynts_evict_stats(self.handle)

    def launch_count(self):
        return dynts_cache_launch_count(self.handle)

    def scores_tensor(self):
        """A torch view (no copy) of the device score accumulator [L, Nb, Hkv, cap]."""
        torch = self.torch
        ptr = dynts_cache_scores(self.handle)
        off = ptr - self.storage.data_ptr()
        n = self.layers * self.batch * self.kv_heads * self.capacity
        return self.storage[off:off + 4 * n].view(torch.float32).view(self.layers, self.batch, self.kv_heads, self.capacity)

    def export_slab(self, layer, seq, head):
        """Host copies (K, V, pos, score) of one slab's n rows."""
        torch = self.torch
        n = self.len(seq)
        K = torch.empty((n, self.head_dim), dtype=self.slab_dtype)
        V = torch.empty((n, self.head_dim), dtype=self.slab_dtype)
        pos = torch.empty((n,), dtype=torch.int32)
        score = torch.empty((n,), dtype=torch.float32)
        m = dynts_cache_export(self.handle, layer, seq, head, K, V, pos, score)
        assert m == n
        return K, V, pos, score

    def import_slab(self, layer, seq, head, K, V, pos, score, n_pinned):
        n = K.shape[0]
        return dynts_cache_import(self.handle, layer, seq, head, K.contiguous(), V.contiguous(),
                                  pos.contiguous(), score.contiguous(), n, n_pinned)
