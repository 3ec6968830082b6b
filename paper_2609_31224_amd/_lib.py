"""ctypes binding of libA2T (include/a2t.h): the same calls, argument marshalling only.

Every step of the KV path runs in the library's HIP kernels.  If libA2T.so is
not built this module raises ImportError; there is no fallback.

Device buffers are torch tensors on the GPU (contiguous, the cache dtype:
torch.float32, or torch.bfloat16 for A2T_BF16 and A2T_MX4) or raw integer device addresses.  Host arrays
are anything numpy can turn into a contiguous array of the right type.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libA2T.so")

A2T_OK = 0
A2T_ERR_INVALID = -1
A2T_ERR_POS = -2
A2T_ERR_CAPACITY = -3
A2T_ERR_STATE = -4
A2T_ERR_OOM = -5
A2T_ERR_HIP = -6
A2T_ERR_NODEV = -7
A2T_F32 = 0
A2T_BF16 = 1
A2T_MX4 = 2
A2T_ALL_LAYERS = -1
A2T_FLAG_HOST_ONLY = 1
A2T_FLAG_NO_WORKSPACE = 2
A2T_FLAG_ROTATED = 4
A2T_RULE_UNIT, A2T_RULE_ROW, A2T_RULE_SINK_RECENT = 0, 1, 2
SEG_PREFIX, SEG_ACOUSTIC, SEG_DELIM, SEG_TEXT, SEG_RESPONSE = 0, 1, 2, 3, 4

EXPORTED = (
    "a2t_cache_create", "a2t_cache_destroy", "a2t_set_stream", "a2t_append",
    "a2t_chunk_attn", "a2t_append_attn", "a2t_append_attn_noalloc", "a2t_decode_attn",
    "a2t_evict", "a2t_evict_rule", "a2t_dev_begin", "a2t_dev_end", "a2t_dev_open",
    "a2t_dev_append_attn", "a2t_dev_evict", "a2t_dev_evict_rule",
    "a2t_stream_info_get", "a2t_resident",
    "a2t_read_layout", "a2t_read_last_evict", "a2t_read_kv", "a2t_read_rows", "a2t_sync",
    "a2t_profile_enable", "a2t_kernel_time", "a2t_profile_reserve", "a2t_status_str",
    "a2t_abi_version", "a2t_distill_create", "a2t_distill_destroy", "a2t_distill_loss",
    "a2t_distill_profile_enable", "a2t_distill_profile_reserve", "a2t_distill_kernel_time",
    "a2t_rope_create", "a2t_rope_destroy", "a2t_rope_set_stream", "a2t_rope_apply",
    "a2t_prompt_create", "a2t_prompt_destroy", "a2t_prompt_set_stream", "a2t_prompt_attn",
    "a2t_prompt_attn_grad", "a2t_prefer_create", "a2t_prefer_destroy", "a2t_prefer_set_stream",
    "a2t_prefer_logp", "a2t_prefer_loss",
)
A2T_ROW_NONE, A2T_ROW_ASR, A2T_ROW_NATIVE = 0, 1, 2
A2T_ROPE_HALF, A2T_ROPE_PAIRS = 0, 1
A2T_ROPE_PLAIN, A2T_ROPE_LINEAR, A2T_ROPE_NTK, A2T_ROPE_YARN = 0, 1, 2, 3
A2T_PROMPT_UNTIL = 1
A2T_PREFER_MAX_PAIRS = 256


class a2t_config(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("n_streams", C.c_int32), ("n_q_heads", C.c_int32),
        ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
        ("unit_rows", C.c_int32), ("kept_rows", C.c_int32), ("max_step_rows", C.c_int32),
        ("flags", C.c_uint32), ("rope_theta", C.c_double), ("attn_scale", C.c_double),
        ("device", C.c_int32), ("reserved", C.c_int32), ("k_pool", C.c_void_p),
        ("v_pool", C.c_void_p),
    ]


class a2t_stream_info(C.Structure):
    _fields_ = [
        ("resident", C.c_int32), ("peak", C.c_int32), ("kept", C.c_int32), ("ring", C.c_int32),
        ("ring_head", C.c_int32), ("cur_unit", C.c_int32), ("last_evicted_unit", C.c_int32),
        ("step_rows", C.c_int32), ("last_pos", C.c_int64), ("evicted_total", C.c_int64),
        ("moved_total", C.c_int64), ("budget_unmet", C.c_int32), ("last_evict_pre", C.c_int32),
    ]


class a2t_rope_config(C.Structure):
    _fields_ = [
        ("head_dim", C.c_int32), ("dtype", C.c_int32), ("rotary_dim", C.c_int32),
        ("layout", C.c_int32), ("scaling", C.c_int32), ("trained_rows", C.c_int32),
        ("theta", C.c_double), ("factor", C.c_double), ("turns_fast", C.c_double),
        ("turns_slow", C.c_double), ("device", C.c_int32), ("reserved", C.c_int32),
    ]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python paper_2609_31224_amd/build.py`")
    # torch ships its own HIP runtime and loads it under the unversioned name.
    # Loading torch first lets libA2T's libamdhip64.so.7 dependency resolve,
    # by SONAME, to that same runtime: one HIP/HSA runtime per process, so
    # torch's device pointers and streams are valid in libA2T.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    lib = C.CDLL(LIB_PATH)
    P, I32, I64, VP = C.POINTER, C.c_int32, C.c_int64, C.c_void_p
    sig = {
        "a2t_cache_create": (C.c_int, [P(a2t_config), VP, P(VP)]),
        "a2t_cache_destroy": (C.c_int, [VP]),
        "a2t_set_stream": (C.c_int, [VP, VP]),
        "a2t_append": (C.c_int, [VP, I32, I32, P(I32), P(I32), VP, VP, P(C.c_uint8), P(I32), P(I32)]),
        "a2t_chunk_attn": (C.c_int, [VP, I32, I32, P(I32), P(I32), VP, VP]),
        "a2t_append_attn": (C.c_int, [VP, I32, I32, P(I32), P(I32), VP, VP, P(C.c_uint8), P(I32),
                                      P(I32), P(I32), VP, VP]),
        "a2t_append_attn_noalloc": (C.c_int, [VP, I32, I32, P(I32), P(I32), VP, VP, P(C.c_uint8),
                                              P(I32), P(I32), P(I32), VP, VP]),
        "a2t_decode_attn": (C.c_int, [VP, I32, I32, P(I32), VP, VP]),
        "a2t_evict": (C.c_int, [VP, I32, P(I32), P(I32), I32, P(I32), P(C.c_uint8)]),
        "a2t_evict_rule": (C.c_int, [VP, I32, P(I32), P(I32), I32, I32, I32, P(I32),
                                     P(C.c_uint8)]),
        "a2t_dev_begin": (C.c_int, [VP]),
        "a2t_dev_end": (C.c_int, [VP]),
        "a2t_dev_open": (C.c_int, [VP, I32, P(I32), VP, VP, VP, VP]),
        "a2t_dev_append_attn": (C.c_int, [VP, I32, VP, VP, VP, VP]),
        "a2t_dev_evict": (C.c_int, [VP, VP, I32, VP, VP]),
        "a2t_dev_evict_rule": (C.c_int, [VP, VP, I32, I32, I32, VP, VP]),
        "a2t_stream_info_get": (C.c_int, [VP, I32, P(a2t_stream_info)]),
        "a2t_resident": (C.c_int, [VP, I32, P(C.c_int32), P(C.c_int32)]),
        "a2t_read_layout": (C.c_int, [VP, I32, P(I32), P(C.c_uint8), P(I32)]),
        "a2t_read_last_evict": (C.c_int, [VP, I32, P(I32), P(C.c_uint8), P(I32)]),
        "a2t_read_kv": (C.c_int, [VP, I32, I32, VP, VP]),
        "a2t_read_rows": (C.c_int, [VP, I32, I32, P(I32), VP, VP]),
        "a2t_sync": (C.c_int, [VP]),
        "a2t_profile_enable": (C.c_int, [VP, C.c_char_p]),
        "a2t_kernel_time": (C.c_int, [VP, C.c_char_p, P(C.c_int64), P(C.c_double)]),
        "a2t_profile_reserve": (C.c_int, [VP, I32]),
        "a2t_status_str": (C.c_char_p, [C.c_int]),
        "a2t_abi_version": (C.c_int, []),
        "a2t_distill_create": (C.c_int, [I32, I32, I32, I32, I32, VP, P(VP)]),
        "a2t_distill_destroy": (C.c_int, [VP]),
        "a2t_distill_loss": (C.c_int, [VP, I32, VP, C.c_int64, VP, C.c_int64, P(C.c_int8), P(I32),
                                       P(C.c_int8), P(C.c_int8), C.c_float, VP, VP]),
        "a2t_distill_profile_enable": (C.c_int, [VP, I32]),
        "a2t_distill_profile_reserve": (C.c_int, [VP, I32]),
        "a2t_distill_kernel_time": (C.c_int, [VP, P(C.c_int64), P(C.c_double)]),
        "a2t_rope_create": (C.c_int, [P(a2t_rope_config), VP, P(VP)]),
        "a2t_rope_destroy": (C.c_int, [VP]),
        "a2t_rope_set_stream": (C.c_int, [VP, VP]),
        "a2t_rope_apply": (C.c_int, [VP, I32, VP, I32, VP, I64, VP, I64, I32, VP, I64, VP, I64, I32]),
        "a2t_prompt_create": (C.c_int, [I32, I32, I32, I32, I32, C.c_double, C.c_uint32, I32, VP, P(VP)]),
        "a2t_prompt_destroy": (C.c_int, [VP]),
        "a2t_prompt_set_stream": (C.c_int, [VP, VP]),
        "a2t_prompt_attn": (C.c_int, [VP, I32, P(I32), VP, I64, VP, I64, VP, I64, VP, VP, VP]),
        "a2t_prompt_attn_grad": (C.c_int, [VP, I32, P(I32), VP, I64, VP, I64, VP, I64, VP, VP, VP, VP,
                                           VP, VP, VP]),
        "a2t_prefer_create": (C.c_int, [I32, I32, I32, I32, VP, P(VP)]),
        "a2t_prefer_destroy": (C.c_int, [VP]),
        "a2t_prefer_set_stream": (C.c_int, [VP, VP]),
        "a2t_prefer_logp": (C.c_int, [VP, I32, VP, I64, VP, VP]),
        "a2t_prefer_loss": (C.c_int, [VP, I32, P(I32), VP, I64, VP, I64, VP, VP, C.c_float, C.c_float,
                                      VP, VP, VP]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


_lib = _load()


class A2TError(RuntimeError):
    def __init__(self, status: int, call: str):
        self.status = status
        super().__init__(f"{call}: {a2t_status_str(status)} ({status})")


def _check(rc: int, call: str) -> None:
    if rc != A2T_OK:
        raise A2TError(rc, call)


def _i32(x) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(x), dtype=np.int32)


def _u8(x) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(x), dtype=np.uint8)


def _p(arr: Optional[np.ndarray], ctype):
    if arr is None:
        return None
    return arr.ctypes.data_as(C.POINTER(ctype))


def _dev(x, what: str, dtype=None) -> Optional[int]:
    """Device address of a torch tensor (validated) or a raw integer address."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    import torch
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what}: expected a GPU torch tensor or a device address")
    if not x.is_cuda:
        raise ValueError(f"{what}: tensor must live on the GPU")
    if not x.is_contiguous():
        raise ValueError(f"{what}: tensor must be contiguous")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{what}: dtype {x.dtype}, cache uses {dtype}")
    return x.data_ptr()


@dataclass
class Cache:
    """Handle returned by a2t_cache_create (plus what marshalling needs)."""
    ptr: C.c_void_p
    config: a2t_config

    @property
    def torch_dtype(self):
        import torch
        return torch.float32 if self.config.dtype == A2T_F32 else torch.bfloat16


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return None
    if isinstance(stream, int):
        return stream
    return int(stream.cuda_stream)


def a2t_abi_version() -> int:
    return _lib.a2t_abi_version()


def a2t_status_str(status: int) -> str:
    return _lib.a2t_status_str(status).decode()


def a2t_cache_create(n_layers: int, n_streams: int, n_q_heads: int, n_kv_heads: int,
                     head_dim: int, dtype: int, unit_rows: int, kept_rows: int,
                     max_step_rows: int, flags: int = 0, rope_theta: float = 0.0,
                     attn_scale: float = 0.0, device: int = 0, stream=None,
                     k_pool=None, v_pool=None) -> Cache:
    """``k_pool``/``v_pool``: optional caller-owned device pools (torch tensors or
    addresses) of L*S*Hkv*(unit_rows+kept_rows)*D elements each (A2T_MX4: that many
    rows of D/2 + D/32 bytes); the caller keeps them alive until a2t_cache_destroy."""
    cfg = a2t_config(n_layers, n_streams, n_q_heads, n_kv_heads, head_dim, dtype, unit_rows,
                     kept_rows, max_step_rows, flags, rope_theta, attn_scale, device, 0,
                     _dev(k_pool, "k_pool"), _dev(v_pool, "v_pool"))
    out = C.c_void_p()
    _check(_lib.a2t_cache_create(C.byref(cfg), _stream_handle(stream), C.byref(out)),
           "a2t_cache_create")
    return Cache(out, cfg)


def a2t_cache_destroy(c: Cache) -> None:
    if c.ptr:
        _check(_lib.a2t_cache_destroy(c.ptr), "a2t_cache_destroy")
        c.ptr = C.c_void_p()


def a2t_set_stream(c: Cache, stream) -> None:
    _check(_lib.a2t_set_stream(c.ptr, _stream_handle(stream)), "a2t_set_stream")


def a2t_append(c: Cache, layer: int, stream_ids: Sequence[int], n_rows: Sequence[int], k, v,
               seg=None, pos=None, unit_id=None) -> None:
    ids, nr = _i32(stream_ids), _i32(n_rows)
    if ids.shape != nr.shape:
        raise ValueError("stream_ids and n_rows differ in length")
    sg = None if seg is None else _u8(seg)
    ps = None if pos is None else _i32(pos)
    un = None if unit_id is None else _i32(unit_id)
    dt = c.torch_dtype if not isinstance(k, (int, type(None))) else None
    rc = _lib.a2t_append(c.ptr, layer, len(ids), _p(ids, C.c_int32), _p(nr, C.c_int32),
                         _dev(k, "k", dt), _dev(v, "v", dt), _p(sg, C.c_uint8),
                         _p(ps, C.c_int32), _p(un, C.c_int32))
    _check(rc, "a2t_append")


def a2t_chunk_attn(c: Cache, layer: int, stream_ids: Sequence[int], n_q: Sequence[int], q, o) -> None:
    ids, nq = _i32(stream_ids), _i32(n_q)
    if ids.shape != nq.shape:
        raise ValueError("stream_ids and n_q differ in length")
    dt = c.torch_dtype if not isinstance(q, int) else None
    rc = _lib.a2t_chunk_attn(c.ptr, layer, len(ids), _p(ids, C.c_int32), _p(nq, C.c_int32),
                             _dev(q, "q", dt), _dev(o, "o", dt))
    _check(rc, "a2t_chunk_attn")


def _append_attn(fn, name, c, layer, stream_ids, n_rows, k, v, seg, pos, unit_id, n_q, q, o):
    ids, nr, nq = _i32(stream_ids), _i32(n_rows), _i32(n_q)
    if not (ids.shape == nr.shape == nq.shape):
        raise ValueError("stream_ids, n_rows and n_q differ in length")
    sg = None if seg is None else _u8(seg)
    ps = None if pos is None else _i32(pos)
    un = None if unit_id is None else _i32(unit_id)
    dt = c.torch_dtype if not isinstance(k, (int, type(None))) else None
    rc = fn(c.ptr, layer, len(ids), _p(ids, C.c_int32), _p(nr, C.c_int32), _dev(k, "k", dt),
            _dev(v, "v", dt), _p(sg, C.c_uint8), _p(ps, C.c_int32), _p(un, C.c_int32),
            _p(nq, C.c_int32), _dev(q, "q", dt), _dev(o, "o", dt))
    _check(rc, name)


def a2t_append_attn(c: Cache, layer: int, stream_ids: Sequence[int], n_rows: Sequence[int], k, v,
                    seg, pos, unit_id, n_q: Sequence[int], q, o) -> None:
    _append_attn(_lib.a2t_append_attn, "a2t_append_attn", c, layer, stream_ids, n_rows, k, v, seg,
                 pos, unit_id, n_q, q, o)


def a2t_append_attn_noalloc(c: Cache, layer: int, stream_ids: Sequence[int],
                            n_rows: Sequence[int], k, v, seg, pos, unit_id, n_q: Sequence[int],
                            q, o) -> None:
    _append_attn(_lib.a2t_append_attn_noalloc, "a2t_append_attn_noalloc", c, layer, stream_ids,
                 n_rows, k, v, seg, pos, unit_id, n_q, q, o)


def a2t_decode_attn(c: Cache, layer: int, stream_ids: Sequence[int], q, o) -> None:
    ids = _i32(stream_ids)
    dt = c.torch_dtype if not isinstance(q, int) else None
    rc = _lib.a2t_decode_attn(c.ptr, layer, len(ids), _p(ids, C.c_int32), _dev(q, "q", dt),
                              _dev(o, "o", dt))
    _check(rc, "a2t_decode_attn")


def a2t_evict(c: Cache, stream_ids: Sequence[int], budget, window: int) -> Tuple[np.ndarray, np.ndarray]:
    ids = _i32(stream_ids)
    b = _i32(np.broadcast_to(np.asarray(budget), ids.shape))
    n_ev = np.zeros(ids.shape, np.int32)
    unmet = np.zeros(ids.shape, np.uint8)
    rc = _lib.a2t_evict(c.ptr, len(ids), _p(ids, C.c_int32), _p(b, C.c_int32), window,
                        _p(n_ev, C.c_int32), _p(unmet, C.c_uint8))
    _check(rc, "a2t_evict")
    return n_ev, unmet.astype(bool)


def a2t_evict_rule(c: Cache, stream_ids: Sequence[int], budget, window: int, rule: int,
                   n_sink: int = 0) -> Tuple[np.ndarray, np.ndarray]:
    ids = _i32(stream_ids)
    b = _i32(np.broadcast_to(np.asarray(budget), ids.shape))
    n_ev = np.zeros(ids.shape, np.int32)
    unmet = np.zeros(ids.shape, np.uint8)
    rc = _lib.a2t_evict_rule(c.ptr, len(ids), _p(ids, C.c_int32), _p(b, C.c_int32), window, rule,
                             n_sink, _p(n_ev, C.c_int32), _p(unmet, C.c_uint8))
    _check(rc, "a2t_evict_rule")
    return n_ev, unmet.astype(bool)


def a2t_dev_begin(c: Cache) -> None:
    _check(_lib.a2t_dev_begin(c.ptr), "a2t_dev_begin")


def a2t_dev_end(c: Cache) -> None:
    _check(_lib.a2t_dev_end(c.ptr), "a2t_dev_end")


def a2t_dev_open(c: Cache, stream_ids: Sequence[int], n_rows, unit_id, seg, pos) -> None:
    """n_rows, unit_id: device int32 [n]; seg: device uint8 [n][max_step_rows];
    pos: device int32 [n][max_step_rows] (torch tensors or addresses)."""
    ids = _i32(stream_ids)
    rc = _lib.a2t_dev_open(c.ptr, len(ids), _p(ids, C.c_int32), _dev(n_rows, "n_rows"),
                           _dev(unit_id, "unit_id"), _dev(seg, "seg"), _dev(pos, "pos"))
    _check(rc, "a2t_dev_open")


def a2t_dev_append_attn(c: Cache, layer: int, k, v, q, o) -> None:
    dt = c.torch_dtype if not isinstance(k, int) else None
    rc = _lib.a2t_dev_append_attn(c.ptr, layer, _dev(k, "k", dt), _dev(v, "v", dt),
                                  _dev(q, "q", dt), _dev(o, "o", dt))
    _check(rc, "a2t_dev_append_attn")


def a2t_dev_evict(c: Cache, budget, window: int, n_evicted=None, budget_unmet=None) -> None:
    """budget: device int32 [n]; n_evicted (int32), budget_unmet (uint8): optional
    device [n] outputs."""
    rc = _lib.a2t_dev_evict(c.ptr, _dev(budget, "budget"), window, _dev(n_evicted, "n_evicted"),
                            _dev(budget_unmet, "budget_unmet"))
    _check(rc, "a2t_dev_evict")


def a2t_dev_evict_rule(c: Cache, budget, window: int, rule: int, n_sink: int = 0, n_evicted=None,
                       budget_unmet=None) -> None:
    """a2t_dev_evict with an a2t_rule (A2T_RULE_*) and, for the sink rule, the sink count."""
    rc = _lib.a2t_dev_evict_rule(c.ptr, _dev(budget, "budget"), window, rule, n_sink,
                                 _dev(n_evicted, "n_evicted"), _dev(budget_unmet, "budget_unmet"))
    _check(rc, "a2t_dev_evict_rule")


def a2t_stream_info_get(c: Cache, stream: int) -> dict:
    info = a2t_stream_info()
    _check(_lib.a2t_stream_info_get(c.ptr, stream, C.byref(info)), "a2t_stream_info_get")
    return {name: getattr(info, name) for name, _ in a2t_stream_info._fields_}


def a2t_resident(c: Cache, stream: int) -> tuple:
    """(resident rows R, peak R) of one stream."""
    n, peak = C.c_int32(), C.c_int32()
    _check(_lib.a2t_resident(c.ptr, stream, C.byref(n), C.byref(peak)), "a2t_resident")
    return n.value, peak.value


def a2t_read_layout(c: Cache, stream: int):
    n = a2t_stream_info_get(c, stream)["resident"]
    pos = np.zeros(n, np.int32)
    seg = np.zeros(n, np.uint8)
    unit = np.zeros(n, np.int32)
    _check(_lib.a2t_read_layout(c.ptr, stream, _p(pos, C.c_int32), _p(seg, C.c_uint8),
                                _p(unit, C.c_int32)), "a2t_read_layout")
    return pos, seg, unit


def a2t_read_last_evict(c: Cache, stream: int):
    n_pre = C.c_int32()
    _check(_lib.a2t_read_last_evict(c.ptr, stream, C.byref(n_pre), None, None),
           "a2t_read_last_evict")
    mask = np.zeros(n_pre.value, np.uint8)
    slot = np.zeros(n_pre.value, np.int32)
    _check(_lib.a2t_read_last_evict(c.ptr, stream, C.byref(n_pre), _p(mask, C.c_uint8),
                                    _p(slot, C.c_int32)), "a2t_read_last_evict")
    return n_pre.value, mask, slot


def a2t_read_kv(c: Cache, layer: int, stream: int):
    """Resident K (rotated) and V of one layer in cache order.  float32 arrays
    for fp32 caches; for bf16 and A2T_MX4 caches the raw 16-bit patterns of the
    bf16 values (uint16)."""
    n = a2t_stream_info_get(c, stream)["resident"]
    shape = (n, c.config.n_kv_heads, c.config.head_dim)
    dt = np.float32 if c.config.dtype == A2T_F32 else np.uint16
    k = np.zeros(shape, dt)
    v = np.zeros(shape, dt)
    _check(_lib.a2t_read_kv(c.ptr, layer, stream, k.ctypes.data, v.ctypes.data), "a2t_read_kv")
    return k, v


def a2t_read_rows(c: Cache, layer: int, stream_ids: Sequence[int], k=None, v=None) -> None:
    """Resident rows of the streams, in cache order, into GPU tensors [rows][Hkv][D] (one
    layer) or [L][rows][Hkv][D] (A2T_ALL_LAYERS) of the cache's input type, rows being the
    sum of the streams' a2t_resident; either may be None.  Tensors too small for them are a
    ValueError.  Asynchronous on the cache's stream."""
    ids = _i32(stream_ids)
    k_ptr = _dev(k, "k", c.torch_dtype if not isinstance(k, int) else None)
    v_ptr = _dev(v, "v", c.torch_dtype if not isinstance(v, int) else None)
    rows = sum(a2t_resident(c, int(s))[0] for s in ids if 0 <= s < c.config.n_streams)
    need = rows * c.config.n_kv_heads * c.config.head_dim * (c.config.n_layers if layer == A2T_ALL_LAYERS else 1)
    for what, x in (("k", k), ("v", v)):
        if x is not None and not isinstance(x, int) and x.numel() < need:
            raise ValueError(f"{what}: {x.numel()} elements, the resident rows have {need}")
    rc = _lib.a2t_read_rows(c.ptr, layer, len(ids), _p(ids, C.c_int32), k_ptr, v_ptr)
    _check(rc, "a2t_read_rows")


def a2t_sync(c: Cache) -> None:
    _check(_lib.a2t_sync(c.ptr), "a2t_sync")


def a2t_profile_enable(c: Cache, kernel_filter: Optional[str]) -> None:
    arg = None if kernel_filter is None else kernel_filter.encode()
    _check(_lib.a2t_profile_enable(c.ptr, arg), "a2t_profile_enable")


def a2t_kernel_time(c: Cache, kernel: str) -> Tuple[int, float]:
    n = C.c_int64()
    ms = C.c_double()
    _check(_lib.a2t_kernel_time(c.ptr, kernel.encode(), C.byref(n), C.byref(ms)), "a2t_kernel_time")
    return n.value, ms.value


def a2t_profile_reserve(c: Cache, n_launches: int) -> None:
    _check(_lib.a2t_profile_reserve(c.ptr, n_launches), "a2t_profile_reserve")


def raw_lib():
    """The ctypes library with argument types set, for callers that marshal
    their arguments once and call the C entry points directly."""
    return _lib


# ---- adaptation objective (Sec. 3.2)
@dataclass
class Distill:
    """Handle returned by a2t_distill_create."""
    ptr: C.c_void_p
    max_rows: int
    vocab: int
    n_added: int
    dtype: int


def a2t_distill_create(max_rows: int, vocab: int, n_added: int, dtype: int, device: int = 0,
                       stream=None) -> Distill:
    out = C.c_void_p()
    _check(_lib.a2t_distill_create(max_rows, vocab, n_added, dtype, device, _stream_handle(stream),
                                   C.byref(out)), "a2t_distill_create")
    return Distill(out, max_rows, vocab, n_added, dtype)


def a2t_distill_destroy(d: Distill) -> None:
    _check(_lib.a2t_distill_destroy(d.ptr), "a2t_distill_destroy")


def a2t_distill_loss(d: Distill, student, teacher, kind, target, dec_group, turn_group,
                     temperature: float, losses, grad=None) -> None:
    """student / teacher / grad: GPU tensors [n_rows][stride] (rows of the
    extended / teacher vocabulary, strides multiples of 8); kind, target,
    dec_group, turn_group: host arrays [n_rows]; losses: GPU float32 [5]."""
    import torch
    dt = torch.float32 if d.dtype == A2T_F32 else torch.bfloat16
    n = int(student.shape[0])
    kd = np.ascontiguousarray(np.asarray(kind), dtype=np.int8)
    tg = _i32(target)
    dg = np.ascontiguousarray(np.asarray(dec_group), dtype=np.int8)
    tu = np.ascontiguousarray(np.asarray(turn_group), dtype=np.int8)
    if not (kd.shape == tg.shape == dg.shape == tu.shape == (n,)):
        raise ValueError("row metadata must have one entry per row")
    rc = _lib.a2t_distill_loss(d.ptr, n, _dev(student, "student", dt), int(student.stride(0)),
                               _dev(teacher, "teacher", dt), int(teacher.stride(0)),
                               _p(kd, C.c_int8), _p(tg, C.c_int32), _p(dg, C.c_int8),
                               _p(tu, C.c_int8), float(temperature),
                               _dev(losses, "losses", torch.float32), _dev(grad, "grad", dt))
    _check(rc, "a2t_distill_loss")


# ---- training on whole sessions: rotary encoding, packed attention, preference loss
def _torch_dtype(dtype: int):
    import torch
    return torch.float32 if dtype == A2T_F32 else torch.bfloat16


def _on(x, what: str, device: int) -> None:
    """x lives on the handle's GPU: another's memory may be out of its reach."""
    if x.get_device() != device:
        where = f" of its handle ({device}), not {x.get_device()}" if x.is_cuda else ""
        raise ValueError(f"{what}: tensor must live on the GPU{where}")


def _rows(x, what: str, dtype, device: int, heads: Optional[int], dim: int, n: Optional[int] = None):
    """(address, row stride) of a GPU tensor [rows][heads][dim] whose rows are dense; the rows may
    be parts of wider ones.  Sizes that do not fit are a ValueError."""
    import torch
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what}: expected a GPU torch tensor")
    _on(x, what, device)
    if x.dtype != dtype:
        raise ValueError(f"{what}: dtype {x.dtype}, the handle uses {dtype}")
    if x.dim() != 3 or x.shape[2] != dim or (heads is not None and x.shape[1] != heads) or (n is not None and x.shape[0] != n):
        want = f"[{'rows' if n is None else n}][{'heads' if heads is None else heads}][{dim}]"
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected {want}")
    if x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != dim):
        raise ValueError(f"{what}: a row's heads must be dense")
    stride = x.stride(0) if x.shape[0] > 1 else max(x.stride(0), (x.shape[1] * dim + 7) // 8 * 8)
    return x.data_ptr(), int(stride)


def _flat(x, what: str, dtype, device: int, numel: int):
    """Address of a contiguous GPU tensor with `numel` elements."""
    if x is None:
        return None
    if isinstance(x, int):
        raise TypeError(f"{what}: expected a GPU torch tensor")
    ptr = _dev(x, what, dtype)
    _on(x, what, device)
    if x.numel() != numel:
        raise ValueError(f"{what}: {x.numel()} elements, expected {numel}")
    return ptr


@dataclass
class Rope:
    """Handle returned by a2t_rope_create."""
    ptr: C.c_void_p
    head_dim: int
    dtype: int
    device: int = 0


def a2t_rope_create(head_dim: int, dtype: int, rotary_dim: int = 0, layout: int = A2T_ROPE_HALF, theta: float = 0.0,
                    scaling: int = A2T_ROPE_PLAIN, factor: float = 1.0, trained_rows: int = 0, turns_fast: float = 32.0,
                    turns_slow: float = 1.0, device: int = 0, stream=None) -> Rope:
    cfg = a2t_rope_config(head_dim, dtype, rotary_dim, layout, scaling, trained_rows, theta, factor, turns_fast,
                          turns_slow, device, 0)
    out = C.c_void_p()
    _check(_lib.a2t_rope_create(C.byref(cfg), _stream_handle(stream), C.byref(out)), "a2t_rope_create")
    return Rope(out, head_dim, dtype, device)


def a2t_rope_destroy(r: Rope) -> None:
    if r.ptr:
        _check(_lib.a2t_rope_destroy(r.ptr), "a2t_rope_destroy")
        r.ptr = C.c_void_p()


def a2t_rope_set_stream(r: Rope, stream) -> None:
    _check(_lib.a2t_rope_set_stream(r.ptr, _stream_handle(stream)), "a2t_rope_set_stream")


def a2t_rope_apply(r: Rope, pos, q=None, k=None, q_out=None, k_out=None, grad: bool = False) -> None:
    """q, k: GPU tensors [rows][heads][D] (either may be None), rotated into q_out, k_out (the input
    itself rotates in place); pos: GPU int32 [rows].  grad=True turns gradients of the outputs back."""
    import torch
    dt, n = _torch_dtype(r.dtype), int(pos.shape[0])
    args = []
    for what, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            if out is not None:
                raise ValueError(f"{what}_out without {what}")
            args += [0, None, 0, None, 0]
            continue
        heads = int(x.shape[1]) if x.dim() == 3 else None
        args += [heads or 0, *_rows(x, what, dt, r.device, None, r.head_dim, n),
                 *_rows(out, what + "_out", dt, r.device, heads, r.head_dim, n)]
    _check(_lib.a2t_rope_apply(r.ptr, n, _flat(pos, "pos", torch.int32, r.device, n), *args, int(bool(grad))),
           "a2t_rope_apply")


@dataclass
class Prompt:
    """Handle returned by a2t_prompt_create."""
    ptr: C.c_void_p
    max_rows: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    dtype: int
    device: int = 0


def a2t_prompt_create(max_rows: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: int, attn_scale: float = 0.0,
                      flags: int = 0, device: int = 0, stream=None) -> Prompt:
    out = C.c_void_p()
    _check(_lib.a2t_prompt_create(max_rows, n_q_heads, n_kv_heads, head_dim, dtype, attn_scale, flags, device,
                                  _stream_handle(stream), C.byref(out)), "a2t_prompt_create")
    return Prompt(out, max_rows, n_q_heads, n_kv_heads, head_dim, dtype, device)


def a2t_prompt_destroy(p: Prompt) -> None:
    if p.ptr:
        _check(_lib.a2t_prompt_destroy(p.ptr), "a2t_prompt_destroy")
        p.ptr = C.c_void_p()


def a2t_prompt_set_stream(p: Prompt, stream) -> None:
    _check(_lib.a2t_prompt_set_stream(p.ptr, _stream_handle(stream)), "a2t_prompt_set_stream")


def _prompt_rows(p: Prompt, seq_rows, q, k, v, until):
    import torch
    rows = _i32(seq_rows)
    n = int(rows.sum(dtype=np.int64))
    dt = _torch_dtype(p.dtype)
    given = []
    for what, x, heads in (("q", q, p.n_q_heads), ("k", k, p.n_kv_heads), ("v", v, p.n_kv_heads)):
        given.append(_rows(x, what, dt, p.device, heads, p.head_dim))
        if x.shape[0] < n:
            raise ValueError(f"{what}: {x.shape[0]} rows, the sequences have {n}")
    if until is not None:
        if not isinstance(until, torch.Tensor):
            raise TypeError("until: expected a GPU torch tensor")
        _dev(until, "until", torch.int32)
        _on(until, "until", p.device)
        if until.numel() < n:
            raise ValueError(f"until: {until.numel()} entries, the sequences have {n} rows")
    return rows, n, dt, given, None if until is None else until.data_ptr()


def _packed(x, what: str, dt, p: Prompt, n: int):
    ptr = _dev(x, what, dt)
    if ptr is None or isinstance(x, int):
        raise TypeError(f"{what}: expected a GPU torch tensor")
    _on(x, what, p.device)
    if x.dim() != 3 or x.shape[0] < n or tuple(x.shape[1:]) != (p.n_q_heads, p.head_dim):
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected [{n}][{p.n_q_heads}][{p.head_dim}]")
    return ptr


def a2t_prompt_attn(p: Prompt, seq_rows: Sequence[int], q, k, v, o, lse=None, until=None) -> None:
    """q, k, v: GPU tensors [rows][heads][D], rows dense; o: GPU [rows][Hq][D]; lse: GPU float32
    [Hq][rows], rows the sum of seq_rows, or None; until: GPU int32 [rows] or None."""
    import torch
    rows, n, dt, given, ut = _prompt_rows(p, seq_rows, q, k, v, until)
    _check(_lib.a2t_prompt_attn(p.ptr, len(rows), _p(rows, C.c_int32), *given[0], *given[1], *given[2], ut,
                                _packed(o, "o", dt, p, n), _flat(lse, "lse", torch.float32, p.device, n * p.n_q_heads)),
           "a2t_prompt_attn")


def a2t_prompt_attn_grad(p: Prompt, seq_rows: Sequence[int], q, k, v, o, lse, d_o, dq, dk, dv, until=None) -> None:
    """Gradients dq, dk, dv from d_o: GPU tensors shaped and strided like q, k, v."""
    import torch
    rows, n, dt, given, ut = _prompt_rows(p, seq_rows, q, k, v, until)
    outs = []
    for what, x, like, (_, stride), heads in (("dq", dq, q, given[0], p.n_q_heads), ("dk", dk, k, given[1], p.n_kv_heads),
                                              ("dv", dv, v, given[2], p.n_kv_heads)):
        ptr, own = _rows(x, what, dt, p.device, heads, p.head_dim)
        if x.shape[0] < n or (own != stride and n > 1):
            raise ValueError(f"{what}: {x.shape[0]} rows with stride {own}, expected {n} with stride {stride}")
        outs.append(ptr)
    if lse is None:
        raise ValueError("lse: the forward pass's")
    _check(_lib.a2t_prompt_attn_grad(p.ptr, len(rows), _p(rows, C.c_int32), *given[0], *given[1], *given[2], ut,
                                     _packed(o, "o", dt, p, n), _flat(lse, "lse", torch.float32, p.device, n * p.n_q_heads),
                                     _packed(d_o, "d_o", dt, p, n), *outs), "a2t_prompt_attn_grad")


@dataclass
class Prefer:
    """Handle returned by a2t_prefer_create."""
    ptr: C.c_void_p
    max_rows: int
    vocab: int
    dtype: int
    device: int = 0


def a2t_prefer_create(max_rows: int, vocab: int, dtype: int, device: int = 0, stream=None) -> Prefer:
    out = C.c_void_p()
    _check(_lib.a2t_prefer_create(max_rows, vocab, dtype, device, _stream_handle(stream), C.byref(out)), "a2t_prefer_create")
    return Prefer(out, max_rows, vocab, dtype, device)


def a2t_prefer_destroy(p: Prefer) -> None:
    if p.ptr:
        _check(_lib.a2t_prefer_destroy(p.ptr), "a2t_prefer_destroy")
        p.ptr = C.c_void_p()


def a2t_prefer_set_stream(p: Prefer, stream) -> None:
    _check(_lib.a2t_prefer_set_stream(p.ptr, _stream_handle(stream)), "a2t_prefer_set_stream")


def _logits(p: Prefer, x, what: str, n: int):
    """(address, row stride) of a GPU tensor [rows][>= vocab] of logits, rows dense."""
    import torch
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{what}: expected a GPU torch tensor")
    _on(x, what, p.device)
    if x.dtype != _torch_dtype(p.dtype):
        raise ValueError(f"{what}: dtype {x.dtype}, the handle uses {_torch_dtype(p.dtype)}")
    if x.dim() != 2 or x.shape[0] < n or x.shape[1] < p.vocab or x.stride(1) != 1:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected [{n}][{p.vocab} or more] with dense rows")
    if x.stride(0) < x.shape[1] and x.shape[0] > 1:
        raise ValueError(f"{what}: rows overlap")
    if what == "grad" and x.stride(0) > (x.shape[1] + 7) // 8 * 8:
        raise ValueError(f"grad: columns {x.shape[1]} to {x.stride(0)} of its rows would be zeroed: pass them, or a tensor of its own")
    # the last row is read (and the gradient's written) in whole chunks of 8 elements up to its stride
    room = x.untyped_storage().nbytes() // x.element_size() - x.storage_offset()
    if room < (n - 1) * x.stride(0) + (x.stride(0) if what == "grad" else (p.vocab + 7) // 8 * 8):
        raise ValueError(f"{what}: the last row ends before its stride does")
    return x.data_ptr(), int(x.stride(0))


def a2t_prefer_logp(p: Prefer, logits, target, logp) -> None:
    """logits: GPU [rows][stride]; target: GPU int32 [rows]; logp: GPU float32 [rows] out."""
    import torch
    n = int(target.shape[0])
    _check(_lib.a2t_prefer_logp(p.ptr, n, *_logits(p, logits, "logits", n), _flat(target, "target", torch.int32, p.device, n),
                                _flat(logp, "logp", torch.float32, p.device, n)), "a2t_prefer_logp")


def a2t_prefer_loss(p: Prefer, answer_rows: Sequence[int], policy, target, losses, reference=None, ref_logp=None,
                    beta: float = 0.1, smoothing: float = 0.0, ratios=None, grad=None) -> None:
    """answer_rows: host, rows of the chosen and the rejected answer of each pair in turn; policy,
    reference: GPU [rows][stride] logits; losses: GPU float32 [3]; ratios: GPU float32, one per answer;
    grad: GPU tensor like policy (or policy itself), zeroed from the vocabulary up to its rows' stride: a
    view of some columns of wider rows is a ValueError."""
    import torch
    rows = _i32(answer_rows)
    if rows.ndim != 1 or len(rows) % 2:
        raise ValueError("answer_rows: two answers a pair")
    n = int(rows.sum(dtype=np.int64))
    ptr, stride = _logits(p, policy, "policy", n)
    ref = (None, 0) if reference is None else _logits(p, reference, "reference", n)
    g = None
    if grad is not None:
        g, own = _logits(p, grad, "grad", n)
        if own != stride:
            raise ValueError(f"grad: stride {own}, the policy's is {stride}")
    _check(_lib.a2t_prefer_loss(p.ptr, len(rows) // 2, _p(rows, C.c_int32), ptr, stride, *ref,
                                _flat(ref_logp, "ref_logp", torch.float32, p.device, n),
                                _flat(target, "target", torch.int32, p.device, n),
                                float(beta), float(smoothing), _flat(losses, "losses", torch.float32, p.device, 3),
                                _flat(ratios, "ratios", torch.float32, p.device, len(rows)), g), "a2t_prefer_loss")
