"""Thin ctypes binding of libs2o.so (the C ABI declared in include/s2o.h).

Argument marshalling only: every step of the path runs in the HIP kernels behind the
library.  PyTorch appears only as the owner of device memory and streams.  There is no
CPU fallback: if the library has not been built, loading raises."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from functools import lru_cache
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libs2o.so")

S2O_OK, S2O_EINVAL, S2O_EUNSUPPORTED, S2O_ESCRATCH, S2O_EHIP = 0, -1, -2, -3, -4

STATIC_SCRATCH_BYTES = 32 << 20

EXPORTS = ("s2o_version", "s2o_strerror", "s2o_last_hip_error", "s2o_plan_sizes", "s2o_plan", "s2o_plan_static",
           "s2o_attention_sizes", "s2o_attention", "s2o_attention_local", "s2o_attention_prefix",
           "s2o_decode_sizes", "s2o_decode", "s2o_key_weights_sizes", "s2o_key_weights", "s2o_evict_sizes", "s2o_evict")


class S2OParams(C.Structure):
    _fields_ = [("struct_size", C.c_int32), ("batch", C.c_int32), ("q_heads", C.c_int32),
                ("kv_heads", C.c_int32), ("seq_len", C.c_int32), ("head_dim", C.c_int32),
                ("seg_len", C.c_int32), ("block_m", C.c_int32), ("block_n", C.c_int32),
                ("use_q_perm", C.c_int32), ("stop_mode", C.c_int32), ("softmax_scale", C.c_float),
                ("max_prefix_tiles", C.c_int32), ("non_causal", C.c_int32),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3),
                ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3)]


class S2OPlanOut(C.Structure):
    _fields_ = [("q_perm", C.c_void_p), ("kv_perm", C.c_void_p), ("s_q", C.c_void_p),
                ("s_k", C.c_void_p), ("q_mean", C.c_void_p), ("k_guide", C.c_void_p),
                ("status", C.c_void_p)]


S2O_BF16, S2O_F16 = 0, 1


class S2ODecodeParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("struct_size", "batch", "branches", "q_heads", "kv_heads", "head_dim", "q_len", "cache_len",
                                         "own_len", "dtype")] + [
                ("softmax_scale", C.c_float), ("reserved", C.c_int32), ("q_stride", C.c_int64 * 4),
                ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3), ("own_k_stride", C.c_int64 * 4),
                ("own_v_stride", C.c_int64 * 4), ("o_stride", C.c_int64 * 4)]


class S2OWeightsParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("struct_size", "batch", "branches", "q_heads", "kv_heads", "head_dim", "q_len", "cache_len",
                                         "dtype", "causal")] + [
                ("softmax_scale", C.c_float), ("reserved", C.c_int32), ("q_stride", C.c_int64 * 4),
                ("k_stride", C.c_int64 * 3)]


class S2OEvictParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("struct_size", "batch", "kv_heads", "head_dim", "cache_len", "keep", "sink", "recent", "dtype",
                                         "reserved")] + [
                ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3), ("out_k_stride", C.c_int64 * 3),
                ("out_v_stride", C.c_int64 * 3)]


class S2OError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"s2o error {code}: {msg}")
        self.code = code


_lib = None


def load_library():
    """Load libs2o.so (once).  Import torch first so that both share one HIP runtime."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with "
                          "`python -m paper_2602_22575_amd.build` (there is no fallback path)")
    import torch  # noqa: F401  (loads libamdhip64 that libs2o.so resolves against)
    lib = C.CDLL(LIB_PATH)
    lib.s2o_version.restype = C.c_int
    lib.s2o_strerror.restype = C.c_char_p
    lib.s2o_strerror.argtypes = [C.c_int]
    lib.s2o_last_hip_error.restype = C.c_int
    szp = C.POINTER(C.c_size_t)
    lib.s2o_plan_sizes.restype = C.c_int
    lib.s2o_plan_sizes.argtypes = [C.POINTER(S2OParams)] + [szp] * 7
    lib.s2o_plan.restype = C.c_int
    lib.s2o_plan.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(S2OParams), C.POINTER(S2OPlanOut),
                             C.c_void_p, C.c_size_t, C.c_void_p]
    lib.s2o_plan_static.restype = C.c_int
    lib.s2o_plan_static.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(S2OParams), C.POINTER(S2OPlanOut), C.c_void_p]
    lib.s2o_attention_sizes.restype = C.c_int
    lib.s2o_attention_sizes.argtypes = [C.POINTER(S2OParams), szp, szp]
    lib.s2o_attention.restype = C.c_int
    lib.s2o_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(S2OParams),
                                  C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.s2o_attention_prefix.restype = C.c_int
    lib.s2o_attention_prefix.argtypes = lib.s2o_attention.argtypes
    lib.s2o_attention_local.restype = C.c_int
    lib.s2o_attention_local.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(S2OParams),
                                        C.c_void_p, C.c_size_t, C.c_void_p]
    vp, st = C.c_void_p, C.c_size_t
    lib.s2o_decode_sizes.argtypes = [C.POINTER(S2ODecodeParams), szp, szp]
    lib.s2o_decode.argtypes = [vp] * 7 + [C.POINTER(S2ODecodeParams), vp, vp, vp, st, vp]
    lib.s2o_key_weights_sizes.argtypes = [C.POINTER(S2OWeightsParams), C.c_int, szp, szp]
    lib.s2o_key_weights.argtypes = [vp] * 4 + [C.POINTER(S2OWeightsParams), vp, vp, vp, st, vp]
    lib.s2o_evict_sizes.argtypes = [C.POINTER(S2OEvictParams), szp]
    lib.s2o_evict.argtypes = [vp] * 4 + [C.POINTER(S2OEvictParams), vp, vp, vp, vp, vp, vp, st, vp]
    for name in ("s2o_decode_sizes", "s2o_decode", "s2o_key_weights_sizes", "s2o_key_weights", "s2o_evict_sizes", "s2o_evict"):
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(rc: int):
    if rc != S2O_OK:
        lib = load_library()
        msg = lib.s2o_strerror(rc).decode()
        if rc == S2O_EHIP:
            msg += f" (hipError {lib.s2o_last_hip_error()})"
        raise S2OError(rc, msg)


def make_params(Z, H, Hkv, L, D, S, BM=64, BN=64, use_q_perm=1, stop_mode=0, softmax_scale=0.0,
                q_stride=(0, 0, 0), k_stride=(0, 0, 0), v_stride=(0, 0, 0),
                o_stride=(0, 0, 0), max_prefix_tiles=0, non_causal=0) -> S2OParams:
    p = S2OParams()
    p.struct_size = C.sizeof(S2OParams)
    p.batch, p.q_heads, p.kv_heads, p.seq_len, p.head_dim = Z, H, Hkv, L, D
    p.seg_len, p.block_m, p.block_n = S, BM, BN
    p.use_q_perm, p.stop_mode, p.softmax_scale = use_q_perm, stop_mode, softmax_scale
    p.max_prefix_tiles, p.non_causal = max_prefix_tiles, non_causal
    for name, val in (("q_stride", q_stride), ("k_stride", k_stride), ("v_stride", v_stride),
                      ("o_stride", o_stride)):
        setattr(p, name, (C.c_int64 * 3)(*val))
    return p


def s2o_plan_sizes(params: S2OParams) -> dict:
    lib = load_library()
    v = [C.c_size_t(0) for _ in range(7)]
    _check(lib.s2o_plan_sizes(C.byref(params), *[C.byref(x) for x in v]))
    names = ("q_perm", "kv_perm", "s_q", "s_k", "q_mean", "k_guide", "scratch")
    return {n: int(x.value) for n, x in zip(names, v)}


def s2o_attention_sizes(params: S2OParams) -> dict:
    lib = load_library()
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib.s2o_attention_sizes(C.byref(params), C.byref(a), C.byref(b)))
    return {"counts": int(a.value), "scratch": int(b.value)}


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_STRIDE_OF = {"Q": "q_stride", "K": "k_stride", "V": "v_stride", "O": "o_stride"}


def _check_qkv(params: S2OParams, **tensors):
    """The library sees only pointers: refuse tensors it would silently misread (wrong dtype,
    another device, or a memory layout that params' strides do not describe)."""
    import torch
    bf16, dev = torch.bfloat16, None
    for name, t in tensors.items():
        if t is None:
            continue
        if t.dtype != bf16 or not t.is_cuda:
            raise ValueError(f"{name}: expected a CUDA bfloat16 tensor, got {t.dtype} on {t.device}")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"{name}: on {t.device}, the other tensors on {dev}")
        stride = getattr(params, _STRIDE_OF[name])
        if stride[0] == 0 and stride[1] == 0 and stride[2] == 0:
            if not t.is_contiguous():
                raise ValueError(f"{name}: params describe a packed [Z,heads,L,D] tensor but this one is not "
                                 "contiguous (pass its strides in params or call .contiguous())")
        elif t.stride(-1) != 1:
            raise ValueError(f"{name}: the last dimension must be contiguous")


def _keep_alive_on(stream, *tensors):
    """Buffers allocated here and handed to kernels on a stream other than torch's current one
    must not be recycled by the caching allocator before that stream has passed them."""
    if stream is None:
        return
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _stream_handle(stream, current_device=None) -> Optional[int]:
    import torch
    if stream is None:
        # torch's own entry leaves out the Stream object around the handle (0.3 instead of 2.9 us a call); it is not
        # a public one and need not be there
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(torch.cuda.current_device() if current_device is None else current_device) or None
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


@dataclass
class Plan:
    q_perm: "object"
    kv_perm: "object"
    s_q: "object" = None
    s_k: "object" = None
    q_mean: "object" = None
    k_guide: "object" = None
    status: "object" = None      # int32[1] on the device: 0, or S2O_PLAN_* bits (see s2o.h)


def s2o_plan(Q, K, params: S2OParams, want_scores: bool = True, scratch=None, stream=None,
             maps=None, static_scratch: bool = False) -> Plan:
    """Step 1.  Q, K: torch CUDA bf16 tensors [Z,H,L,D] / [Z,Hkv,L,D].  Returns device
    tensors; the call is asynchronous on the current (or given) torch stream.
    maps: optional (q_perm [Z,H,N,S], kv_perm [Z,H,max(P,4)]) int32 tensors to write into
    (P = entries of the key rows of one head: S*N(N-1)/2, or N*L when params.non_causal).
    static_scratch: call s2o_plan_static (the library's built-in scratch) instead of s2o_plan."""
    import torch
    lib = load_library()
    _check_qkv(params, Q=Q, K=K)
    scratch_bytes = C.c_size_t(0)
    _check(lib.s2o_plan_sizes(C.byref(params), None, None, None, None, None, None, C.byref(scratch_bytes)))
    dev = Q.device
    Z, H, Hkv, L, D, S = (params.batch, params.q_heads, params.kv_heads, params.seq_len,
                          params.head_dim, params.seg_len)
    N = L // S
    P = N * L if params.non_causal else S * N * (N - 1) // 2
    if maps is not None:
        out = Plan(q_perm=maps[0], kv_perm=maps[1])
        if (out.q_perm.numel() != Z * H * N * S or out.kv_perm.numel() != Z * H * max(P, 4)
                or out.q_perm.dtype != torch.int32 or out.kv_perm.dtype != torch.int32):
            raise ValueError("maps: wrong size or dtype")
    else:
        out = Plan(q_perm=torch.empty((Z, H, N, S), dtype=torch.int32, device=dev),
                   kv_perm=torch.empty((Z, H, max(P, 4)), dtype=torch.int32, device=dev))
    if want_scores:
        out.s_q = torch.empty((Z, H, N, S), dtype=torch.float32, device=dev)
        out.s_k = torch.empty((Z, H, max(P, 4)), dtype=torch.float32, device=dev)
        out.q_mean = torch.empty((Z, H, N, D), dtype=torch.float32, device=dev)
        out.k_guide = torch.empty((Z, Hkv, D), dtype=torch.float32, device=dev)
    own_scratch = scratch is None and not static_scratch
    if own_scratch:
        scratch = torch.empty(scratch_bytes.value, dtype=torch.uint8, device=dev)
    out.status = torch.empty(1, dtype=torch.int32, device=dev)
    _keep_alive_on(stream, scratch if own_scratch else None, out.status, out.s_q, out.s_k, out.q_mean, out.k_guide,
                   None if maps is not None else out.q_perm, None if maps is not None else out.kv_perm)
    po = S2OPlanOut(_ptr(out.q_perm), _ptr(out.kv_perm), _ptr(out.s_q), _ptr(out.s_k),
                    _ptr(out.q_mean), _ptr(out.k_guide), _ptr(out.status))
    if static_scratch:
        _check(lib.s2o_plan_static(Q.data_ptr(), K.data_ptr(), C.byref(params), C.byref(po), _stream_handle(stream)))
    else:
        _check(lib.s2o_plan(Q.data_ptr(), K.data_ptr(), C.byref(params), C.byref(po),
                            scratch.data_ptr(), scratch.numel(), _stream_handle(stream)))
    if P < 4 or maps is not None:                # (the buffers hold at least four entries)
        out.kv_perm = out.kv_perm[:, :, :P]
        if out.s_k is not None:
            out.s_k = out.s_k[:, :, :P]
    out._scratch = scratch  # keep alive until the caller synchronises
    return out


def s2o_attention(Q, K, V, params: S2OParams, q_perm, kv_perm, tau: float, O=None,
                  computed=None, skipped=None, stream=None, scratch=None, two_pass=True):
    """Step 2.  Returns (O [Z,H,L,D] bf16, computed, skipped int32 [Z,H,L/B_M]).
    two_pass: launch Alg. 2 and Alg. 3 separately (needs `scratch`, allocated here if not
    given); False: one fused launch."""
    import torch
    lib = load_library()
    _check_qkv(params, Q=Q, K=K, V=V, O=O)
    sz = s2o_attention_sizes(params)
    dev = Q.device
    Z, H, L, D = params.batch, params.q_heads, params.seq_len, params.head_dim
    fresh = []
    if O is None:
        O = torch.empty((Z, H, L, D), dtype=torch.bfloat16, device=dev)
        fresh.append(O)
    if computed is None:
        computed = torch.empty((Z, H, L // params.block_m), dtype=torch.int32, device=dev)
        fresh.append(computed)
    if skipped is None:
        skipped = torch.empty((Z, H, L // params.block_m), dtype=torch.int32, device=dev)
        fresh.append(skipped)
    if two_pass and scratch is None and sz["scratch"] > 0:
        scratch = torch.empty(sz["scratch"], dtype=torch.uint8, device=dev)
        fresh.append(scratch)
    if not two_pass:
        scratch = None
    _keep_alive_on(stream, *fresh)
    _check(lib.s2o_attention(Q.data_ptr(), K.data_ptr(), V.data_ptr(), C.byref(params),
                             _ptr(q_perm), _ptr(kv_perm), float(tau), O.data_ptr(),
                             computed.data_ptr(), skipped.data_ptr(), _ptr(scratch),
                             0 if scratch is None else scratch.numel(), _stream_handle(stream)))
    return O, computed, skipped


def s2o_attention_local(Q, K, V, params: S2OParams, scratch=None, stream=None):
    """Pass 1 (Alg. 2) alone.  Returns the state buffer (uint8 tensor) s2o_attention_prefix reads."""
    import torch
    lib = load_library()
    _check_qkv(params, Q=Q, K=K, V=V)
    if scratch is None:
        scratch = torch.empty(s2o_attention_sizes(params)["scratch"], dtype=torch.uint8, device=Q.device)
        _keep_alive_on(stream, scratch)
    _check(lib.s2o_attention_local(Q.data_ptr(), K.data_ptr(), V.data_ptr(), C.byref(params),
                                   scratch.data_ptr(), scratch.numel(), _stream_handle(stream)))
    return scratch


def s2o_attention_prefix(Q, K, V, params: S2OParams, q_perm, kv_perm, tau: float, scratch, O=None,
                         computed=None, skipped=None, stream=None):
    """Pass 2 (Alg. 3) alone, resuming from the state s2o_attention_local left in `scratch`
    (None when params.non_causal: there is no state)."""
    import torch
    lib = load_library()
    _check_qkv(params, Q=Q, K=K, V=V, O=O)
    dev = Q.device
    Z, H, L, D = params.batch, params.q_heads, params.seq_len, params.head_dim
    fresh = []
    if O is None:
        O = torch.empty((Z, H, L, D), dtype=torch.bfloat16, device=dev)
        fresh.append(O)
    if computed is None:
        computed = torch.empty((Z, H, L // params.block_m), dtype=torch.int32, device=dev)
        fresh.append(computed)
    if skipped is None:
        skipped = torch.empty((Z, H, L // params.block_m), dtype=torch.int32, device=dev)
        fresh.append(skipped)
    _keep_alive_on(stream, *fresh)
    _check(lib.s2o_attention_prefix(Q.data_ptr(), K.data_ptr(), V.data_ptr(), C.byref(params),
                                    _ptr(q_perm), _ptr(kv_perm), float(tau), O.data_ptr(),
                                    computed.data_ptr(), skipped.data_ptr(), _ptr(scratch),
                                    0 if scratch is None else scratch.numel(), _stream_handle(stream)))
    return O, computed, skipped


# ---- the cache behind a prefill: s2o_decode, s2o_key_weights, s2o_evict

def _dtype_code(dtype) -> int:
    """"bf16" / "f16", the torch dtypes, or S2O_BF16 / S2O_F16."""
    code = {"bf16": S2O_BF16, "f16": S2O_F16, "torch.bfloat16": S2O_BF16, "torch.float16": S2O_F16, "0": S2O_BF16, "1": S2O_F16}.get(str(dtype))
    if code is None:
        raise ValueError(f"dtype: expected bf16 or f16, got {dtype}")
    return code


def _filled_struct(p, strides, **fields):
    p.struct_size = C.sizeof(p)
    for name, val in fields.items():
        setattr(p, name, val)
    for name, val in strides.items():
        kind = type(getattr(p, name))
        if len(val) != kind._length_:
            raise ValueError(f"{name}: expected {kind._length_} strides, got {len(val)}")
        setattr(p, name, kind(*val))
    return p


def make_decode_params(Z, B, H, Hkv, D, T, L, own_len=0, dtype="bf16", softmax_scale=0.0, q_stride=(0,) * 4, k_stride=(0,) * 3,
                       v_stride=(0,) * 3, own_k_stride=(0,) * 4, own_v_stride=(0,) * 4, o_stride=(0,) * 4) -> S2ODecodeParams:
    """Z caches of at most L rows, B sequences on each with T query tokens and at most own_len rows of their own."""
    return _filled_struct(S2ODecodeParams(), dict(q_stride=q_stride, k_stride=k_stride, v_stride=v_stride, own_k_stride=own_k_stride,
                                                  own_v_stride=own_v_stride, o_stride=o_stride),
                          batch=Z, branches=B, q_heads=H, kv_heads=Hkv, head_dim=D, q_len=T, cache_len=L, own_len=own_len,
                          dtype=_dtype_code(dtype), softmax_scale=softmax_scale)


def make_weights_params(Z, B, H, Hkv, D, T, L, dtype="bf16", causal=0, softmax_scale=0.0, q_stride=(0,) * 4,
                        k_stride=(0,) * 3) -> S2OWeightsParams:
    """Z caches of at most L rows, T query tokens of B sequences on each."""
    return _filled_struct(S2OWeightsParams(), dict(q_stride=q_stride, k_stride=k_stride),
                          batch=Z, branches=B, q_heads=H, kv_heads=Hkv, head_dim=D, q_len=T, cache_len=L, dtype=_dtype_code(dtype), causal=causal,
                          softmax_scale=softmax_scale)


def make_evict_params(Z, Hkv, D, L, keep, sink=0, recent=0, dtype="bf16", k_stride=(0,) * 3, v_stride=(0,) * 3, out_k_stride=(0,) * 3,
                      out_v_stride=(0,) * 3) -> S2OEvictParams:
    """Z caches of at most L rows that are cut down to at most `keep`."""
    return _filled_struct(S2OEvictParams(), dict(k_stride=k_stride, v_stride=v_stride, out_k_stride=out_k_stride, out_v_stride=out_v_stride),
                          batch=Z, kv_heads=Hkv, head_dim=D, cache_len=L, keep=keep, sink=sink, recent=recent, dtype=_dtype_code(dtype))


def s2o_decode_sizes(params: S2ODecodeParams) -> dict:
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(load_library().s2o_decode_sizes(C.byref(params), C.byref(a), C.byref(b)))
    return {"lse": int(a.value), "scratch": int(b.value)}


def s2o_key_weights_sizes(params: S2OWeightsParams, with_lse: bool = False) -> dict:
    """with_lse: of a call that is given the queries' lse (a call without it needs more)."""
    a, b = C.c_size_t(0), C.c_size_t(0)
    _check(load_library().s2o_key_weights_sizes(C.byref(params), int(with_lse), C.byref(a), C.byref(b)))
    return {"weights": int(a.value), "scratch": int(b.value)}


def s2o_evict_sizes(params: S2OEvictParams) -> dict:
    b = C.c_size_t(0)
    _check(load_library().s2o_evict_sizes(C.byref(params), C.byref(b)))
    return {"scratch": int(b.value)}


@lru_cache(maxsize=64)
def _decode_layout(raw: bytes):
    """What a call with these parameters (by value) takes: {name: (shape, strides or None for packed)}, scratch bytes."""
    p = S2ODecodeParams.from_buffer_copy(raw)
    scratch = s2o_decode_sizes(p)["scratch"]
    q = (p.batch, p.branches, p.q_heads, p.q_len, p.head_dim)
    k, own = (p.batch, p.kv_heads, p.cache_len, p.head_dim), (p.batch, p.branches, p.kv_heads, p.own_len, p.head_dim)
    shapes = dict(Q=q, O=q, K=k, V=k, own_K=own, own_V=own)
    return _with_strides(p, shapes, Q="q", O="o", K="k", V="v", own_K="own_k", own_V="own_v"), _torch_dtype(p.dtype), scratch


@lru_cache(maxsize=64)
def _weights_layout(raw: bytes, with_lse: bool):
    p = S2OWeightsParams.from_buffer_copy(raw)
    scratch = s2o_key_weights_sizes(p, with_lse)["scratch"]
    shapes = dict(Q=(p.batch, p.branches, p.q_heads, p.q_len, p.head_dim), K=(p.batch, p.kv_heads, p.cache_len, p.head_dim))
    return _with_strides(p, shapes, Q="q", K="k"), _torch_dtype(p.dtype), scratch


@lru_cache(maxsize=64)
def _evict_layout(raw: bytes):
    p = S2OEvictParams.from_buffer_copy(raw)
    scratch = s2o_evict_sizes(p)["scratch"]
    k, out = (p.batch, p.kv_heads, p.cache_len, p.head_dim), (p.batch, p.kv_heads, p.keep, p.head_dim)
    return _with_strides(p, dict(K=k, V=k, out_K=out, out_V=out), K="k", V="v", out_K="out_k", out_V="out_v"), _torch_dtype(p.dtype), scratch


def _torch_dtype(code):
    import torch
    return torch.float16 if code == S2O_F16 else torch.bfloat16


def _with_strides(p, shapes, **fields):
    out = {}
    for name, field in fields.items():
        st = tuple(getattr(p, field + "_stride"))
        out[name] = (shapes[name], st if any(st) else None)
    return out


def _check_layout(name, t, dtype, dev, shape, strides=None):
    """The library sees only pointers: a tensor is what the parameters describe, or refused."""
    if t.dtype is not dtype or not t.is_cuda or t.device != dev:
        raise ValueError(f"{name}: expected a {dtype} tensor on {dev}, got {t.dtype} on {t.device}")
    if t.shape != shape:
        raise ValueError(f"{name}: expected the shape {tuple(shape)}, got {tuple(t.shape)}")
    if strides is None:
        if not t.is_contiguous():
            raise ValueError(f"{name}: expected a packed tensor but this one is not contiguous (pass its strides in params or call "
                             ".contiguous())")
        return
    have = t.stride()
    if have[-1] != 1 or any(n > 1 and a != b for n, a, b in zip(shape, have, strides)):
        raise ValueError(f"{name}: params describe the strides {strides}, but this tensor has {have}")


def _on_device(dev, stream):
    """(handle of the stream that the call goes to, context that makes `dev` the current device or None)."""
    import torch
    if stream is not None and getattr(stream, "device", dev) != dev:
        raise ValueError(f"stream: on {stream.device}, the tensors on {dev}")
    current = torch.cuda.current_device()
    if dev.index == current:
        return _stream_handle(stream, current), None
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    return stream.cuda_stream or None, torch.cuda.device(dev)


def _call(fn, ctx, *args):
    if ctx is None:
        return _check(fn(*args))
    with ctx:
        _check(fn(*args))


def _allocate(stream, dev, allocate):
    """allocate() -> tensors for kernels on `stream`, of memory that is free there: what torch's current stream has freed may still
    be in use by it.  The caller may go on with them on the current stream (once that has waited)."""
    import torch
    if stream is None:
        return allocate()
    with torch.cuda.stream(stream):
        tensors = allocate()
    current = torch.cuda.current_stream(dev)
    for t in tensors:
        if t is not None:
            t.record_stream(current)
    return tensors


def _scratch_for(scratch, size, dev, stream):
    import torch
    if scratch is None and size:
        scratch, = _allocate(stream, dev, lambda: (torch.empty(size, dtype=torch.uint8, device=dev),))
    if scratch is not None and (scratch.device != dev or not scratch.is_contiguous()):
        raise ValueError(f"scratch: expected a contiguous tensor on {dev}")
    return scratch, 0 if scratch is None else scratch.numel() * scratch.element_size()


def s2o_decode(Q, K, V, params: S2ODecodeParams, own_K=None, own_V=None, lens=None, own_lens=None, O=None, lse=None, scratch=None,
               stream=None, want_lse: bool = True):
    """Attention of B sequences that share a cache, each with rows of its own behind it.  Q [Z,B,H,T,D]; K, V [Z,Hkv,L,D] or None
    (params.cache_len 0); own_K, own_V [Z,B,Hkv,Lo,D] or None (params.own_len 0); lens [Z], own_lens [Z,B] int32: filled rows,
    None for all.  Query t of T sees the shared rows and the own ones up to own_lens - T + t.
    Returns (O like Q, lse [Z,B,H,T] fp32 or None); asynchronous on the current (or given) torch stream."""
    import torch
    lib = load_library()
    layout, dtype, size = _decode_layout(bytes(params))
    dev = Q.device
    for name, t in (("Q", Q), ("K", K), ("V", V), ("own_K", own_K), ("own_V", own_V), ("O", O)):
        if t is not None:
            _check_layout(name, t, dtype, dev, *layout[name])
    rows = layout["Q"][0][:4]
    for name, t, kind, shape in (("lens", lens, torch.int32, rows[:1]), ("own_lens", own_lens, torch.int32, rows[:2]), ("lse", lse, torch.float32, rows)):
        if t is not None:
            _check_layout(name, t, kind, dev, shape)
    handle, ctx = _on_device(dev, stream)

    def allocate():
        new, new_lse = O, lse
        if new is None:
            shape, strides = layout["O"]
            if strides is None and layout["Q"][1] is None:
                new = torch.empty_like(Q)                # (packed like it; quicker)
            elif strides is None:
                new = torch.empty(shape, dtype=dtype, device=dev)
            else:
                new = torch.empty_strided(shape, strides + (1,), dtype=dtype, device=dev)
        if new_lse is None and want_lse:
            new_lse = torch.empty(rows, dtype=torch.float32, device=dev)
        return new, new_lse

    O, lse = _allocate(stream, dev, allocate)
    scratch, size = _scratch_for(scratch, size, dev, stream)
    _call(lib.s2o_decode, ctx, Q.data_ptr(), _ptr(K), _ptr(V), _ptr(own_K), _ptr(own_V), _ptr(lens), _ptr(own_lens), C.byref(params),
          O.data_ptr(), _ptr(lse), _ptr(scratch), size, handle)
    return O, lse


def s2o_key_weights(Q, K, params: S2OWeightsParams, lse=None, lens=None, prev=None, out=None, scratch=None, stream=None):
    """Softmax weights of a cache's keys added up over query rows: prev + sum exp(scale <q, k> - lse).  Q [Z,B,H,T,D]; K [Z,Hkv,L,D];
    lse [Z,B,H,T] fp32 (as s2o_decode returns it) or None (of the keys a query sees here); lens [Z] int32 or None; prev
    [Z,Hkv,L] fp32 or None; out like it, may be prev itself (entries behind lens are left as they were; without `out` they start at 0).
    Returns out."""
    import torch
    lib = load_library()
    layout, dtype, size = _weights_layout(bytes(params), lse is not None)
    dev = Q.device
    _check_layout("Q", Q, dtype, dev, *layout["Q"])
    _check_layout("K", K, dtype, dev, *layout["K"])
    shape = layout["K"][0][:3]
    for name, t, kind, s in (("lse", lse, torch.float32, layout["Q"][0][:4]), ("lens", lens, torch.int32, shape[:1]), ("prev", prev, torch.float32, shape),
                             ("out", out, torch.float32, shape)):
        if t is not None:
            _check_layout(name, t, kind, dev, s)
    handle, ctx = _on_device(dev, stream)
    if out is None:
        out, = _allocate(stream, dev, lambda: ((torch.empty if lens is None else torch.zeros)(shape, dtype=torch.float32, device=dev),))
    scratch, size = _scratch_for(scratch, size, dev, stream)
    _call(lib.s2o_key_weights, ctx, Q.data_ptr(), K.data_ptr(), _ptr(lse), _ptr(lens), C.byref(params), _ptr(prev), out.data_ptr(),
          _ptr(scratch), size, handle)
    return out


@dataclass
class Evicted:
    K: "object"
    V: "object"
    weights: "object"            # [Z,Hkv,keep] fp32: the kept rows' weights
    kept: "object"               # [Z,Hkv,keep] int32: their indices in the cache, ascending
    lens: "object"               # [Z] int32: rows that are left


def s2o_evict(K, V, weights, params: S2OEvictParams, lens=None, out_K=None, out_V=None, out_weights=None, kept=None, out_lens=None,
              scratch=None, stream=None) -> Evicted:
    """Cuts caches down to the first params.sink, the last params.recent and the otherwise most heavily weighted rows, params.keep in
    all, in the order they had.  K, V [Z,Hkv,L,D] (both None: the selection alone); weights [Z,Hkv,L] fp32; lens [Z] int32 or None.
    Outputs that are given are written into (out_K, out_V [Z,Hkv,keep,D]; rows behind the new lens are left as they were);
    the others are allocated here, undefined behind the new lens."""
    import torch
    lib = load_library()
    layout, dtype, size = _evict_layout(bytes(params))
    dev = weights.device
    if (K is None) != (V is None):
        raise ValueError("K, V: both or neither")
    if K is None and (out_K is not None or out_V is not None):
        raise ValueError("out_K, out_V: nothing to move into them")
    for name, t in (("K", K), ("V", V), ("out_K", out_K), ("out_V", out_V)):
        if t is not None:
            _check_layout(name, t, dtype, dev, *layout[name])
    rows, left = layout["K"][0][:3], layout["out_K"][0][:3]
    for name, t, kind, s in (("weights", weights, torch.float32, rows), ("lens", lens, torch.int32, rows[:1]), ("out_weights", out_weights, torch.float32, left),
                             ("kept", kept, torch.int32, left), ("out_lens", out_lens, torch.int32, rows[:1])):
        if t is not None:
            _check_layout(name, t, kind, dev, s)
    handle, ctx = _on_device(dev, stream)

    def new(t, shape, kind, strides=None):
        if t is not None:
            return t
        return torch.empty(shape, dtype=kind, device=dev) if strides is None else torch.empty_strided(shape, strides + (1,), dtype=kind, device=dev)

    def allocate():
        k = v = None
        if K is not None:
            (moved, ks), (_, vs) = layout["out_K"], layout["out_V"]
            k, v = new(out_K, moved, dtype, ks), new(out_V, moved, dtype, vs)
        return k, v, new(out_weights, left, torch.float32), new(kept, left, torch.int32), new(out_lens, rows[:1], torch.int32)

    out_K, out_V, out_weights, kept, out_lens = _allocate(stream, dev, allocate)
    scratch, size = _scratch_for(scratch, size, dev, stream)
    _call(lib.s2o_evict, ctx, _ptr(K), _ptr(V), weights.data_ptr(), _ptr(lens), C.byref(params), _ptr(out_K), _ptr(out_V), out_weights.data_ptr(),
          kept.data_ptr(), out_lens.data_ptr(), _ptr(scratch), size, handle)
    return Evicted(out_K, out_V, out_weights, kept, out_lens)
