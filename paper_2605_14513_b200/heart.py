"""Thin Python binding of the C ABI in include/heart.h (argument marshalling only).

Every step of the hot path runs in the CUDA kernels of libheart.so; torch is used
for device memory and streams.  Importing this module loads the library and
fails loudly if it has not been built -- there is no CPU or eager fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("HEART_LIB") or os.path.join(_HERE, "libheart.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_CUDA, ERR_DEVICE_CHECK, ERR_TOO_LARGE, ERR_INFEASIBLE = 0, 1, 2, 3, 4, 5, 6
STATIC_SCRATCH_BYTES = 16 << 20
FORCE_REFRESH, FORCE_DENSE, BLOCK_MEANS_VALID, ESTIMATOR_ANTIDIAG = 1, 2, 4, 8
MAX_BLOCKS = 1024
CACHE_BF16, CACHE_E4M3 = 0, 1

# Every symbol include/heart.h declares.
SYMBOLS = (
    "heart_workspace_bytes", "heart_state_reset", "heart_drift", "heart_predict_mask",
    "heart_block_sparse_attn", "heart_step", "heart_step_host", "heart_get_status", "heart_strerror",
    "heart_last_launch_count", "heart_drift_static", "heart_full_token_drift", "heart_mask_iou",
    "heart_band_error_workspace_bytes", "heart_band_error", "heart_drift_workspace_bytes",
    "heart_assign_thresholds", "heart_cache_workspace_bytes", "heart_cache_write", "heart_cache_read", "heart_cache_attn",
    "heart_cache_extend", "heart_cache_release", "heart_cross_workspace_bytes", "heart_cross_attn",
)


class Config(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("N", C.c_int32), ("D", C.c_int32),
                ("block", C.c_int32),
                ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64),
                ("scale", C.c_double), ("gate_lo", C.c_double), ("gate_hi", C.c_double),
                ("idx_stride", C.c_int32), ("flags", C.c_uint32)]


class StateStruct(C.Structure):
    _fields_ = [("anchor_q", C.c_void_p), ("anchor_k", C.c_void_p), ("has_anchor", C.c_void_p),
                ("mask_bits", C.c_void_p), ("kv_idx", C.c_void_p), ("kv_cnt", C.c_void_p)]


class CacheConfig(C.Structure):
    _fields_ = ([(x, C.c_int32) for x in ("S", "T", "Hq", "Hkv", "D", "page", "n_pages", "table_stride", "kind", "max_new", "causal",
                                          "window", "sink")] + [("flags", C.c_uint32)] +
                [(x, C.c_int64) for x in ("q_stride_t", "q_stride_h", "kv_stride_t", "kv_stride_h", "pool_stride_page", "pool_stride_h",
                                          "pool_stride_t")] + [("scale", C.c_double)])


class CacheStruct(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class CrossConfig(C.Structure):
    _fields_ = ([(x, C.c_int32) for x in ("S", "T", "Tk", "Hq", "Hkv", "D", "max_q")] + [("flags", C.c_uint32)] +
                [(x, C.c_int64) for x in ("q_stride_t", "q_stride_h", "kv_stride_t", "kv_stride_h")] + [("scale", C.c_double)])


class HeartError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"heart error {code}: {lib().heart_strerror(code).decode()}")


_lib = None


def lib():
    """The loaded libheart.so (raises if it is missing: build it with build.py)."""
    global _lib
    if _lib is None:
        _lib = load(_LIB_PATH)
    return _lib


def load(path):
    """Loads a build of the library and declares its signatures (the tests use this for the
    test-hook build; everything else goes through lib())."""
    if True:
        if not os.path.exists(path):
            raise ImportError(f"{path} not found: run `python -m paper_2605_14513_b200.build` "
                              "(or __graft_entry__.build()) -- there is no fallback path")
        l = C.CDLL(path)
        l.heart_workspace_bytes.restype = C.c_size_t
        l.heart_workspace_bytes.argtypes = [C.POINTER(Config)]
        l.heart_drift_workspace_bytes.restype = C.c_size_t
        l.heart_drift_workspace_bytes.argtypes = [C.POINTER(Config)]
        l.heart_strerror.restype = C.c_char_p
        l.heart_strerror.argtypes = [C.c_int]
        l.heart_last_launch_count.restype = C.c_int
        vp = C.c_void_p
        l.heart_state_reset.argtypes = [C.POINTER(Config), C.POINTER(StateStruct), vp]
        l.heart_drift.argtypes = [C.POINTER(Config), vp, vp, vp, C.POINTER(StateStruct), vp, vp, vp, vp]
        l.heart_predict_mask.argtypes = [C.POINTER(Config), vp, vp, vp, vp, C.POINTER(StateStruct), vp, vp]
        l.heart_block_sparse_attn.argtypes = [C.POINTER(Config), vp, vp, vp, vp, vp, vp, vp, vp, vp]
        l.heart_step.argtypes = [C.POINTER(Config), vp, vp, vp, vp, vp, C.POINTER(StateStruct), vp, vp, vp, vp, vp, vp]
        l.heart_step_host.argtypes = [C.POINTER(Config), vp, vp, vp, vp, vp, C.POINTER(StateStruct)] + [vp] * 9
        l.heart_get_status.argtypes = [vp, vp, C.POINTER(C.c_int32)]
        l.heart_drift_static.argtypes = [C.POINTER(Config), vp, vp, vp, C.POINTER(StateStruct), vp, vp, vp]
        l.heart_drift_static.restype = C.c_int
        l.heart_full_token_drift.argtypes = [C.POINTER(Config)] + [vp] * 7
        l.heart_full_token_drift.restype = C.c_int
        l.heart_mask_iou.argtypes = [C.POINTER(Config)] + [vp] * 5
        l.heart_mask_iou.restype = C.c_int
        l.heart_band_error_workspace_bytes.argtypes = [C.c_int32] * 4
        l.heart_band_error_workspace_bytes.restype = C.c_size_t
        l.heart_band_error.argtypes = [vp, vp] + [C.c_int32] * 4 + [C.POINTER(C.c_double), C.c_double, vp, vp, vp]
        l.heart_band_error.restype = C.c_int
        l.heart_assign_thresholds.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_double, vp, C.POINTER(C.c_double),
                                              C.POINTER(C.c_double), C.POINTER(C.c_int32)]
        l.heart_assign_thresholds.restype = C.c_int
        l.heart_cache_workspace_bytes.argtypes = [C.POINTER(CacheConfig)]
        l.heart_cache_workspace_bytes.restype = C.c_size_t
        l.heart_cache_write.argtypes = [C.POINTER(CacheConfig), vp, vp, C.POINTER(CacheStruct)] + [vp] * 5
        l.heart_cache_read.argtypes = [C.POINTER(CacheConfig), C.POINTER(CacheStruct)] + [vp] * 7
        l.heart_cache_attn.argtypes = [C.POINTER(CacheConfig), vp, C.POINTER(CacheStruct)] + [vp] * 7
        l.heart_cache_extend.argtypes = [C.POINTER(CacheConfig)] + [vp] * 11
        l.heart_cache_release.argtypes = [C.POINTER(CacheConfig)] + [vp] * 9
        l.heart_cross_workspace_bytes.argtypes = [C.POINTER(CrossConfig)]
        l.heart_cross_workspace_bytes.restype = C.c_size_t
        l.heart_cross_attn.argtypes = [C.POINTER(CrossConfig)] + [vp] * 10
        for fn in ("heart_state_reset", "heart_drift", "heart_predict_mask", "heart_block_sparse_attn",
                   "heart_step", "heart_step_host", "heart_get_status", "heart_cache_write", "heart_cache_read", "heart_cache_attn",
                   "heart_cache_extend", "heart_cache_release", "heart_cross_attn"):
            getattr(l, fn).restype = C.c_int
    return l


def _ptr(t):
    return None if t is None else t.data_ptr()  # (every pointer argument is declared c_void_p)


def _stream():
    # the raw handle: building a torch.cuda.Stream object for it costs as much as a kernel launch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(rc):
    if rc != OK:
        raise HeartError(rc)


def _with_flags(cfg, flags):
    c = Config.from_buffer_copy(cfg)
    c.flags = flags
    return c


def n_blocks(N, block):
    return (N + block - 1) // block


def make_config(B, H, N, block, D=128, scale=0.0, gate_lo=0.0, gate_hi=1.0, idx_stride=None, flags=0,
                strides=(0, 0, 0)) -> Config:
    nb = n_blocks(N, block)
    return Config(B, H, N, D, block, strides[0], strides[1], strides[2], scale, gate_lo, gate_hi,
                  idx_stride if idx_stride is not None else nb, flags)


def config_for(x: torch.Tensor, block, **kw) -> Config:
    """Config for a [B, H, N, D] bf16 tensor (strides taken from the tensor)."""
    assert x.dim() == 4 and x.dtype == torch.bfloat16 and x.stride(3) == 1
    B, H, N, D = x.shape
    return make_config(B, H, N, block, D=D, strides=(x.stride(0), x.stride(1), x.stride(2)), **kw)


class State:
    """Caller-owned TMR state of one layer (device tensors + the C struct that points at them)."""

    def __init__(self, cfg: Config, device="cuda"):
        R, nb = cfg.B * cfg.H, n_blocks(cfg.N, cfg.block)
        self.R, self.nb, self.W = R, nb, (nb + 31) // 32
        self.anchor_q = torch.zeros((R, cfg.D), dtype=torch.float64, device=device)
        self.anchor_k = torch.zeros((R, cfg.D), dtype=torch.float64, device=device)
        self.has_anchor = torch.zeros(R, dtype=torch.uint8, device=device)
        self.mask_bits = torch.zeros((R, nb, self.W), dtype=torch.int32, device=device)
        self.kv_idx = torch.full((R, nb, cfg.idx_stride), -1, dtype=torch.int32, device=device)
        self.kv_cnt = torch.zeros((R, nb), dtype=torch.int32, device=device)
        self.struct = StateStruct(*(t.data_ptr() for t in self.tensors()))

    def tensors(self):
        return (self.anchor_q, self.anchor_k, self.has_anchor, self.mask_bits, self.kv_idx, self.kv_cnt)

    def state_dict(self):
        return {k: getattr(self, k).clone() for k in ("anchor_q", "anchor_k", "has_anchor", "mask_bits", "kv_idx", "kv_cnt")}

    def load_state_dict(self, d):
        for k, v in d.items():
            getattr(self, k).copy_(v)


def workspace_bytes(cfg: Config) -> int:
    return int(lib().heart_workspace_bytes(C.byref(cfg)))


def drift_workspace_bytes(cfg: Config) -> int:
    """The leading part of the workspace that heart_drift alone touches."""
    return int(lib().heart_drift_workspace_bytes(C.byref(cfg)))


def new_workspace(cfg: Config, device="cuda") -> torch.Tensor:
    n = workspace_bytes(cfg)
    if n == 0:
        raise HeartError(ERR_UNSUPPORTED)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def heart_state_reset(cfg, st: State):
    _check(lib().heart_state_reset(C.byref(cfg), C.byref(st.struct), _stream()))


def heart_drift(cfg, Q, K, delta, st: State, ws, drift_out=None, refresh_out=None):
    _check(lib().heart_drift(C.byref(cfg), _ptr(Q), _ptr(K), _ptr(delta), C.byref(st.struct), _ptr(drift_out),
                             _ptr(refresh_out), _ptr(ws), _stream()))


def heart_predict_mask(cfg, Q, K, tau, st: State, ws, refresh=None, means_valid=False):
    """means_valid: pass HEART_BLOCK_MEANS_VALID for this call (heart_drift has just run on the same
    Q, K and workspace), so the pass over Q and K is not repeated."""
    if means_valid:
        cfg = _with_flags(cfg, cfg.flags | BLOCK_MEANS_VALID)
    _check(lib().heart_predict_mask(C.byref(cfg), _ptr(Q), _ptr(K), _ptr(tau), _ptr(refresh), C.byref(st.struct),
                                    _ptr(ws), _stream()))


def heart_block_sparse_attn(cfg, Q, K, V, kv_idx, kv_cnt, O, ws, lse=None):
    _check(lib().heart_block_sparse_attn(C.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(kv_idx), _ptr(kv_cnt),
                                         _ptr(O), _ptr(lse), _ptr(ws), _stream()))


def heart_step(cfg, Q, K, V, delta, tau, st: State, O, ws, lse=None, drift_out=None, refresh_out=None):
    _check(lib().heart_step(C.byref(cfg), _ptr(Q), _ptr(K), _ptr(V), _ptr(delta), _ptr(tau), C.byref(st.struct),
                            _ptr(O), _ptr(lse), _ptr(drift_out), _ptr(refresh_out), _ptr(ws), _stream()))


def heart_step_host(cfg, Qh, Kh, Vh, delta, tau, st: State, Oh, staging, ws, drift_host=None, refresh_host=None):
    """Host-buffer step: Qh/Kh/Vh/Oh (and the optional drift/refresh) are CPU tensors, ideally pinned;
    `staging` = (Q_dev, K_dev, V_dev, O_dev) device tensors.  Asynchronous on the current stream."""
    for t in (Qh, Kh, Vh, Oh):
        assert t.device.type == "cpu" and t.is_contiguous()
    _check(lib().heart_step_host(C.byref(cfg), _ptr(Qh), _ptr(Kh), _ptr(Vh), _ptr(delta), _ptr(tau),
                                 C.byref(st.struct), _ptr(Oh), _ptr(drift_host), _ptr(refresh_host),
                                 _ptr(staging[0]), _ptr(staging[1]), _ptr(staging[2]), _ptr(staging[3]), _ptr(ws),
                                 _stream()))


def heart_drift_static(cfg, Q, K, delta, st: State, drift_out=None, refresh_out=None):
    """heart_drift for callers that cannot allocate: scratch comes from the library's built-in
    16 MiB array (shapes that need more raise ERR_TOO_LARGE).  Calls on one device must not overlap."""
    _check(lib().heart_drift_static(C.byref(cfg), _ptr(Q), _ptr(K), _ptr(delta), C.byref(st.struct),
                                    _ptr(drift_out), _ptr(refresh_out), _stream()))


# ---- A paged cache of keys and values, and attention over it (include/heart.h has the definitions).


def make_cache_config(S, T, Hq, Hkv, page, n_pages, table_stride, kind=CACHE_BF16, D=128, max_new=0, causal=0, window=0, sink=0, scale=0.0,
                      q_strides=(0, 0), kv_strides=(0, 0), pool_strides=(0, 0, 0)) -> CacheConfig:
    """S sequences, T rows of the packed tensors.  max_new, the most new tokens of a sequence, selects the kernel: 0 (not known) is right for any
    lengths, but slow where there are few (say 1 for a step of single tokens).  Strides in elements: (token, head) of Q and O, (token, head) of the
    packed K and V, (page, head, token) of the pools; zeros select the contiguous layouts."""
    return CacheConfig(S, T, Hq, Hkv, D, page, n_pages, table_stride, kind, max_new, causal, window, sink, 0, *q_strides, *kv_strides,
                       *pool_strides, scale)


_cache_fields = struct.Struct("=13iI7qd").unpack_from  # all of a CacheConfig at once: a third of the time of reading it field by field


def _cache_layout(cfg):
    """What a cache's pools depend on: Hkv, D, page, n_pages, kind, and their strides (those of contiguous pools where they are zeros)."""
    f = _cache_fields(cfg)
    Hkv, D, page, n_pages = f[3:7]
    return (Hkv, D, page, n_pages, f[8]) + (f[18:21] if any(f[18:21]) else (Hkv * page * D, page * D, D))


class Cache:
    """Caller-owned pools of a paged cache (device tensors + the C struct that points at them): new ones, zero-filled, or the
    tensors given.  k, v: [n_pages, Hkv, page, D] elements as cfg lays them out, bf16 or float8_e4m3fn; k_scale, v_scale
    (e4m3): uint8 [n_pages, Hkv, page]."""

    def __init__(self, cfg: CacheConfig, k=None, v=None, k_scale=None, v_scale=None, device="cuda"):
        e4m3 = cfg.kind == CACHE_E4M3
        shape = (cfg.n_pages, cfg.Hkv, cfg.page)
        dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16

        def new(*a):
            return torch.zeros(a, dtype=torch.uint8 if e4m3 else dtype, device=device).view(dtype)

        self.k, self.v = (new(*shape, cfg.D) if x is None else x for x in (k, v))
        self.k_scale, self.v_scale = ((torch.zeros(shape, dtype=torch.uint8, device=device) if x is None and e4m3 else x)
                                      for x in (k_scale, v_scale))
        strides = (cfg.pool_stride_page, cfg.pool_stride_h, cfg.pool_stride_t)
        for x in (self.k, self.v):
            plain = (cfg.Hkv * cfg.page * cfg.D, cfg.page * cfg.D, cfg.D)
            if (x.dtype != dtype or tuple(x.shape) != shape + (cfg.D,) or not x.is_cuda or x.device != self.k.device or x.stride(3) != 1 or
                    any(n > 1 and have != want for n, have, want in zip(shape, x.stride(), strides if any(strides) else plain))):
                raise ValueError(f"a pool has to be {dtype} {shape + (cfg.D,)} on a GPU, in cfg's layout: got {x.dtype} {tuple(x.shape)}, strides {x.stride()}")
        for x in (self.k_scale, self.v_scale) if e4m3 else ():
            if x.dtype != torch.uint8 or tuple(x.shape) != shape or x.device != self.k.device or not x.is_contiguous():
                raise ValueError(f"scales have to be contiguous uint8 {shape} beside the pools: got {x.dtype} {tuple(x.shape)}")
        self.device = self.k.get_device()
        self.layout, self.fields = _cache_layout(cfg), _cache_fields(cfg)
        self.struct = CacheStruct(*(None if x is None else x.data_ptr() for x in (self.k, self.v, self.k_scale, self.v_scale)))
        self.ref = C.byref(self.struct)


def cache_workspace_bytes(cfg: CacheConfig) -> int:
    return int(lib().heart_cache_workspace_bytes(C.byref(cfg)))


def new_cache_workspace(cfg: CacheConfig, device="cuda") -> torch.Tensor:
    n = cache_workspace_bytes(cfg)
    if n == 0:
        raise HeartError(ERR_UNSUPPORTED)
    return torch.zeros(n, dtype=torch.uint8, device=device)


@functools.lru_cache(maxsize=256)
def _cache_workspace_bytes(S, T, Hq, Hkv):
    """What the size of a workspace goes by."""
    return cache_workspace_bytes(make_cache_config(S, T, Hq, Hkv, 64, 1, 1))


def _has_strides(x, T, heads, stride_t, stride_h):
    """Whether x can be a packed tensor of these strides: all that they reach is x's, and x, where it is [T, heads, D] or
    [heads, T, D] (behind ones), has them itself."""
    room = x.untyped_storage().nbytes() // x.element_size() - x.storage_offset()
    if x.stride(-1) != 1 or stride_t < 0 or stride_h < 0 or (T - 1) * stride_t + (heads - 1) * stride_h + 128 > room:
        return False
    if x.dim() < 3 or x.shape[-3:].numel() != x.numel():
        return True
    have = tuple(zip(x.shape, x.stride()))[-3:-1]
    return any(all(n == m and (n == 1 or a == b) for (n, a), (m, b) in zip(have, want))
               for want in (((T, stride_t), (heads, stride_h)), ((heads, stride_h), (T, stride_t))))


def _cache_call(cfg, cache, query, tensors, page_table, row_start, kv_len, ws):
    """Checks what the library cannot see (types, sizes, devices).  query: the packed `tensors` are Q and O."""
    device = cache.device
    f = _cache_fields(cfg)
    S, T, Hq, Hkv = f[:4]
    stride_t, stride_h = f[14:16] if query else f[16:18]
    if f != cache.fields and _cache_layout(cfg) != cache.layout:
        raise ValueError("the cache was made for a config with other pools (Hkv, D, page, n_pages, kind or strides)")
    heads = Hq if query else Hkv
    n = T * heads * 128
    for x in tensors:
        if (x.dtype is not torch.bfloat16 or x.numel() != n or x.get_device() != device or
                not (_has_strides(x, T, heads, stride_t, stride_h) if stride_t else x.is_contiguous())):
            raise ValueError(f"packed tensors have to be bf16, {T} rows x {heads} heads x 128, beside the cache, contiguous or with their strides in the "
                             f"config: got {x.dtype} {tuple(x.shape)}, strides {x.stride()}, on {x.device}")
    for x, n in ((page_table, S * f[7]), (row_start, S + 1), (kv_len, S)):
        if x.dtype is not torch.int32 or x.numel() != n or x.get_device() != device or not x.is_contiguous():
            raise ValueError(f"page_table, row_start and kv_len have to be contiguous int32 of {S} x {cfg.table_stride}, {S + 1} and {S} "
                             f"entries beside the cache: got {x.dtype} {tuple(x.shape)} on {x.device}")
    if ws.get_device() != device or not ws.is_contiguous() or ws.nbytes < _cache_workspace_bytes(S, T, Hq, Hkv):
        raise ValueError(f"the workspace has to have cache_workspace_bytes(cfg) = {cache_workspace_bytes(cfg)} bytes beside the cache")


def _launch(call, device, *args):
    """The call on the device's current stream."""
    if device == torch._C._cuda_getDevice():
        rc = call(*args, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            rc = call(*args, torch._C._cuda_getCurrentRawStream(device))
    if rc != OK:
        raise HeartError(rc)


def heart_cache_write(cfg, K, V, cache: Cache, page_table, row_start, kv_len, ws):
    """Stores the packed rows of K and V (bf16 [T, Hkv, D]), the last tokens of their sequences, in their pages."""
    _cache_call(cfg, cache, False, (K, V), page_table, row_start, kv_len, ws)
    _launch(lib().heart_cache_write, cache.device, C.byref(cfg), K.data_ptr(), V.data_ptr(), cache.ref, page_table.data_ptr(), row_start.data_ptr(),
            kv_len.data_ptr(), ws.data_ptr())


def heart_cache_read(cfg, cache: Cache, page_table, row_start, kv_len, K_out, V_out, ws):
    """The last tokens of the sequences out of their pages into the packed rows of K_out and V_out (bf16 [T, Hkv, D])."""
    _cache_call(cfg, cache, False, (K_out, V_out), page_table, row_start, kv_len, ws)
    _launch(lib().heart_cache_read, cache.device, C.byref(cfg), cache.ref, page_table.data_ptr(), row_start.data_ptr(), kv_len.data_ptr(),
            K_out.data_ptr(), V_out.data_ptr(), ws.data_ptr())


def heart_cache_attn(cfg, Q, cache: Cache, page_table, row_start, kv_len, O, ws, lse=None):
    """Attention of the packed rows of Q (bf16 [T, Hq, D]), the last tokens of their sequences, over the sequences' pages
    into O; lse: optional fp32 [T, Hq]."""
    _cache_call(cfg, cache, True, (Q, O), page_table, row_start, kv_len, ws)
    if lse is not None and (lse.dtype is not torch.float32 or lse.numel() != cfg.T * cfg.Hq or lse.get_device() != cache.device or not lse.is_contiguous()):
        raise ValueError(f"lse has to be contiguous fp32 [{cfg.T}, {cfg.Hq}] beside the cache: got {lse.dtype} {tuple(lse.shape)} on {lse.device}")
    _launch(lib().heart_cache_attn, cache.device, C.byref(cfg), Q.data_ptr(), cache.ref, page_table.data_ptr(), row_start.data_ptr(), kv_len.data_ptr(),
            O.data_ptr(), _ptr(lse), ws.data_ptr())


def _table_call(fields, names, tensors, sizes, ws):
    """Checks the int32 arrays of a table call and the workspace: on one device, which it returns."""
    device, i32 = ws.get_device(), torch.int32
    for x, n in zip(tensors, sizes):
        if x.dtype is not i32 or x.numel() != n or x.get_device() != device or not x.is_contiguous():
            name = names.split()[next(i for i, y in enumerate(tensors) if y is x)]
            raise ValueError(f"{name} has to be contiguous {i32} of {n} entries beside the workspace: got {x.dtype} {tuple(x.shape)} on {x.device}")
    if device < 0 or not ws.is_contiguous() or ws.nbytes < _cache_workspace_bytes(*fields[:4]):
        raise ValueError(f"the workspace has to have cache_workspace_bytes(cfg) = {_cache_workspace_bytes(*fields[:4])} bytes on a GPU")
    return device


def heart_cache_extend(cfg, new_len, kv_len, free_pages, free_count, page_table, row_start, ws, slots=None, kv_len_out=None, free_count_out=None):
    """Gives the sequences (kv_len: int32 [S]) pages for new_len more tokens from the stack free_pages (int32 [n_pages], free_count [1] of them) and
    writes page_table, row_start and, if given, slots (int64 [T]).  Lengths and count go to kv_len_out and free_count_out, or are updated in place."""
    f = _cache_fields(cfg)
    S = f[0]
    tensors = (new_len, kv_len, free_pages, free_count, page_table, row_start, kv_len if kv_len_out is None else kv_len_out,
               free_count if free_count_out is None else free_count_out)
    device = _table_call(f, "new_len kv_len free_pages free_count page_table row_start kv_len_out free_count_out", tensors,
                         (S, S, f[6], 1, S * f[7], S + 1, S, 1), ws)
    if slots is not None and (slots.dtype is not torch.int64 or slots.numel() != f[1] or slots.get_device() != device or not slots.is_contiguous()):
        raise ValueError(f"slots has to be contiguous {torch.int64} of {f[1]} entries beside the workspace: got {slots.dtype} {tuple(slots.shape)} on {slots.device}")
    _launch(lib().heart_cache_extend, device, C.byref(cfg), *[x.data_ptr() for x in tensors], _ptr(slots), ws.data_ptr())


def heart_cache_release(cfg, ended, kv_len, free_pages, free_count, page_table, ws, kv_len_out=None, free_count_out=None):
    """Puts the pages of the sequences with ended (uint8 [S]) back on the stack; lengths (0 for those) and count as in heart_cache_extend."""
    f = _cache_fields(cfg)
    S = f[0]
    tensors = (kv_len, free_pages, free_count, page_table, kv_len if kv_len_out is None else kv_len_out, free_count if free_count_out is None else free_count_out)
    device = _table_call(f, "kv_len free_pages free_count page_table kv_len_out free_count_out", tensors, (S, f[6], 1, S * f[7], S, 1), ws)
    if ended.dtype is not torch.uint8 or ended.numel() != S or ended.get_device() != device or not ended.is_contiguous():
        raise ValueError(f"ended has to be contiguous {torch.uint8} of {S} entries beside the workspace: got {ended.dtype} {tuple(ended.shape)} on {ended.device}")
    _launch(lib().heart_cache_release, device, C.byref(cfg), ended.data_ptr(), *[x.data_ptr() for x in tensors], ws.data_ptr())


# ---- Cross attention: to states of another length.


def make_cross_config(S, T, Tk, Hq, Hkv, max_q=0, D=128, scale=0.0, q_strides=(0, 0), kv_strides=(0, 0)) -> CrossConfig:
    """S sequences, T rows of Q and O, Tk rows of K and V.  max_q, the most queries of a sequence, selects the kernel: 0 (not known) is right for
    any lengths, but slow where there are few (say 1 for a step of single tokens).  Strides in elements: (token, head) of Q and O, and of K and V; zeros
    select the contiguous layouts."""
    return CrossConfig(S, T, Tk, Hq, Hkv, D, max_q, 0, *q_strides, *kv_strides, scale)


def cross_workspace_bytes(cfg: CrossConfig) -> int:
    return int(lib().heart_cross_workspace_bytes(C.byref(cfg)))


def new_cross_workspace(cfg: CrossConfig, device="cuda") -> torch.Tensor:
    n = cross_workspace_bytes(cfg)
    if n == 0:
        raise HeartError(ERR_UNSUPPORTED)
    return torch.zeros(n, dtype=torch.uint8, device=device)


_cross_fields = struct.Struct("=7iI4qd").unpack_from


@functools.lru_cache(maxsize=1)
def _cross_workspace_bytes():
    """(It has one size.)"""
    return cross_workspace_bytes(make_cross_config(1, 1, 1, 1, 1))


def heart_cross_attn(cfg, Q, K, V, q_start, k_start, k_len, O, ws, lse=None):
    """Attention of the packed rows of Q (bf16 [T, Hq, D], sequence s from q_start[s] to q_start[s + 1]) over the rows k_start[s] .. + k_len[s]
    of K and V (bf16 [Tk, Hkv, D]) into O; lse: optional fp32 [T, Hq].  q_start, k_start, k_len: int32 on the GPU, [S + 1], [S], [S]."""
    S, T, Tk, Hq, Hkv, _, _, _, qt, qh, kt, kh, _ = _cross_fields(cfg)
    device = Q.get_device()
    for x, rows, heads, t, h in ((Q, T, Hq, qt, qh), (O, T, Hq, qt, qh), (K, Tk, Hkv, kt, kh), (V, Tk, Hkv, kt, kh)):
        if (x.dtype is not torch.bfloat16 or x.numel() != rows * heads * 128 or x.get_device() != device or
                not (_has_strides(x, rows, heads, t, h) if t else x.is_contiguous())):
            raise ValueError(f"packed tensors have to be bf16, {rows} rows x {heads} heads x 128, on one GPU, contiguous or with their strides in the "
                             f"config: got {x.dtype} {tuple(x.shape)}, strides {x.stride()}, on {x.device}")
    for x, n in ((q_start, S + 1), (k_start, S), (k_len, S)):
        if x.dtype is not torch.int32 or x.numel() != n or x.get_device() != device or not x.is_contiguous():
            raise ValueError(f"q_start, k_start and k_len have to be contiguous int32 of {S + 1}, {S} and {S} entries beside Q: got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
    if lse is not None and (lse.dtype is not torch.float32 or lse.numel() != T * Hq or lse.get_device() != device or not lse.is_contiguous()):
        raise ValueError(f"lse has to be contiguous fp32 [{T}, {Hq}] beside Q: got {lse.dtype} {tuple(lse.shape)} on {lse.device}")
    if device < 0 or ws.get_device() != device or not ws.is_contiguous() or ws.nbytes < _cross_workspace_bytes():
        raise ValueError(f"the workspace has to have cross_workspace_bytes(cfg) = {cross_workspace_bytes(cfg)} bytes beside Q, on a GPU")
    _launch(lib().heart_cross_attn, device, C.byref(cfg), Q.data_ptr(), K.data_ptr(), V.data_ptr(), q_start.data_ptr(), k_start.data_ptr(),
            k_len.data_ptr(), O.data_ptr(), _ptr(lse), ws.data_ptr())


def heart_full_token_drift(cfg, Qa, Ka, Qb, Kb, drift_out, ws):
    """Full-token drift (Eq. full-token drift) between a cached step (Qa, Ka) and the current one
    (Qb, Kb) into drift_out [R] fp64."""
    _check(lib().heart_full_token_drift(C.byref(cfg), _ptr(Qa), _ptr(Ka), _ptr(Qb), _ptr(Kb), _ptr(drift_out),
                                        _ptr(ws), _stream()))


def heart_mask_iou(cfg, mask_a, mask_b, iou_out, counts_out=None):
    """Block-mask IoU per head between two [R, n_b, W] bit masks (Observation I) into iou_out [R] fp64;
    counts_out: optional int64 [R, 2] = (intersection, union)."""
    _check(lib().heart_mask_iou(C.byref(cfg), _ptr(mask_a), _ptr(mask_b), _ptr(iou_out), _ptr(counts_out),
                                _stream()))


def heart_band_error(y_sparse, y_dense, weights=(1.0, 0.5, 0.01, 0.01), eps=1e-10):
    """Four-band 3-D DFT calibration error of y_sparse against y_dense (fp32 [C, T, H, W] on the GPU).
    Returns a device tensor of 6 doubles: (e, E_LL, E_LH, E_HL, E_HH, denominator)."""
    assert y_sparse.dtype == torch.float32 and y_dense.dtype == torch.float32
    assert y_sparse.is_contiguous() and y_dense.is_contiguous() and y_sparse.shape == y_dense.shape
    Cc, T, H, W = y_sparse.shape
    nbytes = lib().heart_band_error_workspace_bytes(Cc, T, H, W)
    if nbytes == 0:
        raise HeartError(ERR_INVALID)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=y_sparse.device)
    out = torch.empty(6, dtype=torch.float64, device=y_sparse.device)
    w = (C.c_double * 4)(*weights)
    _check(lib().heart_band_error(_ptr(y_sparse), _ptr(y_dense), Cc, T, H, W, w, float(eps), _ptr(out), _ptr(ws),
                                  _stream()))
    return out


def heart_assign_thresholds(E, S, S_min):
    """One threshold candidate per head under a mean-sparsity budget (host-side, exact).
    E, S: [n_heads, n_candidates] float64 numpy arrays.  Returns (choice int32 [n_heads], objective,
    mean sparsity, proved_optimal) or None when no assignment meets the budget."""
    import numpy as np

    E = np.ascontiguousarray(E, np.float64)
    S = np.ascontiguousarray(S, np.float64)
    M, K = E.shape
    assert S.shape == (M, K)
    choice = np.empty(M, np.int32)
    obj, ms, proved = C.c_double(0), C.c_double(0), C.c_int32(0)
    rc = lib().heart_assign_thresholds(E.ctypes.data_as(C.c_void_p), S.ctypes.data_as(C.c_void_p), M, K,
                                       float(S_min), choice.ctypes.data_as(C.c_void_p), C.byref(obj), C.byref(ms),
                                       C.byref(proved))
    if rc == ERR_INFEASIBLE:
        return None
    _check(rc)
    return choice, obj.value, ms.value, bool(proved.value)


def heart_get_status(ws) -> int:
    code = C.c_int32(0)
    _check(lib().heart_get_status(_ptr(ws), _stream(), C.byref(code)))
    return code.value


def heart_last_launch_count() -> int:
    return int(lib().heart_last_launch_count())
