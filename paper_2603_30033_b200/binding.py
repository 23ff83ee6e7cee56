"""Thin ctypes binding of libtucker_attn.so (the C ABI declared in include/tucker_attn.h).

Only argument marshalling happens here: tensors are checked for device / dtype / contiguity,
their pointers and the current CUDA stream are handed to the library, and every step of the
computation runs in the library's kernels.  torch is used for device memory and streams
only.  If the library has not been built, loading raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
# TUCKER_ATTN_LIB=checked selects the twin built with -DTA_BOUNDS_CHECK (device-side range checks on every
# global index, reported through the device error word); anything else, or nothing, the normal library.
LIB_PATH = os.path.join(_HERE, "libtucker_attn_checked.so" if os.environ.get("TUCKER_ATTN_LIB") == "checked"
                        else "libtucker_attn.so")

TA_OK = 0
TA_DTYPE_F32, TA_DTYPE_BF16 = 0, 1
TA_FLAG_FORCE_GENERIC = 1
TA_WORKSPACE_NONE = 1           # a workspace query's answer: the call needs none
TA_FLAG_FMA_ATTENTION, TA_FLAG_SEPARATE_QUERIES, TA_FLAG_SEPARATE_OUTPUT_GEMMS = 0x200, 0x400, 0x800
TA_DEVERR_WAIT_TIMEOUT, TA_DEVERR_BAD_CACHE_LEN, TA_DEVERR_BAD_INDEX, TA_DEVERR_BAD_PAGE = 1, 2, 4, 8

EXPORTS = (
    "tucker_attn_fwd_workspace_bytes", "tucker_attn_decode_workspace_bytes", "tucker_attn_fwd",
    "tucker_attn_decode", "tucker_attn_status_string", "tucker_attn_last_device_error",
    "tucker_attn_last_path", "tucker_attn_last_launch_count", "tucker_attn_set_profile_events",
    "tucker_attn_decode_static", "tucker_attn_selftest_wait_timeout", "tucker_attn_sync_status",
    "tucker_attn_bounds_checked", "tucker_attn_selftest_cluster_wait",
    "tucker_cache_append_paged", "tucker_cache_append_paged_workspace_bytes", "tucker_attn_decode_paged", "tucker_attn_decode_paged_workspace_bytes",
    "tucker_attn_decode_prefix", "tucker_attn_decode_prefix_workspace_bytes",
    "tucker_cache_append_paged_q8", "tucker_cache_append_paged_q8_workspace_bytes", "tucker_cache_store_paged_q8",
    "tucker_cache_read_paged_q8", "tucker_attn_decode_paged_q8", "tucker_attn_decode_paged_q8_workspace_bytes",
    "tucker_attn_decode_prefix_q8", "tucker_attn_decode_prefix_q8_workspace_bytes",
    "tucker_pack_gqa", "tucker_pack_mha", "tucker_pack_mla",
    "tucker_hosvd_workspace_bytes", "tucker_hosvd_init", "tucker_mha_weight_tensors", "tucker_probe_plane_mix", "tucker_probe_mma_rate",
)
TA_STATIC_SCRATCH_BYTES = 16 << 20


class TuckerAttnDesc(ctypes.Structure):
    """Mirror of `tucker_attn_desc`."""
    _fields_ = [
        ("B", ctypes.c_int32), ("N", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_H", ctypes.c_int32),
        ("r1", ctypes.c_int32), ("r2", ctypes.c_int32), ("r3", ctypes.c_int32),
        ("t1", ctypes.c_int32), ("t2", ctypes.c_int32), ("t3", ctypes.c_int32),
        ("causal", ctypes.c_int32), ("rope", ctypes.c_int32), ("rope_base", ctypes.c_float),
        ("pos0", ctypes.c_int32), ("scale", ctypes.c_float), ("dtype", ctypes.c_int32),
        ("flags", ctypes.c_int32),
    ]


class TuckerPagedCache(ctypes.Structure):
    """Mirror of `tucker_paged_cache`."""
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
        ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
    ]


class TuckerPagedCacheQ8(ctypes.Structure):
    """Mirror of `tucker_paged_cache_q8`."""
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("Ks", ctypes.c_void_p), ("Vs", ctypes.c_void_p),
        ("block_table", ctypes.c_void_p),
        ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
    ]


class TuckerAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where} failed: {status_string(status)} ({status})")


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2603_30033_b200.build` "
            "(needs nvcc); this package has no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(TuckerAttnDesc)
    lib.tucker_attn_fwd_workspace_bytes.restype = sz
    lib.tucker_attn_fwd_workspace_bytes.argtypes = [dp]
    lib.tucker_attn_decode_workspace_bytes.restype = sz
    lib.tucker_attn_decode_workspace_bytes.argtypes = [dp, i32]
    lib.tucker_attn_fwd.restype = ctypes.c_int
    lib.tucker_attn_fwd.argtypes = [dp] + [vp] * 12 + [i32, vp, sz, vp]
    lib.tucker_attn_decode.restype = ctypes.c_int
    lib.tucker_attn_decode.argtypes = [dp] + [vp] * 11 + [i32, vp, i32, vp, vp, sz, vp]
    lib.tucker_attn_decode_static.restype = ctypes.c_int
    lib.tucker_attn_decode_static.argtypes = [dp] + [vp] * 11 + [i32, vp, i32, vp, vp]
    # descriptor and cache by address: packed bytes or a structure by reference
    lib.tucker_cache_append_paged.restype = ctypes.c_int
    lib.tucker_cache_append_paged.argtypes = [vp] + [vp] * 3 + [vp, vp, vp, i32, vp, sz, vp]
    lib.tucker_cache_append_paged_workspace_bytes.restype = sz
    lib.tucker_cache_append_paged_workspace_bytes.argtypes = [vp, vp, i32]
    lib.tucker_attn_decode_paged_workspace_bytes.restype = sz
    lib.tucker_attn_decode_paged_workspace_bytes.argtypes = [vp, vp]
    lib.tucker_attn_decode_paged.restype = ctypes.c_int
    lib.tucker_attn_decode_paged.argtypes = [vp] + [vp] * 9 + [vp, vp, i32, vp, vp, sz, vp]
    lib.tucker_attn_decode_prefix_workspace_bytes.restype = sz
    lib.tucker_attn_decode_prefix_workspace_bytes.argtypes = [vp, vp, i32]
    lib.tucker_attn_decode_prefix.restype = ctypes.c_int
    lib.tucker_attn_decode_prefix.argtypes = [vp] + [vp] * 9 + [vp, vp, vp, i32, i32, vp, vp, sz, vp]
    for name in ("cache_append_paged", "attn_decode_paged", "attn_decode_prefix"):       # the 8-bit cache's: the same arguments
        for tail in ("", "_workspace_bytes"):
            q8, like = getattr(lib, f"tucker_{name}_q8{tail}"), getattr(lib, f"tucker_{name}{tail}")
            q8.restype, q8.argtypes = like.restype, like.argtypes
    lib.tucker_cache_store_paged_q8.restype = ctypes.c_int
    lib.tucker_cache_store_paged_q8.argtypes = [vp] * 6 + [i32, vp]
    lib.tucker_cache_read_paged_q8.restype = ctypes.c_int
    lib.tucker_cache_read_paged_q8.argtypes = [vp] * 4 + [i32, vp, vp, vp]
    lib.tucker_attn_status_string.restype = ctypes.c_char_p
    lib.tucker_attn_status_string.argtypes = [ctypes.c_int]
    lib.tucker_attn_last_device_error.restype = ctypes.c_int
    lib.tucker_attn_last_device_error.argtypes = [vp]
    lib.tucker_attn_sync_status.restype = ctypes.c_int
    lib.tucker_attn_sync_status.argtypes = [vp]
    lib.tucker_attn_bounds_checked.restype = ctypes.c_int
    lib.tucker_attn_last_path.restype = ctypes.c_int
    lib.tucker_attn_last_launch_count.restype = ctypes.c_int
    lib.tucker_attn_set_profile_events.restype = ctypes.c_int
    lib.tucker_attn_set_profile_events.argtypes = [vp, vp]
    lib.tucker_attn_selftest_wait_timeout.restype = ctypes.c_int
    lib.tucker_attn_selftest_wait_timeout.argtypes = [i32, vp, vp]
    lib.tucker_attn_selftest_cluster_wait.restype = ctypes.c_int
    lib.tucker_attn_selftest_cluster_wait.argtypes = [i32, vp, vp]
    lib.tucker_pack_gqa.restype = ctypes.c_int
    lib.tucker_pack_gqa.argtypes = [i32] * 4 + [vp] * 13
    lib.tucker_pack_mha.restype = ctypes.c_int
    lib.tucker_pack_mha.argtypes = [i32] * 3 + [vp] * 13
    lib.tucker_pack_mla.restype = ctypes.c_int
    lib.tucker_pack_mla.argtypes = [i32] * 5 + [vp] * 16
    lib.tucker_hosvd_workspace_bytes.restype = sz
    lib.tucker_hosvd_workspace_bytes.argtypes = [i32] * 4
    lib.tucker_hosvd_init.restype = ctypes.c_int
    lib.tucker_hosvd_init.argtypes = [i32] * 5 + [vp] * 7 + [sz, vp]
    lib.tucker_mha_weight_tensors.restype = ctypes.c_int
    lib.tucker_mha_weight_tensors.argtypes = [i32] * 2 + [vp] * 7
    lib.tucker_probe_mma_rate.restype = ctypes.c_int
    lib.tucker_probe_mma_rate.argtypes = [i32] * 4 + [vp] * 2
    lib.tucker_probe_plane_mix.restype = ctypes.c_int
    lib.tucker_probe_plane_mix.argtypes = [i32] * 3 + [vp] * 4
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().tucker_attn_status_string(int(status)).decode()


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return TA_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return TA_DTYPE_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")


def _check(t, name, shape, dtype, device):
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.device == device and t.is_contiguous():
        return
    if t.device != device or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def make_desc(*, B, N, d_model, n_H, r, t, causal, rope, rope_base=10000.0, pos0=0, scale=0.0,
              dtype=TA_DTYPE_BF16, flags=0) -> TuckerAttnDesc:
    return TuckerAttnDesc(int(B), int(N), int(d_model), int(n_H), int(r[0]), int(r[1]), int(r[2]),
                          int(t[0]), int(t[1]), int(t[2]), int(bool(causal)), int(bool(rope)),
                          float(rope_base), int(pos0), float(scale), int(dtype), int(flags))


def fwd_workspace_bytes(desc: TuckerAttnDesc) -> int:
    return int(load_library().tucker_attn_fwd_workspace_bytes(ctypes.byref(desc)))


def decode_workspace_bytes(desc: TuckerAttnDesc, Lmax: int) -> int:
    return int(load_library().tucker_attn_decode_workspace_bytes(ctypes.byref(desc), int(Lmax)))


def alloc_workspace(nbytes: int, device):
    """Device scratch buffer (256-byte aligned by the torch allocator)."""
    torch = _torch()
    return torch.empty(nbytes if nbytes > 256 else 256, dtype=torch.uint8, device=device)


def _enter_device(cuda, device):
    """Makes `device` current if it is not, and returns what to leave afterwards (None: nothing).  `with torch.cuda.device(device)`
    around every call costs several microseconds."""
    if cuda.current_device() == device.index:
        return None
    ctx = cuda.device(device)
    ctx.__enter__()
    return ctx


def _stream_ptr(device) -> int:
    raw = getattr(_torch()._C, "_cuda_getCurrentRawStream", None)      # the handle alone, without a Stream object around it
    if raw is not None and device.index is not None:
        return int(raw(device.index))
    return int(_torch().cuda.current_stream(device).cuda_stream)


def _weights_check(w, d_model, n_H, dtype, device):
    C, U1, U2, U3, Ct, Ut1, Ut2, Ut3 = w
    if C.dim() != 3 or Ct.dim() != 3:
        raise ValueError("cores must be 3-way tensors")
    r = tuple(C.shape)
    t = tuple(Ct.shape)
    _check(C, "C", r, dtype, device)
    _check(U1, "U1", (n_H, r[0]), dtype, device)
    _check(U2, "U2", (d_model, r[1]), dtype, device)
    _check(U3, "U3", (d_model, r[2]), dtype, device)
    _check(Ct, "Ct", t, dtype, device)
    _check(Ut1, "Ut1", (n_H, t[0]), dtype, device)
    _check(Ut2, "Ut2", (d_model, t[1]), dtype, device)
    _check(Ut3, "Ut3", (d_model, t[2]), dtype, device)
    return r, t


def tucker_attn_fwd(X, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, *, n_H: int, causal: bool, rope: bool,
                    rope_base: float = 10000.0, pos0: int = 0, scale: float = 0.0, out=None,
                    Kcache=None, Vcache=None, workspace=None, flags: int = 0):
    """Prefill forward (same name and argument meaning as the C entry point).  X [B, N, d];
    returns Y [B, N, d].  Kcache [B, Lmax, r3] / Vcache [B, Lmax, t3], when given, receive the
    rotated latent keys and the latent values in rows 0..N-1."""
    torch = _torch()
    lib = load_library()
    if X.dim() != 3:
        raise ValueError("X must be [B, N, d_model]")
    B, N, d = X.shape
    dev, dt = X.device, X.dtype
    _check(X, "X", (B, N, d), dt, dev)
    r, t = _weights_check((C, U1, U2, U3, Ct, Ut1, Ut2, Ut3), d, n_H, dt, dev)
    desc = make_desc(B=B, N=N, d_model=d, n_H=n_H, r=r, t=t, causal=causal, rope=rope, rope_base=rope_base,
                     pos0=pos0, scale=scale, dtype=_dtype_code(X), flags=flags)
    if out is None:
        out = torch.empty_like(X)
    _check(out, "out", (B, N, d), dt, dev)
    Lmax = 0
    kp = vp = None
    if (Kcache is None) != (Vcache is None):
        raise ValueError("pass both caches or neither")
    if Kcache is not None:
        Lmax = Kcache.shape[1]
        _check(Kcache, "Kcache", (B, Lmax, r[2]), dt, dev)
        _check(Vcache, "Vcache", (B, Lmax, t[2]), dt, dev)
        kp, vp = Kcache.data_ptr(), Vcache.data_ptr()
    need = lib.tucker_attn_fwd_workspace_bytes(ctypes.byref(desc))
    if workspace is None:
        workspace = alloc_workspace(need, dev)
    with torch.cuda.device(dev):
        rc = lib.tucker_attn_fwd(ctypes.byref(desc), X.data_ptr(), C.data_ptr(), U1.data_ptr(), U2.data_ptr(),
                                 U3.data_ptr(), Ct.data_ptr(), Ut1.data_ptr(), Ut2.data_ptr(), Ut3.data_ptr(),
                                 out.data_ptr(), kp, vp, int(Lmax), workspace.data_ptr(), workspace.numel(),
                                 _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_fwd")
    return out


def tucker_attn_decode(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kcache, Vcache, cache_len, *, n_H: int,
                       rope: bool, rope_base: float = 10000.0, scale: float = 0.0, append: bool = True,
                       out=None, workspace=None, flags: int = 0):
    """One cached decode step (same name and argument meaning as the C entry point).
    x [B, d]; Kcache [B, Lmax, r3] (rotated keys); Vcache [B, Lmax, t3]; cache_len int32 [B] on
    the device.  Returns y [B, d]."""
    torch = _torch()
    lib = load_library()
    if x.dim() != 2:
        raise ValueError("x must be [B, d_model]")
    B, d = x.shape
    dev, dt = x.device, x.dtype
    _check(x, "x", (B, d), dt, dev)
    r, t = _weights_check((C, U1, U2, U3, Ct, Ut1, Ut2, Ut3), d, n_H, dt, dev)
    Lmax = Kcache.shape[1]
    _check(Kcache, "Kcache", (B, Lmax, r[2]), dt, dev)
    _check(Vcache, "Vcache", (B, Lmax, t[2]), dt, dev)
    _check(cache_len, "cache_len", (B,), torch.int32, dev)
    desc = make_desc(B=B, N=1, d_model=d, n_H=n_H, r=r, t=t, causal=True, rope=rope, rope_base=rope_base,
                     pos0=0, scale=scale, dtype=_dtype_code(x), flags=flags)
    if out is None:
        out = torch.empty_like(x)
    _check(out, "out", (B, d), dt, dev)
    need = lib.tucker_attn_decode_workspace_bytes(ctypes.byref(desc), int(Lmax))
    if workspace is None:
        workspace = alloc_workspace(need, dev)
    with torch.cuda.device(dev):
        rc = lib.tucker_attn_decode(ctypes.byref(desc), x.data_ptr(), C.data_ptr(), U1.data_ptr(), U2.data_ptr(),
                                    U3.data_ptr(), Ct.data_ptr(), Ut1.data_ptr(), Ut2.data_ptr(), Ut3.data_ptr(),
                                    Kcache.data_ptr(), Vcache.data_ptr(), int(Lmax), cache_len.data_ptr(),
                                    int(bool(append)), out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                    _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_decode")
    return out


def tucker_attn_decode_static(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kcache, Vcache, cache_len, out, *, n_H: int,
                              rope: bool, rope_base: float = 10000.0, scale: float = 0.0, append: bool = True,
                              flags: int = 0):
    """Decode step for callers that cannot allocate: same arguments and result as
    tucker_attn_decode, but the output tensor `out` [B, d] is mandatory and no workspace is
    passed -- the library uses its built-in static scratch array (TA_STATIC_SCRATCH_BYTES).
    Neither this wrapper nor the C entry point allocates device memory.  Raises
    TuckerAttnError("workspace too small") when the problem needs more scratch than that.
    Calls share the one array: do not let two of them overlap on the GPU."""
    torch = _torch()
    lib = load_library()
    if x.dim() != 2:
        raise ValueError("x must be [B, d_model]")
    B, d = x.shape
    dev, dt = x.device, x.dtype
    _check(x, "x", (B, d), dt, dev)
    r, t = _weights_check((C, U1, U2, U3, Ct, Ut1, Ut2, Ut3), d, n_H, dt, dev)
    Lmax = Kcache.shape[1]
    _check(Kcache, "Kcache", (B, Lmax, r[2]), dt, dev)
    _check(Vcache, "Vcache", (B, Lmax, t[2]), dt, dev)
    _check(cache_len, "cache_len", (B,), torch.int32, dev)
    _check(out, "out", (B, d), dt, dev)
    desc = make_desc(B=B, N=1, d_model=d, n_H=n_H, r=r, t=t, causal=True, rope=rope, rope_base=rope_base,
                     pos0=0, scale=scale, dtype=_dtype_code(x), flags=flags)
    with torch.cuda.device(dev):
        rc = lib.tucker_attn_decode_static(ctypes.byref(desc), x.data_ptr(), C.data_ptr(), U1.data_ptr(),
                                           U2.data_ptr(), U3.data_ptr(), Ct.data_ptr(), Ut1.data_ptr(),
                                           Ut2.data_ptr(), Ut3.data_ptr(), Kcache.data_ptr(), Vcache.data_ptr(),
                                           int(Lmax), cache_len.data_ptr(), int(bool(append)), out.data_ptr(),
                                           _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_decode_static")
    return out


# The serving calls are short and are made once per layer and token, so their host time counts: the structures are packed in one
# call, and the usual outcome of the argument checks is decided in one expression (the checks one by one name the culprit).
_DESC_PACK = struct.Struct("=12ififii").pack
_CACHE_PACK = struct.Struct("=QQQiii4x").pack
_CACHE_Q8_PACK = struct.Struct("=QQQQQiii4x").pack


def _check_all(items, dtype, device):
    for t, name, shape in items:
        _check(t, name, shape, dtype, device)


def tucker_cache_append_paged(X, U3, Ut3, Kpages, Vpages, block_table, cache_len, tok_start, *, rope: bool,
                              rope_base: float = 10000.0, pos0: int = 0, workspace=None, flags: int = 0) -> None:
    """Appends a ragged batch of tokens to a paged cache (same name and argument meaning as the C entry point).
    X [T, d]: rows tok_start[b] .. tok_start[b + 1] - 1 are the new tokens of sequence b; Kpages [n_pages, page_size, r3],
    Vpages [n_pages, page_size, t3] (the same tensor: one shared latent pool, with U3 and Ut3 the same tensor);
    block_table [B, max_pages], cache_len [B] and tok_start [B + 1] int32 on the device."""
    torch = _torch()
    lib = load_library()
    if X.dim() != 2 or cache_len.dim() != 1 or U3.dim() != 2 or Ut3.dim() != 2 or Kpages.dim() != 3 or block_table.dim() != 2:
        raise ValueError("X must be [T, d_model], U3 and Ut3 [d_model, rank], Kpages [n_pages, page_size, r3], "
                         "block_table [B, max_pages] and cache_len [B]")
    T, d = X.shape
    r3, t3 = U3.shape[1], Ut3.shape[1]
    n_pages, page_size, _ = Kpages.shape
    B, max_pages = block_table.shape
    dt, dev = X.dtype, X.device
    i32, idx = torch.int32, dev.index
    code = _dtype_code(X)
    if not (X.is_cuda and dt is U3.dtype is Ut3.dtype is Kpages.dtype is Vpages.dtype
            and i32 is block_table.dtype is cache_len.dtype is tok_start.dtype
            and idx == U3.get_device() == Ut3.get_device() == Kpages.get_device() == Vpages.get_device()
            == block_table.get_device() == cache_len.get_device() == tok_start.get_device()
            and U3.shape == (d, r3) and Ut3.shape == (d, t3) and Kpages.shape == (n_pages, page_size, r3)
            and Vpages.shape == (n_pages, page_size, t3) and cache_len.shape == (B,) and tok_start.shape == (B + 1,)
            and X.is_contiguous() and U3.is_contiguous() and Ut3.is_contiguous() and Kpages.is_contiguous()
            and Vpages.is_contiguous() and block_table.is_contiguous() and cache_len.is_contiguous()
            and tok_start.is_contiguous()):
        B = cache_len.shape[0]
        _check_all(((X, "X", (T, d)), (U3, "U3", (d, r3)), (Ut3, "Ut3", (d, t3)), (Kpages, "Kpages", (n_pages, page_size, r3)),
                    (Vpages, "Vpages", (n_pages, page_size, t3))), dt, dev)
        _check_all(((block_table, "block_table", (B, max_pages)), (cache_len, "cache_len", (B,)),
                    (tok_start, "tok_start", (B + 1,))), i32, dev)
    desc = _DESC_PACK(B, 1, d, 1, 1, 1, r3, 1, 1, t3, 1, bool(rope), rope_base, pos0, 0.0, code, flags)
    cache = _CACHE_PACK(Kpages.data_ptr(), Vpages.data_ptr(), block_table.data_ptr(), n_pages, page_size, max_pages)
    other = _enter_device(torch.cuda, dev)
    try:
        if workspace is None:                          # the size goes by the current device's number of SMs
            workspace = alloc_workspace(lib.tucker_cache_append_paged_workspace_bytes(desc, cache, T), dev)
        else:
            _check(workspace, "workspace", workspace.shape, torch.uint8, dev)
        rc = lib.tucker_cache_append_paged(desc, X.data_ptr(), U3.data_ptr(), Ut3.data_ptr(), cache, cache_len.data_ptr(),
                                           tok_start.data_ptr(), T, workspace.data_ptr(), workspace.numel(), _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_cache_append_paged")


def tucker_attn_decode_prefix(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Vpages, block_table, cache_len, prefix_table,
                              prefix_len: int, *, n_H: int, rope: bool, rope_base: float = 10000.0, scale: float = 0.0,
                              append: bool = True, out=None, workspace=None, flags: int = 0):
    """One decode step for a batch whose sequences share a stored prefix (same name and argument meaning as the C entry
    point).  x [B, d]; pools, block_table and cache_len as for tucker_cache_append_paged (the sequences' own part);
    prefix_table int32 [>= ceil(prefix_len / page_size)] on the device (None when prefix_len is 0).  Returns y [B, d]."""
    torch = _torch()
    lib = load_library()
    if x.dim() != 2 or C.dim() != 3 or Ct.dim() != 3 or Kpages.dim() != 3 or block_table.dim() != 2:
        raise ValueError("x must be [B, d_model], the cores 3-way tensors, Kpages [n_pages, page_size, r3] and block_table "
                         "[B, max_pages]")
    B, d = x.shape
    r1, r2, r3 = C.shape
    t1, t2, t3 = Ct.shape
    n_pages, page_size, _ = Kpages.shape
    max_pages = block_table.shape[1]
    dt, dev = x.dtype, x.device
    i32, idx = torch.int32, dev.index
    code = _dtype_code(x)
    if out is None:
        out = torch.empty_like(x)
    if not (x.is_cuda and dt is C.dtype is U1.dtype is U2.dtype is U3.dtype is Ct.dtype is Ut1.dtype is Ut2.dtype is Ut3.dtype
            is Kpages.dtype is Vpages.dtype is out.dtype and i32 is block_table.dtype is cache_len.dtype
            and idx == C.get_device() == U1.get_device() == U2.get_device() == U3.get_device() == Ct.get_device()
            == Ut1.get_device() == Ut2.get_device() == Ut3.get_device() == Kpages.get_device() == Vpages.get_device()
            == out.get_device() == block_table.get_device() == cache_len.get_device()
            and U1.shape == (n_H, r1) and U2.shape == (d, r2) and U3.shape == (d, r3) and Ut1.shape == (n_H, t1)
            and Ut2.shape == (d, t2) and Ut3.shape == (d, t3) and Kpages.shape == (n_pages, page_size, r3)
            and Vpages.shape == (n_pages, page_size, t3) and out.shape == (B, d) and block_table.shape == (B, max_pages)
            and cache_len.shape == (B,)
            and x.is_contiguous() and C.is_contiguous() and U1.is_contiguous() and U2.is_contiguous() and U3.is_contiguous()
            and Ct.is_contiguous() and Ut1.is_contiguous() and Ut2.is_contiguous() and Ut3.is_contiguous()
            and Kpages.is_contiguous() and Vpages.is_contiguous() and out.is_contiguous() and block_table.is_contiguous()
            and cache_len.is_contiguous()):
        _check_all(((x, "x", (B, d)), (C, "C", (r1, r2, r3)), (U1, "U1", (n_H, r1)), (U2, "U2", (d, r2)), (U3, "U3", (d, r3)),
                    (Ct, "Ct", (t1, t2, t3)), (Ut1, "Ut1", (n_H, t1)), (Ut2, "Ut2", (d, t2)), (Ut3, "Ut3", (d, t3)),
                    (Kpages, "Kpages", (n_pages, page_size, r3)), (Vpages, "Vpages", (n_pages, page_size, t3)),
                    (out, "out", (B, d))), dt, dev)
        _check_all(((block_table, "block_table", (B, max_pages)), (cache_len, "cache_len", (B,))), i32, dev)
    prefix_len = int(prefix_len)
    if prefix_len < 0:
        raise ValueError("prefix_len must not be negative")
    prefix_ptr = None
    if prefix_len > 0:
        if prefix_table is None or prefix_table.dim() != 1 or prefix_table.shape[0] * page_size < prefix_len:
            raise ValueError("prefix_table must hold the ceil(prefix_len / page_size) pages of the prefix")
        _check(prefix_table, "prefix_table", prefix_table.shape, i32, dev)
        prefix_ptr = prefix_table.data_ptr()
    desc = _DESC_PACK(B, 1, d, n_H, r1, r2, r3, t1, t2, t3, 1, bool(rope), rope_base, 0, scale, code, flags)
    cache = _CACHE_PACK(Kpages.data_ptr(), Vpages.data_ptr(), block_table.data_ptr(), n_pages, page_size, max_pages)
    ws_ptr, ws_bytes = None, 0
    other = _enter_device(torch.cuda, dev)
    try:
        if workspace is not None:
            _check(workspace, "workspace", workspace.shape, torch.uint8, dev)
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
        else:
            need = lib.tucker_attn_decode_prefix_workspace_bytes(desc, cache, prefix_len)
            if need != TA_WORKSPACE_NONE:
                workspace = alloc_workspace(need, dev)
                ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
        rc = lib.tucker_attn_decode_prefix(desc, x.data_ptr(), C.data_ptr(), U1.data_ptr(), U2.data_ptr(), U3.data_ptr(),
                                           Ct.data_ptr(), Ut1.data_ptr(), Ut2.data_ptr(), Ut3.data_ptr(), cache,
                                           cache_len.data_ptr(), prefix_ptr, prefix_len, bool(append), out.data_ptr(),
                                           ws_ptr, ws_bytes, _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_decode_prefix")
    return out


def tucker_attn_decode_paged(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Vpages, block_table, cache_len, *, n_H: int,
                             rope: bool, rope_base: float = 10000.0, scale: float = 0.0, append: bool = True, out=None,
                             workspace=None, flags: int = 0):
    """One cached decode step over a paged cache (same name and argument meaning as the C entry point): the step of
    tucker_attn_decode_prefix without a prefix.  Returns y [B, d]."""
    return tucker_attn_decode_prefix(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Vpages, block_table, cache_len, None, 0,
                                     n_H=n_H, rope=rope, rope_base=rope_base, scale=scale, append=append, out=out,
                                     workspace=workspace, flags=flags)


# ---- the paged cache held in 8 bits ------------------------------------------------------------------------------------
#
# Pools Kpages [n_pages, page_size, r3], Vpages [n_pages, page_size, t3] of dtype torch.float8_e4m3fn, scales Kscale, Vscale
# [n_pages, page_size] of dtype torch.float8_e8m0fnu: a row stands for its codes times its scale.  One shared latent pool: the
# same tensors for keys and values.

def _q8_cache(Kpages, Kscale, Vpages, Vscale, block_table, r3: int, t3: int, dev):
    """Checks the tensors of an 8-bit cache; returns the packed structure."""
    torch = _torch()
    if Kpages.dim() != 3 or block_table.dim() != 2:
        raise ValueError("Kpages must be [n_pages, page_size, r3] and block_table [B, max_pages]")
    n_pages, page_size, _ = Kpages.shape
    e4, e8, idx = torch.float8_e4m3fn, torch.float8_e8m0fnu, dev.index
    if not (e4 is Kpages.dtype is Vpages.dtype and e8 is Kscale.dtype is Vscale.dtype and block_table.dtype is torch.int32
            and idx == Kpages.get_device() == Vpages.get_device() == Kscale.get_device() == Vscale.get_device()
            == block_table.get_device()
            and Kpages.shape == (n_pages, page_size, r3) and Vpages.shape == (n_pages, page_size, t3)
            and Kscale.shape == Vscale.shape == (n_pages, page_size)
            and Kpages.is_contiguous() and Vpages.is_contiguous() and Kscale.is_contiguous() and Vscale.is_contiguous()
            and block_table.is_contiguous()):
        _check_all(((Kpages, "Kpages", (n_pages, page_size, r3)), (Vpages, "Vpages", (n_pages, page_size, t3))), e4, dev)
        _check_all(((Kscale, "Kscale", (n_pages, page_size)), (Vscale, "Vscale", (n_pages, page_size))), e8, dev)
        _check(block_table, "block_table", block_table.shape, torch.int32, dev)
    return _CACHE_Q8_PACK(Kpages.data_ptr(), Vpages.data_ptr(), Kscale.data_ptr(), Vscale.data_ptr(), block_table.data_ptr(),
                          n_pages, page_size, block_table.shape[1])


def tucker_cache_append_paged_q8(X, U3, Ut3, Kpages, Kscale, Vpages, Vscale, block_table, cache_len, tok_start, *, rope: bool,
                                 rope_base: float = 10000.0, pos0: int = 0, workspace=None, flags: int = 0) -> None:
    """tucker_cache_append_paged into an 8-bit cache (same name and argument meaning as the C entry point): every row is
    quantised on its way to its page."""
    torch = _torch()
    lib = load_library()
    if X.dim() != 2 or cache_len.dim() != 1 or U3.dim() != 2 or Ut3.dim() != 2:
        raise ValueError("X must be [T, d_model], U3 and Ut3 [d_model, rank] and cache_len [B]")
    T, d = X.shape
    r3, t3, B = U3.shape[1], Ut3.shape[1], cache_len.shape[0]
    dt, dev, i32 = X.dtype, X.device, torch.int32
    code = _dtype_code(X)
    idx = dev.index
    if not (X.is_cuda and dt is U3.dtype is Ut3.dtype and i32 is cache_len.dtype is tok_start.dtype
            and idx == U3.get_device() == Ut3.get_device() == cache_len.get_device() == tok_start.get_device()
            and U3.shape[0] == Ut3.shape[0] == d and tok_start.shape == (B + 1,)
            and X.is_contiguous() and U3.is_contiguous() and Ut3.is_contiguous() and cache_len.is_contiguous() and tok_start.is_contiguous()):
        _check_all(((X, "X", (T, d)), (U3, "U3", (d, r3)), (Ut3, "Ut3", (d, t3))), dt, dev)
        _check_all(((cache_len, "cache_len", (B,)), (tok_start, "tok_start", (B + 1,))), i32, dev)
    cache = _q8_cache(Kpages, Kscale, Vpages, Vscale, block_table, r3, t3, dev)
    if block_table.shape[0] != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected {B} rows")
    desc = _DESC_PACK(B, 1, d, 1, 1, 1, r3, 1, 1, t3, 1, bool(rope), rope_base, pos0, 0.0, code, flags)
    other = _enter_device(torch.cuda, dev)
    try:
        if workspace is None:                          # the size goes by the current device's number of SMs
            workspace = alloc_workspace(lib.tucker_cache_append_paged_q8_workspace_bytes(desc, cache, T), dev)
        else:
            _check(workspace, "workspace", workspace.shape, torch.uint8, dev)
        rc = lib.tucker_cache_append_paged_q8(desc, X.data_ptr(), U3.data_ptr(), Ut3.data_ptr(), cache, cache_len.data_ptr(),
                                              tok_start.data_ptr(), T, workspace.data_ptr(), workspace.numel(), _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_cache_append_paged_q8")


def _q8_rows(Krows, Vrows, Kpages, Kscale, Vpages, Vscale, block_table, slots, tok_start, slots_name):
    """Checks the arguments of the store and the read; returns (descriptor, cache, T, device)."""
    torch = _torch()
    if Krows.dim() != 2 or Vrows.dim() != 2 or slots.dim() != 1:
        raise ValueError(f"Krows must be [T, r3], Vrows [T, t3] and {slots_name} [B]")
    (T, r3), t3, B = Krows.shape, Vrows.shape[1], slots.shape[0]
    dt, dev = Krows.dtype, Krows.device
    code = _dtype_code(Krows)
    if not (Krows.is_cuda and dt is Vrows.dtype and slots.dtype is tok_start.dtype is torch.int32
            and dev.index == Vrows.get_device() == slots.get_device() == tok_start.get_device()
            and Vrows.shape[0] == T and tok_start.shape == (B + 1,)
            and Krows.is_contiguous() and Vrows.is_contiguous() and slots.is_contiguous() and tok_start.is_contiguous()):
        _check_all(((Krows, "Krows", (T, r3)), (Vrows, "Vrows", (T, t3))), dt, dev)
        _check_all(((slots, slots_name, (B,)), (tok_start, "tok_start", (B + 1,))), torch.int32, dev)
    cache = _q8_cache(Kpages, Kscale, Vpages, Vscale, block_table, r3, t3, dev)
    if block_table.shape[0] != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected {B} rows")
    return _DESC_PACK(B, 1, 1, 1, 1, 1, r3, 1, 1, t3, 1, 0, 0.0, 0, 0.0, code, 0), cache, T, dev


def tucker_cache_store_paged_q8(Krows, Vrows, Kpages, Kscale, Vpages, Vscale, block_table, cache_len, tok_start) -> None:
    """Quantises latent rows that exist already (Krows [T, r3], Vrows [T, t3], as the cache is to hold them) into the slots
    that follow each sequence's cached ones (same name and argument meaning as the C entry point)."""
    torch = _torch()
    lib = load_library()
    desc, cache, T, dev = _q8_rows(Krows, Vrows, Kpages, Kscale, Vpages, Vscale, block_table, cache_len, tok_start, "cache_len")
    other = _enter_device(torch.cuda, dev)
    try:
        rc = lib.tucker_cache_store_paged_q8(desc, Krows.data_ptr(), Vrows.data_ptr(), cache, cache_len.data_ptr(),
                                             tok_start.data_ptr(), T, _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_cache_store_paged_q8")


def tucker_cache_read_paged_q8(Kpages, Kscale, Vpages, Vscale, block_table, slot_start, tok_start, Krows, Vrows) -> None:
    """Reads cached rows back into rows tok_start[b] .. tok_start[b + 1] - 1 of Krows [T, r3] and Vrows [T, t3]: the slots of
    sequence b from slot_start[b] on (same name and argument meaning as the C entry point)."""
    torch = _torch()
    lib = load_library()
    desc, cache, T, dev = _q8_rows(Krows, Vrows, Kpages, Kscale, Vpages, Vscale, block_table, slot_start, tok_start, "slot_start")
    other = _enter_device(torch.cuda, dev)
    try:
        rc = lib.tucker_cache_read_paged_q8(desc, cache, slot_start.data_ptr(), tok_start.data_ptr(), T, Krows.data_ptr(),
                                            Vrows.data_ptr(), _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_cache_read_paged_q8")


def tucker_attn_decode_prefix_q8(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Kscale, Vpages, Vscale, block_table, cache_len,
                                 prefix_table, prefix_len: int, *, n_H: int, rope: bool, rope_base: float = 10000.0,
                                 scale: float = 0.0, append: bool = True, out=None, workspace=None, flags: int = 0):
    """tucker_attn_decode_prefix over an 8-bit cache (same name and argument meaning as the C entry point).  Returns y [B, d]."""
    torch = _torch()
    lib = load_library()
    if x.dim() != 2 or C.dim() != 3 or Ct.dim() != 3:
        raise ValueError("x must be [B, d_model] and the cores 3-way tensors")
    B, d = x.shape
    r1, r2, r3 = C.shape
    t1, t2, t3 = Ct.shape
    dt, dev = x.dtype, x.device
    i32, idx = torch.int32, dev.index
    code = _dtype_code(x)
    if out is None:
        out = torch.empty_like(x)
    if not (x.is_cuda and dt is C.dtype is U1.dtype is U2.dtype is U3.dtype is Ct.dtype is Ut1.dtype is Ut2.dtype is Ut3.dtype
            is out.dtype and cache_len.dtype is i32
            and idx == C.get_device() == U1.get_device() == U2.get_device() == U3.get_device() == Ct.get_device()
            == Ut1.get_device() == Ut2.get_device() == Ut3.get_device() == out.get_device() == cache_len.get_device()
            and U1.shape == (n_H, r1) and U2.shape == (d, r2) and U3.shape == (d, r3) and Ut1.shape == (n_H, t1)
            and Ut2.shape == (d, t2) and Ut3.shape == (d, t3) and out.shape == (B, d) and cache_len.shape == (B,)
            and x.is_contiguous() and C.is_contiguous() and U1.is_contiguous() and U2.is_contiguous() and U3.is_contiguous()
            and Ct.is_contiguous() and Ut1.is_contiguous() and Ut2.is_contiguous() and Ut3.is_contiguous()
            and out.is_contiguous() and cache_len.is_contiguous()):
        _check_all(((x, "x", (B, d)), (C, "C", (r1, r2, r3)), (U1, "U1", (n_H, r1)), (U2, "U2", (d, r2)), (U3, "U3", (d, r3)),
                    (Ct, "Ct", (t1, t2, t3)), (Ut1, "Ut1", (n_H, t1)), (Ut2, "Ut2", (d, t2)), (Ut3, "Ut3", (d, t3)),
                    (out, "out", (B, d))), dt, dev)
        _check(cache_len, "cache_len", (B,), i32, dev)
    cache = _q8_cache(Kpages, Kscale, Vpages, Vscale, block_table, r3, t3, dev)
    if block_table.shape[0] != B:
        raise ValueError(f"block_table has shape {tuple(block_table.shape)}, expected {B} rows")
    prefix_len = int(prefix_len)
    if prefix_len < 0:
        raise ValueError("prefix_len must not be negative")
    prefix_ptr = None
    if prefix_len > 0:
        if prefix_table is None or prefix_table.dim() != 1 or prefix_table.shape[0] * Kpages.shape[1] < prefix_len:
            raise ValueError("prefix_table must hold the ceil(prefix_len / page_size) pages of the prefix")
        _check(prefix_table, "prefix_table", prefix_table.shape, i32, dev)
        prefix_ptr = prefix_table.data_ptr()
    desc = _DESC_PACK(B, 1, d, n_H, r1, r2, r3, t1, t2, t3, 1, bool(rope), rope_base, 0, scale, code, flags)
    ws_ptr, ws_bytes = None, 0
    other = _enter_device(torch.cuda, dev)
    try:
        if workspace is not None:
            _check(workspace, "workspace", workspace.shape, torch.uint8, dev)
            ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
        else:
            need = lib.tucker_attn_decode_prefix_q8_workspace_bytes(desc, cache, prefix_len)
            if need != TA_WORKSPACE_NONE:
                workspace = alloc_workspace(need, dev)
                ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel()
        rc = lib.tucker_attn_decode_prefix_q8(desc, x.data_ptr(), C.data_ptr(), U1.data_ptr(), U2.data_ptr(), U3.data_ptr(),
                                              Ct.data_ptr(), Ut1.data_ptr(), Ut2.data_ptr(), Ut3.data_ptr(), cache,
                                              cache_len.data_ptr(), prefix_ptr, prefix_len, bool(append), out.data_ptr(),
                                              ws_ptr, ws_bytes, _stream_ptr(dev))
    finally:
        if other is not None:
            other.__exit__(None, None, None)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_decode_prefix_q8")
    return out


def tucker_attn_decode_paged_q8(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Kscale, Vpages, Vscale, block_table, cache_len, *,
                                n_H: int, rope: bool, rope_base: float = 10000.0, scale: float = 0.0, append: bool = True,
                                out=None, workspace=None, flags: int = 0):
    """tucker_attn_decode_paged over an 8-bit cache (same name and argument meaning as the C entry point): the step of
    tucker_attn_decode_prefix_q8 without a prefix.  Returns y [B, d]."""
    return tucker_attn_decode_prefix_q8(x, C, U1, U2, U3, Ct, Ut1, Ut2, Ut3, Kpages, Kscale, Vpages, Vscale, block_table, cache_len,
                                        None, 0, n_H=n_H, rope=rope, rope_base=rope_base, scale=scale, append=append, out=out,
                                        workspace=workspace, flags=flags)


_PACK_KEYS = ("C", "U1", "U2", "U3", "Ct", "Ut1", "Ut2", "Ut3")


def _pack_outputs(shapes, like, out=None):
    torch = _torch()
    if out is None:
        return [torch.empty(sh, dtype=like.dtype, device=like.device) for sh in shapes]
    if len(out) != len(shapes):
        raise ValueError(f"out must hold {len(shapes)} tensors (C, U1, U2, U3, Ct, Ut1, Ut2, Ut3)")
    for name, t, sh in zip(_PACK_KEYS, out, shapes):
        _check(t, name, sh, like.dtype, like.device)
    return list(out)


def tucker_pack_gqa(WQ, WKg, WVg, WO, *, n_H: int, n_G: int, out=None):
    """GQA / MQA (n_G = n_H: MHA) weights as Tucker-attention weights; returns the list
    [C, U1, U2, U3, Ct, Ut1, Ut2, Ut3] of new device tensors (ranks (n_H, d, n_G d_H))."""
    torch = _torch()
    lib = load_library()
    d = WQ.shape[0]
    dev, dt = WQ.device, WQ.dtype
    if d % n_H or not (1 <= n_G <= n_H):
        raise ValueError("d_model must be a multiple of n_H and 1 <= n_G <= n_H")
    w = n_G * (d // n_H)
    _check(WQ, "WQ", (d, d), dt, dev)
    _check(WKg, "WKg", (d, w), dt, dev)
    _check(WVg, "WVg", (d, w), dt, dev)
    _check(WO, "WO", (d, d), dt, dev)
    outs = _pack_outputs([(n_H, d, w), (n_H, n_H), (d, d), (d, w), (n_H, d, w), (n_H, n_H), (d, d), (d, w)], WQ, out)
    with torch.cuda.device(dev):
        rc = lib.tucker_pack_gqa(int(d), int(n_H), int(n_G), _dtype_code(WQ), WQ.data_ptr(), WKg.data_ptr(),
                                 WVg.data_ptr(), WO.data_ptr(), *[o.data_ptr() for o in outs], _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_pack_gqa")
    return outs


def tucker_pack_mha(WQ, WK, WV, WO, *, n_H: int, out=None):
    """MHA weights as Tucker-attention weights (ranks (n_H, d, d)); see tucker_pack_gqa."""
    torch = _torch()
    lib = load_library()
    d = WQ.shape[0]
    dev, dt = WQ.device, WQ.dtype
    if d % n_H:
        raise ValueError("d_model must be a multiple of n_H")
    for name, t in (("WQ", WQ), ("WK", WK), ("WV", WV), ("WO", WO)):
        _check(t, name, (d, d), dt, dev)
    outs = _pack_outputs([(n_H, d, d), (n_H, n_H), (d, d), (d, d), (n_H, d, d), (n_H, n_H), (d, d), (d, d)], WQ, out)
    with torch.cuda.device(dev):
        rc = lib.tucker_pack_mha(int(d), int(n_H), _dtype_code(WQ), WQ.data_ptr(), WK.data_ptr(), WV.data_ptr(),
                                 WO.data_ptr(), *[o.data_ptr() for o in outs], _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_pack_mha")
    return outs


def tucker_pack_mla(WDQ, WUQ, WDKV, WUK, WDV, WUV, WO, *, n_H: int, out=None):
    """MLA (no RoPE) weights as Tucker-attention weights (ranks (n_H, dcq, dck) and
    (n_H, d, dck)); pass WDKV as WDV for a shared key / value latent."""
    torch = _torch()
    lib = load_library()
    d, dcq = WDQ.shape
    dck = WDKV.shape[1]
    dev, dt = WDQ.device, WDQ.dtype
    if d % n_H:
        raise ValueError("d_model must be a multiple of n_H")
    _check(WDQ, "WDQ", (d, dcq), dt, dev)
    _check(WUQ, "WUQ", (dcq, d), dt, dev)
    _check(WDKV, "WDKV", (d, dck), dt, dev)
    _check(WUK, "WUK", (dck, d), dt, dev)
    _check(WDV, "WDV", (d, dck), dt, dev)
    _check(WUV, "WUV", (dck, d), dt, dev)
    _check(WO, "WO", (d, d), dt, dev)
    outs = _pack_outputs([(n_H, dcq, dck), (n_H, n_H), (d, dcq), (d, dck), (n_H, d, dck), (n_H, n_H), (d, d), (d, dck)],
                         WDQ, out)
    with torch.cuda.device(dev):
        rc = lib.tucker_pack_mla(int(d), int(n_H), int(dcq), int(dck), _dtype_code(WDQ), WDQ.data_ptr(), WUQ.data_ptr(),
                                 WDKV.data_ptr(), WUK.data_ptr(), WDV.data_ptr(), WUV.data_ptr(), WO.data_ptr(),
                                 *[o.data_ptr() for o in outs], _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_pack_mla")
    return outs


def tucker_mha_weight_tensors(WQ, WK, WV, WO, *, n_H: int):
    """The two n_H x d x d weight tensors of MHA weights (fp32): W[i] = WQ_i WK_i^T, Wt[i] = (WV_i WO_i)^T."""
    torch = _torch()
    d = WQ.shape[0]
    dev = WQ.device
    if d % n_H:
        raise ValueError("d_model must be a multiple of n_H")
    for name, t in (("WQ", WQ), ("WK", WK), ("WV", WV), ("WO", WO)):
        _check(t, name, (d, d), torch.float32, dev)
    W = torch.empty(n_H, d, d, dtype=torch.float32, device=dev)
    Wt = torch.empty_like(W)
    with torch.cuda.device(dev):
        rc = load_library().tucker_mha_weight_tensors(int(d), int(n_H), WQ.data_ptr(), WK.data_ptr(), WV.data_ptr(),
                                                      WO.data_ptr(), W.data_ptr(), Wt.data_ptr(), _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_mha_weight_tensors")
    return W, Wt


def tucker_hosvd_init(W, ranks, *, workspace=None):
    """HOSVD of one weight tensor W [n_H, d, d] (fp32): returns (C [r1, r2, r3], U1 [n_H, r1], U2 [d, r2],
    U3 [d, r3], spectra), spectra = the singular values of the mode-1, mode-2 and mode-3 unfoldings
    ([n_H], [d], [d], each descending)."""
    torch = _torch()
    lib = load_library()
    if W.dim() != 3 or W.shape[1] != W.shape[2]:
        raise ValueError("W must be [n_H, d, d]")
    n_H, d, _ = W.shape
    dev = W.device
    _check(W, "W", (n_H, d, d), torch.float32, dev)
    r1, r2, r3 = (int(r) for r in ranks)
    f = dict(dtype=torch.float32, device=dev)
    C, U1 = torch.empty(r1, r2, r3, **f), torch.empty(n_H, r1, **f)
    U2, U3 = torch.empty(d, r2, **f), torch.empty(d, r3, **f)
    spectra = torch.empty(n_H + 2 * d, **f)
    need = int(lib.tucker_hosvd_workspace_bytes(int(d), int(n_H), r2, r3))
    if need == 0:
        raise ValueError("invalid sizes for tucker_hosvd_init")
    if workspace is None:
        workspace = alloc_workspace(need, dev)
    with torch.cuda.device(dev):
        rc = lib.tucker_hosvd_init(int(d), int(n_H), r1, r2, r3, W.data_ptr(), C.data_ptr(), U1.data_ptr(), U2.data_ptr(),
                                   U3.data_ptr(), spectra.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                   _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_hosvd_init")
    return C, U1, U2, U3, (spectra[:n_H], spectra[n_H:n_H + d], spectra[n_H + d:])


def probe_mma_rate(mode: int, N: int, iters: int = 256, n_blocks: int = 148) -> float:
    """Cycles per tcgen05.mma 128 x N x 16 for an operand source / layout (see tucker_probe_mma_rate): the
    slowest block's count divided by the number of MMAs."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device())
    cycles = torch.zeros(n_blocks, dtype=torch.int64, device=dev)
    rc = load_library().tucker_probe_mma_rate(int(mode), int(N), int(iters), int(n_blocks), cycles.data_ptr(),
                                              _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_probe_mma_rate")
    torch.cuda.synchronize()
    return float(cycles.max().item()) / (iters * 8)


def probe_plane_mix(tiles: int, r1: int, n_blocks: int = 148):
    """Runs the plane-mixing probe (see tucker_probe_plane_mix); returns (median cycles per tile over the
    blocks, kernel milliseconds by CUDA events)."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device())
    u1 = torch.randn(2, r1, device=dev, dtype=torch.float32)
    cycles = torch.zeros(n_blocks, dtype=torch.int64, device=dev)
    sink = torch.zeros(n_blocks * 256, dtype=torch.float32, device=dev)
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    ms = 0.0
    for _ in range(2):      # the second run is the measured one
        e0.record()
        rc = load_library().tucker_probe_plane_mix(int(tiles), int(r1), int(n_blocks), u1.data_ptr(), cycles.data_ptr(),
                                                   sink.data_ptr(), _stream_ptr(dev))
        e1.record()
        if rc != TA_OK:
            raise TuckerAttnError(rc, "tucker_probe_plane_mix")
        torch.cuda.synchronize()
        ms = e0.elapsed_time(e1)
    return float(cycles.median().item()) / tiles, ms


def selftest_wait_timeout(budget_us: int = 2000, device=None):
    """Runs the library's bounded-wait self-test; returns the int32 tensor [first wait returned,
    second wait returned, second wait's duration / 1024 cycles] (read it after synchronising)."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    out = torch.full((3,), -1, dtype=torch.int32, device=dev)
    with torch.cuda.device(dev):
        rc = load_library().tucker_attn_selftest_wait_timeout(int(budget_us), out.data_ptr(), _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_selftest_wait_timeout")
    return out


def selftest_cluster_wait(budget_us: int = 2000, device=None):
    """Runs the self-test of the bounded waits within a cluster; returns the int32 tensor [the wait returned, what was
    sent late had come when the block ended] (read it after synchronising)."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    out = torch.full((2,), -1, dtype=torch.int32, device=dev)
    with torch.cuda.device(dev):
        rc = load_library().tucker_attn_selftest_cluster_wait(int(budget_us), out.data_ptr(), _stream_ptr(dev))
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_selftest_cluster_wait")
    return out


def last_device_error(device=None) -> int:
    """Synchronises the current stream and returns-and-clears the device error word."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    with torch.cuda.device(dev):
        return int(load_library().tucker_attn_last_device_error(_stream_ptr(dev)))


def sync_status(device=None) -> int:
    """Synchronises the current stream and folds the device error word into a status code (and clears
    it): TA_OK, or TA_ERR_DEVICE_TIMEOUT (-5) / TA_ERR_INVALID_ARG (-1) / TA_ERR_CUDA (-4)."""
    torch = _torch()
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    with torch.cuda.device(dev):
        return int(load_library().tucker_attn_sync_status(_stream_ptr(dev)))


def bounds_checked() -> bool:
    """True when the loaded library was built with -DTA_BOUNDS_CHECK."""
    return bool(load_library().tucker_attn_bounds_checked())


def last_path() -> int:
    return int(load_library().tucker_attn_last_path())


def last_launch_count() -> int:
    return int(load_library().tucker_attn_last_launch_count())


def set_profile_events(start=None, stop=None) -> None:
    """Registers two torch.cuda.Event(enable_timing=True) objects (already recorded once, so
    that their handles exist) to be recorded around the dominant kernel of later calls;
    call with no arguments to unregister."""
    lib = load_library()
    if start is None and stop is None:
        rc = lib.tucker_attn_set_profile_events(None, None)
    else:
        rc = lib.tucker_attn_set_profile_events(start.cuda_event, stop.cuda_event)
    if rc != TA_OK:
        raise TuckerAttnError(rc, "tucker_attn_set_profile_events")
