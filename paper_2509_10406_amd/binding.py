"""ctypes binding of libmuse.so: argument marshalling only.

Same names as the C ABI (include/muse.h).  PyTorch supplies device memory and the
stream; every step of the path runs in the library's kernels.  There is no
fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmuse.so")
_lib = None

FP32, BF16 = 0, 1
FLAG_KEEP_FWD_STATE = 1
FLAG_FROZEN_WEIGHTS = 2
FLAG_STREAMING_KMEANS = 4
FLAG_BALANCED_ASSIGN = 8
FLAG_DIPOLE = 16
WS_CLUSTER, WS_FWD, WS_BWD, WS_EXACT_FWD, WS_EXACT_BWD = range(5)
SYMBOLS = ["muse_workspace_bytes", "muse_cluster", "muse_kmeans_stream", "muse_fwd", "muse_bwd", "exact_attn_fwd", "exact_attn_bwd",
           "exact_attn_bwd_static", "muse_packed_workspace_bytes", "exact_attn_packed_fwd", "exact_attn_packed_bwd",
           "exact_attn_cache_append", "muse_cache_workspace_bytes", "exact_attn_cache_fwd", "muse_profile_enable",
           "muse_profile_report", "muse_probe_peaks", "muse_strerror"]
STATIC_SCRATCH_BYTES = 64 << 20


class MuseError(RuntimeError):
    pass


class _Params(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("B", "Hq", "Hkv", "N", "D", "Cq", "Ck", "r", "k2", "block", "kmeans_iters", "dtype", "grad_dtype",
                 "causal")] + [("flags", C.c_uint32), ("scale", C.c_float)]


@dataclass
class Params:
    B: int
    Hq: int
    Hkv: int
    N: int
    D: int
    Cq: int = 1
    Ck: int = 1
    r: int = 0
    k2: int = 1
    block: int = 0
    kmeans_iters: int = 10
    dtype: int = BF16
    grad_dtype: int = FP32
    causal: int = 1
    flags: int = 0
    scale: float = 0.0

    def c(self) -> _Params:
        return _Params(self.B, self.Hq, self.Hkv, self.N, self.D, self.Cq, self.Ck, self.r, self.k2, self.block,
                       self.kmeans_iters, self.dtype, self.grad_dtype, self.causal, self.flags, self.scale)

    @property
    def Bs(self) -> int:
        return self.block if self.block else self.N // 8

    @property
    def nb(self) -> int:
        return self.N // self.Bs

    @property
    def k2e(self) -> int:
        return self.k2 if self.k2 > 0 else max(self.nb - 1, 1)

    @property
    def eff_scale(self) -> float:
        return self.scale if self.scale > 0 else 1.0 / math.sqrt(self.D)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32

    @property
    def torch_grad_dtype(self):
        return torch.bfloat16 if self.grad_dtype == BF16 else torch.float32


def load():
    """Loads libmuse.so; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MuseError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        lib = C.CDLL(LIB_PATH)
        lib.muse_strerror.restype = C.c_char_p
        lib.muse_strerror.argtypes = [C.c_int]
        for n in SYMBOLS[:-1]:
            getattr(lib, n).restype = C.c_int
        ptr, size = C.c_void_p, C.c_size_t
        lib.muse_packed_workspace_bytes.argtypes = [ptr, C.c_int, ptr]
        lib.muse_cache_workspace_bytes.argtypes = [ptr, ptr]
        lib.exact_attn_packed_fwd.argtypes = [ptr] * 8 + [size, ptr]
        lib.exact_attn_packed_bwd.argtypes = [ptr] * 12 + [size, ptr]
        lib.exact_attn_cache_append.argtypes = [ptr] * 11
        lib.exact_attn_cache_fwd.argtypes = [ptr] * 12 + [size, ptr]
        _lib = lib
    return _lib


def muse_strerror(code: int) -> str:
    return load().muse_strerror(code).decode()


def _check(rc: int, what: str):
    if rc != 0:
        raise MuseError(f"{what}: {muse_strerror(rc)} ({rc})")


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def muse_workspace_bytes(p: Params, which: int):
    mn, pref = C.c_size_t(0), C.c_size_t(0)
    pc = p.c()
    _check(load().muse_workspace_bytes(C.byref(pc), C.c_int(which), C.byref(mn), C.byref(pref)), "muse_workspace_bytes")
    return mn.value, pref.value


_ws_cache: dict = {}


def workspace(p: Params, which: int, device="cuda", limit_bytes: int | None = None) -> torch.Tensor:
    """A cached uint8 device buffer of the preferred size (capped by limit_bytes, never below the minimum)."""
    mn, pref = muse_workspace_bytes(p, which)
    size = pref if limit_bytes is None else max(mn, min(pref, limit_bytes))
    # under MUSE_FLAG_KEEP_FWD_STATE the backward must be handed the very buffer the forward filled
    shared = (p.flags & FLAG_KEEP_FWD_STATE) and which in (WS_FWD, WS_BWD)
    device = torch.device(device)
    if device.index is None:   # "cuda" and "cuda:<current>" are one device: one buffer
        device = torch.device(device.type, torch.cuda.current_device())
    key = (str(device), "fwd+bwd" if shared else which)
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < size:
        _ws_cache.pop(key, None)
        buf = torch.empty(size, dtype=torch.uint8, device=device)
        _ws_cache[key] = buf
    return buf


def free_workspaces():
    _ws_cache.clear()


def muse_cluster(p: Params, Q, K, q_init_idx, k_init_idx, q_centroids=None, k_centroids=None, ws=None):
    """Returns (q_centroids, q_assign, k_centroids, k_assign); a side is skipped when its tensor is None."""
    dev = (Q if Q is not None else K).device
    ws = ws if ws is not None else workspace(p, WS_CLUSTER, dev)
    qa = ka = None
    if Q is not None:
        if q_centroids is None:
            q_centroids = torch.empty(p.B, p.Hq, p.Cq, p.D, dtype=torch.float32, device=dev)
        qa = torch.empty(p.B, p.Hq, p.N, dtype=torch.int32, device=dev)
    if K is not None:
        if k_centroids is None:
            k_centroids = torch.empty(p.B, p.Hkv, p.Ck, p.D, dtype=torch.float32, device=dev)
        ka = torch.empty(p.B, p.Hkv, p.N, dtype=torch.int32, device=dev)
    pc = p.c()
    _check(load().muse_cluster(C.byref(pc), _ptr(Q), _ptr(K), _ptr(q_init_idx), _ptr(k_init_idx), _ptr(q_centroids),
                               _ptr(qa), _ptr(k_centroids), _ptr(ka), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "muse_cluster")
    return q_centroids, qa, k_centroids, ka


def muse_kmeans_stream(p: Params, side: int, X, init_idx, centroids=None, ws=None):
    """The streaming centroid pass alone.  side 0: query rows, 1: key rows.
    Returns (centroids, stream_assign, counts)."""
    dev = X.device
    H, Cn = (p.Hkv, p.Ck) if side else (p.Hq, p.Cq)
    ws = ws if ws is not None else workspace(p, WS_CLUSTER, dev)
    if centroids is None:
        centroids = torch.empty(p.B, H, Cn, p.D, dtype=torch.float32, device=dev)
    sa = torch.empty(p.B, H, p.N, dtype=torch.int32, device=dev)
    cnt = torch.empty(p.B, H, Cn, dtype=torch.float32, device=dev)
    pc = p.c()
    _check(load().muse_kmeans_stream(C.byref(pc), C.c_int(side), _ptr(X), _ptr(init_idx), _ptr(centroids), _ptr(sa),
                                     _ptr(cnt), _ptr(ws), C.c_size_t(ws.numel()), _stream()), "muse_kmeans_stream")
    return centroids, sa, cnt


def muse_fwd(p: Params, Q, K, V, q_centroids, q_assign, k_assign, ws=None, out=None):
    """Returns (O, LSE, sel_clusters, sel_blocks)."""
    dev = Q.device
    ws = ws if ws is not None else workspace(p, WS_FWD, dev)
    if out is None:
        O = torch.empty(p.B, p.Hq, p.N, p.D, dtype=p.torch_dtype, device=dev)
        LSE = torch.empty(p.B, p.Hq, p.N, dtype=torch.float32, device=dev)
        selc = torch.empty(p.B, p.Hq, p.N, max(p.r, 1), dtype=torch.int32, device=dev)
        selb = torch.empty(p.B, p.Hq, p.N, max(p.r, 1), p.k2e, dtype=torch.int32, device=dev)
    else:
        O, LSE, selc, selb = out
    pc = p.c()
    _check(load().muse_fwd(C.byref(pc), _ptr(Q), _ptr(K), _ptr(V), _ptr(q_centroids), _ptr(q_assign), _ptr(k_assign),
                           _ptr(O), _ptr(LSE), _ptr(selc), _ptr(selb), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "muse_fwd")
    return O, LSE, selc, selb


def muse_bwd(p: Params, Q, K, V, O, LSE, dO, q_centroids, q_assign, k_assign, sel_clusters, sel_blocks, ws=None,
             out=None):
    """Returns (dQ, dK, dV)."""
    dev = Q.device
    ws = ws if ws is not None else workspace(p, WS_BWD, dev)
    if out is None:
        dQ = torch.empty(p.B, p.Hq, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
        dK = torch.empty(p.B, p.Hkv, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
        dV = torch.empty(p.B, p.Hkv, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
    else:
        dQ, dK, dV = out
    pc = p.c()
    _check(load().muse_bwd(C.byref(pc), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(dO), _ptr(q_centroids),
                           _ptr(q_assign), _ptr(k_assign), _ptr(sel_clusters), _ptr(sel_blocks), _ptr(dQ), _ptr(dK),
                           _ptr(dV), _ptr(ws), C.c_size_t(ws.numel()), _stream()), "muse_bwd")
    return dQ, dK, dV


def exact_attn_fwd(p: Params, Q, K, V, ws=None, out=None):
    """Returns (O, LSE)."""
    dev = Q.device
    ws = ws if ws is not None else workspace(p, WS_EXACT_FWD, dev)
    if out is None:
        O = torch.empty(p.B, p.Hq, p.N, p.D, dtype=p.torch_dtype, device=dev)
        LSE = torch.empty(p.B, p.Hq, p.N, dtype=torch.float32, device=dev)
    else:
        O, LSE = out
    pc = p.c()
    _check(load().exact_attn_fwd(C.byref(pc), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(ws),
                                 C.c_size_t(ws.numel()), _stream()), "exact_attn_fwd")
    return O, LSE


def exact_attn_bwd(p: Params, Q, K, V, O, LSE, dO, ws=None, out=None):
    """Returns (dQ, dK, dV)."""
    dev = Q.device
    ws = ws if ws is not None else workspace(p, WS_EXACT_BWD, dev)
    if out is None:
        dQ = torch.empty(p.B, p.Hq, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
        dK = torch.empty(p.B, p.Hkv, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
        dV = torch.empty(p.B, p.Hkv, p.N, p.D, dtype=p.torch_grad_dtype, device=dev)
    else:
        dQ, dK, dV = out
    pc = p.c()
    _check(load().exact_attn_bwd(C.byref(pc), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(dO), _ptr(dQ),
                                 _ptr(dK), _ptr(dV), _ptr(ws), C.c_size_t(ws.numel()), _stream()), "exact_attn_bwd")
    return dQ, dK, dV


def exact_attn_bwd_static(p: Params, Q, K, V, O, LSE, dO, out):
    """exact_attn_bwd on the library's static scratch: no workspace, nothing allocated by the call.
    out = (dQ, dK, dV), allocated by the caller beforehand."""
    dQ, dK, dV = out
    pc = p.c()
    _check(load().exact_attn_bwd_static(C.byref(pc), _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(LSE), _ptr(dO), _ptr(dQ),
                                        _ptr(dK), _ptr(dV), _stream()), "exact_attn_bwd_static")
    return dQ, dK, dV


# ---- packed sequences and the paged 8-bit cache ------------------------------------------------------------------
class _Rows(C.Structure):
    _fields_ = [("token", C.c_int64), ("head", C.c_int64)]


class _PackedParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("S", "Hq", "Hkv", "D", "T", "max_len", "dtype", "grad_dtype")] + \
               [("flags", C.c_uint32), ("scale", C.c_float)] + [(n, _Rows) for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")]


class _CacheParams(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("S", "Hq", "Hkv", "D", "T", "pages", "page", "table_cols", "max_new", "dtype")] + \
               [("flags", C.c_uint32), ("scale", C.c_float)] + [(n, _Rows) for n in ("q", "k", "v", "o")]


@dataclass(frozen=True)
class PackedParams:
    """S sequences packed into T rows; max_len: a bound on their lengths (0: none is known)."""
    S: int
    Hq: int
    Hkv: int
    T: int
    D: int
    max_len: int = 0
    dtype: int = BF16
    grad_dtype: int = FP32
    scale: float = 0.0

    def __post_init__(self):
        object.__setattr__(self, "_c", _PackedParams(self.S, self.Hq, self.Hkv, self.D, self.T, self.max_len, self.dtype,
                                                     self.grad_dtype, 0, self.scale))

    torch_dtype = Params.torch_dtype
    torch_grad_dtype = Params.torch_grad_dtype


@dataclass(frozen=True)
class CacheParams:
    """S sequences with T new tokens; a cache of `pages` pages of `page` tokens; max_new: a bound on a sequence's new tokens (0: none)."""
    S: int
    Hq: int
    Hkv: int
    T: int
    D: int
    pages: int
    page: int
    table_cols: int
    max_new: int = 0
    dtype: int = BF16
    scale: float = 0.0

    def __post_init__(self):
        object.__setattr__(self, "_c", _CacheParams(self.S, self.Hq, self.Hkv, self.D, self.T, self.pages, self.page, self.table_cols,
                                                    self.max_new, self.dtype, 0, self.scale))

    torch_dtype = Params.torch_dtype


@dataclass(frozen=True, eq=False)
class KVCache:
    """k [pages, Hkv, page, D] and v [pages, Hkv, D, page] of e4m3 bytes (uint8), k_scale and v_scale [pages, Hkv] fp32.  A call takes the
    tensors as they are at that moment: their storage may have been replaced since (a cache that was moved out and back)."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    def __post_init__(self):
        dev = _on_gpu(self.k)
        if self.k.dim() != 4:
            raise MuseError(f"cache.k: expected [pages, Hkv, page, D], got {list(self.k.shape)}")
        self._addresses(*self.k.shape, dev)

    def _addresses(self, pages, Hkv, page, D, dev):
        return (_whole(self.k, "cache.k", (pages, Hkv, page, D), torch.uint8, dev),
                _whole(self.v, "cache.v", (pages, Hkv, D, page), torch.uint8, dev),
                _whole(self.k_scale, "cache.k_scale", (pages, Hkv), torch.float32, dev),
                _whole(self.v_scale, "cache.v_scale", (pages, Hkv), torch.float32, dev))


def kv_cache(p: CacheParams, device="cuda") -> KVCache:
    """An empty cache (its contents are those of a page without tokens: they do not count)."""
    return KVCache(torch.zeros(p.pages, p.Hkv, p.page, p.D, dtype=torch.uint8, device=device),
                   torch.zeros(p.pages, p.Hkv, p.D, p.page, dtype=torch.uint8, device=device),
                   torch.ones(p.pages, p.Hkv, device=device), torch.ones(p.pages, p.Hkv, device=device))


def _packed_rows(rows: _Rows, t, what, T, H, D, dtype, dev):
    """The strides of a [T, H, D] tensor into `rows`; its address."""
    if t.shape != (T, H, D) or t.dtype != dtype or t.device != dev:
        raise MuseError(f"{what}: expected {dtype} [{T}, {H}, {D}] on {dev}, got {t.dtype} {list(t.shape)} on {t.device}")
    st = t.stride()
    if st[2] != 1:
        raise MuseError(f"{what}: the elements of a row must be adjacent (strides {st})")
    rows.token, rows.head = st[0], st[1]
    return t.data_ptr()


def _whole(t, what, shape, dtype, dev):
    """The address of a contiguous tensor."""
    if t.shape != shape or t.dtype != dtype or t.device != dev or not t.is_contiguous():
        raise MuseError(f"{what}: expected contiguous {dtype} {list(shape)} on {dev}, got {t.dtype} {list(t.shape)} "
                        f"(strides {t.stride()}) on {t.device}")
    return t.data_ptr()


def _packed_call(name, dev, pc, *args):
    """Calls an entry point on the current stream of the tensors' device."""
    stream = torch._C._cuda_getCurrentRawStream(dev.index)  # without the object that torch.cuda.current_stream makes: a microsecond
    if dev.index == torch._C._cuda_getDevice():
        rc = getattr(load(), name)(C.byref(pc), *args, stream)
    else:
        with torch.cuda.device(dev):
            rc = getattr(load(), name)(C.byref(pc), *args, stream)
    if rc:
        _check(rc, name)


def _scratch(bytes_, ws, dev):
    """(address, size) of the caller's workspace, or of one from torch's allocator: a call's own, so that calls on several streams
    and captured graphs do not meet in it."""
    if ws is None:
        ws = torch.empty(bytes_, dtype=torch.uint8, device=dev) if bytes_ else None
    elif ws.device != dev or not ws.is_contiguous():
        raise MuseError(f"workspace: expected a contiguous tensor on {dev}")
    return (ws, ws.data_ptr(), ws.numel() * ws.element_size()) if ws is not None else (None, 0, 0)


def _on_gpu(t):
    if not t.is_cuda:
        raise MuseError("device-resident tensors only")
    return t.device


def muse_packed_workspace_bytes(p: PackedParams, which: int) -> int:
    """Scratch of exact_attn_packed_fwd (WS_EXACT_FWD) or exact_attn_packed_bwd (WS_EXACT_BWD) for [T, H, D] tensors."""
    got, pc = C.c_size_t(0), _PackedParams.from_buffer_copy(p._c)
    for n in ("q", "o", "dout", "dq"):
        getattr(pc, n).token, getattr(pc, n).head = p.Hq * p.D, p.D
    for n in ("k", "v", "dk", "dv"):
        getattr(pc, n).token, getattr(pc, n).head = p.Hkv * p.D, p.D
    _check(load().muse_packed_workspace_bytes(C.byref(pc), which, C.byref(got)), "muse_packed_workspace_bytes")
    return got.value


def _packed_bytes(p: PackedParams, which: int) -> int:
    """muse_packed_workspace_bytes, asked once per params."""
    key = "_ws%d" % which
    got = p.__dict__.get(key)
    if got is None:
        got = muse_packed_workspace_bytes(p, which)
        object.__setattr__(p, key, got)
    return got


def exact_attn_packed_fwd(p: PackedParams, Q, K, V, cu_seqlens, ws=None, out=None):
    """Exact causal attention of packed sequences.  Q [T, Hq, D], K and V [T, Hkv, D] in any strides whose rows are adjacent elements at
    16-byte boundaries, cu_seqlens [S + 1] int32.  Returns (O [T, Hq, D], LSE [Hq, T]); out: tensors to write them into.  Rows of no sequence
    keep what out holds there; without out they are not initialised."""
    dev = _on_gpu(Q)
    O, LSE = out if out is not None else (torch.empty(p.T, p.Hq, p.D, dtype=p.torch_dtype, device=dev),
                                          torch.empty(p.Hq, p.T, dtype=torch.float32, device=dev))
    t, pc = p.torch_dtype, _PackedParams.from_buffer_copy(p._c)
    ptrs = (_packed_rows(pc.q, Q, "Q", p.T, p.Hq, p.D, t, dev), _packed_rows(pc.k, K, "K", p.T, p.Hkv, p.D, t, dev),
            _packed_rows(pc.v, V, "V", p.T, p.Hkv, p.D, t, dev), _whole(cu_seqlens, "cu_seqlens", (p.S + 1,), torch.int32, dev),
            _packed_rows(pc.o, O, "O", p.T, p.Hq, p.D, t, dev), _whole(LSE, "LSE", (p.Hq, p.T), torch.float32, dev))
    keep, at, size = _scratch(_packed_bytes(p, WS_EXACT_FWD), ws, dev)
    _packed_call("exact_attn_packed_fwd", dev, pc, *ptrs, at, size)
    return O, LSE


def exact_attn_packed_bwd(p: PackedParams, Q, K, V, cu_seqlens, O, LSE, dO, ws=None, out=None):
    """The gradient of exact_attn_packed_fwd.  Returns (dQ, dK, dV) of grad_dtype, shaped as Q, K, V; out: tensors to write them into.  Rows of
    no sequence (padding) keep what out holds there; without out they are not initialised: a caller that sums over all rows gives zeros."""
    dev = _on_gpu(Q)
    t, gt, pc = p.torch_dtype, p.torch_grad_dtype, _PackedParams.from_buffer_copy(p._c)
    dQ, dK, dV = out if out is not None else (torch.empty(p.T, h, p.D, dtype=gt, device=dev) for h in (p.Hq, p.Hkv, p.Hkv))
    ptrs = (_packed_rows(pc.q, Q, "Q", p.T, p.Hq, p.D, t, dev), _packed_rows(pc.k, K, "K", p.T, p.Hkv, p.D, t, dev),
            _packed_rows(pc.v, V, "V", p.T, p.Hkv, p.D, t, dev), _whole(cu_seqlens, "cu_seqlens", (p.S + 1,), torch.int32, dev),
            _packed_rows(pc.o, O, "O", p.T, p.Hq, p.D, t, dev), _whole(LSE, "LSE", (p.Hq, p.T), torch.float32, dev),
            _packed_rows(pc.dout, dO, "dO", p.T, p.Hq, p.D, t, dev), _packed_rows(pc.dq, dQ, "dQ", p.T, p.Hq, p.D, gt, dev),
            _packed_rows(pc.dk, dK, "dK", p.T, p.Hkv, p.D, gt, dev), _packed_rows(pc.dv, dV, "dV", p.T, p.Hkv, p.D, gt, dev))
    keep, at, size = _scratch(_packed_bytes(p, WS_EXACT_BWD), ws, dev)
    _packed_call("exact_attn_packed_bwd", dev, pc, *ptrs, at, size)
    return dQ, dK, dV


def _cache_ptrs(p: CacheParams, cu_new, kv_lens, table, cache: KVCache, dev):
    return ((_whole(cu_new, "cu_new", (p.S + 1,), torch.int32, dev) if cu_new is not None else 0,
             _whole(kv_lens, "kv_lens", (p.S,), torch.int32, dev), _whole(table, "table", (p.S, p.table_cols), torch.int32, dev)),
            cache._addresses(p.pages, p.Hkv, p.page, p.D, dev))


def exact_attn_cache_append(p: CacheParams, K, V, cu_new, kv_lens, table, cache: KVCache):
    """Stores the new tokens' K and V [T, Hkv, D] into the cache.  cu_new [S + 1] (None: one token per sequence), kv_lens [S] (the new
    tokens included) and table [S, table_cols] are int32."""
    dev = _on_gpu(K)
    pc = _CacheParams.from_buffer_copy(p._c)
    kp, vp = (_packed_rows(getattr(pc, n), x, n.upper(), p.T, p.Hkv, p.D, p.torch_dtype, dev) for n, x in (("k", K), ("v", V)))
    index, held = _cache_ptrs(p, cu_new, kv_lens, table, cache, dev)
    _packed_call("exact_attn_cache_append", dev, pc, kp, vp, *index, *held)


def muse_cache_workspace_bytes(p: CacheParams) -> int:
    got = C.c_size_t(0)
    _check(load().muse_cache_workspace_bytes(C.byref(p._c), C.byref(got)), "muse_cache_workspace_bytes")
    return got.value


def exact_attn_cache_fwd(p: CacheParams, Q, cu_new, kv_lens, table, cache: KVCache, ws=None, out=None):
    """Causal attention of the new tokens' queries Q [T, Hq, D] to their sequences' cached tokens.  Returns (O [T, Hq, D], LSE [Hq, T]); out:
    tensors to write them into, its LSE may be None.  Rows of no sequence keep what out holds there; without out they are not initialised."""
    dev = _on_gpu(Q)
    O, LSE = out if out is not None else (torch.empty(p.T, p.Hq, p.D, dtype=p.torch_dtype, device=dev),
                                          torch.empty(p.Hq, p.T, dtype=torch.float32, device=dev))
    t, pc = p.torch_dtype, _CacheParams.from_buffer_copy(p._c)
    qp, op = (_packed_rows(r, x, n, p.T, p.Hq, p.D, t, dev) for r, x, n in ((pc.q, Q, "Q"), (pc.o, O, "O")))
    index, held = _cache_ptrs(p, cu_new, kv_lens, table, cache, dev)
    need = p.__dict__.get("_ws")
    if need is None:
        need = muse_cache_workspace_bytes(p)
        object.__setattr__(p, "_ws", need)
    keep, at, size = _scratch(need, ws, dev)
    _packed_call("exact_attn_cache_fwd", dev, pc, qp, *index, *held, op,
                 _whole(LSE, "LSE", (p.Hq, p.T), torch.float32, dev) if LSE is not None else 0, at, size)
    return O, LSE


def muse_profile_enable(on: bool):
    _check(load().muse_profile_enable(C.c_int(1 if on else 0)), "muse_profile_enable")


def muse_profile_report() -> dict:
    """{kernel name: (launches, total ms)} of everything launched since muse_profile_enable(True)."""
    buf = C.create_string_buffer(1 << 16)
    _check(load().muse_profile_report(buf, C.c_size_t(len(buf))), "muse_profile_report")
    out = {}
    for line in buf.value.decode().splitlines():
        name, cnt, ms = line.split()
        out[name] = (int(cnt), float(ms))
    return out


def muse_probe_peaks(buf) -> dict:
    """{"copy_GBps", "mfma_bf16_TFLOPs"}: what a plain copy inside the device tensor `buf` (>= 1 GiB, overwritten) and
    a loop of independent bf16 MFMAs reach on this device."""
    gbps, tfl = C.c_double(0.0), C.c_double(0.0)
    _check(load().muse_probe_peaks(_ptr(buf), C.c_size_t(buf.numel() * buf.element_size()), C.byref(gbps), C.byref(tfl),
                                   _stream()), "muse_probe_peaks")
    return {"copy_GBps": gbps.value, "mfma_bf16_TFLOPs": tfl.value}


def params_for(w, **kw) -> Params:
    """Params of a workload from paper_2509_10406_amd.inputs."""
    d = dict(B=w.B, Hq=w.Hq, Hkv=w.Hkv, N=w.N, D=w.D, Cq=w.Cq, Ck=w.Ck, r=w.r, k2=w.k2, block=w.block,
             kmeans_iters=w.kmeans_iters, dtype=BF16 if w.dtype == "bf16" else FP32, grad_dtype=FP32)
    d.update(kw)
    return Params(**d)
