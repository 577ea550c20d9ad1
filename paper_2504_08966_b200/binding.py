"""ctypes binding of libpact.so: argument marshalling only, every step runs in the CUDA kernels.

Function names follow include/pact.h.  Tensors are torch CUDA tensors; the binding passes their
data pointers and the current stream.  There is no fallback: if the library is missing or the
device is not a B200-class GPU the calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpact.so")

PACT_BF16, PACT_F32 = 0, 1
N_COUNTERS = 16
CNT = {"n_out": 0, "q": 1, "C": 2, "r": 3, "discarded": 4, "sweeps": 5, "band_dc": 6,
       "band_adc": 7, "status": 8, "m": 9}
FLAG_CENTER_ONLY, FLAG_NO_NORM, FLAG_NORM_ONLY = 1, 2, 4

EXPORTS = ["pact_create", "pact_destroy", "pact_workspace_bytes", "pact_status_string",
           "pact_last_cuda_error", "pact_importance", "pact_prune", "pact_dbdpc",
           "pact_prune_static", "pact_reincorporate", "pact_merge", "pact_reduce", "pact_reduce_host",
           "pact_host_staging_bytes", "pact_launch_count", "pact_profile_enable", "pact_profile_read",
           "pact_profile_stage_name", "pact_graph_create", "pact_graph_launch", "pact_graph_destroy",
           "pact_key_spread", "pact_set_wait_limits", "pact_cache_plan", "pact_cache_write", "pact_page_select",
           "pact_paged_attention", "pact_paged_workspace_bytes"]


class Params(C.Structure):
    _fields_ = [("lam", C.c_double), ("d_c", C.c_float), ("d_n", C.c_float), ("alpha", C.c_float),
                ("n_prune", C.c_int32), ("flags", C.c_uint32)]


class ImageDesc(C.Structure):
    _fields_ = [("H", C.c_void_p), ("ldH", C.c_int64), ("K_euti", C.c_void_p), ("ldKe", C.c_int64),
                ("Q_euti", C.c_void_p), ("ldQ", C.c_int64), ("K_clu", C.c_void_p), ("ldKc", C.c_int64),
                ("P", C.c_void_p), ("n_total", C.c_int32), ("vis_start", C.c_int32), ("N", C.c_int32),
                ("reserved", C.c_int32), ("H_out", C.c_void_p), ("ldHo", C.c_int64),
                ("P_out", C.c_void_p), ("size_out", C.c_void_p), ("label", C.c_void_p),
                ("score", C.c_void_p), ("keep", C.c_void_p), ("counters", C.c_void_p),
                ("logw_out", C.c_void_p)]


class PagedCacheDesc(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("k_page", C.c_int64), ("k_head", C.c_int64), ("k_row", C.c_int64),
                ("v_page", C.c_int64), ("v_head", C.c_int64), ("v_row", C.c_int64), ("logw", C.c_void_p),
                ("bounds", C.c_void_p), ("w_max", C.c_void_p), ("n_pages", C.c_int32), ("page_rows", C.c_int32)]


# pact_plan, pact_new_rows and pact_query of pact.h: packed into a buffer of the context, a tenth of the time of as many ctypes arguments
_PLAN = struct.Struct("@4iPPPqPPPPPPqiiP")
_NEW_ROWS = struct.Struct("@PPqqPPqP")
_QUERY = struct.Struct("@PqqPPiiPiiifPqqPPPN")

_lib = None


def lib():
    """Loads libpact.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2504_08966_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
        L.pact_create.argtypes = [C.POINTER(vp), i32, i32, i32, i32, i32, i32]
        L.pact_destroy.argtypes = [vp]
        L.pact_workspace_bytes.argtypes = [vp, i32, i32]
        L.pact_workspace_bytes.restype = sz
        L.pact_status_string.argtypes = [i32]
        L.pact_status_string.restype = C.c_char_p
        L.pact_last_cuda_error.argtypes = [vp]
        L.pact_last_cuda_error.restype = C.c_char_p
        L.pact_importance.argtypes = [vp, C.POINTER(ImageDesc), C.POINTER(Params), vp, vp, sz, vp]
        L.pact_prune.argtypes = [vp, vp, i32, C.POINTER(Params), vp, vp, vp, vp, vp, sz, vp]
        L.pact_prune_static.argtypes = [vp, i32, C.POINTER(Params), vp, vp, vp, vp, vp]
        L.pact_dbdpc.argtypes = [vp, vp, i64, i32, vp, vp, C.POINTER(Params), vp, vp, vp, vp, vp, vp, sz, vp]
        L.pact_reincorporate.argtypes = [vp, vp, i64, i32, vp, vp, vp, vp, C.POINTER(Params), vp, vp, vp,
                                         vp, sz, vp]
        L.pact_key_spread.argtypes = [vp, C.POINTER(vp), i32, i64, i32, C.c_float, vp, vp, vp, sz, vp]
        L.pact_merge.argtypes = [vp, C.POINTER(ImageDesc), vp, vp, vp, C.POINTER(Params), vp, sz, vp]
        L.pact_reduce.argtypes = [vp, C.POINTER(ImageDesc), i32, C.POINTER(Params), i32, vp, sz, vp]
        L.pact_reduce_host.argtypes = [vp, C.POINTER(ImageDesc), C.POINTER(Params), vp, sz, vp, sz, vp]
        L.pact_host_staging_bytes.argtypes = [vp, i32, i32]
        L.pact_host_staging_bytes.restype = sz
        L.pact_graph_create.argtypes = [vp, C.POINTER(ImageDesc), i32, C.POINTER(Params), i32, vp, sz, C.POINTER(vp)]
        L.pact_graph_launch.argtypes = [vp, vp]
        L.pact_graph_destroy.argtypes = [vp]
        L.pact_launch_count.argtypes = [vp]
        L.pact_set_wait_limits.argtypes = [vp, i32, i32]
        L.pact_launch_count.restype = C.c_longlong
        L.pact_profile_enable.argtypes = [vp, i32]
        L.pact_profile_read.argtypes = [vp, C.POINTER(C.c_float), i32]
        L.pact_profile_stage_name.argtypes = [i32]
        L.pact_profile_stage_name.restype = C.c_char_p
        pc = C.POINTER(PagedCacheDesc)
        L.pact_cache_plan.argtypes = [vp, vp, vp]
        L.pact_cache_write.argtypes = [vp, pc, vp, vp]
        L.pact_page_select.argtypes = [vp, pc, vp, vp]
        L.pact_paged_attention.argtypes = [vp, pc, vp, vp]
        L.pact_paged_workspace_bytes.argtypes = [vp, i32, i32]
        L.pact_paged_workspace_bytes.restype = sz
        for name in EXPORTS:
            if getattr(L, name).restype is C.c_int:
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


class PactError(RuntimeError):
    pass


def _check(ctx, status: int):
    if status != 0:
        L = lib()
        msg = L.pact_status_string(status).decode()
        if status == -4 and ctx is not None:
            msg += ": " + L.pact_last_cuda_error(ctx).decode()
        raise PactError(f"pact status {status}: {msg}")


def _ptr(t):
    """Address of a tensor (ctypes takes plain integers for the pointer arguments and fields), None for None."""
    return None if t is None else t.data_ptr()


def _stream_getter():
    """Handle of the current stream of the current device, without a Stream object around it (3 us of a call) where this
    version of torch has the two functions for that."""
    private = getattr(torch, "_C", None)
    raw, device = getattr(private, "_cuda_getCurrentRawStream", None), getattr(private, "_cuda_getDevice", None)
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


_stream = _stream_getter()


def _dt(dtype) -> int:
    if dtype == torch.bfloat16:
        return PACT_BF16
    if dtype == torch.float32:
        return PACT_F32
    raise PactError(f"unsupported dtype {dtype}")


def make_params(lam=0.5, d_c=0.3, d_n=2.0, alpha=1.5, n_prune=-1, flags=0) -> Params:
    return Params(float(lam), float(d_c), float(d_n), float(alpha), int(n_prune), int(flags))


@dataclass
class DeviceImage:
    """Device tensors of one image plus its output buffers (all owned by the caller)."""
    H: torch.Tensor
    K_euti: torch.Tensor
    Q_euti: torch.Tensor
    K_clu: torch.Tensor
    P: torch.Tensor
    vis_start: int
    N: int
    H_out: torch.Tensor
    P_out: torch.Tensor
    size_out: torch.Tensor
    label: torch.Tensor
    score: torch.Tensor
    keep: torch.Tensor
    counters: torch.Tensor
    logw_out: torch.Tensor = None

    def desc(self) -> ImageDesc:
        return ImageDesc(_ptr(self.H), self.H.stride(0), _ptr(self.K_euti), self.K_euti.stride(0),
                         _ptr(self.Q_euti), self.Q_euti.stride(0), _ptr(self.K_clu), self.K_clu.stride(0),
                         _ptr(self.P), self.H.shape[0], self.vis_start, self.N, 0,
                         _ptr(self.H_out), self.H_out.stride(0), _ptr(self.P_out), _ptr(self.size_out),
                         _ptr(self.label), _ptr(self.score), _ptr(self.keep), _ptr(self.counters),
                         _ptr(self.logw_out))


def device_image(img, out_dtype, device="cuda") -> DeviceImage:
    """Uploads a workloads.Image and allocates its outputs."""
    H = img.H.to(device)
    K = img.K.to(device)
    Kc = K if img.K_clu is None else img.K_clu.to(device)
    n_total, d = H.shape
    return DeviceImage(H, K, img.Q.to(device), Kc, img.P.to(device), img.vis_start, img.N,
                       torch.empty((n_total, d), dtype=out_dtype, device=device),
                       torch.empty(n_total, dtype=torch.int32, device=device),
                       torch.empty(n_total, dtype=torch.int32, device=device),
                       torch.empty(img.N, dtype=torch.int32, device=device),
                       torch.empty(img.N, dtype=torch.float32, device=device),
                       torch.empty(img.N, dtype=torch.uint8, device=device),
                       torch.zeros(N_COUNTERS, dtype=torch.int32, device=device),
                       torch.empty(n_total, dtype=torch.float32, device=device))


class Graph:
    """A recorded pact_reduce; launch() replays it on the current stream.  Keeps the tensors it
    points at alive."""

    def __init__(self, ctx, handle, images, ws):
        self._ctx, self.handle, self._images, self._ws = ctx, handle, images, ws

    def launch(self):
        _check(self._ctx.handle, self._ctx._L.pact_graph_launch(self.handle, _stream()))

    def close(self):
        if self.handle:
            self._ctx._L.pact_graph_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _strides(t, what: str):
    """Strides of a tensor whose last axis is contiguous; an axis of one element gets the stride that it would have if packed."""
    shape, st = t.shape, list(t.stride())
    if st[-1] != 1 and shape[-1] != 1:
        raise PactError(f"{what}: the last axis has to be contiguous")
    st[-1] = 1
    for i in range(len(st) - 2, -1, -1):
        if shape[i] == 1:
            st[i] = max([st[j] * shape[j] for j in range(len(st)) if shape[j] > 1 or j == len(st) - 1])
    return st


class PagedCache:
    """One layer's paged cache, the tensors of pact_paged_cache in pact.h: K, V [n_pages, n_kvh, page_rows, d_h] (any strides with a contiguous last
    axis; rows before heads is a transposed view), logw [n_pages, page_rows] fp32, bounds [n_pages, n_kvh, 2, d_h], w_max [n_pages] fp32.  The
    caller owns them; the handle keeps them alive."""

    def __init__(self, K, V, logw=None, bounds=None, w_max=None):
        if K.dim() != 4 or V.shape != K.shape or V.dtype != K.dtype:
            raise PactError("K and V are [n_pages, n_kvh, page_rows, d_h] of one type")
        self.K, self.V, self.logw, self.bounds, self.w_max = K, V, logw, bounds, w_max
        self.n_pages, self.n_kvh, self.page_rows, self.d_h = K.shape
        self.dtype, self.device = K.dtype, K.get_device()
        for t, dtype, shape, what in ((logw, torch.float32, (self.n_pages, self.page_rows), "logw"), (w_max, torch.float32, (self.n_pages,), "w_max"),
                                      (bounds, K.dtype, (self.n_pages, self.n_kvh, 2, self.d_h), "bounds")):
            if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()):
                raise PactError(f"{what}: a contiguous {dtype} tensor of shape {shape} is wanted")
        if any(t is not None and t.get_device() != self.device for t in (V, logw, bounds, w_max)):
            raise PactError("the tensors of a cache are on one device")
        k, v = _strides(K, "K"), _strides(V, "V")
        self.desc = PagedCacheDesc(_ptr(K), _ptr(V), k[0], k[1], k[2], v[0], v[1], v[2], _ptr(logw), _ptr(bounds), _ptr(w_max),
                                   self.n_pages, self.page_rows)
        self.ref = C.byref(self.desc)
        self.kind = (self.n_kvh, self.d_h, self.dtype, self.device)


PRUNE_STATIC_MAX_N = 65536


def pact_prune_static(score, params: Params, keep, kept_idx, pruned_idx, counts):
    """pact_prune without context or workspace, for callers that may not allocate device memory.
    score.numel() <= PRUNE_STATIC_MAX_N."""
    _check(None, lib().pact_prune_static(_ptr(score), score.numel(), C.byref(params), _ptr(keep), _ptr(kept_idx),
                                         _ptr(pruned_idx), _ptr(counts), _stream()))


class Context:
    """Owns a pact_ctx and a caller-side workspace tensor."""

    def __init__(self, d, n_qh, n_kvh, d_h, in_dtype=torch.bfloat16, out_dtype=torch.bfloat16):
        self._L = lib()
        self.handle = C.c_void_p()
        self.in_dtype, self.out_dtype = in_dtype, out_dtype
        self.d, self.n_qh, self.n_kvh, self.d_h = d, n_qh, n_kvh, d_h
        _check(None, self._L.pact_create(C.byref(self.handle), d, n_qh, n_kvh, d_h, _dt(in_dtype), _dt(out_dtype)))
        self.ws = None
        self._need = {}                      # (max_batch, max_N) -> workspace bytes, asked from the library once
        self.device = torch.cuda.current_device()
        self._paged_ws = []                  # workspaces of the paged cache's calls: address, size, tensor; the last one is in use
        self._paged_need = {}
        self._make_args()

    def close(self):
        if self.handle:
            self._L.pact_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, max_batch, max_N) -> int:
        return int(self._L.pact_workspace_bytes(self.handle, max_batch, max_N))

    def ensure_workspace(self, max_batch, max_N):
        need = self._need.get((max_batch, max_N))
        if need is None:
            if len(self._need) >= 4096:
                self._need.clear()
            need = self._need[(max_batch, max_N)] = self.workspace_bytes(max_batch, max_N)
        if self.ws is None or self.ws.numel() < need:
            self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self.ws

    def _ws(self):
        return self.ws.data_ptr(), self.ws.numel()

    # ---- stage calls ------------------------------------------------------------------
    def pact_importance(self, im: DeviceImage, params: Params, score: torch.Tensor):
        self.ensure_workspace(1, im.N)
        d = im.desc()
        w, n = self._ws()
        _check(self.handle, self._L.pact_importance(self.handle, C.byref(d), C.byref(params), _ptr(score), w, n, _stream()))

    def pact_prune(self, score, params: Params, keep, kept_idx, pruned_idx, counts):
        N = score.numel()
        self.ensure_workspace(1, N)
        w, n = self._ws()
        _check(self.handle, self._L.pact_prune(self.handle, _ptr(score), N, C.byref(params), _ptr(keep),
                                               _ptr(kept_idx), _ptr(pruned_idx), _ptr(counts), w, n, _stream()))

    def pact_dbdpc(self, K, idx, q_dev, params: Params, rho, center_idx, C_dev, label, counters=None):
        N = K.shape[0]
        self.ensure_workspace(1, N)
        w, n = self._ws()
        _check(self.handle, self._L.pact_dbdpc(self.handle, _ptr(K), K.stride(0), N, _ptr(idx), _ptr(q_dev),
                                               C.byref(params), _ptr(rho), _ptr(center_idx), _ptr(C_dev),
                                               _ptr(label), _ptr(counters), w, n, _stream()))

    def pact_reincorporate(self, K, pruned_idx, m_dev, center_idx, C_dev, params: Params, label, r_dev,
                           counters=None):
        N = K.shape[0]
        self.ensure_workspace(1, N)
        w, n = self._ws()
        _check(self.handle, self._L.pact_reincorporate(self.handle, _ptr(K), K.stride(0), N, _ptr(pruned_idx),
                                                       _ptr(m_dev), _ptr(center_idx), _ptr(C_dev),
                                                       C.byref(params), _ptr(label), _ptr(r_dev),
                                                       _ptr(counters), w, n, _stream()))

    def pact_key_spread(self, K_layers, threshold: float, max_dist, layer_out=None):
        """K_layers: list of [N, d_k] key matrices (same N and row stride), one per layer."""
        N, ld = K_layers[0].shape[0], K_layers[0].stride(0)
        assert all(K.shape[0] == N and K.stride(0) == ld for K in K_layers)
        self.ensure_workspace(min(len(K_layers), 16), N)
        arr = (C.c_void_p * len(K_layers))(*[K.data_ptr() for K in K_layers])
        w, n = self._ws()
        _check(self.handle, self._L.pact_key_spread(self.handle, arr, len(K_layers), ld, N, float(threshold),
                                                    _ptr(max_dist), _ptr(layer_out), w, n, _stream()))

    def pact_merge(self, im: DeviceImage, label, center_idx, C_dev, params: Params):
        self.ensure_workspace(1, im.N)
        d = im.desc()
        w, n = self._ws()
        _check(self.handle, self._L.pact_merge(self.handle, C.byref(d), _ptr(label), _ptr(center_idx),
                                               _ptr(C_dev), C.byref(params), w, n, _stream()))

    # ---- the whole step -----------------------------------------------------------------
    def pact_reduce(self, images, params):
        """images: list of DeviceImage; params: one Params or a list with one per image."""
        B = len(images)
        self.ensure_workspace(B, max(im.N for im in images))
        arr = (ImageDesc * B)(*[im.desc() for im in images])
        if isinstance(params, Params):
            parr, stride = (Params * 1)(params), 0
        else:
            parr, stride = (Params * B)(*params), 1
        w, n = self._ws()
        _check(self.handle, self._L.pact_reduce(self.handle, arr, B, parr, stride, w, n, _stream()))

    def pact_graph_create(self, images, params):
        """Records pact_reduce(images, params) as a replayable graph (see Graph)."""
        B = len(images)
        self.ensure_workspace(B, max(im.N for im in images))
        arr = (ImageDesc * B)(*[im.desc() for im in images])
        if isinstance(params, Params):
            parr, stride = (Params * 1)(params), 0
        else:
            parr, stride = (Params * B)(*params), 1
        w, n = self._ws()
        h = C.c_void_p()
        _check(self.handle, self._L.pact_graph_create(self.handle, arr, B, parr, stride, w, n, C.byref(h)))
        return Graph(self, h, images, self.ws)

    # ---- the paged cache ------------------------------------------------------------------
    # (A call of a decoding step takes the GPU a few microseconds, and looking at nine tensors one function call each takes as long: the methods test
    # everything in one expression and ask _explain only when it fails.)
    def _make_args(self):
        self._args = C.create_string_buffer(max(_PLAN.size, _NEW_ROWS.size, _QUERY.size))
        self._args_at = C.addressof(self._args)
        self._kind = (self.n_kvh, self.d_h, self.in_dtype, self.device)

    def _explain(self, cache, *wanted):
        """Raises for the first of these that is not what is wanted: (tensor or None, dtype, shape, what), dense or, for [.., heads, d_h], strided."""
        if cache is not None and cache.kind != self._kind:
            raise PactError(f"the cache is not one of {self.n_kvh} key heads of {self.d_h} {self.in_dtype} on cuda:{self.device}")
        for t, dtype, shape, strided, what in wanted:
            if t is None:
                continue
            if t.dtype != dtype or t.get_device() != self.device or t.ndim != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
                raise PactError(f"{what}: a {dtype} tensor of shape [{', '.join('..' if n is None else str(n) for n in shape)}] on cuda:{self.device} is wanted")
            if not t.is_contiguous() if not strided else t.stride()[-1] != 1 and t.shape[-1] != 1:
                raise PactError(f"{what}: {'a contiguous tensor is wanted' if not strided else 'the last axis has to be contiguous'}")
        raise PactError("the arguments do not fit together")

    def _paged_workspace(self, B, max_pages):
        """Address and size of the workspace.  One that is outgrown is kept: a captured graph may hold its address.  (So that they are few, the next one is twice as
        large, up to 64 MB; beyond that it is as large as needed.)"""
        need = self._paged_need.get((B, max_pages))
        if need is None:
            if len(self._paged_need) >= 4096:
                self._paged_need.clear()
            need = self._paged_need[(B, max_pages)] = int(self._L.pact_paged_workspace_bytes(self.handle, B, max_pages))
        have = self._paged_ws[-1] if self._paged_ws else None
        if have is None or have[1] < need:
            size = max(need, min(2 * have[1], 64 << 20) if have else 0)   # (never less than what the attention's parts need, which does not depend on B or max_pages)
            ws = torch.empty(size, dtype=torch.uint8, device=self._cuda())
            self._paged_ws.append((ws.data_ptr(), size, ws))
        return self._paged_ws[-1]

    def _cuda(self):
        return torch.device("cuda", self.device)

    def pact_cache_plan(self, page_rows, block_table, length, n_new, free_pages, n_free, length_out, n_free_out, row_start=None, slot=None,
                        n_rows=None, row_stride=0, status=None):
        """Pages and slots of the rows that come next (pact_cache_plan in pact.h).  block_table [B, max_pages], length, length_out [B], n_new [B] (may be a
        strided view, such as the N_OUT column of the counters of a batch; negative: the request has ended), free_pages [n_pages], n_free, n_free_out
        [1], row_start [B + 1], all int32; slot [n_rows] int64; n_rows: rows that the caller has room for, where slot is not given."""
        i32, dev = torch.int32, self.device
        B, W = block_table.shape if block_table.ndim == 2 else (-1, None)
        n_pages = free_pages.numel()
        if slot is not None:
            room = slot.numel()
            if n_rows is not None and n_rows != room:
                raise PactError("n_rows is the length of slot")
            n_rows = room
        elif n_rows is None:
            raise PactError("slot or n_rows is wanted")
        if not (block_table.dtype is i32 and block_table.get_device() == dev and block_table.is_contiguous()
                and length.dtype is i32 and length.get_device() == dev and length.numel() == B and length.is_contiguous()
                and n_new.dtype is i32 and n_new.get_device() == dev and n_new.numel() == B and n_new.ndim == 1
                and free_pages.dtype is i32 and free_pages.get_device() == dev and free_pages.is_contiguous()
                and n_free.dtype is i32 and n_free.get_device() == dev and n_free.numel() == 1
                and length_out.dtype is i32 and length_out.get_device() == dev and length_out.numel() == B and length_out.is_contiguous()
                and n_free_out.dtype is i32 and n_free_out.get_device() == dev and n_free_out.numel() == 1
                and (row_start is None or row_start.dtype is i32 and row_start.get_device() == dev and row_start.numel() == B + 1 and row_start.is_contiguous())
                and (slot is None or slot.dtype is torch.int64 and slot.get_device() == dev and slot.is_contiguous())
                and (status is None or status.dtype is i32 and status.get_device() == dev and status.numel() == 1)):
            self._explain(None, (block_table, i32, (None, None), False, "block_table"), (length, i32, (B,), False, "length"), (n_new, i32, (B,), True, "n_new"),
                          (free_pages, i32, (None,), False, "free_pages"), (n_free, i32, (1,), False, "n_free"), (length_out, i32, (B,), False, "length_out"),
                          (n_free_out, i32, (1,), False, "n_free_out"), (row_start, i32, (B + 1,), False, "row_start"), (slot, torch.int64, (None,), False, "slot"),
                          (status, i32, (1,), False, "status"))
        _PLAN.pack_into(self._args, 0, page_rows, n_pages, B, W, block_table.data_ptr(), length.data_ptr(), n_new.data_ptr(), n_new.stride()[0] if B > 1 else 1,
                        free_pages.data_ptr(), n_free.data_ptr(), length_out.data_ptr(), n_free_out.data_ptr(), 0 if row_start is None else row_start.data_ptr(),
                        0 if slot is None else slot.data_ptr(), n_rows, row_stride, 0, 0 if status is None else status.data_ptr())
        r = self._L.pact_cache_plan(self.handle, self._args_at, _stream())
        if r:
            _check(self.handle, r)

    def pact_cache_write(self, cache: PagedCache, K_new, V_new, logw_new, slot, status=None):
        """Rows K_new, V_new [n, n_kvh, d_h] (alike in their strides) and logw_new [n] fp32 (None: 0) into slot [n] int64."""
        dtype, dev, heads, d_h = self.in_dtype, self.device, self.n_kvh, self.d_h
        n = slot.numel()
        shape = (n, heads, d_h)
        strides = K_new.stride()
        if not (cache.kind == self._kind and K_new.shape == shape and K_new.dtype is dtype and K_new.get_device() == dev
                and V_new.shape == shape and V_new.dtype is dtype and V_new.get_device() == dev and V_new.stride() == strides and (strides[2] == 1 or d_h == 1)
                and slot.dtype is torch.int64 and slot.get_device() == dev and slot.is_contiguous()
                and (logw_new is None or logw_new.dtype is torch.float32 and logw_new.get_device() == dev and logw_new.numel() == n and logw_new.is_contiguous())
                and (status is None or status.dtype is torch.int32 and status.get_device() == dev and status.numel() == 1)):
            if V_new.shape == K_new.shape and V_new.stride() != strides:
                raise PactError("K_new and V_new have the same strides")
            self._explain(cache, (K_new, dtype, (None, heads, d_h), True, "K_new"), (V_new, dtype, K_new.shape, True, "V_new"),
                          (slot, torch.int64, (K_new.shape[0],), False, "slot"), (logw_new, torch.float32, (n,), False, "logw_new"), (status, torch.int32, (1,), False, "status"))
        # the stride of an axis of one element is anything: the one that it would have if packed
        ld_head = strides[1] if heads > 1 else d_h
        _NEW_ROWS.pack_into(self._args, 0, K_new.data_ptr(), V_new.data_ptr(), strides[0] if n > 1 else ld_head * heads, ld_head, 0 if logw_new is None else logw_new.data_ptr(),
                            slot.data_ptr(), n, 0 if status is None else status.data_ptr())
        r = self._L.pact_cache_write(self.handle, cache.ref, self._args_at, _stream())
        if r:
            _check(self.handle, r)

    def pact_page_select(self, cache: PagedCache, Q, block_table, length, selected, n_first=1, n_last=1, scale=None, status=None):
        """Places of the pages that each request's token attends to, into selected [B, n_kvh, n_select] int32.  Q [B, n_qh, d_h]; scale: 1 / sqrt(d_h) if not given."""
        i32, dev, heads, d_h = torch.int32, self.device, self.n_qh, self.d_h
        B, W = block_table.shape if block_table.ndim == 2 else (-1, None)
        n_select = selected.shape[-1]
        q = Q.stride()
        if not (cache.kind == self._kind and Q.shape == (B, heads, d_h) and Q.dtype is self.in_dtype and Q.get_device() == dev and (q[2] == 1 or d_h == 1)
                and block_table.dtype is i32 and block_table.get_device() == dev and block_table.is_contiguous()
                and length.dtype is i32 and length.get_device() == dev and length.numel() == B and length.is_contiguous()
                and selected.dtype is i32 and selected.get_device() == dev and selected.shape == (B, self.n_kvh, n_select) and selected.is_contiguous()
                and (status is None or status.dtype is i32 and status.get_device() == dev and status.numel() == 1)):
            self._explain(cache, (block_table, i32, (None, None), False, "block_table"), (Q, self.in_dtype, (B, heads, d_h), True, "Q"), (length, i32, (B,), False, "length"),
                          (selected, i32, (B, self.n_kvh, None), False, "selected"), (status, i32, (1,), False, "status"))
        w, n, _ = self._paged_workspace(B, W)
        qh = q[1] if heads > 1 else d_h
        _QUERY.pack_into(self._args, 0, Q.data_ptr(), q[0] if B > 1 else qh * heads, qh, block_table.data_ptr(), length.data_ptr(), B, W, selected.data_ptr(), n_select, n_first, n_last,
                         d_h ** -0.5 if scale is None else scale, 0, 0, 0, 0, 0 if status is None else status.data_ptr(), w, n)
        r = self._L.pact_page_select(self.handle, cache.ref, self._args_at, _stream())
        if r:
            _check(self.handle, r)

    def pact_paged_attention(self, cache: PagedCache, Q, block_table, length, out, lse=None, selected=None, scale=None, status=None):
        """Attention of one token per request, Q [B, n_qh, d_h] -> out [B, n_qh, d_h] (the context's output type), lse [B, n_qh] fp32, over the cached rows or
        those of the pages in selected [B, n_kvh, n_select]; scale: 1 / sqrt(d_h) if not given."""
        i32, dev, heads, d_h = torch.int32, self.device, self.n_qh, self.d_h
        B, W = block_table.shape if block_table.ndim == 2 else (-1, None)
        shape = (B, heads, d_h)
        q, o = Q.stride(), out.stride()
        if not (cache.kind == self._kind and Q.shape == shape and Q.dtype is self.in_dtype and Q.get_device() == dev and (q[2] == 1 or d_h == 1)
                and out.shape == shape and out.dtype is self.out_dtype and out.get_device() == dev and (o[2] == 1 or d_h == 1)
                and block_table.dtype is i32 and block_table.get_device() == dev and block_table.is_contiguous()
                and length.dtype is i32 and length.get_device() == dev and length.numel() == B and length.is_contiguous()
                and (lse is None or lse.dtype is torch.float32 and lse.get_device() == dev and lse.numel() == B * heads and lse.is_contiguous())
                and (selected is None or selected.dtype is i32 and selected.get_device() == dev and selected.ndim == 3 and selected.shape[:2] == (B, self.n_kvh) and selected.is_contiguous())
                and (status is None or status.dtype is i32 and status.get_device() == dev and status.numel() == 1)):
            self._explain(cache, (block_table, i32, (None, None), False, "block_table"), (Q, self.in_dtype, shape, True, "Q"), (out, self.out_dtype, shape, True, "out"),
                          (length, i32, (B,), False, "length"), (lse, torch.float32, (B, heads), False, "lse"), (selected, i32, (B, self.n_kvh, None), False, "selected"),
                          (status, i32, (1,), False, "status"))
        w, n, _ = self._paged_ws[-1] if self._paged_ws else self._paged_workspace(1, 1)   # (any is large enough for the parts)
        qh, oh = (q[1], o[1]) if heads > 1 else (d_h, d_h)
        q0, o0 = (q[0], o[0]) if B > 1 else (qh * heads, oh * heads)
        _QUERY.pack_into(self._args, 0, Q.data_ptr(), q0, qh, block_table.data_ptr(), length.data_ptr(), B, W, 0 if selected is None else selected.data_ptr(),
                         0 if selected is None else selected.shape[2], 0, 0, d_h ** -0.5 if scale is None else scale, out.data_ptr(), o0, oh,
                         0 if lse is None else lse.data_ptr(), 0 if status is None else status.data_ptr(), w, n)
        r = self._L.pact_paged_attention(self.handle, cache.ref, self._args_at, _stream())
        if r:
            _check(self.handle, r)

    def set_wait_limits(self, barrier_polls: int = 0, center_sweeps: int = 0):
        """Bounds of the device-side waits (0 = default); see pact_set_wait_limits in pact.h."""
        _check(self.handle, self._L.pact_set_wait_limits(self.handle, int(barrier_polls), int(center_sweeps)))

    def launch_count(self) -> int:
        return int(self._L.pact_launch_count(self.handle))

    def profile_enable(self, on: bool):
        _check(self.handle, self._L.pact_profile_enable(self.handle, 1 if on else 0))

    def profile_read(self) -> dict:
        """Per-kernel milliseconds of the last profiled pact_reduce (waits for it to finish)."""
        buf = (C.c_float * 16)()
        n = self._L.pact_profile_read(self.handle, buf, 16)
        return {self._L.pact_profile_stage_name(i).decode(): float(buf[i]) for i in range(n)}

    def host_staging_bytes(self, n_total, N) -> int:
        return int(self._L.pact_host_staging_bytes(self.handle, n_total, N))

    def pact_reduce_host(self, host: dict, params: Params, staging: torch.Tensor):
        """host: dict of pinned CPU tensors H, K_euti, Q_euti, K_clu, P, H_out, P_out, size_out,
        label, counters (and optionally logw_out) plus vis_start, N.  Copies in, reduces, copies the valid rows out."""
        self.ensure_workspace(1, host["N"])
        H = host["H"]
        d = ImageDesc(_ptr(H), H.stride(0), _ptr(host["K_euti"]), host["K_euti"].stride(0),
                      _ptr(host["Q_euti"]), host["Q_euti"].stride(0), _ptr(host["K_clu"]),
                      host["K_clu"].stride(0), _ptr(host["P"]), H.shape[0], host["vis_start"], host["N"], 0,
                      _ptr(host["H_out"]), host["H_out"].stride(0), _ptr(host["P_out"]),
                      _ptr(host["size_out"]), _ptr(host.get("label")), None, None, _ptr(host["counters"]),
                      _ptr(host.get("logw_out")))
        w, n = self._ws()
        _check(self.handle, self._L.pact_reduce_host(self.handle, C.byref(d), C.byref(params),
                                                     _ptr(staging), staging.numel(), w, n, _stream()))
