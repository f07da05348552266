"""ctypes binding of the Sol-Attn C ABI (``include/sol_attn.h``).

Argument marshalling only: every step of the path runs in the CUDA library.  Tensors are
torch CUDA tensors (bf16 ``[B, H, N, d]``, contiguous); torch provides device memory and
streams, nothing else.  The functions mirror the C entry points by name.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SOL_ATTN_LIB", os.path.join(_PKG, "libsol_attn.so"))   # override: profiling build

SOL_OK = 0
SOL_ERR_INVALID_ARG = -1
SOL_ERR_UNSUPPORTED_SHAPE = -2
SOL_ERR_UNSUPPORTED_ARCH = -3
SOL_ERR_WORKSPACE = -4
SOL_ERR_CUDA = -5
SOL_ERR_DEVICE_TIMEOUT = -6
SOL_ERR_SCRATCH_LIMIT = -7
SOL_ERR_STATIC_SCRATCH = -8

SOL_MODE_SOL, SOL_MODE_DENSE, SOL_MODE_EXACT_ONLY = 0, 1, 2
SOL_IMPL_AUTO, SOL_IMPL_TCGEN05, SOL_IMPL_MMA_SYNC = 0, 1, 2
SOL_EST_MOMENTS, SOL_EST_DIAGONAL = 0, 1
SOL_LAYOUT_BHND, SOL_LAYOUT_BNHD = 0, 1
SOL_ROUTING_FUSED, SOL_ROUTING_PREPASS = 0, 1
SOL_ROUTE_TOPK, SOL_ROUTE_TOPP = 0, 1
SOL_TYPE_BF16, SOL_TYPE_FP16 = 0, 1

EXPORTS = [
    "sol_attn_status_string", "sol_attn_workspace_bytes", "sol_attn_workspace_view",
    "sol_attn_bind_workspace", "sol_attn_pool", "sol_attn_forward", "sol_attn_dense",
    "sol_attn_forward_ex", "sol_attn_forward_host", "sol_attn_read_device_status",
    "sol_attn_launch_count", "sol_attn_thresholds_static", "sol_attn_thresholds_static_max_floats",
    "sol_attn_route_materialized", "sol_attn_thresholds", "sol_attn_debug_set_wait", "sol_attn_route_mask",
    "sol_attn_block_tables", "sol_attn_qk_norm_rope", "sol_attn_cache_bytes", "sol_attn_cache_append", "sol_attn_cache_read",
    "sol_attn_cache_attention", "sol_attn_cache_workspace_bytes", "sol_attn_cache_read_status",
]


class SolAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _WsView(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in
                ("status", "qbar", "kc", "vc", "mu", "sigma", "tau", "total_bytes")] + \
               [("n_q_blocks", ctypes.c_int32), ("n_k_blocks", ctypes.c_int32)]


class _Args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p),
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("d", ctypes.c_int32),
        ("block_q", ctypes.c_int32), ("block_k", ctypes.c_int32),
        ("threshold", ctypes.c_float), ("scale", ctypes.c_float),
        ("mode", ctypes.c_int32), ("impl", ctypes.c_int32), ("skip_pool", ctypes.c_int32),
        ("tau_override", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("counts", ctypes.c_void_p), ("mask_out", ctypes.c_void_p),
        ("stream", ctypes.c_void_p),
        ("estimator", ctypes.c_int32), ("forced_blocks", ctypes.c_void_p),
        ("layout", ctypes.c_int32), ("routing", ctypes.c_int32),
    ]


class _Cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int32) for n in ("pages", "page_size", "Hk", "d", "k_exp", "v_exp")]


class _TablesArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("old_lens", "new_lens", "free_pages", "free_count", "block_tables", "cu_q", "kv_lens",
                                               "slots", "positions", "result")] + \
               [("table_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("requests", "max_blocks", "max_tokens", "free_capacity", "page_size")] + \
               [("stream", ctypes.c_void_p)]


class _NormArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out")] + \
               [(n, ctypes.c_int64 * 3) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")] + \
               [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight", "cos", "sin", "positions")] + \
               [(n, ctypes.c_int32) for n in ("batch", "tokens", "Hq", "Hk", "d", "rot", "interleaved", "table_rows", "type")] + \
               [("eps", ctypes.c_float), ("stream", ctypes.c_void_p)]


class _CacheArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "out", "lse")] + \
               [("q_stride", ctypes.c_int64 * 2), ("out_stride", ctypes.c_int64 * 2), ("table_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("cu_q", "kv_lens", "block_tables")] + [("cache", _Cache)] + \
               [(n, ctypes.c_int32) for n in ("tokens", "requests", "max_blocks", "max_q", "Hq", "type", "causal")] + \
               [("scale", ctypes.c_float), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("stream", ctypes.c_void_p)]


# The same layouts for struct.pack, which is several times as fast as building a ctypes structure: a call's host time is what bounds
# the smallest calls.
_PACK_CACHE, _PACK_TABLES = struct.Struct("@P6i"), struct.Struct("@10Pq5iP")
_PACK_NORM, _PACK_ATTENTION = struct.Struct("@4P12q5P9ifP"), struct.Struct("@3P5q3PP6i7ifPNP")
_PACK_TWO = struct.Struct("@2q")

_lib = None


def lib() -> ctypes.CDLL:
    """Load the CUDA library; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2607_24027_b200.build` "
                          "(there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    L.sol_attn_status_string.restype = ctypes.c_char_p
    L.sol_attn_status_string.argtypes = [ctypes.c_int32]
    L.sol_attn_workspace_bytes.restype = ctypes.c_size_t
    L.sol_attn_workspace_bytes.argtypes = [ctypes.c_int] * 6
    L.sol_attn_workspace_view.restype = ctypes.c_int32
    L.sol_attn_workspace_view.argtypes = [ctypes.c_int] * 6 + [ctypes.POINTER(_WsView)]
    L.sol_attn_bind_workspace.restype = ctypes.c_int32
    L.sol_attn_bind_workspace.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    L.sol_attn_pool.restype = ctypes.c_int32
    L.sol_attn_pool.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
    L.sol_attn_thresholds.restype = ctypes.c_int32
    L.sol_attn_thresholds.argtypes = [ctypes.c_int] * 6 + [ctypes.c_float] * 2 + [ctypes.c_int, ctypes.c_void_p]
    L.sol_attn_forward.restype = ctypes.c_int32
    L.sol_attn_forward.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
    L.sol_attn_dense.restype = ctypes.c_int32
    L.sol_attn_dense.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int] * 4 + [ctypes.c_void_p]
    L.sol_attn_forward_ex.restype = ctypes.c_int32
    L.sol_attn_forward_ex.argtypes = [ctypes.POINTER(_Args)]
    L.sol_attn_forward_host.restype = ctypes.c_int32
    L.sol_attn_forward_host.argtypes = [ctypes.c_void_p] * 8 + [ctypes.c_int] * 6 + [ctypes.c_float, ctypes.c_void_p]
    L.sol_attn_read_device_status.restype = ctypes.c_int32
    L.sol_attn_read_device_status.argtypes = [ctypes.c_void_p]
    L.sol_attn_launch_count.restype = ctypes.c_int64
    L.sol_attn_launch_count.argtypes = []
    L.sol_attn_route_mask.restype = ctypes.c_int32
    L.sol_attn_route_mask.argtypes = [ctypes.c_int] * 6 + [ctypes.c_float] + [ctypes.c_void_p] * 4
    L.sol_attn_thresholds_static.restype = ctypes.c_int32
    L.sol_attn_thresholds_static.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 5 + [ctypes.c_float] * 2 + \
                                            [ctypes.c_void_p] * 4
    L.sol_attn_thresholds_static_max_floats.restype = ctypes.c_size_t
    L.sol_attn_thresholds_static_max_floats.argtypes = []
    L.sol_attn_route_materialized.restype = ctypes.c_int32
    L.sol_attn_route_materialized.argtypes = [ctypes.c_void_p] * 2 + [ctypes.c_int] * 5 + [ctypes.c_float, ctypes.c_int,
                                                                                           ctypes.c_float] + \
                                             [ctypes.c_void_p] * 5
    L.sol_attn_block_tables.restype = ctypes.c_int32
    L.sol_attn_block_tables.argtypes = [ctypes.c_void_p]        # (structures packed by hand)
    L.sol_attn_qk_norm_rope.restype = ctypes.c_int32
    L.sol_attn_qk_norm_rope.argtypes = [ctypes.c_void_p]
    L.sol_attn_cache_bytes.restype = ctypes.c_size_t
    L.sol_attn_cache_bytes.argtypes = [ctypes.c_int] * 4
    for f in (L.sol_attn_cache_append, L.sol_attn_cache_read):
        f.restype = ctypes.c_int32
        f.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
    L.sol_attn_cache_attention.restype = ctypes.c_int32
    L.sol_attn_cache_attention.argtypes = [ctypes.c_void_p]
    L.sol_attn_cache_workspace_bytes.restype = ctypes.c_size_t
    L.sol_attn_cache_workspace_bytes.argtypes = [ctypes.c_int] * 4
    L.sol_attn_cache_read_status.restype = ctypes.c_int32
    L.sol_attn_cache_read_status.argtypes = [ctypes.c_void_p] * 2
    L.sol_attn_debug_set_wait.restype = None
    L.sol_attn_debug_set_wait.argtypes = [ctypes.c_int64, ctypes.c_int32]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().sol_attn_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != SOL_OK:
        raise SolAttnError(status, where)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # 0.1 us; torch.cuda.current_stream() takes 3


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dims(q: torch.Tensor):
    if q.dim() != 4 or not q.is_contiguous() or q.dtype != torch.bfloat16 or not q.is_cuda:
        raise ValueError("expected a contiguous CUDA bf16 tensor of shape [B, H, N, d]")
    return tuple(int(x) for x in q.shape)


# ----------------------------------------------------------------------------- workspace
def sol_attn_workspace_bytes(B, H, N, d, block_q, block_k) -> int:
    return int(lib().sol_attn_workspace_bytes(B, H, N, d, block_q, block_k))


@dataclass
class Workspace:
    """A device workspace plus typed views of the pre-attention results inside it."""
    buf: torch.Tensor            # uint8
    counts: torch.Tensor         # int32 [B, H, Nq]
    shape: tuple                 # (B, H, N, d, block_q, block_k)
    view: _WsView

    def _f32(self, off, *shape):
        n = 1
        for s in shape:
            n *= s
        return self.buf[off:off + 4 * n].view(torch.float32).view(*shape)

    @property
    def qbar(self):
        B, H, _, d, _, _ = self.shape
        return self._f32(self.view.qbar, B, H, self.view.n_q_blocks, d)

    @property
    def kc(self):
        B, H, _, d, _, _ = self.shape
        return self._f32(self.view.kc, B, H, self.view.n_k_blocks, d)

    @property
    def vc(self):
        B, H, _, d, _, _ = self.shape
        return self._f32(self.view.vc, B, H, self.view.n_k_blocks, d)

    def _per_q(self, off):
        B, H = self.shape[:2]
        return self._f32(off, B, H, self.view.n_q_blocks)

    @property
    def mu(self):
        return self._per_q(self.view.mu)

    @property
    def sigma(self):
        return self._per_q(self.view.sigma)

    @property
    def tau(self):
        return self._per_q(self.view.tau)


def make_workspace(B, H, N, d, block_q, block_k, device="cuda") -> Workspace:
    """Allocate (with torch) a workspace and counts array for one problem shape."""
    view = _WsView()
    _check(lib().sol_attn_workspace_view(B, H, N, d, block_q, block_k, ctypes.byref(view)), "sol_attn_workspace_view")
    buf = torch.empty(view.total_bytes + 1024, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 1024
    buf = buf[off:off + view.total_bytes]
    counts = torch.zeros(B, H, view.n_q_blocks, dtype=torch.int32, device=device)
    return Workspace(buf=buf, counts=counts, shape=(B, H, N, d, block_q, block_k), view=view)


def sol_attn_bind_workspace(ws: Optional[Workspace]):
    if ws is None:
        _check(lib().sol_attn_bind_workspace(None, 0, None), "sol_attn_bind_workspace")
    else:
        _check(lib().sol_attn_bind_workspace(ws.buf.data_ptr(), ws.buf.numel(), ws.counts.data_ptr()),
               "sol_attn_bind_workspace")


# ----------------------------------------------------------------------------- entry points
def sol_attn_pool(q, k, v, block_q, block_k, threshold, stream=None):
    B, H, N, d = _dims(k)
    _check(lib().sol_attn_pool(_ptr(q), _ptr(k), _ptr(v), B, H, N, d, block_q, block_k,
                               float(threshold), _stream(stream)), "sol_attn_pool")


def sol_attn_forward(q, k, v, out, block_q, block_k, threshold, stream=None):
    B, H, N, d = _dims(q)
    _check(lib().sol_attn_forward(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, N, d, block_q, block_k,
                                  float(threshold), _stream(stream)), "sol_attn_forward")


def sol_attn_dense(q, k, v, out, stream=None):
    B, H, N, d = _dims(q)
    _check(lib().sol_attn_dense(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, N, d, _stream(stream)),
           "sol_attn_dense")


def sol_attn_forward_ex(q, k, v, out, ws: Workspace, block_q, block_k, threshold=0.0, scale=0.0,
                        mode=SOL_MODE_SOL, impl=SOL_IMPL_AUTO, skip_pool=False, tau_override=None,
                        counts=None, mask_out=None, stream=None, estimator=SOL_EST_MOMENTS, forced_blocks=None,
                        layout=SOL_LAYOUT_BHND, routing=SOL_ROUTING_FUSED):
    """``layout=SOL_LAYOUT_BNHD``: q, k, v and out are [B, N, H, d] tensors (heads interleaved)."""
    B, H, N, d = _dims(q)
    if layout == SOL_LAYOUT_BNHD:
        H, N = N, H
    a = _Args(q=_ptr(q), k=_ptr(k), v=_ptr(v), out=_ptr(out), B=B, H=H, N=N, d=d,
              block_q=block_q, block_k=block_k, threshold=float(threshold), scale=float(scale),
              mode=mode, impl=impl, skip_pool=int(skip_pool), tau_override=_ptr(tau_override),
              workspace=ws.buf.data_ptr(), workspace_bytes=ws.buf.numel(),
              counts=_ptr(counts if counts is not None else ws.counts), mask_out=_ptr(mask_out),
              stream=_stream(stream), estimator=int(estimator), forced_blocks=_ptr(forced_blocks),
              layout=int(layout), routing=int(routing))
    _check(lib().sol_attn_forward_ex(ctypes.byref(a)), "sol_attn_forward_ex")


def sol_attn_forward_host(hq, hk, hv, hout, dq, dk, dv, dout, block_q, block_k, threshold, stream=None):
    B, H, N, d = _dims(dq)
    _check(lib().sol_attn_forward_host(hq.data_ptr(), hk.data_ptr(), hv.data_ptr(), hout.data_ptr(),
                                       _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dout), B, H, N, d,
                                       block_q, block_k, float(threshold), _stream(stream)),
           "sol_attn_forward_host")


def sol_attn_thresholds_static(qbar, kc, threshold, mu, sigma, tau, scale=0.0, stream=None):
    """mu, sigma, tau (fp32 [B, H, Nq], caller-owned) from pooled queries / keys (fp32 [B, H, N*, d]) without
    any device allocation: the pooled-key moments go to an array built into the library."""
    B, H, Nq, d = (int(x) for x in qbar.shape)
    Nk = int(kc.shape[2])
    for t in (qbar, kc, mu, sigma, tau):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("expected contiguous CUDA fp32 tensors")
    _check(lib().sol_attn_thresholds_static(_ptr(qbar), _ptr(kc), B, H, Nq, Nk, d, float(scale), float(threshold),
                                            _ptr(mu), _ptr(sigma), _ptr(tau), _stream(stream)),
           "sol_attn_thresholds_static")


def sol_attn_thresholds(B, H, N, d, block_q, block_k, threshold, scale=0.0, estimator=SOL_EST_MOMENTS, stream=None):
    """Recompute mu, sigma, tau in the bound workspace from the pooled tensors already there."""
    _check(lib().sol_attn_thresholds(B, H, N, d, block_q, block_k, float(threshold), float(scale), int(estimator),
                                     _stream(stream)), "sol_attn_thresholds")


def sol_attn_route_mask(B, H, N, d, block_q, block_k, mask, scale=0.0, tau_override=None, forced_blocks=None, stream=None):
    """Eq. (4) decisions of the bound workspace's pooled tensors and thresholds, one bit per block pair, into ``mask``
    (int32 / uint32 [B, H, Nq, ceil(Nk / 32)])."""
    _check(lib().sol_attn_route_mask(B, H, N, d, block_q, block_k, float(scale), _ptr(tau_override), _ptr(forced_blocks),
                                     _ptr(mask), _stream(stream)), "sol_attn_route_mask")


def sol_attn_route_materialized(qbar, kc, policy, param, proxy_map, tau, order=None, counts=None, scale=0.0,
                                stream=None):
    """Top-k / top-p routing over a proxy map written to ``proxy_map`` (fp32 [B, H, Nq, Nk]); fills ``tau``
    (fp32 [B, H, Nq], usable as ``tau_override``), optionally ``order`` (int32 [B, H, Nq, Nk]) and ``counts``."""
    B, H, Nq, d = (int(x) for x in qbar.shape)
    Nk = int(kc.shape[2])
    for t in (qbar, kc, proxy_map, tau):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("expected contiguous CUDA fp32 tensors")
    for t in (order, counts):
        if t is not None and (t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous()):
            raise ValueError("expected contiguous CUDA int32 tensors")
    if proxy_map.numel() != B * H * Nq * Nk or tau.numel() != B * H * Nq:
        raise ValueError("proxy_map / tau have the wrong size")
    _check(lib().sol_attn_route_materialized(_ptr(qbar), _ptr(kc), B, H, Nq, Nk, d, float(scale), int(policy),
                                             float(param), _ptr(proxy_map), _ptr(order), _ptr(tau), _ptr(counts),
                                             _stream(stream)),
           "sol_attn_route_materialized")


def sol_attn_thresholds_static_max_floats() -> int:
    return int(lib().sol_attn_thresholds_static_max_floats())


def sol_attn_read_device_status(stream=None) -> int:
    return int(lib().sol_attn_read_device_status(_stream(stream)))


def sol_attn_launch_count() -> int:
    return int(lib().sol_attn_launch_count())


def sol_attn_debug_set_wait(wait_cycles: int = 0, withhold_tile: int = -1):
    """Testing hook: bound of the kernel's device-side waits (SM clocks, <= 0: default) and the tile per CTA
    whose completion signal is withheld (< 0: none)."""
    lib().sol_attn_debug_set_wait(int(wait_cycles), int(withhold_tile))


# ----------------------------------------------------------------------------- cache of keys and values in 4 bits
# What the library cannot see is checked here: types, shapes, and that everything lies on the current device (a call takes its device and
# its stream from there).
_TYPES = {torch.bfloat16: SOL_TYPE_BF16, torch.float16: SOL_TYPE_FP16}
_I32, _F32, _U8 = torch.int32, torch.float32, torch.uint8


def _here(stream):
    """(current device, address of the stream: the given one, or the device's current one)"""
    dev = torch.cuda.current_device()
    if stream is None and _raw_stream is not None:
        return dev, _raw_stream(dev)
    if stream is not None and stream.device.index != dev:
        raise ValueError(f"the stream is not one of the current device ({dev})")
    return dev, _stream(stream)


def _flat(dev, dtype, name, t, shape) -> int:
    """The address of a contiguous tensor of this type and shape on device `dev`; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {list(shape)} on the current CUDA device")
    return t.data_ptr()


def _table(dev, t, B):
    """(address, distance of its rows, columns) of a block table of B requests."""
    if t.dtype is not _I32 or t.get_device() != dev or t.dim() != 2 or t.shape[0] != B or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"block_tables: expected an int32 tensor of {B} contiguous rows on the current CUDA device")
    columns = t.shape[1]
    return t.data_ptr(), t.stride(0) if B > 1 else columns, columns


def _heads(dev, name, t, shape, dtype):
    """(address, strides) of a tensor of this shape whose channels are contiguous."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        raise ValueError(f"{name}: expected a {dtype} tensor of shape {list(shape)} on the current CUDA device")
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"{name}: the channels are not contiguous")
    return t.data_ptr(), st


def _type(dtype) -> int:
    kind = _TYPES.get(dtype)
    if kind is None:
        raise ValueError(f"expected bf16 or fp16 tensors, got {dtype}")
    return kind


def sol_attn_block_tables(old_lens, new_lens, free_pages, free_count, block_tables, cu_q, kv_lens, slots, result, page_size,
                          positions=None, stream=None):
    """Pages, slots and positions of this step's tokens: int32 tensors ``old_lens``, ``new_lens``, ``kv_lens`` [requests], ``cu_q``
    [requests + 1], ``block_tables`` [requests, max_blocks], ``slots`` and ``positions`` [max_tokens], ``free_count`` [1], ``result`` [2]."""
    (dev, st), B, n, free = _here(stream), old_lens.shape[0], slots.shape[0], free_pages.shape[0]
    table, table_stride, columns = _table(dev, block_tables, B)
    per_request, per_token = (B,), (n,)
    a = _PACK_TABLES.pack(_flat(dev, _I32, "old_lens", old_lens, per_request), _flat(dev, _I32, "new_lens", new_lens, per_request),
                          _flat(dev, _I32, "free_pages", free_pages, (free,)), _flat(dev, _I32, "free_count", free_count, (1,)), table,
                          _flat(dev, _I32, "cu_q", cu_q, (B + 1,)), _flat(dev, _I32, "kv_lens", kv_lens, per_request),
                          _flat(dev, _I32, "slots", slots, per_token), _flat(dev, _I32, "positions", positions, per_token),
                          _flat(dev, _I32, "result", result, (2,)), table_stride, B, columns, n, free, page_size, st)
    _check(lib().sol_attn_block_tables(a), "sol_attn_block_tables")


def sol_attn_qk_norm_rope(q, k, q_out, k_out, cos, sin, positions=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                          layout=SOL_LAYOUT_BNHD, stream=None):
    """RMS norm of each head and position rotation of ``q`` and ``k`` (either may be None, with its output): [B, N, H, d], or
    [B, H, N, d] with ``layout=SOL_LAYOUT_BHND``, bf16 or fp16, any strides that are multiples of 8 with contiguous channels.
    ``cos``, ``sin``: fp32 [rows, rot / 2], or None for no rotation; ``positions``: int32 [B, N]; weights: fp32 [d]."""
    x = q if q is not None else k
    if x is None or (q is None) != (q_out is None) or (k is None) != (k_out is None) or (cos is None) != (sin is None):
        raise ValueError("expected q, k or both, each with its output, and cos with sin")
    (dev, st), dtype, shape = _here(stream), x.dtype, x.shape
    kind = _type(dtype)
    if len(shape) != 4:
        raise ValueError("expected tensors of four dimensions")
    token, head = (1, 2) if layout == SOL_LAYOUT_BNHD else (2, 1)
    B, N, d = shape[0], shape[token], shape[3]
    q_at = qo_at = k_at = ko_at = Hq = Hk = 0
    qs = qos = ks = kos = (0, 0, 0)
    if q is not None:
        Hq = q.shape[head]
        of = (B, N, Hq, d) if head == 2 else (B, Hq, N, d)
        (q_at, a), (qo_at, b) = _heads(dev, "q", q, of, dtype), _heads(dev, "q_out", q_out, of, dtype)
        qs, qos = (a[0], a[token], a[head]), (b[0], b[token], b[head])
    if k is not None:
        Hk = k.shape[head]
        of = (B, N, Hk, d) if head == 2 else (B, Hk, N, d)
        (k_at, a), (ko_at, b) = _heads(dev, "k", k, of, dtype), _heads(dev, "k_out", k_out, of, dtype)
        ks, kos = (a[0], a[token], a[head]), (b[0], b[token], b[head])
    table = (0, 0) if cos is None else cos.shape
    rows, half = table
    a = _PACK_NORM.pack(q_at, k_at, qo_at, ko_at, *qs, *ks, *qos, *kos, _flat(dev, _F32, "q_weight", q_weight, (d,)),
                        _flat(dev, _F32, "k_weight", k_weight, (d,)), _flat(dev, _F32, "cos", cos, table), _flat(dev, _F32, "sin", sin, table),
                        _flat(dev, _I32, "positions", positions, (B, N)), B, N, Hq, Hk, d, 2 * half, bool(interleaved), rows, kind, eps, st)
    _check(lib().sol_attn_qk_norm_rope(a), "sol_attn_qk_norm_rope")


@dataclass
class Cache:
    """Pages of keys and values held in 4 bits (see ``sol_attn_cache`` in the header)."""
    data: torch.Tensor           # uint8
    pages: int
    page_size: int
    heads: int                   # key / value heads
    d: int
    k_exp: int = 0
    v_exp: int = 0

    def __post_init__(self):
        self._sized()

    def _sized(self):
        self._shape = self.pages, self.page_size, self.heads, self.d
        self.bytes = sol_attn_cache_bytes(*self._shape)
        if self.bytes == 0:
            raise SolAttnError(SOL_ERR_UNSUPPORTED_SHAPE, "sol_attn_cache_bytes")

    def c(self, dev: int):
        """The members of ``sol_attn_cache``."""
        if self._shape != (self.pages, self.page_size, self.heads, self.d):      # (they may have been changed since)
            self._sized()
        t = self.data
        if t.dtype is not _U8 or t.get_device() != dev or not t.is_contiguous() or t.numel() < self.bytes:
            raise ValueError(f"cache: expected a contiguous uint8 tensor of {self.bytes} bytes on the current CUDA device")
        return t.data_ptr(), self.pages, self.page_size, self.heads, self.d, self.k_exp, self.v_exp


def sol_attn_cache_bytes(pages, page_size, heads, d) -> int:
    return int(lib().sol_attn_cache_bytes(pages, page_size, heads, d))


def make_cache(pages, page_size, heads, d, k_exp=0, v_exp=0, device="cuda") -> Cache:
    """Allocate (with torch) an empty cache."""
    n = sol_attn_cache_bytes(pages, page_size, heads, d)
    return Cache(torch.zeros(n, dtype=torch.uint8, device=device), pages, page_size, heads, d, k_exp, v_exp)


def _cache_rows(cache, k, v, slots, stream):
    (dev, st), x, n = _here(stream), k if k is not None else v, slots.shape[0]
    if x is None:
        raise ValueError("expected k, v or both")
    shape, dtype = (n, cache.heads, cache.d), x.dtype
    kind = _type(dtype)
    k_at, ks = (0, (0, 0)) if k is None else _heads(dev, "k", k, shape, dtype)
    v_at, vs = (0, (0, 0)) if v is None else _heads(dev, "v", v, shape, dtype)
    return (_PACK_CACHE.pack(*cache.c(dev)), k_at, v_at, _PACK_TWO.pack(ks[0], ks[1]), _PACK_TWO.pack(vs[0], vs[1]),
            _flat(dev, _I32, "slots", slots, (n,)), n, kind, st)


def sol_attn_cache_append(k, v, slots, cache: Cache, stream=None):
    """Write keys and values [tokens, heads, d] (bf16 or fp16, contiguous channels) to their ``slots`` (int32 [tokens])."""
    if k is None or v is None:
        raise ValueError("expected k and v")
    _check(lib().sol_attn_cache_append(*_cache_rows(cache, k, v, slots, stream)), "sol_attn_cache_append")


def sol_attn_cache_read(cache: Cache, slots, k_out, v_out, stream=None):
    """Read what ``slots`` hold into ``k_out`` and ``v_out`` [tokens, heads, d] (either may be None)."""
    _check(lib().sol_attn_cache_read(*_cache_rows(cache, k_out, v_out, slots, stream)), "sol_attn_cache_read")


def sol_attn_cache_workspace_bytes(max_q, heads, kv_heads, d) -> int:
    return int(lib().sol_attn_cache_workspace_bytes(max_q, heads, kv_heads, d))


def make_cache_workspace(max_q, heads, kv_heads, d, device="cuda") -> torch.Tensor:
    """Allocate (with torch) the zeroed workspace of ``sol_attn_cache_attention``, for up to ``max_q`` queries a request."""
    n = sol_attn_cache_workspace_bytes(max_q, heads, kv_heads, d)
    if n == 0:
        raise SolAttnError(SOL_ERR_UNSUPPORTED_SHAPE, "sol_attn_cache_workspace_bytes")
    buf = torch.zeros(n + 1024, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 1024
    return buf[off:off + n]


def sol_attn_cache_attention(q, cu_q, kv_lens, block_tables, cache: Cache, out, max_q, workspace, lse=None, causal=True, scale=0.0,
                             stream=None):
    """Attention of ``q`` [tokens, heads, d] (request b: rows cu_q[b] to cu_q[b + 1]) over the first kv_lens[b] tokens of each
    request's pages, into ``out`` (as q) and ``lse`` (fp32 [tokens, heads])."""
    (dev, st), shape, dtype, B = _here(stream), q.shape, q.dtype, kv_lens.shape[0]
    kind = _type(dtype)
    if len(shape) != 3 or shape[2] != cache.d:
        raise ValueError("expected q of three dimensions, and the cache's d")
    (q_at, qs), (o_at, os_) = _heads(dev, "q", q, shape, dtype), _heads(dev, "out", out, shape, dtype)
    table, table_stride, columns = _table(dev, block_tables, B)
    if workspace.dtype is not _U8 or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous uint8 tensor on the current CUDA device")
    a = _PACK_ATTENTION.pack(q_at, o_at, _flat(dev, _F32, "lse", lse, shape[:2]), qs[0], qs[1], os_[0], os_[1], table_stride,
                             _flat(dev, _I32, "cu_q", cu_q, (B + 1,)), _flat(dev, _I32, "kv_lens", kv_lens, (B,)), table, *cache.c(dev), shape[0],
                             B, columns, max_q, shape[1], kind, bool(causal), scale, workspace.data_ptr(), workspace.numel(), st)
    _check(lib().sol_attn_cache_attention(a), "sol_attn_cache_attention")


def sol_attn_cache_read_status(workspace, stream=None) -> int:
    dev, st = _here(stream)
    if workspace.dtype is not _U8 or workspace.get_device() != dev or workspace.numel() < 1024:
        raise ValueError("workspace: expected the uint8 tensor of sol_attn_cache_attention on the current CUDA device")
    return int(lib().sol_attn_cache_read_status(workspace.data_ptr(), st))


def mask_words(n_k_blocks: int) -> int:
    return (n_k_blocks + 31) // 32
