"""Python binding of libbitcos: the C ABI's functions under the same names.

Argument marshalling only -- every step of the GEMV runs in the HIP kernels of
libbitcos.so; packing runs in its C++ host code.  Host arrays are numpy;
device buffers are torch tensors (torch supplies device memory and streams).
Sizes of device buffers are checked here, before the call, because the C ABI
takes plain pointers.
"""

from __future__ import annotations

import ctypes
import math

import numpy as np

from . import _native as N
from ._native import (FMT_BIT2, FMT_BITCOS, FMT_TRIT5, LaunchInfo, Layout, X_BF16, X_I8,  # noqa: F401
                      Y_F32, Y_F32_ADD, Y_I32_RAW, Y_I32_RAW_ADD)


_torch = None


def _t():
    """torch, imported by the first call that takes device tensors."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _ptr(a: np.ndarray) -> ctypes.c_void_p:
    return ctypes.c_void_p(a.ctypes.data)


def _w(w) -> np.ndarray:
    w = np.ascontiguousarray(w)
    if w.dtype != np.int8 or w.ndim != 2:
        raise ValueError("W must be a 2-D int8 array")
    return w


def _scales(s) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(s).view(np.uint16) if np.asarray(s).dtype == np.float16
                                else np.asarray(s, dtype=np.uint16)).reshape(-1)


def num_scales(L: Layout) -> int:
    return L.n * (L.k // 128) if L.group == 128 else 1


# ---------------------------------------------------------------------------
# plan / pack / unpack (host)
# ---------------------------------------------------------------------------

def bitcos_plan(w, group: int = 128, unit_rows: int = 0) -> Layout:
    w = _w(w)
    L = Layout()
    N.check(N.lib().bitcos_plan(_ptr(w), w.shape[0], w.shape[1], group, unit_rows, ctypes.byref(L)),
            "bitcos_plan")
    return L


def trit5_plan(w, group: int = 128) -> Layout:
    w = _w(w)
    L = Layout()
    N.check(N.lib().trit5_plan(_ptr(w), w.shape[0], w.shape[1], group, ctypes.byref(L)), "trit5_plan")
    return L


def bit2_plan(w, group: int = 128) -> Layout:
    w = _w(w)
    L = Layout()
    N.check(N.lib().bit2_plan(_ptr(w), w.shape[0], w.shape[1], group, ctypes.byref(L)), "bit2_plan")
    return L


def _pack(fn: str, w, scales, L: Layout) -> np.ndarray:
    w = _w(w)
    s = _scales(scales)
    if w.shape != (L.n, L.k) or s.size != num_scales(L):
        raise ValueError("W or scales do not match the layout")
    out = np.empty(L.total_bytes, dtype=np.uint8)
    N.check(getattr(N.lib(), fn)(_ptr(w), _ptr(s), ctypes.byref(L), _ptr(out), out.nbytes), fn)
    return out


def bitcos_pack(w, scales, L: Layout) -> np.ndarray:
    return _pack("bitcos_pack", w, scales, L)


def trit5_pack(w, scales, L: Layout) -> np.ndarray:
    return _pack("trit5_pack", w, scales, L)


def bit2_pack(w, scales, L: Layout) -> np.ndarray:
    return _pack("bit2_pack", w, scales, L)


def _unpack(fn: str, L: Layout, blob) -> tuple[np.ndarray, np.ndarray]:
    blob = np.ascontiguousarray(blob, dtype=np.uint8)
    w = np.empty((L.n, L.k), dtype=np.int8)
    s = np.empty(num_scales(L), dtype=np.uint16)
    N.check(getattr(N.lib(), fn)(ctypes.byref(L), _ptr(blob), blob.nbytes, _ptr(w), _ptr(s)), fn)
    return w, s


def bitcos_unpack(L: Layout, blob):
    return _unpack("bitcos_unpack", L, blob)


def trit5_unpack(L: Layout, blob):
    return _unpack("trit5_unpack", L, blob)


def bit2_unpack(L: Layout, blob):
    return _unpack("bit2_unpack", L, blob)


def plan_and_pack(fmt: int, w, scales, group: int = 128, unit_rows: int = 0):
    """(layout, host blob) for one of the three formats."""
    if fmt == FMT_BITCOS:
        L = bitcos_plan(w, group, unit_rows)
        return L, bitcos_pack(w, scales, L)
    if fmt == FMT_TRIT5:
        L = trit5_plan(w, group)
        return L, trit5_pack(w, scales, L)
    if fmt == FMT_BIT2:
        L = bit2_plan(w, group)
        return L, bit2_pack(w, scales, L)
    raise ValueError(f"unknown format {fmt}")


def bitcos_pack_device(w_dev, scales_dev, group: int = 128, unit_rows: int = 0, stream=None):
    """(layout, device blob) packed on the GPU from device tensors: W int8 [n][k]
    and fp16 scales ([n][k/128] or [1]).  Same bytes as the host packer."""
    import torch
    if w_dev.dtype != torch.int8 or w_dev.dim() != 2 or not w_dev.is_cuda or not w_dev.is_contiguous():
        raise ValueError("w_dev must be a contiguous 2-D int8 CUDA tensor")
    if scales_dev.dtype not in (torch.float16, torch.int16) or not scales_dev.is_cuda or not scales_dev.is_contiguous():
        raise ValueError("scales_dev must be a contiguous fp16 CUDA tensor")
    n, k = w_dev.shape
    ws_bytes = N.lib().bitcos_plan_device_workspace(n)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=w_dev.device)
    L = Layout()
    h = _stream_handle(stream)
    N.check(N.lib().bitcos_plan_device(ctypes.c_void_p(w_dev.data_ptr()), n, k, group, unit_rows,
                                       ctypes.c_void_p(ws.data_ptr()), ws_bytes, ctypes.byref(L), h),
            "bitcos_plan_device")
    if scales_dev.numel() != num_scales(L):
        raise ValueError(f"scales_dev has {scales_dev.numel()} values, layout needs {num_scales(L)}")
    blob = torch.empty(L.total_bytes, dtype=torch.uint8, device=w_dev.device)
    N.check(N.lib().bitcos_pack_device(ctypes.c_void_p(w_dev.data_ptr()), ctypes.c_void_p(scales_dev.data_ptr()),
                                       ctypes.byref(L), ctypes.c_void_p(ws.data_ptr()), ws_bytes,
                                       ctypes.c_void_p(blob.data_ptr()), L.total_bytes, h),
            "bitcos_pack_device")
    return L, blob


def bitcos_pack_device_noalloc(w_dev, scales_dev, dst_dev, group: int = 128, unit_rows: int = 0, stream=None):
    """Layout of W packed on the GPU into the caller's dst_dev (a uint8 cuda
    tensor), with the library's fixed per-GPU workspace: no device memory is
    allocated by the call.  Raises BitcosError(E_SPACE) if dst_dev is too
    small (its .status tells; the layout needed is in the exception's
    `layout`)."""
    import torch
    if w_dev.dtype != torch.int8 or w_dev.dim() != 2 or not w_dev.is_cuda or not w_dev.is_contiguous():
        raise ValueError("w_dev must be a contiguous 2-D int8 CUDA tensor")
    if scales_dev.dtype not in (torch.float16, torch.int16) or not scales_dev.is_cuda or not scales_dev.is_contiguous():
        raise ValueError("scales_dev must be a contiguous fp16 CUDA tensor")
    if dst_dev.dtype != torch.uint8 or not dst_dev.is_cuda or not dst_dev.is_contiguous():
        raise ValueError("dst_dev must be a contiguous uint8 CUDA tensor")
    n, k = w_dev.shape
    ns = n * (k // 128) if group == 128 else 1
    if scales_dev.numel() != ns:
        raise ValueError(f"scales_dev has {scales_dev.numel()} values, the layout needs {ns}")
    L = Layout()
    st = N.lib().bitcos_pack_device_noalloc(ctypes.c_void_p(w_dev.data_ptr()), ctypes.c_void_p(scales_dev.data_ptr()),
                                            n, k, group, unit_rows, ctypes.byref(L),
                                            ctypes.c_void_p(dst_dev.data_ptr()), dst_dev.numel(),
                                            _stream_handle(stream))
    if st:
        err = N.BitcosError(st, "bitcos_pack_device_noalloc")
        err.layout = L
        raise err
    return L


# ---------------------------------------------------------------------------
# GEMV (device)
# ---------------------------------------------------------------------------

_GEMV = {FMT_BITCOS: "bitcos_gemv", FMT_TRIT5: "trit5_gemv", FMT_BIT2: "bit2_gemv"}


def _stream_handle(stream, dev=None):
    """The hipStream_t of `stream` (None: torch's current one) as an int.  The
    current stream's handle is read directly where torch offers it: building a
    torch Stream object for it takes 3 us, as long as the launch itself.  With
    `dev`, the GPU of the call's tensors, that has to be the current one, which
    a launch goes to, and the stream's."""
    torch = _t()
    if stream is not None:
        if dev is not None and (torch.cuda.current_device() != dev or getattr(stream, "device_index", dev) != dev):
            raise ValueError(f"the tensors are on cuda:{dev}, the current device or the stream's is another")
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    here = torch.cuda.current_device()
    if dev is not None and here != dev:
        raise ValueError(f"the tensors are on cuda:{dev}, the current device is cuda:{here}")
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(here)


def gemv(L: Layout, blob_dev, x, y, xscale=None, y_mode: int = Y_F32, stream=None):
    """Enqueue y = (S (.) W) x for the layout's format on `stream`.

    blob_dev: uint8 cuda tensor of >= L.total_bytes; x: int8 or bfloat16 cuda
    tensor [m, k] (or [k]); y: float32 (Y_F32, Y_F32_ADD) or int32 (Y_I32_RAW,
    Y_I32_RAW_ADD) cuda tensor [m, n] (or [n]), overwritten or (the _ADD modes)
    added onto; xscale: None or float32 cuda tensor [m, k/128].
    """
    torch = _t()
    m = x.shape[0] if x.dim() == 2 else 1
    if x.dtype == torch.int8:
        xd = X_I8
    elif x.dtype == torch.bfloat16:
        xd = X_BF16
    else:
        raise TypeError("x must be int8 or bfloat16")
    for t, nm in ((blob_dev, "blob"), (x, "x"), (y, "y")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{nm} must be a contiguous cuda tensor")
    k = L.k
    if blob_dev.dtype != torch.uint8 or blob_dev.numel() < L.total_bytes:
        raise ValueError("blob_dev must be uint8 with at least total_bytes elements")
    if x.numel() != m * k:
        raise ValueError("x has the wrong size")
    want_y = torch.int32 if y_mode in (Y_I32_RAW, Y_I32_RAW_ADD) else torch.float32
    if y.dtype != want_y or y.numel() != m * L.n:
        raise ValueError("y has the wrong dtype or size")
    xs_ptr = None
    if xscale is not None:
        if (not xscale.is_cuda or xscale.dtype != torch.float32 or not xscale.is_contiguous()
                or xscale.numel() != m * (k // 128) or k % 128):
            raise ValueError("xscale must be a contiguous float32 cuda tensor [m, k/128]")
        xs_ptr = xscale.data_ptr()
    name = _GEMV[L.format]
    st = getattr(N.lib(), name)(ctypes.byref(L), blob_dev.data_ptr(), m, x.data_ptr(), xd, xs_ptr, y.data_ptr(), y_mode,
                                _stream_handle(stream))
    if st:
        N.check(st, name)
    return y


def bitcos_gemv(L, blob_dev, x, y, xscale=None, y_mode=Y_F32, stream=None):
    assert L.format == FMT_BITCOS
    return gemv(L, blob_dev, x, y, xscale, y_mode, stream)


def trit5_gemv(L, blob_dev, x, y, xscale=None, y_mode=Y_F32, stream=None):
    assert L.format == FMT_TRIT5
    return gemv(L, blob_dev, x, y, xscale, y_mode, stream)


def bit2_gemv(L, blob_dev, x, y, xscale=None, y_mode=Y_F32, stream=None):
    assert L.format == FMT_BIT2
    return gemv(L, blob_dev, x, y, xscale, y_mode, stream)


def describe(L: Layout, m: int = 1, x_dtype: int = X_I8) -> LaunchInfo:
    info = LaunchInfo()
    N.check(N.lib().bitcos_describe(ctypes.byref(L), m, x_dtype, ctypes.byref(info)), "bitcos_describe")
    return info


def add_partials(y, parts, stream=None):
    """Enqueue y += parts[0] + parts[1] + ... (fp32, in that order) on
    `stream`: the partial outputs of a split row's later column blocks.
    y: contiguous float32 cuda tensor of n elements; parts: contiguous float32
    cuda tensor [nparts, ...] of nparts * n elements."""
    torch = _t()
    for t, nm in ((y, "y"), (parts, "parts")):
        if not t.is_cuda or not t.is_contiguous() or t.dtype != torch.float32:
            raise ValueError(f"{nm} must be a contiguous float32 cuda tensor")
    n = y.numel()
    if parts.dim() < 1 or parts.shape[0] < 1 or parts.numel() != parts.shape[0] * n:
        raise ValueError("parts must hold nparts slices of y's size")
    N.check(N.lib().bitcos_add_partials(y.data_ptr(), parts.data_ptr(), int(parts.shape[0]), n,
                                        _stream_handle(stream)), "bitcos_add_partials")
    return y


def quantize_activations(x, q, scale, stream=None):
    """Device int8 quantisation of bf16 activations per group of 128 (see bitcos.h)."""
    torch = _t()
    if x.dtype != torch.bfloat16 or q.dtype != torch.int8 or scale.dtype != torch.float32:
        raise TypeError("x bfloat16, q int8, scale float32")
    for t in (x, q, scale):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("contiguous cuda tensors required")
    m = x.shape[0] if x.dim() == 2 else 1
    k = x.numel() // m
    if q.numel() != m * k or scale.numel() != m * (k // 128) or k % 128:
        raise ValueError("q must be [m, k] and scale [m, k/128], k % 128 == 0")
    N.check(N.lib().bitcos_quantize_act(x.data_ptr(), m, k, q.data_ptr(), scale.data_ptr(), _stream_handle(stream)),
            "bitcos_quantize_act")
    return q, scale


class Batch:
    """A list of GEMVs of one format and tile, run as one persistent launch.

    Holds the host table and its device copy; the device buffers it points to
    (blobs, activations, outputs) must outlive it.  Every GEMV takes the same
    number m of activation rows: xs[i] is [m, k] (or [k] for m = 1) and ys[i]
    [m, n]; m > 1 runs the small-batch kernel.
    """

    def __init__(self, layouts, blobs_dev, xs, ys, xscales=None, y_mode: int = Y_F32):
        import torch
        count = len(layouts)
        if not (count == len(blobs_dev) == len(xs) == len(ys)) or count < 1:
            raise ValueError("layouts, blobs, xs and ys must have the same non-zero length")
        x_dtype = X_I8 if xs[0].dtype == torch.int8 else X_BF16
        m = xs[0].shape[0] if xs[0].dim() == 2 else 1
        arr = (Layout * count)(*layouts)
        for L, b, x, y in zip(layouts, blobs_dev, xs, ys):
            _check_gemv_buffers(L, b, x, y, None, y_mode, m)
        if xscales is not None:
            for L, xs_ in zip(layouts, xscales):
                if xs_ is not None:
                    _check_xscale(L, xs_, m)
        P = ctypes.c_void_p
        blobs = (P * count)(*[b.data_ptr() for b in blobs_dev])
        xp = (P * count)(*[x.data_ptr() for x in xs])
        yp = (P * count)(*[y.data_ptr() for y in ys])
        sp = None if xscales is None else (P * count)(*[0 if s is None else s.data_ptr() for s in xscales])
        nbytes = N.lib().bitcos_batch_bytes(count)
        self.host = np.zeros(nbytes, dtype=np.uint8)
        N.check(N.lib().bitcos_batch_build(count, m, arr, blobs, xp, sp, yp, x_dtype, y_mode,
                                           _ptr(self.host), nbytes), "bitcos_batch_build")
        self._host_ptr = self.host.ctypes.data  # self.host is this object's own and never reallocated
        self.dev = torch.from_numpy(self.host).cuda()
        self.count = count
        self.m = m
        self._keep = (layouts, blobs_dev, xs, ys, xscales)

    def run(self, stream=None):
        st = N.lib().bitcos_gemv_batch(self._host_ptr, self.dev.data_ptr(), _stream_handle(stream))
        if st:
            N.check(st, "bitcos_gemv_batch")


def _check_gemv_buffers(L, blob_dev, x, y, xscale, y_mode, m=1):
    import torch
    for t, nm in ((blob_dev, "blob"), (x, "x"), (y, "y")):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{nm} must be a contiguous cuda tensor")
    if blob_dev.dtype != torch.uint8 or blob_dev.numel() < L.total_bytes:
        raise ValueError("blob_dev must be uint8 with at least total_bytes elements")
    if x.numel() != m * L.k or x.dtype not in (torch.int8, torch.bfloat16):
        raise ValueError("x must be int8 or bfloat16 with m * k elements")
    want_y = torch.int32 if y_mode in (Y_I32_RAW, Y_I32_RAW_ADD) else torch.float32
    if y.dtype != want_y or y.numel() != m * L.n:
        raise ValueError("y has the wrong dtype or size")


def _check_xscale(L, xscale, m):
    import torch
    if (not xscale.is_cuda or xscale.dtype != torch.float32 or not xscale.is_contiguous()
            or xscale.numel() != m * (L.k // 128) or L.k % 128):
        raise ValueError("xscale must be a contiguous float32 cuda tensor [m, k/128]")


# ---------------------------------------------------------------------------
# Paged key/value cache (device)
# ---------------------------------------------------------------------------

_I32_MAX = 2**31 - 1  # a larger number would reach the C ABI's 32 bits as another one


class KVCache:
    """A paged cache of one layer: views of the caller's device tensors.

    k, v: [pages, kv_heads, page_size, head_dim], bfloat16 or int8, any strides
    with the head's values next to each other (a cache kept as [pages,
    page_size, kv_heads, head_dim] is passed as its transpose(1, 2)); with
    int8, k_scale and v_scale: contiguous float32 [pages, kv_heads, page_size].
    Slot s is token s % page_size of page s // page_size.
    """

    def __init__(self, k, v, k_scale=None, v_scale=None):
        torch = _t()
        if k.dtype not in (torch.bfloat16, torch.int8) or v.dtype != k.dtype:
            raise TypeError("k and v must both be bfloat16 or both int8")
        if k.dim() != 4 or v.shape != k.shape or not k.is_cuda or v.device != k.device:
            raise ValueError("k and v must be cuda tensors [pages, kv_heads, page_size, head_dim] of one shape")
        if k.numel() == 0 or k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("k and v must hold something, a head's values next to each other")
        scales = (k_scale, v_scale)
        if k.dtype == torch.int8:
            for s in scales:
                if (s is None or s.dtype != torch.float32 or s.device != k.device or not s.is_contiguous()
                        or s.shape != k.shape[:3]):
                    raise ValueError("an int8 cache needs contiguous float32 scales [pages, kv_heads, page_size]")
        elif any(s is not None for s in scales):
            raise ValueError("a bfloat16 cache has no scales")
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        if self.pages * self.page_size > _I32_MAX or self.kv_heads > _I32_MAX:
            raise ValueError("a cache holds fewer than 2^31 slots")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self._dev = k.device, k.get_device()
        P = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.desc = N.KVCacheDesc(N.KV_I8 if k.dtype == torch.int8 else N.KV_BF16, *k.shape, 0, k.stride()[:3], v.stride()[:3],
                                  k.data_ptr(), v.data_ptr(), P(k_scale), P(v_scale))
        self._ref = ctypes.byref(self.desc)

    @classmethod
    def empty(cls, pages: int, kv_heads: int, page_size: int, head_dim: int, dtype=None, device="cuda"):
        """A cache of new tensors (contents undefined), bfloat16 unless `dtype` is torch.int8."""
        torch = _t()
        dtype = dtype or torch.bfloat16
        shape = (pages, kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        if dtype != torch.int8:
            return cls(k, v)
        return cls(k, v, *(torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2)))


class StepPlan:
    """Outputs of kv_plan for a step of at most max_tokens new tokens of `requests` requests:
    cu_q int32 [requests + 1], kv_len int32 [requests], slots and positions int32 [max_tokens],
    ring_state int64 [2], counts int32 [4] (tokens, pages taken, pages given back, requests
    refused).  kv_len and ring_state are the next step's inputs, so an engine keeps two plans
    and takes them in turn.  The tensors stay the ones made here, on a GPU."""

    def __init__(self, requests: int, max_tokens: int, device="cuda"):
        torch = _t()
        if torch.device(device).type != "cuda":
            raise ValueError("a plan's tensors are written by a kernel: device must be a GPU")
        new = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt, device=device)  # noqa: E731
        self.requests, self.max_tokens = requests, max_tokens
        self.cu_q, self.kv_len = new(requests + 1), new(requests)
        self.slots, self.positions = new(max_tokens), new(max_tokens)
        self.ring_state, self.counts = new(2, torch.int64), new(4)
        self._dev = self.cu_q.get_device()
        self._out = tuple(t.data_ptr() for t in (self.cu_q, self.kv_len, self.slots, self.positions, self.ring_state, self.counts))


def _i32(t, dev, name, n=None):
    """The address of a contiguous int32 tensor on GPU `dev`, of n elements (None: any number)."""
    if t.dtype is not _torch.int32 or t.get_device() != dev or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be a contiguous int32 tensor on cuda:{dev}" + ("" if n is None else f" of {n} elements"))
    return t.data_ptr()


_stride_arrays = {}  # strides {token, head, 1} -> the array that the C ABI takes


def _rows(t, dev, name, shape):
    """The address and strides of a [tokens, heads, dim] tensor on GPU `dev`, a head's values next to each other."""
    st = t.stride()
    arr = _stride_arrays.get(st)
    if t.shape != shape or t.get_device() != dev or (arr is None and st[2] != 1):
        raise ValueError(f"{name} must be a tensor {list(shape)} on cuda:{dev}, a head's values next to each other")
    if arr is None:
        if len(_stride_arrays) > 1000:
            _stride_arrays.clear()
        arr = _stride_arrays[st] = N._I64x2(*st[:2])
    return t.data_ptr(), arr


def kv_plan(kv_len, new_len, table, ring, ring_state, page_size: int, plan: StepPlan, stream=None) -> StepPlan:
    """Enqueue the planning of a step on `stream`: pages, slots and positions of the new tokens
    (see bitcos_kv.h).  kv_len, new_len: int32 [requests]; table: int32 [requests, width]; ring:
    int32 [ring places]; ring_state: int64 [2]; `plan` receives the results, table and ring are
    updated in place.  All of them are on the plan's GPU, the current one."""
    torch = _t()
    n, dev = plan.requests, plan._dev
    if table.dim() != 2 or table.shape[0] != n or ring.dim() != 1:
        raise ValueError("table must be [requests, width] and ring 1-D")
    if page_size > _I32_MAX:
        raise ValueError("page_size must be below 2^31")
    if ring_state.dtype is not torch.int64 or ring_state.get_device() != dev or not ring_state.is_contiguous() or ring_state.numel() != 2:
        raise ValueError(f"ring_state must be a contiguous int64 tensor [2] on cuda:{dev}")
    st = N.lib().bitcos_kv_plan(_i32(kv_len, dev, "kv_len", n), _i32(new_len, dev, "new_len", n), n, _i32(table, dev, "table"),
                                table.shape[1], _i32(ring, dev, "ring"), ring.numel(), ring_state.data_ptr(), page_size,
                                plan.max_tokens, *plan._out, _stream_handle(stream, dev))
    if st:
        N.check(st, "bitcos_kv_plan")
    return plan


def kv_append(cache: KVCache, k, v, slots, q=None, q_out=None, rope=None, positions=None, stream=None):
    """Enqueue the storing of k and v ([tokens, kv_heads, head_dim], both float32 or both
    bfloat16) at slots (int32 [tokens or more]) of the cache, on `stream`.

    q, q_out: [tokens, q_heads, head_dim] of k's type and bfloat16: the queries as
    paged_attention reads them.  rope: None, or (cos, sin), contiguous float32 [positions,
    rotated values / 2]; q and k are then rotated by positions (int32 [tokens or more]).  All
    of them are on the cache's GPU, the current one."""
    torch = _t()
    tokens, dev = k.shape[0], cache._dev
    dtype = k.dtype
    if dtype is torch.float32:
        act = N.ACT_F32
    elif dtype is torch.bfloat16:
        act = N.ACT_BF16
    else:
        raise TypeError("k must be float32 or bfloat16")
    if v.dtype is not dtype or (q is not None and q.dtype is not dtype):
        raise TypeError("q, k and v must be of one type")
    shape = (tokens, cache.kv_heads, cache.head_dim)
    kp, ks = _rows(k, dev, "k", shape)
    vp, vs = _rows(v, dev, "v", shape)
    at = _i32(slots, dev, "slots")
    if slots.numel() < tokens:
        raise ValueError("slots must have an entry for every token")
    hq = 0
    qp = qs = op = os_ = None
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q must be [tokens, q_heads, head_dim]")
        hq = q.shape[1]
        shape = (tokens, hq, cache.head_dim)
        qp, qs = _rows(q, dev, "q", shape)
        if q_out is None or q_out.dtype is not torch.bfloat16:
            raise TypeError("q_out must be bfloat16")
        op, os_ = _rows(q_out, dev, "q_out", shape)
    rot = places = 0
    cp = sp = pp = None
    if rope is not None:
        cos, sin = rope
        angles = cos.shape
        if (len(angles) != 2 or sin.shape != angles or cos.dtype is not torch.float32 or sin.dtype is not torch.float32
                or cos.get_device() != dev or sin.get_device() != dev or not (cos.is_contiguous() and sin.is_contiguous())):
            raise ValueError(f"rope must be two contiguous float32 tensors [positions, rotated values / 2] on cuda:{dev}")
        if positions is None:
            raise ValueError("rope needs positions")
        pp = _i32(positions, dev, "positions")
        if positions.numel() < tokens:
            raise ValueError("positions must have an entry for every token")
        places, rot = angles[0], 2 * angles[1]
        cp, sp = cos.data_ptr(), sin.data_ptr()
    if tokens == 0:
        return
    st = N.lib().bitcos_kv_append(cache._ref, tokens, act, kp, ks, vp, vs, at, hq, qp, qs, op, os_, rot, cp, sp, places, pp,
                                  _stream_handle(stream, dev))
    if st:
        N.check(st, "bitcos_kv_append")


def paged_attention_workspace(cache: KVCache, tokens: int, requests: int, q_heads: int, max_q: int, max_kv: int) -> int:
    """Bytes of the workspace that paged_attention needs for these counts."""
    if max(tokens, requests, q_heads, max_q, max_kv) > _I32_MAX:
        raise ValueError("counts must be below 2^31")
    n = N.lib().bitcos_paged_attn_workspace(cache._ref, tokens, requests, q_heads, max_q, max_kv)
    if n == 0:
        raise ValueError("counts must be positive, and the cache's heads of 8 to 256 values in steps of 8")
    return n


def paged_attention(q, cache: KVCache, table, kv_len, cu_q, out, workspace, *, max_q: int, max_kv: int, scale=None,
                    causal: bool = True, window: int = 0, lse=None, stream=None):
    """Enqueue out = softmax(scale q k^T) v of the step's tokens over the cache, on `stream`
    (see bitcos_kv.h).

    q, out: bfloat16 [tokens, q_heads, head_dim]; table: int32 [requests, width]; kv_len: int32
    [requests], the new tokens included; cu_q: int32 [requests + 1]; max_q, max_kv: what the host
    knows of the most new tokens and the most keys of a request; workspace: uint8 of
    paged_attention_workspace bytes; scale: 1 / sqrt(head_dim) unless given; window: keys that a
    query sees at most (0: all); lse: None or float32 [tokens, q_heads].  All of them are on the
    cache's GPU, the current one."""
    torch = _t()
    dim, dev = cache.head_dim, cache._dev
    if q.dtype is not torch.bfloat16 or out.dtype is not torch.bfloat16:
        raise TypeError("q and out must be bfloat16")
    shape = q.shape
    if len(shape) != 3 or shape[2] != dim:
        raise ValueError("q must be [tokens, q_heads, head_dim]")
    tokens, hq, _ = shape
    qp, qs = _rows(q, dev, "q", shape)
    op, os_ = _rows(out, dev, "out", shape)
    if table.dim() != 2 or table.shape[0] < 1:
        raise ValueError("table must be [requests, width]")
    if max_q > _I32_MAX or max_kv > _I32_MAX or window > _I32_MAX:
        raise ValueError("max_q, max_kv and window must be below 2^31")
    n, width = table.shape
    if workspace.dtype is not torch.uint8 or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{dev}")
    lp = None
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.get_device() != dev or not lse.is_contiguous() or lse.shape != shape[:2]:
            raise ValueError(f"lse must be a contiguous float32 tensor [tokens, q_heads] on cuda:{dev}")
        lp = lse.data_ptr()
    tp, kp, cp = _i32(table, dev, "table"), _i32(kv_len, dev, "kv_len", n), _i32(cu_q, dev, "cu_q", n + 1)
    if tokens == 0:
        return out
    st = N.lib().bitcos_paged_attn(cache._ref, tokens, n, hq, qp, qs, tp, width, kp, cp, max_q, max_kv,
                                   1.0 / math.sqrt(dim) if scale is None else scale, causal, window, op, os_, lp,
                                   workspace.data_ptr(), workspace.numel(), _stream_handle(stream, dev))
    if st:
        N.check(st, "bitcos_paged_attn")
    return out
