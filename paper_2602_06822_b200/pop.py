"""Thin ctypes binding over the C ABI in ``include/pop.h`` (same names, argument
marshalling only: every step of the path runs in the library's CUDA kernels).

PyTorch is used for device memory and streams.  There is no CPU fallback: if
``libpop.so`` has not been built, or no CUDA device is present, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple, Optional, Tuple

import numpy as np

POP_OK = 0
POP_ERR_INVALID_ARG = -1
POP_ERR_UNSUPPORTED = -2
POP_ERR_ALLOC = -3
POP_ERR_CUDA = -4
POP_ERR_TIMEOUT = -5
POP_MAX_BATCH = 8
POP_F32, POP_BF16 = 0, 1
POP_NOALLOC_MAX_N = 32768
POP_KV_TILE, POP_KV_GROUP, POP_KV_MAX_REQUESTS = 16, 64, 4096

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpop.so")


class Ratios(C.Structure):
    _fields_ = [("retained", C.c_double), ("candidate", C.c_double), ("pruned", C.c_double)]


class Config(C.Structure):
    _fields_ = [("decode_kernel", C.c_int), ("launch_mode", C.c_int), ("wait_budget_us", C.c_uint),
                ("slab_cache_bytes", C.c_ulonglong)]


class KVCacheDesc(C.Structure):
    """pop_kv_cache_t"""
    _fields_ = [("pages", C.c_void_p), ("n_pages", C.c_int), ("page_size", C.c_int), ("n_kv_heads", C.c_int), ("head_dim", C.c_int)]


POP_DECODE_AUTO, POP_DECODE_FUSED, POP_DECODE_SIMPLE = 0, 1, 2
POP_LAUNCH_PDL, POP_LAUNCH_COOPERATIVE, POP_LAUNCH_PLAIN = 0, 1, 2


class PopError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = f"{where}: {status_string(status)}"
        if status in (POP_ERR_CUDA, POP_ERR_ALLOC, POP_ERR_TIMEOUT):
            msg += f" [{lib().pop_last_cuda_error().decode()}]"
        super().__init__(msg)


_lib = None

# name -> (restype, argtypes); mirrors include/pop.h
_P = C.c_void_p
SIGNATURES = {
    "pop_version": (C.c_char_p, []),
    "pop_status_string": (C.c_char_p, [C.c_int]),
    "pop_last_cuda_error": (C.c_char_p, []),
    "pop_kernel_launch_count": (C.c_ulonglong, []),
    "pop_get_config": (C.c_int, [C.POINTER(Config)]),
    "pop_set_config": (C.c_int, [C.POINTER(Config)]),
    "pop_release_cached_memory": (C.c_int, []),
    "pop_region_sizes": (C.c_int, [C.c_int, Ratios] + [C.POINTER(C.c_int)] * 4),
    "pop_prefill_partition": (C.c_int, [_P, C.c_int, C.c_int, _P, _P, _P, C.c_int, C.c_int, Ratios, _P,
                                        C.POINTER(_P)]),
    "pop_weights_prepare": (C.c_int, [_P, _P, _P, C.c_int, C.c_int, C.c_int, _P, C.POINTER(_P)]),
    "pop_prefill_partition_prepared": (C.c_int, [_P, C.c_int, _P, Ratios, _P, C.POINTER(_P)]),
    "pop_prefill_partition_probe": (C.c_int, [_P, C.c_int, C.c_int, _P, Ratios, _P, C.POINTER(_P)]),
    "pop_weights_destroy": (C.c_int, [_P]),
    "pop_prefill_partition_with_output": (C.c_int, [_P, C.c_int, _P, Ratios, C.c_int, _P, _P, C.POINTER(_P)]),
    "pop_partition_from_indices": (C.c_int, [_P, _P, _P, C.c_int, C.c_int, C.c_int, _P, C.c_int, _P, C.c_int,
                                             _P, C.POINTER(_P)]),
    "pop_partition_sizes": (C.c_int, [_P] + [C.POINTER(C.c_int)] * 3),
    "pop_partition_indices": (C.c_int, [_P] + [C.POINTER(_P)] * 3),
    "pop_partition_scores": (C.c_int, [_P, C.POINTER(_P)]),
    "pop_partition_score_bounds": (C.c_int, [_P, C.POINTER(_P)]),
    "pop_partition_streamed_scores": (C.c_int, [_P, C.POINTER(_P)]),
    "pop_partition_shape": (C.c_int, [_P, C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_int)]),
    "pop_partition_check": (C.c_int, [_P]),
    "pop_partition_destroy": (C.c_int, [_P]),
    "pop_decode_step": (C.c_int, [_P, _P, C.c_int, C.c_int, _P, _P, _P, _P]),
    "pop_prefill_scores_noalloc": (C.c_int, [_P, C.c_int, C.c_int, _P, _P, _P, C.c_int, C.c_int, _P, _P]),
    "pop_kv_page_bytes": (C.c_int, [C.c_int, C.c_int, C.c_int, C.POINTER(C.c_size_t)]),
    "pop_kv_plan": (C.c_int, [_P, _P, C.c_int, C.c_int, _P, C.c_int, _P, _P, _P, C.c_int, C.c_int, _P, _P, _P, _P, _P, _P]),
    "pop_kv_append": (C.c_int, [C.POINTER(KVCacheDesc), _P, C.c_longlong, _P, C.c_longlong, C.c_int, _P, C.c_int, _P]),
    "pop_kv_read": (C.c_int, [C.POINTER(KVCacheDesc), _P, C.c_int, C.c_int, _P, _P, _P]),
    "pop_kv_attention_workspace": (C.c_int, [C.POINTER(C.c_size_t)]),
    "pop_kv_attention_check": (C.c_int, [_P, _P]),
    "pop_kv_attention": (C.c_int, [C.POINTER(KVCacheDesc), _P, C.c_longlong, C.c_int, C.c_int, C.c_int, _P, _P, C.c_int, _P, C.c_int,
                                   C.c_float, C.c_int, C.c_int, _P, _P, _P, C.c_size_t, _P]),
}


def lib() -> C.CDLL:
    """Loads libpop.so (built by ``__graft_entry__.build()``); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def version() -> str:
    return lib().pop_version().decode()


def kernel_launch_count() -> int:
    return int(lib().pop_kernel_launch_count())


def status_string(status: int) -> str:
    return lib().pop_status_string(status).decode()


def _check(status: int, where: str):
    if status != POP_OK:
        raise PopError(status, where)


def get_config() -> Config:
    c = Config()
    _check(lib().pop_get_config(C.byref(c)), "pop_get_config")
    return c


def set_config(**fields) -> Config:
    """pop_set_config with the named fields replaced (decode_kernel, launch_mode, wait_budget_us, slab_cache_bytes);
    returns the settings that were in force before."""
    old = get_config()
    new = Config(old.decode_kernel, old.launch_mode, old.wait_budget_us, old.slab_cache_bytes)
    for k, v in fields.items():
        if k not in dict(Config._fields_):
            raise KeyError(k)
        setattr(new, k, v)
    _check(lib().pop_set_config(C.byref(new)), "pop_set_config")
    return old


def release_cached_memory():
    _kv_workspaces.clear()              # (their memory goes back to torch, in the order of the streams that they were made on)
    _check(lib().pop_release_cached_memory(), "pop_release_cached_memory")


def region_sizes(N: int, ratios) -> Tuple[int, int, int, int]:
    """(n_ret, n_cand, n_pruned, k_default) - host only."""
    out = [C.c_int() for _ in range(4)]
    _check(lib().pop_region_sizes(N, Ratios(*ratios), *[C.byref(o) for o in out]), "pop_region_sizes")
    return tuple(o.value for o in out)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:                  # asked once: the question costs more than some of the calls
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2602_06822_b200 needs a CUDA device (there is no CPU path)")
        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return POP_F32
    if t.dtype == torch.bfloat16:
        return POP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream_ptr(stream=None) -> int:
    if stream is None:
        torch = _torch()
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


class _DevView:
    """Minimal __cuda_array_interface__ carrier for a raw device pointer."""

    def __init__(self, ptr: int, n: int, typestr: str):
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": typestr, "data": (int(ptr), False),
                                         "version": 2, "strides": None}


class Partition:
    """Owner of a ``pop_partition_t*``."""

    def __init__(self, handle: int, device):
        self._h = C.c_void_p(handle)
        self.device = device
        n = [C.c_int() for _ in range(3)]
        _check(lib().pop_partition_sizes(self._h, *[C.byref(v) for v in n]), "pop_partition_sizes")
        self.n_ret, self.n_cand, self.n_pruned = (v.value for v in n)
        s = [C.c_int() for _ in range(3)]
        _check(lib().pop_partition_shape(self._h, *[C.byref(v) for v in s]), "pop_partition_shape")
        self.d, self.N, self.dtype_code = (v.value for v in s)

    @property
    def handle(self) -> C.c_void_p:
        if self._h is None:
            raise RuntimeError("partition destroyed")
        return self._h

    def _view(self, ptr: int, n: int, typestr: str):
        """torch view (no copy) of a device array owned by the partition."""
        torch = _torch()
        if n == 0:
            return torch.empty(0, device=self.device, dtype={"<i4": torch.int32, "<f8": torch.float64, "<f4": torch.float32}[typestr])
        return torch.as_tensor(_DevView(ptr, n, typestr), device=self.device)

    def indices_device(self):
        """(R, C, P) channel ids as int32 CUDA tensors that alias the partition's arrays."""
        p = [C.c_void_p() for _ in range(3)]
        _check(lib().pop_partition_indices(self.handle, *[C.byref(v) for v in p]), "pop_partition_indices")
        return (self._view(p[0].value, self.n_ret, "<i4"), self._view(p[1].value, self.n_cand, "<i4"),
                self._view(p[2].value, self.n_pruned, "<i4"))

    def indices(self) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
        """(R, C, P) channel ids as host int32 arrays (synchronises)."""
        return tuple(t.cpu().numpy() for t in self.indices_device())

    def scores(self) -> np.ndarray:
        """Prefill importance scores I_i as a host float64 array (synchronises)."""
        p = C.c_void_p()
        _check(lib().pop_partition_scores(self.handle, C.byref(p)), "pop_partition_scores")
        return self._view(p.value, self.N, "<f8").cpu().numpy()

    def score_bounds(self) -> np.ndarray:
        """Bound of |scores()[i] - exact I_i| per channel as a host float64 array (synchronises)."""
        p = C.c_void_p()
        _check(lib().pop_partition_score_bounds(self.handle, C.byref(p)), "pop_partition_score_bounds")
        return self._view(p.value, self.N, "<f8").cpu().numpy()

    def streamed_scores(self):
        """(score, bound) of every candidate as the streaming kernel's last step saw them: two host float32
        arrays (synchronises); raises PopError(POP_ERR_UNSUPPORTED) for partitions served by another kernel."""
        p = C.c_void_p()
        _check(lib().pop_partition_streamed_scores(self.handle, C.byref(p)), "pop_partition_streamed_scores")
        pairs = self._view(p.value, 2 * self.n_cand, "<f4").cpu().numpy().reshape(self.n_cand, 2)
        return pairs[:, 0].copy(), pairs[:, 1].copy()

    def check(self):
        _check(lib().pop_partition_check(self.handle), "pop_partition_check")

    def destroy(self):
        if self._h is not None:
            _torch().cuda.synchronize(self.device)
            lib().pop_partition_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def prefill_partition(X, Wg, Wu, Wd, ratios, stream=None) -> Partition:
    """pop_prefill_partition: X [L, d], Wg/Wu [N, d], Wd [d, N] CUDA tensors of one dtype."""
    for t in (X, Wg, Wu, Wd):
        if not (t.is_cuda and t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
    L, d = X.shape
    N = Wg.shape[0]
    if tuple(Wg.shape) != (N, d) or tuple(Wu.shape) != (N, d) or tuple(Wd.shape) != (d, N):
        raise ValueError("shape mismatch")
    dt = _dtype_code(X)
    if any(_dtype_code(t) != dt for t in (Wg, Wu, Wd)):
        raise TypeError("dtype mismatch")
    out = C.c_void_p()
    _check(lib().pop_prefill_partition(X.data_ptr(), L, d, Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), N, dt,
                                       Ratios(*ratios), _stream_ptr(stream), C.byref(out)),
           "pop_prefill_partition")
    return Partition(out.value, X.device)


class Weights:
    """Owner of a ``pop_weights_t*`` (pop_weights_prepare).  Keeps references to the weight tensors, which the
    library reads again at every prefill that uses the object."""

    def __init__(self, Wg, Wu, Wd, stream=None):
        for t in (Wg, Wu, Wd):
            if not (t.is_cuda and t.is_contiguous()):
                raise ValueError("tensors must be contiguous CUDA tensors")
        N, d = Wg.shape
        if tuple(Wu.shape) != (N, d) or tuple(Wd.shape) != (d, N):
            raise ValueError("shape mismatch")
        dt = _dtype_code(Wg)
        if any(_dtype_code(t) != dt for t in (Wu, Wd)):
            raise TypeError("dtype mismatch")
        self.tensors = (Wg, Wu, Wd)
        self.device = Wg.device
        out = C.c_void_p()
        _check(lib().pop_weights_prepare(Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), N, d, dt, _stream_ptr(stream),
                                         C.byref(out)), "pop_weights_prepare")
        self._h = out

    def prefill_partition(self, X, ratios, stream=None) -> "Partition":
        """pop_prefill_partition_prepared: X [L, d] -> partition, with this weight set's statistics."""
        if not (X.is_cuda and X.is_contiguous()) or _dtype_code(X) != _dtype_code(self.tensors[0]):
            raise ValueError("X must be a contiguous CUDA tensor of the weights' dtype")
        if X.shape[1] != self.tensors[0].shape[1]:
            raise ValueError("shape mismatch")
        out = C.c_void_p()
        _check(lib().pop_prefill_partition_prepared(X.data_ptr(), X.shape[0], self._h, Ratios(*ratios), _stream_ptr(stream),
                                                    C.byref(out)), "pop_prefill_partition_prepared")
        return Partition(out.value, X.device)

    def prefill_partition_probe(self, X, ratios, token_stride: int, stream=None) -> "Partition":
        """pop_prefill_partition_probe: the partition from every token_stride-th row of X [L, d]."""
        if not (X.is_cuda and X.is_contiguous()) or _dtype_code(X) != _dtype_code(self.tensors[0]):
            raise ValueError("X must be a contiguous CUDA tensor of the weights' dtype")
        if X.shape[1] != self.tensors[0].shape[1]:
            raise ValueError("shape mismatch")
        out = C.c_void_p()
        _check(lib().pop_prefill_partition_probe(X.data_ptr(), X.shape[0], int(token_stride), self._h, Ratios(*ratios),
                                                 _stream_ptr(stream), C.byref(out)), "pop_prefill_partition_probe")
        return Partition(out.value, X.device)

    def prefill_partition_with_output(self, X, ratios, k: int, Y=None, stream=None):
        """pop_prefill_partition_with_output: (partition, Y [L, d]) - the partition and the prompt's own block output
        over Retained + the k best Candidates by prefill score."""
        torch = _torch()
        if not (X.is_cuda and X.is_contiguous()) or _dtype_code(X) != _dtype_code(self.tensors[0]):
            raise ValueError("X must be a contiguous CUDA tensor of the weights' dtype")
        if Y is None:
            Y = torch.empty_like(X)
        out = C.c_void_p()
        _check(lib().pop_prefill_partition_with_output(X.data_ptr(), X.shape[0], self._h, Ratios(*ratios), k, Y.data_ptr(),
                                                       _stream_ptr(stream), C.byref(out)), "pop_prefill_partition_with_output")
        return Partition(out.value, X.device), Y

    def destroy(self):
        if self._h is not None:
            _torch().cuda.synchronize(self.device)
            lib().pop_weights_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def partition_from_indices(Wg, Wu, Wd, ret: np.ndarray, cand: np.ndarray, stream=None) -> Partition:
    for t in (Wg, Wu, Wd):
        if not (t.is_cuda and t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
    N, d = Wg.shape
    ret = np.ascontiguousarray(ret, dtype=np.int32)
    cand = np.ascontiguousarray(cand, dtype=np.int32)
    out = C.c_void_p()
    _check(lib().pop_partition_from_indices(Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), N, d, _dtype_code(Wg),
                                            ret.ctypes.data, ret.size, cand.ctypes.data, cand.size,
                                            _stream_ptr(stream), C.byref(out)),
           "pop_partition_from_indices")
    return Partition(out.value, Wg.device)


def decode_step(part: Partition, x, k: int, y=None, mask_out=None, sel_out=None, stream=None):
    """pop_decode_step: x [B, d] -> y [B, d]; optional mask_out uint8 [n_cand], sel_out int32 [k]."""
    torch = _torch()
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if not (x.is_cuda and x.is_contiguous()):
        raise ValueError("x must be a contiguous CUDA tensor")
    B, d = x.shape
    if d != part.d or _dtype_code(x) != part.dtype_code:
        raise ValueError("x does not match the partition")
    if y is None:
        y = torch.empty_like(x)
    _check(lib().pop_decode_step(part.handle, x.data_ptr(), B, k, y.data_ptr(),
                                 None if mask_out is None else mask_out.data_ptr(),
                                 None if sel_out is None else sel_out.data_ptr(), _stream_ptr(stream)),
           "pop_decode_step")
    return y


def prefill_scores_noalloc(X, Wg, Wu, Wd, out, stream=None):
    """pop_prefill_scores_noalloc: the prefill scores I_i written into ``out`` (a float64 CUDA
    tensor of N elements that the caller already owns).  The library call allocates nothing: its
    temporaries live in a fixed array inside the library, shared by all calls on the device."""
    torch = _torch()
    for t in (X, Wg, Wu, Wd, out):
        if not (t.is_cuda and t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")
    L, d = X.shape
    N = Wg.shape[0]
    if out.dtype != torch.float64 or out.numel() != N:
        raise ValueError("out must be a float64 tensor of N elements")
    _check(lib().pop_prefill_scores_noalloc(X.data_ptr(), L, d, Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), N,
                                            _dtype_code(X), out.data_ptr(), _stream_ptr(stream)),
           "pop_prefill_scores_noalloc")
    return out


# ---------------------------------------------------------------------------------------------------------------------
# The paged 4-bit key / value cache (pop_kv_*).  The tensors of a call have to be on the current device.
# ---------------------------------------------------------------------------------------------------------------------

def kv_page_bytes(page_size: int, n_kv_heads: int, head_dim: int) -> int:
    """Bytes of one page of one layer - host only."""
    out = C.c_size_t()
    _check(lib().pop_kv_page_bytes(page_size, n_kv_heads, head_dim, C.byref(out)), "pop_kv_page_bytes")
    return out.value


def kv_pages(n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """Uninitialised memory for one layer's cache: uint8 [n_pages, n_kv_heads, page_size / 16, tile bytes], the tensor that
    the calls below take as ``pages``."""
    per_tile = kv_page_bytes(POP_KV_TILE, 1, head_dim)
    kv_page_bytes(page_size, n_kv_heads, head_dim)
    return _torch().empty(n_pages, n_kv_heads, page_size // POP_KV_TILE, per_tile, dtype=_torch().uint8, device=device)


def _kv_desc(pages) -> KVCacheDesc:
    if pages.dim() != 4 or not pages.is_cuda or not pages.is_contiguous() or pages.element_size() != 1:
        raise ValueError("pages must be a contiguous uint8 CUDA tensor as kv_pages() makes it")
    n, h, tiles, nbytes = pages.shape
    per_group = 2 * 512 + POP_KV_TILE * 8
    if nbytes % per_group:
        raise ValueError("pages must be a contiguous uint8 CUDA tensor as kv_pages() makes it")
    return KVCacheDesc(pages.data_ptr(), n, tiles * POP_KV_TILE, h, nbytes // per_group * POP_KV_GROUP)


def _on_current_device(stream, *tensors):
    """The kernels run on the current device and follow the addresses they are given there: a tensor (or a stream) of another device, or of the
    host, must not reach them."""
    here = _torch()._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:                    # (-1 on the host)
            raise ValueError(f"all tensors of a call must be on the current CUDA device ({here}), one is on {t.device}")
    if stream is not None and getattr(stream, "device_index", here) != here:
        raise ValueError(f"the stream is not one of the current CUDA device ({here})")


def _ints(t, dtype, what, dim=1):
    if t.dtype != dtype or t.dim() != dim or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of {dim} dimension(s)")


def _rows(t, heads: int, dim: int, what: str) -> int:
    """Token stride (in elements) of [tokens, heads, dim] whose heads lie one after another."""
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim:
        raise ValueError(f"{what} must be [tokens, {heads}, {dim}]")
    s = t.stride()
    if t.shape[0] and (s[2] != 1 or (heads > 1 and s[1] != dim)):
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    return s[0] if t.shape[0] > 1 else heads * dim


def _used_on(stream, *tensors):
    """Tells the caching allocator that tensors made here for the current stream are used on another one."""
    if stream is not None and stream != _torch().cuda.current_stream():
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _no_gradient(*tensors):
    """The cache has no backward pass (its values are rounded to 4 bits): a gradient must not end here unnoticed."""
    for t in tensors:
        if t.requires_grad and _torch().is_grad_enabled():
            raise ValueError("the 4-bit cache has no backward pass: detach() what requires a gradient, or call under torch.no_grad()")


class KVPlan(NamedTuple):
    q_indptr: object      # int32 [requests + 1]
    kv_lens: object       # int32 [requests]
    slots: object         # int64 [tokens]
    positions: object     # int32 [tokens]
    state: object         # int32 [2]: head and count of the ring of free pages after this step
    info: object          # int32 [2]: new tokens; pages wanted and not given


def kv_plan(ctx_lens, new_lens, block_table, ring, state, page_size: int, n_tokens: int, state_out=None, stream=None) -> KVPlan:
    """pop_kv_plan: block table (updated in place), slot map and lengths of one step.  ``state_out`` defaults to ``state``
    (updated in place)."""
    torch = _torch()
    i32 = torch.int32
    for t, w in ((ctx_lens, "ctx_lens"), (new_lens, "new_lens"), (ring, "ring"), (state, "state")):
        _ints(t, i32, w)
    _ints(block_table, i32, "block_table", 2)
    if state_out is None:
        state_out = state
    else:
        _ints(state_out, i32, "state_out")
    R, dev = ctx_lens.shape[0], ctx_lens.device
    if new_lens.shape[0] != R or block_table.shape[0] != R or state.shape[0] < 2 or state_out.shape[0] < 2:
        raise ValueError("shape mismatch")
    _on_current_device(stream, ctx_lens, new_lens, block_table, ring, state, state_out)
    ints = torch.empty(2 * R + 3 + n_tokens, dtype=i32, device=dev)      # one allocation for the int32 outputs
    slots = torch.empty(n_tokens, dtype=torch.int64, device=dev)
    at = ints.data_ptr()
    _check(lib().pop_kv_plan(ctx_lens.data_ptr(), new_lens.data_ptr(), R, page_size, ring.data_ptr(), ring.shape[0], state.data_ptr(),
                             state_out.data_ptr(), block_table.data_ptr(), block_table.shape[1], n_tokens, at, at + 4 * (R + 1),
                             slots.data_ptr(), at + 4 * (2 * R + 3), at + 4 * (2 * R + 1), _stream_ptr(stream)), "pop_kv_plan")
    _used_on(stream, ints, slots)
    q_indptr, kv_lens, info, positions = ints.split_with_sizes((R + 1, R, 2, n_tokens))
    return KVPlan(q_indptr, kv_lens, slots, positions, state_out, info)


def kv_append(pages, k, v, slots, stream=None):
    """pop_kv_append: k, v [T, n_kv_heads, head_dim] (token rows may be strided) quantised into the slots (int64 [T])."""
    desc = _kv_desc(pages)
    ks, vs = _rows(k, desc.n_kv_heads, desc.head_dim, "k"), _rows(v, desc.n_kv_heads, desc.head_dim, "v")
    _ints(slots, _torch().int64, "slots")
    if k.shape[0] != v.shape[0] or slots.shape[0] != k.shape[0]:
        raise ValueError("k, v and slots must have one length")
    if k.dtype != v.dtype:
        raise TypeError("dtype mismatch")
    _on_current_device(stream, pages, k, v, slots)
    _no_gradient(k, v)
    _check(lib().pop_kv_append(C.byref(desc), k.data_ptr(), ks, v.data_ptr(), vs, _dtype_code(k), slots.data_ptr(), k.shape[0],
                               _stream_ptr(stream)), "pop_kv_append")


def kv_read(pages, slots, dtype, stream=None):
    """pop_kv_read: (k, v) [T, n_kv_heads, head_dim] of ``dtype``, the values that the slots hold."""
    torch = _torch()
    desc = _kv_desc(pages)
    _ints(slots, torch.int64, "slots")
    _on_current_device(stream, pages, slots)
    k = torch.empty(slots.shape[0], desc.n_kv_heads, desc.head_dim, dtype=dtype, device=pages.device)
    v = torch.empty_like(k)
    _check(lib().pop_kv_read(C.byref(desc), slots.data_ptr(), slots.shape[0], _dtype_code(k), k.data_ptr(), v.data_ptr(),
                             _stream_ptr(stream)), "pop_kv_read")
    _used_on(stream, k, v)
    return k, v


def kv_workspace(device="cuda"):
    """A workspace for kv_attention, zeroed on the current stream.  Calls that share one must not run at the same time: it is for one stream, one
    cache or one captured graph."""
    n = C.c_size_t()
    _check(lib().pop_kv_attention_workspace(C.byref(n)), "pop_kv_attention_workspace")
    return _torch().zeros(n.value, dtype=_torch().uint8, device=device)


_kv_workspaces = {}


def _kv_workspace(device: int, stream):
    """The workspace of a call that was given none: the one kept for its (device, stream).  A call that is being captured gets one of its own, as the
    graph may be replayed on any stream, beside other work of this one."""
    torch = _torch()
    if stream is not None:                                              # made on the stream that uses it
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream.cuda_stream)
        with torch.cuda.stream(stream):
            return _kv_workspace(device, None)
    if torch._C._cuda_isCurrentStreamCapturing():
        return kv_workspace(device)
    key = (device, torch._C._cuda_getCurrentRawStream(device))
    ws = _kv_workspaces.get(key)
    if ws is None:
        ws = _kv_workspaces[key] = kv_workspace(device)
    return ws


def kv_attention(pages, q, block_table, q_indptr, kv_lens, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                 out=None, lse_out=None, workspace=None, stream=None):
    """pop_kv_attention: q [T, n_heads, head_dim] (token rows may be strided) over the cache -> out [T, n_heads, head_dim].
    ``scale`` defaults to 1 / sqrt(head_dim); ``lse_out`` float32 [T, n_heads] receives the logarithms of the softmax sums.
    ``workspace`` (kv_workspace()) defaults to one kept for the stream, or, in a call that is being captured into a graph, to one that the graph
    zeroes for every such call: a captured step should bring its own."""
    torch = _torch()
    desc = _kv_desc(pages)
    T, heads = q.shape[0], q.shape[1]
    qs = _rows(q, heads, desc.head_dim, "q")
    _ints(block_table, torch.int32, "block_table", 2)
    _ints(q_indptr, torch.int32, "q_indptr")
    _ints(kv_lens, torch.int32, "kv_lens")
    R = kv_lens.shape[0]
    if block_table.shape[0] != R or q_indptr.shape[0] != R + 1:
        raise ValueError("block_table, q_indptr and kv_lens must be of one number of requests")
    _on_current_device(stream, pages, q, block_table, q_indptr, kv_lens, out, lse_out, workspace)
    _no_gradient(q)
    made = out is None
    if made:
        out = torch.empty(T, heads, desc.head_dim, dtype=q.dtype, device=q.device)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor of q's shape and dtype")
    if lse_out is not None and (lse_out.dtype != torch.float32 or tuple(lse_out.shape) != (T, heads) or not lse_out.is_contiguous()):
        raise ValueError("lse_out must be a contiguous float32 tensor [tokens, heads]")
    window = int(window)
    if not 0 <= window < 2**31:                              # (what a C int holds: -1 is refused, 2^31 - 1 hides nothing)
        window = -1 if window < 0 else 2**31 - 1
    st = _stream_ptr(stream)
    if workspace is None:
        workspace = _kv_workspace(q.get_device(), stream)
    _check(lib().pop_kv_attention(C.byref(desc), q.data_ptr(), qs, _dtype_code(q), heads, T, q_indptr.data_ptr(), kv_lens.data_ptr(), R,
                                  block_table.data_ptr(), block_table.shape[1], desc.head_dim ** -0.5 if scale is None else scale,
                                  int(causal), window, out.data_ptr(), None if lse_out is None else lse_out.data_ptr(),
                                  workspace.data_ptr(), workspace.numel() * workspace.element_size(), st), "pop_kv_attention")
    if made:
        _used_on(stream, out)
    return out


def kv_attention_check(device="cuda", workspace=None, stream=None):
    """pop_kv_attention_check for the workspace given, or the one kept for the stream: synchronises, raises PopError if a wait ran out.  (KVCache
    has a check() of its own.  A captured call that was given no workspace cannot be checked.)"""
    st = _stream_ptr(stream)
    if workspace is None:
        workspace = _kv_workspace(_torch().empty(0, device=device).get_device(), stream)
    _on_current_device(stream, workspace)
    _check(lib().pop_kv_attention_check(workspace.data_ptr(), st), "pop_kv_attention_check")


class KVCache:
    """A decoder's paged 4-bit cache: the pages of its layers, the block table of its requests, the ring of free pages and the attention's
    workspace.  One step of all requests is ``plan()`` once, then ``append()`` and ``attend()`` in every layer; everything stays on the device
    and keeps its addresses, so a step can be captured into a CUDA graph (``plan`` with a fixed number of tokens).  A cache is for one stream at a
    time; several caches, and graphs of them, may run side by side."""

    def __init__(self, n_layers: int, n_requests: int, max_tokens: int, n_kv_heads: int, head_dim: int, page_size: int = 64,
                 n_pages: Optional[int] = None, device="cuda"):
        torch = _torch()
        self.page_size = page_size
        max_blocks = -(-max_tokens // page_size)
        self.max_tokens = max_blocks * page_size                  # of a request: what its row of the block table has place for
        self.n_pages = n_requests * max_blocks if n_pages is None else n_pages
        self.pages = [kv_pages(self.n_pages, page_size, n_kv_heads, head_dim, device) for _ in range(n_layers)]
        i32 = dict(dtype=torch.int32, device=device)
        self.block_table = torch.empty(n_requests, max_blocks, **i32)
        self.ring = torch.empty(self.n_pages, **i32)
        self.state = torch.empty(2, **i32)
        self.lens = torch.empty(n_requests, **i32)
        self.workspace = kv_workspace(device)
        self.step: Optional[KVPlan] = None
        self.reset()

    def reset(self):
        """All requests empty, all pages free."""
        torch = _torch()
        self.block_table.fill_(-1)
        torch.arange(self.n_pages, out=self.ring)
        self.state.copy_(torch.tensor([0, self.n_pages], dtype=torch.int32))
        self.lens.zero_()
        self.step = None

    def plan(self, new_lens, n_tokens: int) -> KVPlan:
        """The step's plan (kv_plan): new_lens int32 [requests] tokens each request gets (negative: it has finished), n_tokens in all.
        ``step.info[1]`` counts pages that were wanted and not there."""
        self.step = kv_plan(self.lens, new_lens, self.block_table, self.ring, self.state, self.page_size, n_tokens)
        self.lens.copy_(self.step.kv_lens)
        return self.step

    def append(self, layer: int, k, v):
        kv_append(self.pages[layer], k, v, self.step.slots)

    def attend(self, layer: int, q, **kw):
        kw.setdefault("workspace", self.workspace)
        return kv_attention(self.pages[layer], q, self.block_table, self.step.q_indptr, self.step.kv_lens, **kw)

    def check(self):
        """Synchronises the current stream; raises PopError if a wait of one of the cache's attention calls up to here ran out since the last check,
        whichever stream or graph it ran in."""
        kv_attention_check(workspace=self.workspace)
