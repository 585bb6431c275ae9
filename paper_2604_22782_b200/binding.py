"""Binding of ``libskv.so``: same names as the C entry points, argument marshalling only, through ctypes; the entry
points of a serving step, which are a few microseconds long, through ``_calls.so`` (csrc/skv_calls.cpp) where their
arguments are plain.  Tensors are torch CUDA tensors (torch is used for device
memory and streams, nothing else)."""
from __future__ import annotations

import ctypes
import functools
import os
import re
import subprocess
import warnings
from typing import List, Optional, Sequence

import torch

from . import build as _build

_HERE = os.path.dirname(os.path.abspath(__file__))
_HEADER = os.path.join(_HERE, "..", "include", "skv.h")

SKV_OK = 0
SKV_ERR_ARG, SKV_ERR_ROUTING, SKV_ERR_UNSUPPORTED, SKV_ERR_NOMEM = -1, -2, -3, -4
SKV_ERR_LAYER, SKV_ERR_CUDA, SKV_ERR_TIMEOUT, SKV_ERR_BOUNDS = -5, -6, -7, -8
SKV_ERR_TOO_LARGE = -9
SKV_STATIC_SCRATCH_BYTES = 8 << 20


def lib_path() -> str:
    return _build.LIB


def _load() -> ctypes.CDLL:
    path = _build.LIB
    if not os.path.exists(path):
        try:
            _build.build()
        except Exception as e:  # no silent fallback: the CUDA library is the product
            raise ImportError(f"libskv.so is missing and could not be built with nvcc: {e}") from e
    return ctypes.CDLL(path)


lib = _load()


class _Declines:
    """Stands in for the marshalling extension where there is none: every call is declined."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_calls():
    """The marshalling extension, which only saves time: without it every call goes through the ctypes form beside it."""
    try:
        if not os.path.exists(_build.CALLS):
            _build.build_calls()
        from . import _calls
        if _calls.torch_version != torch.__version__:
            raise ImportError(f"built for torch {_calls.torch_version}, this is {torch.__version__}")
        if not hasattr(_calls, "connect_pages"):
            raise ImportError("built from an earlier version of its source")
    except (ImportError, OSError, subprocess.SubprocessError) as e:
        warnings.warn(f"_calls.so is not used: {e}.  The serving step's calls go through ctypes, which takes 4 to 6 us more for each; "
                      f"python -m {__package__}.build --force builds it", RuntimeWarning, stacklevel=2)
        return _Declines()
    _calls.connect(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.skv_is_owner, lib.skv_rope_append, lib.skv_plan_step, lib.skv_plan_release, lib.skv_decode_attn_window,
        lib.skv_prefill_attn_window)))
    _calls.connect_pages(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.skv_index_pages, lib.skv_select_pages, lib.skv_decode_attn_pages, lib.skv_prefill_attn_pages)))
    return _calls


_calls = _load_calls()
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)

_vp, _i32p, _i64p, _szp = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)
_int, _i64, _f32, _sz = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t

lib.skv_strerror.restype = ctypes.c_char_p
lib.skv_strerror.argtypes = [_int]
lib.skv_routing_from_owners.argtypes = [_int, _i32p, _int, _i32p]
lib.skv_routing_groups.argtypes = [_int, _int, _i32p]
lib.skv_routing_rcla.argtypes = [_int, ctypes.c_double, _vp, _vp, _i32p]
lib.skv_routing_rdcla.argtypes = [_int, _int, ctypes.c_double, _vp, _i32p]
lib.skv_cache_pool_bytes.argtypes = [_int, _i32p, _int, _int, _int, _i64, _szp]
lib.skv_cache_create.argtypes = [ctypes.POINTER(_vp), _int, _i32p, _int, _int, _int, _i64, _vp, _sz, _vp]
lib.skv_cache_create_fp8.argtypes = lib.skv_cache_create.argtypes
lib.skv_cache_pool_bytes_fp8.argtypes = [_int, _i32p, _int, _int, _int, _i64, _szp]
lib.skv_gather_fp8.argtypes = [_vp, _int, _i64p, _i64, _vp, _vp, _vp, _vp, _vp]
lib.skv_cache_destroy.restype = None
lib.skv_cache_destroy.argtypes = [_vp]
lib.skv_layer_owner.argtypes = [_vp, _int]
lib.skv_is_owner.argtypes = [_vp, _int]
lib.skv_cache_stats.argtypes = [_vp, ctypes.POINTER(_int), _szp, _szp, _szp]
lib.skv_append.argtypes = [_vp, _int, _vp, _vp, _i64p, _i64, _vp]
lib.skv_gather.argtypes = [_vp, _int, _i64p, _i64, _vp, _vp, _vp]
lib.skv_decode_workspace_bytes.argtypes = [_vp, _int, _int, _szp]
lib.skv_decode_attn.argtypes = [_vp, _int, _vp, _i32p, _i32p, _vp, _int, _int, _int, _f32, _vp, _sz, _vp]
lib.skv_decode_attn_static.argtypes = [_vp, _int, _vp, _i32p, _i32p, _vp, _int, _int, _int, _f32, _vp]
lib.skv_prefill_attn.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _vp, _int, _int, _int, _int, _f32, _vp]
lib.skv_prefill_attn_src.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _vp, _int, _int, _int, _int, _f32, _vp]
lib.skv_rope_create.argtypes = [ctypes.POINTER(_vp), _int, _vp, _vp, _int, _int]
lib.skv_rope_destroy.restype = None
lib.skv_rope_destroy.argtypes = [_vp]
lib.skv_rope_append.argtypes = [_vp, _int, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _i32p, _i64, _i64p, _i64, _int, _vp]
lib.skv_plan_step.argtypes = [_vp, _i32p, _int, _i32p, _i32p, _int, _i32p, _int, _i32p, _i64, _i64p, _i32p, _i32p, _i32p, _i32p, _vp]
lib.skv_plan_release.argtypes = [_vp, _i32p, _int, _i32p, _i32p, _int, _i32p, _int, _i32p, _i32p, _vp]
lib.skv_decode_attn_window.argtypes = [_vp, _int, _vp, _i32p, _i32p, _vp, _int, _int, _int, _int, _int, _f32, _vp, _sz, _vp]
lib.skv_prefill_attn_window.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _vp, _int, _int, _int, _int, _int, _int, _f32, _vp]
lib.skv_page_index_bytes.argtypes = [_vp, _szp]
lib.skv_set_page_index.argtypes = [_vp, _vp, _sz, _vp]
lib.skv_index_pages.argtypes = [_vp, _int, _i32p, _i32p, _i32p, _int, _int, _int, _vp]
lib.skv_page_list_width.argtypes = [_int, _int, _int, _int, ctypes.POINTER(_int)]
lib.skv_select_pages.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _i32p, _i32p] + [_int] * 9 + [_vp]
lib.skv_decode_attn_pages.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _i32p, _vp] + [_int] * 4 + [_f32, _vp]
lib.skv_prefill_attn_pages.argtypes = [_vp, _int, _vp, _i32p, _i32p, _i32p, _i32p, _i32p, _vp] + [_int] * 6 + [_f32, _vp]
lib.skv_decode_splitk.argtypes = [_vp, _int, _vp, _i32p, _i32p, _int, _int, _int, _f32, _vp, _sz, _vp]
lib.skv_decode_merge.argtypes = [_vp, _vp, _int, _int, _vp, _sz, _vp]
lib.skv_decode_step.argtypes = [_vp, _vp, _vp, _vp, _i64p, _i32p, _i32p, _vp, _int, _int, _int, _f32, _vp, _sz, _vp]
lib.skv_decode_step_staging_bytes.argtypes = [_vp, _int, _int, _int, _szp]
lib.skv_decode_step_host.argtypes = [_vp, _vp, _vp, _vp, _i64p, _i32p, _i32p, _vp, _int, _int, _int, _f32,
                                     _vp, _sz, _vp]
lib.skv_get_status.argtypes = [_vp, _vp, ctypes.POINTER(_int)]
lib.skv_set_decode_variant.argtypes = [_vp, _int]
lib.skv_set_decode_tuning.argtypes = [_vp, _int, _int, _int]
lib.skv_set_prefill_variant.argtypes = [_vp, _int]
lib.skv_prefill_scratch_bytes.argtypes = [_vp, _szp]
lib.skv_set_prefill_scratch.argtypes = [_vp, _vp, _sz]
lib.skv_set_decode_overlap.argtypes = [_vp, _int]
lib.skv_set_decode_l2_reuse.argtypes = [_vp, _int]
lib.skv_set_decode_early_fetch.argtypes = [_vp, _int]
lib.skv_set_decode_worker.argtypes = [_vp, _int, _int, _int, _int]
lib.skv_set_decode_merge.argtypes = [_vp, _int]
lib.skv_set_host_step.argtypes = [_vp, _int, _int]
lib.skv_set_trace_buffer.argtypes = [_vp, _vp, _sz]
lib.skv_decode_worker_count.argtypes = [_vp]
lib.skv_launch_count.argtypes = [_vp, ctypes.POINTER(_i64)]
lib.skv_plan_worker_range.argtypes = [_i64, _int, _int, ctypes.POINTER(_i64), ctypes.POINTER(_i64)]
lib.skv_plan_worker_of.argtypes = [_i64, _int, _i64]


def exported_symbols() -> List[str]:
    """Names of the functions ``include/skv.h`` declares."""
    with open(_HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(skv_[a-z_0-9]+)\s*\(", text)))


class SkvError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {skv_strerror(status)} ({status})")


def skv_strerror(status: int) -> str:
    return lib.skv_strerror(status).decode()


def _check(rc: int, what: str) -> None:
    if rc != SKV_OK:
        raise SkvError(rc, what)


def _i32_array(xs: Sequence[int]):
    return (ctypes.c_int32 * len(xs))(*[int(x) for x in xs])


def skv_routing_from_owners(n_layers: int, owners: Sequence[int]) -> List[int]:
    out = (ctypes.c_int32 * max(n_layers, 1))()
    _check(lib.skv_routing_from_owners(n_layers, _i32_array(list(owners)), len(owners), out), "skv_routing_from_owners")
    return list(out)[:n_layers]


def skv_routing_groups(n_layers: int, g: int) -> List[int]:
    out = (ctypes.c_int32 * max(n_layers, 1))()
    _check(lib.skv_routing_groups(n_layers, g, out), "skv_routing_groups")
    return list(out)[:n_layers]


def _f64_array(xs: Sequence[float]):
    return (ctypes.c_double * len(xs))(*xs)


def skv_routing_rcla(p_self: float, u: Sequence[float], v: Sequence[float]) -> List[int]:
    n = len(u)
    out = (ctypes.c_int32 * n)()
    _check(lib.skv_routing_rcla(n, p_self, _f64_array(list(u)), _f64_array(list(v)), out), "skv_routing_rcla")
    return list(out)


def skv_routing_rdcla(k: int, p_self: float, u: Sequence[float]) -> List[int]:
    n = len(u)
    out = (ctypes.c_int32 * n)()
    _check(lib.skv_routing_rdcla(n, k, p_self, _f64_array(list(u)), out), "skv_routing_rdcla")
    return list(out)


def skv_cache_pool_bytes(r: Sequence[int], kv_heads: int, head_dim: int, page_size: int, max_pages: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib.skv_cache_pool_bytes(len(r), _i32_array(r), kv_heads, head_dim, page_size, max_pages,
                                    ctypes.byref(out)), "skv_cache_pool_bytes")
    return out.value


def skv_cache_pool_bytes_fp8(r: Sequence[int], kv_heads: int, head_dim: int, page_size: int, max_pages: int) -> int:
    out = _sz(0)
    _check(lib.skv_cache_pool_bytes_fp8(len(r), _i32_array(r), kv_heads, head_dim, page_size, max_pages,
                                        ctypes.byref(out)), "skv_cache_pool_bytes_fp8")
    return out.value


def skv_page_list_width(top: int, first_pages: int, last_pages: int, run: int = 1) -> int:
    """Entries of a list that ``skv_select_pages`` writes at most."""
    out = _int(0)
    _check(lib.skv_page_list_width(_i32("top", top), _i32("first_pages", first_pages), _i32("last_pages", last_pages), _i32("run", run),
                                   ctypes.byref(out)), "skv_page_list_width")
    return out.value


def skv_plan_worker_range(n_blocks: int, n_workers: int, w: int):
    b, e = _i64(0), _i64(0)
    _check(lib.skv_plan_worker_range(n_blocks, n_workers, w, ctypes.byref(b), ctypes.byref(e)),
           "skv_plan_worker_range")
    return b.value, e.value


def skv_plan_worker_of(n_blocks: int, n_workers: int, x: int) -> int:
    rc = lib.skv_plan_worker_of(n_blocks, n_workers, x)
    if rc < 0:
        raise SkvError(rc, "skv_plan_worker_of")
    return rc


@functools.lru_cache(None)
def _has_cuda() -> bool:
    return torch.cuda.is_available()


def _stream_ptr(stream) -> int:
    if stream is None:
        # (torch.cuda.current_stream() builds a Stream object first: 4 us against 0.2 us)
        return _raw_stream(torch.cuda.current_device()) if _has_cuda() else 0
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _arg(name: str, t: Optional[torch.Tensor], dtype, shape=None, min_numel: Optional[int] = None,
         cuda: Optional[bool] = True) -> Optional[torch.Tensor]:
    """Checks a tensor argument before its raw pointer goes to the library: dtype, device (cuda=None: either),
    contiguity, and an exact shape or a minimum number of elements.  The kernels trust the sizes they are
    given, so a wrong one here would be an out-of-bounds access there."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if cuda is not None and t.is_cuda != cuda:
        raise ValueError(f"{name}: expected a {'CUDA' if cuda else 'host'} tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if min_numel is not None and t.numel() < min_numel:
        raise ValueError(f"{name}: needs at least {min_numel} elements, has {t.numel()}")
    return t


def _i32(name: str, x: int) -> int:
    """ctypes cuts an int to its low 32 bits without a word."""
    if not -(1 << 31) <= x < (1 << 31):
        raise ValueError(f"{name}: {x} is not a 32-bit integer")
    return x


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _checked(name: str, t: torch.Tensor, dtype, shape, device: int) -> int:
    """The pointer of a dense tensor on the current device; `_arg` says what is wrong with another one.  (These calls
    are a few microseconds long: what is asked of a tensor is asked once.)"""
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous() and t.shape == shape:
        return t.data_ptr()
    _arg(name, t, dtype, shape)
    raise ValueError(f"{name}: is on {t.device}, the current device is cuda:{device}")


def _rows(name: str, t: torch.Tensor, n: int, heads: int, dim: int, device: int):
    """Pointer and row stride (elements) of bf16 rows [n][heads][dim] whose heads are dense and whose rows may be further
    apart (a slice of a fused projection)."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name}: expected {torch.bfloat16}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name}: expected a tensor on cuda:{device}, got {t.device}")
    if t.shape != (n, heads, dim):
        raise ValueError(f"{name}: expected shape {(n, heads, dim)}, got {tuple(t.shape)}")
    row, head, one = t.stride()
    if n <= 1:                      # (a single row's stride says nothing)
        row = heads * dim
    if n and heads and (one != 1 or (heads > 1 and head != dim) or row < heads * dim):
        raise ValueError(f"{name}: the rows' heads must be dense")
    return t.data_ptr(), row


class SkvRope:
    """Handle of a rotary embedding: ``inv_freq`` radians per position of every frequency (half the rotary dims),
    ``axis`` which of the ``n_axes`` positions of a token turns it (None: the first)."""

    def __init__(self, inv_freq: Sequence[float], axis: Optional[Sequence[int]] = None, n_axes: int = 1,
                 adjacent_pairs: bool = False):
        inv_freq = [float(x) for x in inv_freq]
        if axis is not None and len(axis) != len(inv_freq):
            raise ValueError(f"axis: expected {len(inv_freq)} entries, got {len(axis)}")
        self.rotary_dim, self.n_axes = 2 * len(inv_freq), n_axes
        self._h = _vp()
        _check(lib.skv_rope_create(ctypes.byref(self._h), self.rotary_dim, _f64_array(inv_freq),
                                   None if axis is None else _i32_array(axis), n_axes, int(bool(adjacent_pairs))), "skv_rope_create")
        self._handle = self._h.value

    def close(self):
        if getattr(self, "_h", None):
            lib.skv_rope_destroy(self._h)
            self._h = self._handle = None

    __del__ = close


class SkvCache:
    """Handle of one routed cache.  ``device_pool`` is a torch uint8 CUDA tensor
    of at least ``skv_cache_pool_bytes`` bytes that the caller keeps alive; pass
    ``allocate=True`` to let this wrapper allocate it with torch, or
    ``accounting_only=True`` for a handle without device memory."""

    def __init__(self, r: Sequence[int], kv_heads: int, head_dim: int, page_size: int, max_pages: int,
                 device_pool: Optional[torch.Tensor] = None, allocate: bool = False,
                 accounting_only: bool = False, stream=None, fp8: bool = False):
        self.fp8 = fp8
        create = lib.skv_cache_create_fp8 if fp8 else lib.skv_cache_create
        self.r = [int(x) for x in r]
        self.n_layers = len(self.r)
        self.kv_heads, self.head_dim, self.page_size, self.max_pages = kv_heads, head_dim, page_size, max_pages
        self._h = _vp()
        self.pool = None
        if accounting_only:
            rc = create(ctypes.byref(self._h), self.n_layers, _i32_array(self.r), kv_heads, head_dim,
                        page_size, max_pages, None, 0, None)
            _check(rc, "skv_cache_create")
            self._handle = self._h.value
            return
        need = (skv_cache_pool_bytes_fp8 if fp8 else skv_cache_pool_bytes)(self.r, kv_heads, head_dim, page_size, max_pages)
        if device_pool is None:
            if not allocate:
                raise ValueError("pass device_pool, allocate=True or accounting_only=True")
            device_pool = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert device_pool.is_cuda and device_pool.dtype == torch.uint8 and device_pool.is_contiguous()
        self.pool = device_pool
        rc = create(ctypes.byref(self._h), self.n_layers, _i32_array(self.r), kv_heads, head_dim,
                    page_size, max_pages, device_pool.data_ptr(), device_pool.numel(), _stream_ptr(stream))
        _check(rc, "skv_cache_create")
        self._handle = self._h.value

    # -- lifetime
    def close(self):
        if getattr(self, "_h", None):
            lib.skv_cache_destroy(self._h)
            self._h = self._handle = None

    __del__ = close

    # -- introspection
    def skv_layer_owner(self, layer: int) -> int:
        rc = lib.skv_layer_owner(self._h, layer)
        if rc < 0:
            raise SkvError(rc, "skv_layer_owner")
        return rc

    def skv_is_owner(self, layer: int) -> bool:
        rc = lib.skv_is_owner(self._h, layer)
        if rc < 0:
            raise SkvError(rc, "skv_is_owner")
        return bool(rc)

    def skv_cache_stats(self) -> dict:
        n = _int(0)
        pb, kb, bt = _sz(0), _sz(0), _sz(0)
        _check(lib.skv_cache_stats(self._h, ctypes.byref(n), ctypes.byref(pb), ctypes.byref(kb), ctypes.byref(bt)),
               "skv_cache_stats")
        return {"n_owners": n.value, "page_bytes": pb.value, "kv_bytes": kb.value, "bytes_per_token": bt.value}

    # -- Update
    def skv_append(self, layer: int, K: Optional[torch.Tensor], V: Optional[torch.Tensor],
                   slot_map: Optional[torch.Tensor], n_tokens: Optional[int] = None, stream=None) -> None:
        if n_tokens is None:
            n_tokens = 0 if slot_map is None else slot_map.numel()
        row = (n_tokens, self.kv_heads, self.head_dim)
        _arg("K", K, torch.bfloat16, row)
        _arg("V", V, torch.bfloat16, row)
        _arg("slot_map", slot_map, torch.int64, min_numel=n_tokens)
        rc = lib.skv_append(self._h, layer, _ptr(K), _ptr(V), _ptr(slot_map), n_tokens, _stream_ptr(stream))
        _check(rc, "skv_append")

    def skv_gather(self, layer: int, slot_ids: torch.Tensor, K_out: torch.Tensor, V_out: torch.Tensor,
                   stream=None) -> None:
        n = slot_ids.numel()
        _arg("slot_ids", slot_ids, torch.int64)
        _arg("K_out", K_out, torch.bfloat16, (n, self.kv_heads, self.head_dim))
        _arg("V_out", V_out, torch.bfloat16, (n, self.kv_heads, self.head_dim))
        rc = lib.skv_gather(self._h, layer, _ptr(slot_ids), slot_ids.numel(), _ptr(K_out), _ptr(V_out),
                            _stream_ptr(stream))
        _check(rc, "skv_gather")

    def skv_gather_fp8(self, layer: int, slot_ids: torch.Tensor, K_codes: torch.Tensor, V_codes: torch.Tensor,
                       K_scales: torch.Tensor, V_scales: torch.Tensor, stream=None) -> None:
        rc = lib.skv_gather_fp8(self._h, layer, _ptr(slot_ids), slot_ids.numel(), _ptr(K_codes), _ptr(V_codes),
                                _ptr(K_scales), _ptr(V_scales), _stream_ptr(stream))
        _check(rc, "skv_gather_fp8")

    def skv_rope_append(self, layer: int, rope: SkvRope, Q: Optional[torch.Tensor], Q_out: Optional[torch.Tensor],
                        K: Optional[torch.Tensor], V: Optional[torch.Tensor], positions: torch.Tensor,
                        slot_map: Optional[torch.Tensor], stream=None) -> None:
        """Q, Q_out [n][q_heads][head_dim], K, V [n][kv_heads][head_dim] with any row stride; positions [n] or
        [n_axes][n] int32; slot_map [n] int64.  On a layer that is not an owner K, V, slot_map are not used."""
        rc = _calls.rope_append(self._handle, self.pool, self.head_dim, self.kv_heads, rope.n_axes, layer, rope._handle, Q, Q_out, K, V,
                                positions, slot_map, stream)
        if rc is not None:
            return _check(rc, "skv_rope_append") if rc else None
        device = self._current_device()
        n = positions.shape[-1] if positions.dim() else -1
        axes = 1 if positions.dim() == 1 else positions.shape[0] if positions.dim() == 2 else -1
        if positions.dtype is not torch.int32:
            raise TypeError("positions: expected an int32 tensor")
        if positions.get_device() != device:
            raise ValueError(f"positions: expected a tensor on cuda:{device}, got {positions.device}")
        if axes != rope.n_axes or (n > 1 and positions.stride(-1) != 1):
            raise ValueError(f"positions: expected [{rope.n_axes}][n] with dense rows, got {tuple(positions.shape)}")
        if (Q is None) != (Q_out is None):
            raise ValueError("Q and Q_out go together")
        q_heads = 0 if Q is None else Q.shape[1] if Q.dim() == 3 else -1
        q, qs = (None, 0) if Q is None else _rows("Q", Q, n, q_heads, self.head_dim, device)
        o, os_ = (None, 0) if Q is None else _rows("Q_out", Q_out, n, q_heads, self.head_dim, device)
        k = v = slots = None
        ks = vs = 0
        if 0 <= layer < self.n_layers and self.r[layer] == layer and K is not None and V is not None and slot_map is not None:
            k, ks = _rows("K", K, n, self.kv_heads, self.head_dim, device)
            v, vs = _rows("V", V, n, self.kv_heads, self.head_dim, device)
            slots = _checked("slot_map", slot_map, torch.int64, (n,), device)
        rc = lib.skv_rope_append(self._h, layer, rope._h, q, qs, o, os_, k, ks, v, vs, positions.data_ptr(),
                                 positions.stride(0) if axes > 1 else n, slots, n, q_heads, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_rope_append")

    # -- a step's tables
    def skv_plan_step(self, page_table: torch.Tensor, seq_lens: torch.Tensor, new_lens: torch.Tensor,
                      free_pages: torch.Tensor, n_free: torch.Tensor, slot_map: torch.Tensor, cu_q_lens: torch.Tensor,
                      seq_lens_out: torch.Tensor, n_free_out: torch.Tensor, positions: Optional[torch.Tensor] = None,
                      stream=None) -> None:
        """page_table [batch][width], seq_lens, new_lens, seq_lens_out [batch], free_pages [capacity], n_free, n_free_out [1],
        cu_q_lens [batch+1], positions [max_tokens]: int32; slot_map [max_tokens]: int64."""
        rc = _calls.plan_step(self._handle, self.pool, page_table, seq_lens, new_lens, free_pages, n_free, slot_map, cu_q_lens, seq_lens_out,
                              n_free_out, positions, stream)
        if rc is not None:
            return _check(rc, "skv_plan_step") if rc else None
        device, i32 = self._current_device(), torch.int32
        if seq_lens.dim() != 1:
            raise ValueError("seq_lens: expected [batch]")
        batch = seq_lens.shape[0]
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        row, width, capacity, tokens = (batch,), page_table.shape[1], free_pages.numel(), slot_map.numel()
        pos = None
        if positions is not None:
            if positions.numel() < tokens:
                raise ValueError(f"positions: needs at least {tokens} elements, has {positions.numel()}")
            pos = _checked("positions", positions, i32, positions.shape, device)
        rc = lib.skv_plan_step(self._h, _checked("page_table", page_table, i32, (batch, width), device), width,
                               _checked("seq_lens", seq_lens, i32, row, device), _checked("new_lens", new_lens, i32, row, device), batch,
                               _checked("free_pages", free_pages, i32, (capacity,), device), capacity,
                               _checked("n_free", n_free, i32, (1,), device), tokens,
                               _checked("slot_map", slot_map, torch.int64, (tokens,), device), pos,
                               _checked("cu_q_lens", cu_q_lens, i32, (batch + 1,), device),
                               _checked("seq_lens_out", seq_lens_out, i32, row, device),
                               _checked("n_free_out", n_free_out, i32, (1,), device), _stream_ptr(stream))
        if rc:
            _check(rc, "skv_plan_step")

    def skv_plan_release(self, page_table: torch.Tensor, first_page: torch.Tensor, end_page: torch.Tensor,
                         free_pages: torch.Tensor, n_free: torch.Tensor, n_free_out: torch.Tensor, stream=None) -> None:
        rc = _calls.plan_release(self._handle, self.pool, page_table, first_page, end_page, free_pages, n_free, n_free_out, stream)
        if rc is not None:
            return _check(rc, "skv_plan_release") if rc else None
        device, i32 = self._current_device(), torch.int32
        if page_table.dim() != 2:
            raise ValueError(f"page_table: expected [batch][width], got {tuple(page_table.shape)}")
        batch, width = page_table.shape
        capacity = free_pages.numel()
        rc = lib.skv_plan_release(self._h, _checked("page_table", page_table, i32, (batch, width), device), width,
                                  _checked("first_page", first_page, i32, (batch,), device),
                                  _checked("end_page", end_page, i32, (batch,), device), batch,
                                  _checked("free_pages", free_pages, i32, (capacity,), device), capacity,
                                  _checked("n_free", n_free, i32, (1,), device), _checked("n_free_out", n_free_out, i32, (1,), device),
                                  _stream_ptr(stream))
        if rc:
            _check(rc, "skv_plan_release")

    def _current_device(self) -> int:
        """The current device, to which launches go: it has to be the pool's.  (-2, where no tensor is, for a handle
        without memory, which launches nothing.)"""
        if self.pool is None:
            return -2
        device = torch.cuda.current_device()
        if self.pool.get_device() != device:
            raise ValueError(f"the cache's pool is on {self.pool.device}, the current device is cuda:{device}")
        return device

    # -- Load + Attn
    def _decode_args(self, Q, page_table, seq_lens, out):
        """Shapes of one decode-attention call: Q, out [batch][q_heads][head_dim] bf16; page_table
        [batch][width] int32; seq_lens [batch] int32, all on the device."""
        if Q.dim() != 3 or Q.shape[2] != self.head_dim:
            raise ValueError(f"Q: expected [batch][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        batch, q_heads = Q.shape[0], Q.shape[1]
        _arg("Q", Q, torch.bfloat16)
        if out is not None:
            _arg("out", out, torch.bfloat16, Q.shape)
        _arg("page_table", page_table, torch.int32)
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        _arg("seq_lens", seq_lens, torch.int32, (batch,))
        return batch, q_heads

    def skv_decode_workspace_bytes(self, batch: int, q_heads: int) -> int:
        out = _sz(0)
        _check(lib.skv_decode_workspace_bytes(self._h, batch, q_heads, ctypes.byref(out)),
               "skv_decode_workspace_bytes")
        return out.value

    def skv_decode_attn(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                        out: torch.Tensor, workspace: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        batch, q_heads = self._decode_args(Q, page_table, seq_lens, out)
        _arg("workspace", workspace, torch.uint8)
        rc = lib.skv_decode_attn(self._h, layer, _ptr(Q), _ptr(page_table), _ptr(seq_lens), _ptr(out), batch,
                                 q_heads, page_table.shape[1], scale, _ptr(workspace), _nbytes(workspace),
                                 _stream_ptr(stream))
        _check(rc, "skv_decode_attn")

    def skv_decode_attn_window(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                               out: torch.Tensor, workspace: torch.Tensor, window: int, sinks: int = 0,
                               scale: float = 0.0, stream=None) -> None:
        rc = _calls.decode_attn_window(self._handle, self.pool, self.head_dim, layer, Q, page_table, seq_lens, out, workspace, window, sinks,
                                       scale, stream)
        if rc is not None:
            return _check(rc, "skv_decode_attn_window") if rc else None
        device, bf16, i32 = self._current_device(), torch.bfloat16, torch.int32
        if Q.dim() != 3 or Q.shape[2] != self.head_dim:
            raise ValueError(f"Q: expected [batch][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        batch, q_heads, _ = shape = Q.shape
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        width, nbytes = page_table.shape[1], workspace.numel()
        rc = lib.skv_decode_attn_window(self._h, layer, _checked("Q", Q, bf16, shape, device),
                                        _checked("page_table", page_table, i32, (batch, width), device),
                                        _checked("seq_lens", seq_lens, i32, (batch,), device), _checked("out", out, bf16, shape, device),
                                        batch, q_heads, width, _i32("window", window), _i32("sinks", sinks), scale,
                                        _checked("workspace", workspace, torch.uint8, (nbytes,), device), nbytes, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_decode_attn_window")

    def skv_decode_attn_static(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                               out: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        """skv_decode_attn without a workspace argument, for callers that cannot allocate device memory:
        the scratch is a fixed SKV_STATIC_SCRATCH_BYTES area inside the library (shared by all calls on
        the device; calls that overlap on the GPU race on it)."""
        batch, q_heads = self._decode_args(Q, page_table, seq_lens, out)
        rc = lib.skv_decode_attn_static(self._h, layer, _ptr(Q), _ptr(page_table), _ptr(seq_lens), _ptr(out),
                                        batch, q_heads, page_table.shape[1], scale, _stream_ptr(stream))
        _check(rc, "skv_decode_attn_static")

    def _prefill_args(self, Q, cu_q_lens, page_table, seq_lens, out):
        if Q.dim() != 3 or Q.shape[2] != self.head_dim:
            raise ValueError(f"Q: expected [n_q][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        batch = seq_lens.shape[0]
        _arg("Q", Q, torch.bfloat16)
        _arg("out", out, torch.bfloat16, Q.shape)
        _arg("cu_q_lens", cu_q_lens, torch.int32, (batch + 1,))
        _arg("page_table", page_table, torch.int32)
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        _arg("seq_lens", seq_lens, torch.int32, (batch,))
        return batch, Q.shape[1]

    def skv_prefill_attn(self, layer: int, Q: torch.Tensor, cu_q_lens: torch.Tensor, page_table: torch.Tensor,
                         seq_lens: torch.Tensor, out: torch.Tensor, max_q_len: int, scale: float = 0.0,
                         stream=None) -> None:
        batch, q_heads = self._prefill_args(Q, cu_q_lens, page_table, seq_lens, out)
        rc = lib.skv_prefill_attn(self._h, layer, _ptr(Q), _ptr(cu_q_lens), _ptr(page_table), _ptr(seq_lens),
                                  _ptr(out), batch, max_q_len, q_heads, page_table.shape[1], scale,
                                  _stream_ptr(stream))
        _check(rc, "skv_prefill_attn")

    def skv_prefill_attn_window(self, layer: int, Q: torch.Tensor, cu_q_lens: torch.Tensor, page_table: torch.Tensor,
                                seq_lens: torch.Tensor, out: torch.Tensor, max_q_len: int, window: int, sinks: int = 0,
                                scale: float = 0.0, stream=None) -> None:
        rc = _calls.prefill_attn_window(self._handle, self.pool, self.head_dim, layer, Q, cu_q_lens, page_table, seq_lens, out, max_q_len,
                                        window, sinks, scale, stream)
        if rc is not None:
            return _check(rc, "skv_prefill_attn_window") if rc else None
        device, bf16, i32 = self._current_device(), torch.bfloat16, torch.int32
        if Q.dim() != 3 or Q.shape[2] != self.head_dim:
            raise ValueError(f"Q: expected [n_q][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        if seq_lens.dim() != 1:
            raise ValueError("seq_lens: expected [batch]")
        batch = seq_lens.shape[0]
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        shape, width = Q.shape, page_table.shape[1]
        rc = lib.skv_prefill_attn_window(self._h, layer, _checked("Q", Q, bf16, shape, device),
                                         _checked("cu_q_lens", cu_q_lens, i32, (batch + 1,), device),
                                         _checked("page_table", page_table, i32, (batch, width), device),
                                         _checked("seq_lens", seq_lens, i32, (batch,), device), _checked("out", out, bf16, shape, device),
                                         batch, _i32("max_q_len", max_q_len), shape[1], width, _i32("window", window), _i32("sinks", sinks),
                                         scale, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_prefill_attn_window")

    def skv_prefill_attn_src(self, src_layer: int, Q: torch.Tensor, cu_q_lens: torch.Tensor, page_table: torch.Tensor,
                             seq_lens: torch.Tensor, out: torch.Tensor, max_q_len: int, scale: float = 0.0,
                             stream=None) -> None:
        batch, q_heads = self._prefill_args(Q, cu_q_lens, page_table, seq_lens, out)
        rc = lib.skv_prefill_attn_src(self._h, src_layer, _ptr(Q), _ptr(cu_q_lens), _ptr(page_table), _ptr(seq_lens),
                                      _ptr(out), batch, max_q_len, q_heads, page_table.shape[1], scale,
                                      _stream_ptr(stream))
        _check(rc, "skv_prefill_attn_src")

    def skv_decode_splitk(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                          workspace: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        batch, q_heads = self._decode_args(Q, page_table, seq_lens, None)
        _arg("workspace", workspace, torch.uint8)
        rc = lib.skv_decode_splitk(self._h, layer, _ptr(Q), _ptr(page_table), _ptr(seq_lens), batch, q_heads,
                                   page_table.shape[1], scale, _ptr(workspace), _nbytes(workspace),
                                   _stream_ptr(stream))
        _check(rc, "skv_decode_splitk")

    def skv_decode_merge(self, out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
        batch, q_heads = out.shape[0], out.shape[1]
        _arg("out", out, torch.bfloat16, (batch, q_heads, self.head_dim))
        _arg("workspace", workspace, torch.uint8)
        rc = lib.skv_decode_merge(self._h, _ptr(out), batch, q_heads, _ptr(workspace),
                                  _nbytes(workspace), _stream_ptr(stream))
        _check(rc, "skv_decode_merge")

    def skv_decode_step(self, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, slot_map: torch.Tensor,
                        page_table: torch.Tensor, seq_lens: torch.Tensor, out: torch.Tensor,
                        workspace: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        batch, q_heads = Q.shape[1], Q.shape[2]
        self._step_args(Q, K, V, slot_map, page_table, seq_lens, out, cuda=True)
        _arg("workspace", workspace, torch.uint8)
        rc = lib.skv_decode_step(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(slot_map), _ptr(page_table),
                                 _ptr(seq_lens), _ptr(out), batch, q_heads, page_table.shape[1], scale,
                                 _ptr(workspace), _nbytes(workspace), _stream_ptr(stream))
        _check(rc, "skv_decode_step")

    def _step_args(self, Q, K, V, slot_map, page_table, seq_lens, out, cuda):
        """Shapes of one whole step: Q, out [n_layers][batch][q_heads][head_dim]; K, V
        [n_owners][batch][kv_heads][head_dim]; slot_map [batch] int64; page_table [batch][width]; seq_lens [batch]."""
        if Q.dim() != 4 or Q.shape[0] != self.n_layers or Q.shape[3] != self.head_dim:
            raise ValueError(f"Q: expected [{self.n_layers}][batch][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        batch = Q.shape[1]
        n_owners = sum(1 for l, s in enumerate(self.r) if s == l)
        _arg("Q", Q, torch.bfloat16, cuda=cuda)
        _arg("out", out, torch.bfloat16, Q.shape, cuda=cuda)
        _arg("K", K, torch.bfloat16, (n_owners, batch, self.kv_heads, self.head_dim), cuda=cuda)
        _arg("V", V, torch.bfloat16, (n_owners, batch, self.kv_heads, self.head_dim), cuda=cuda)
        _arg("slot_map", slot_map, torch.int64, (batch,), cuda=cuda)
        _arg("page_table", page_table, torch.int32, cuda=cuda)
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        _arg("seq_lens", seq_lens, torch.int32, (batch,), cuda=cuda)

    def skv_decode_step_staging_bytes(self, batch: int, q_heads: int, pt_stride: int) -> int:
        out = _sz(0)
        _check(lib.skv_decode_step_staging_bytes(self._h, batch, q_heads, pt_stride, ctypes.byref(out)),
               "skv_decode_step_staging_bytes")
        return out.value

    def skv_decode_step_host(self, hQ: torch.Tensor, hK: torch.Tensor, hV: torch.Tensor, h_slot_map: torch.Tensor,
                             h_page_table: torch.Tensor, h_seq_lens: torch.Tensor, h_out: torch.Tensor,
                             staging: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        batch, q_heads = hQ.shape[1], hQ.shape[2]
        self._step_args(hQ, hK, hV, h_slot_map, h_page_table, h_seq_lens, h_out, cuda=False)
        _arg("staging", staging, torch.uint8)
        rc = lib.skv_decode_step_host(self._h, _ptr(hQ), _ptr(hK), _ptr(hV), _ptr(h_slot_map), _ptr(h_page_table),
                                      _ptr(h_seq_lens), _ptr(h_out), batch, q_heads, h_page_table.shape[1], scale,
                                      _ptr(staging), _nbytes(staging), _stream_ptr(stream))
        _check(rc, "skv_decode_step_host")

    # -- attention over selected pages
    def skv_page_index_bytes(self) -> int:
        out = _sz(0)
        _check(lib.skv_page_index_bytes(self._h, ctypes.byref(out)), "skv_page_index_bytes")
        return out.value

    def skv_set_page_index(self, memory: Optional[torch.Tensor], stream=None) -> None:
        """Give (or, with None, take back) the memory of the page index, uint8; it is zero-filled, and has to stay alive
        while it is set."""
        _arg("memory", memory, torch.uint8)
        if memory is not None and memory.get_device() != self._current_device():
            raise ValueError(f"memory: is on {memory.device}, the cache is elsewhere")
        _check(lib.skv_set_page_index(self._h, _ptr(memory), 0 if memory is None else _nbytes(memory), _stream_ptr(stream)),
               "skv_set_page_index")
        self._page_index = memory

    def skv_index_pages(self, layer: int, page_table: torch.Tensor, seq_lens: torch.Tensor, cu_q_lens: Optional[torch.Tensor] = None,
                        max_q_len: int = 1, stream=None) -> None:
        """page_table [batch][width], seq_lens [batch], cu_q_lens [batch+1] (None: one new token per sequence): int32."""
        rc = _calls.index_pages(self._handle, self.pool, layer, page_table, seq_lens, cu_q_lens, max_q_len, stream)
        if rc is not None:
            return _check(rc, "skv_index_pages") if rc else None
        device = self._current_device()
        batch, table, width, lens, cu = self._page_args(page_table, seq_lens, cu_q_lens, device)
        rc = lib.skv_index_pages(self._h, _i32("layer", layer), table, lens, cu, batch, _i32("max_q_len", max_q_len), width, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_index_pages")

    def skv_select_pages(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor, lists: torch.Tensor,
                         counts: torch.Tensor, top: int, first_pages: int = 1, last_pages: int = 1,
                         cu_q_lens: Optional[torch.Tensor] = None, max_q_len: int = 1, run: int = 1, stream=None) -> None:
        """Q [n_q][q_heads][head_dim]; lists [batch * ceil(max_q_len / run)][kv_heads][width] and counts [...][kv_heads] int32
        are written; without cu_q_lens one row per sequence."""
        rc = _calls.select_pages(self._handle, self.pool, self.head_dim, self.kv_heads, layer, Q, cu_q_lens, page_table, seq_lens, lists, counts,
                                 max_q_len, run, top, first_pages, last_pages, stream)
        if rc is not None:
            return _check(rc, "skv_select_pages") if rc else None
        device = self._current_device()
        batch, table, width, lens, cu = self._page_args(page_table, seq_lens, cu_q_lens, device)
        heads, q = self._query_rows(Q, batch if cu is None else None, device)
        ls, ct, entries = self._list_args(lists, counts, batch, _i32("max_q_len", max_q_len), _i32("run", run), device)
        rc = lib.skv_select_pages(self._h, _i32("layer", layer), q, cu, table, lens, ls, ct, batch, max_q_len, heads, width, run, _i32("top", top),
                                  _i32("first_pages", first_pages), _i32("last_pages", last_pages), entries, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_select_pages")

    def skv_decode_attn_pages(self, layer: int, Q: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor, lists: torch.Tensor,
                              counts: torch.Tensor, out: torch.Tensor, scale: float = 0.0, stream=None) -> None:
        """lists [batch][kv_heads][width], counts [batch][kv_heads]: int32, as skv_select_pages writes them."""
        rc = _calls.decode_attn_pages(self._handle, self.pool, self.head_dim, self.kv_heads, layer, Q, page_table, seq_lens, lists, counts, out,
                                      scale, stream)
        if rc is not None:
            return _check(rc, "skv_decode_attn_pages") if rc else None
        device = self._current_device()
        batch, table, width, lens, _ = self._page_args(page_table, seq_lens, None, device)
        heads, q = self._query_rows(Q, batch, device)
        ls, ct, entries = self._list_args(lists, counts, batch, 1, 1, device)
        rc = lib.skv_decode_attn_pages(self._h, _i32("layer", layer), q, table, lens, ls, ct, _checked("out", out, torch.bfloat16, Q.shape, device),
                                       batch, heads, width, entries, scale, _stream_ptr(stream))
        if rc:
            _check(rc, "skv_decode_attn_pages")

    def skv_prefill_attn_pages(self, layer: int, Q: torch.Tensor, cu_q_lens: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                               lists: torch.Tensor, counts: torch.Tensor, out: torch.Tensor, max_q_len: int, run: int = 1, scale: float = 0.0,
                               stream=None) -> None:
        rc = _calls.prefill_attn_pages(self._handle, self.pool, self.head_dim, self.kv_heads, layer, Q, cu_q_lens, page_table, seq_lens, lists,
                                       counts, out, max_q_len, run, scale, stream)
        if rc is not None:
            return _check(rc, "skv_prefill_attn_pages") if rc else None
        device = self._current_device()
        batch, table, width, lens, cu = self._page_args(page_table, seq_lens, cu_q_lens, device)
        heads, q = self._query_rows(Q, None, device)
        ls, ct, entries = self._list_args(lists, counts, batch, _i32("max_q_len", max_q_len), _i32("run", run), device)
        rc = lib.skv_prefill_attn_pages(self._h, _i32("layer", layer), q, cu, table, lens, ls, ct,
                                        _checked("out", out, torch.bfloat16, Q.shape, device), batch, max_q_len, heads, width, run, entries, scale,
                                        _stream_ptr(stream))
        if rc:
            _check(rc, "skv_prefill_attn_pages")

    def _page_args(self, page_table, seq_lens, cu_q_lens, device):
        """Batch, table pointer and width, pointers of the lengths and of the row offsets (None where there are none)."""
        i32 = torch.int32
        if seq_lens.dim() != 1:
            raise ValueError("seq_lens: expected [batch]")
        batch = seq_lens.shape[0]
        if page_table.dim() != 2 or page_table.shape[0] != batch:
            raise ValueError(f"page_table: expected [{batch}][width], got {tuple(page_table.shape)}")
        width = page_table.shape[1]
        return (batch, _checked("page_table", page_table, i32, (batch, width), device), width, _checked("seq_lens", seq_lens, i32, (batch,), device),
                None if cu_q_lens is None else _checked("cu_q_lens", cu_q_lens, i32, (batch + 1,), device))

    def _query_rows(self, Q, rows, device):
        if Q.dim() != 3 or Q.shape[2] != self.head_dim or (rows is not None and Q.shape[0] != rows):
            raise ValueError(f"Q: expected [{'n_q' if rows is None else rows}][q_heads][{self.head_dim}], got {tuple(Q.shape)}")
        return Q.shape[1], _checked("Q", Q, torch.bfloat16, Q.shape, device)

    def _list_args(self, lists, counts, batch, max_q_len, run, device):
        """Pointers of the lists and counts, entries of a list."""
        if max_q_len < 1 or run < 1:
            raise ValueError("max_q_len and run: at least 1")
        n = batch * -(-max_q_len // run)
        if lists.dim() != 3 or lists.shape[:2] != (n, self.kv_heads):
            raise ValueError(f"lists: expected [{n}][{self.kv_heads}][width], got {tuple(lists.shape)}")
        return (_checked("lists", lists, torch.int32, lists.shape, device), _checked("counts", counts, torch.int32, (n, self.kv_heads), device),
                lists.shape[2])

    # -- status, tuning, counters
    def skv_get_status(self, stream=None) -> int:
        st = _int(0)
        _check(lib.skv_get_status(self._h, _stream_ptr(stream), ctypes.byref(st)), "skv_get_status")
        return st.value

    def skv_set_decode_variant(self, variant: int) -> None:
        _check(lib.skv_set_decode_variant(self._h, variant), "skv_set_decode_variant")

    def skv_set_decode_tuning(self, warps_per_cta: int = 0, stages: int = 0, ctas_per_sm: int = 0) -> None:
        _check(lib.skv_set_decode_tuning(self._h, warps_per_cta, stages, ctas_per_sm), "skv_set_decode_tuning")

    def skv_prefill_scratch_bytes(self) -> int:
        out = _sz(0)
        _check(lib.skv_prefill_scratch_bytes(self._h, ctypes.byref(out)), "skv_prefill_scratch_bytes")
        return out.value

    def skv_set_prefill_scratch(self, scratch: Optional[torch.Tensor]) -> None:
        """Give (or, with None, take back) the area in which pre-fill calls on an FP8 cache keep a bf16 copy of
        the pages they reach; the tensor must stay alive while it is set."""
        _arg("scratch", scratch, torch.uint8)
        self._prefill_scratch = scratch
        _check(lib.skv_set_prefill_scratch(self._h, _ptr(scratch), 0 if scratch is None else _nbytes(scratch)),
               "skv_set_prefill_scratch")

    def skv_set_prefill_variant(self, variant: int) -> None:
        _check(lib.skv_set_prefill_variant(self._h, variant), "skv_set_prefill_variant")

    def skv_set_decode_overlap(self, enabled: int) -> None:
        _check(lib.skv_set_decode_overlap(self._h, enabled), "skv_set_decode_overlap")

    def skv_set_decode_worker(self, mode: int, consumers: int = 0, stages: int = 0, ctas_per_sm: int = 0) -> None:
        _check(lib.skv_set_decode_worker(self._h, mode, consumers, stages, ctas_per_sm), "skv_set_decode_worker")

    def skv_set_decode_early_fetch(self, enabled: int) -> None:
        _check(lib.skv_set_decode_early_fetch(self._h, enabled), "skv_set_decode_early_fetch")

    def skv_set_decode_merge(self, mode: int) -> None:
        _check(lib.skv_set_decode_merge(self._h, mode), "skv_set_decode_merge")

    def skv_set_decode_l2_reuse(self, keep_percent: int) -> None:
        _check(lib.skv_set_decode_l2_reuse(self._h, keep_percent), "skv_set_decode_l2_reuse")

    def skv_set_host_step(self, groups: int, ramp: int) -> None:
        _check(lib.skv_set_host_step(self._h, groups, ramp), "skv_set_host_step")

    def skv_set_trace_buffer(self, buf: Optional[torch.Tensor]) -> None:
        _check(lib.skv_set_trace_buffer(self._h, _ptr(buf), 0 if buf is None else buf.numel() * buf.element_size()),
               "skv_set_trace_buffer")

    def skv_decode_worker_count(self) -> int:
        rc = lib.skv_decode_worker_count(self._h)
        if rc < 0:
            raise SkvError(rc, "skv_decode_worker_count")
        return rc

    def skv_launch_count(self) -> int:
        out = _i64(0)
        _check(lib.skv_launch_count(self._h, ctypes.byref(out)), "skv_launch_count")
        return out.value
