"""ctypes binding of libflashcache.so: argument marshalling only.

Every step of the path runs in the library's HIP kernels; torch is used for
device memory and for the current stream handle.  There is no fallback: if the
library has not been built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

# FLASHCACHE_LIBRARY names another build of the same library (bench.py --library sets it for the
# experiment builds of build.py); unset, the product library beside this file is loaded.
_LIB_PATH = os.environ.get("FLASHCACHE_LIBRARY") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "libflashcache.so")

FC_OK, FC_EINVAL, FC_EUNSUPPORTED, FC_EWORKSPACE, FC_EBUDGET, FC_EHIP = range(6)
FC_F32, FC_BF16 = 0, 1
FC_PATH_AUTO, FC_PATH_DENSE, FC_PATH_FFT, FC_PATH_BASIS, FC_PATH_STREAM, FC_PATH_RESAMPLE = range(6)
PATHS = {"auto": FC_PATH_AUTO, "dense": FC_PATH_DENSE, "fft": FC_PATH_FFT,
         "basis": FC_PATH_BASIS, "stream": FC_PATH_STREAM, "resample": FC_PATH_RESAMPLE}

EXPORTED_SYMBOLS = (
    "flashcache_cutoff_r", "flashcache_total_budget", "flashcache_resolve_path", "flashcache_realisation",
    "flashcache_workspace_bytes", "flashcache_select_workspace_bytes", "flashcache_prepare",
    "flashcache_workspace_error", "flashcache_score", "flashcache_score_layer", "flashcache_lowpass_energy",
    "flashcache_allocate",
    "flashcache_select_gather", "flashcache_select_gather_shared", "flashcache_select_gather_paged",
    "flashcache_decode_workspace_bytes", "flashcache_decode_attention",
    "flashcache_decode_attention_paged", "flashcache_decode_static_scratch_bytes",
    "flashcache_decode_attention_static", "flashcache_status_string",
    "flashcache_rotary_prepare", "flashcache_rotary", "flashcache_assign_pages", "flashcache_mx_page_bytes",
    "flashcache_mx_store", "flashcache_mx_load", "flashcache_select_gather_mx", "flashcache_mx_decode_workspace_bytes",
    "flashcache_mx_decode_attention",
    "flashcache_profile_enable", "flashcache_profile_read",
)


class FcKvDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
        ("n_tokens", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("stride_b", ctypes.c_int64), ("stride_l", ctypes.c_int64),
        ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64),
    ]


MAX_ROTARY_PAIRS = 128
FC_ROTARY_PLAIN, FC_ROTARY_LINEAR, FC_ROTARY_BASE, FC_ROTARY_PARTS = range(4)
ROTARY_SCALINGS = {"none": FC_ROTARY_PLAIN, "linear": FC_ROTARY_LINEAR, "base": FC_ROTARY_BASE, "parts": FC_ROTARY_PARTS}


class FcRotarySpec(ctypes.Structure):
    _fields_ = [
        ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("scaling", ctypes.c_int32),
        ("original_tokens", ctypes.c_int32), ("streams", ctypes.c_int32), ("stream_pairs", ctypes.c_int32 * 4),
        ("reserved", ctypes.c_int32), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
        ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double), ("magnitude", ctypes.c_double),
    ]


class FcRotaryPlan(ctypes.Structure):
    _fields_ = [
        ("magic", ctypes.c_uint32), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
        ("streams", ctypes.c_int32), ("stream_end", ctypes.c_int32 * 4), ("magnitude", ctypes.c_float),
        ("reserved", ctypes.c_int32), ("turns", ctypes.c_uint64 * MAX_ROTARY_PAIRS),
    ]


class FcHeadsDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("tokens", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64),
        ("out_stride_b", ctypes.c_int64), ("out_stride_t", ctypes.c_int64), ("out_stride_h", ctypes.c_int64),
    ]


class FcRowsDesc(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("rows", ctypes.c_int64), ("stride_b", ctypes.c_int64), ("stride_r", ctypes.c_int64),
    ]


class FlashCacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it first "
            "(python -c 'import __graft_entry__ as g; g.build()'); there is no fallback path")
    lib = ctypes.CDLL(_LIB_PATH)
    c_desc_p = ctypes.POINTER(FcKvDesc)
    vp, i32, i64, sz, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_double
    lib.flashcache_cutoff_r.argtypes, lib.flashcache_cutoff_r.restype = [i32, dbl], i32
    lib.flashcache_total_budget.argtypes, lib.flashcache_total_budget.restype = [i32, i32, dbl], i64
    lib.flashcache_resolve_path.argtypes, lib.flashcache_resolve_path.restype = [c_desc_p, i32, i32], i32
    lib.flashcache_realisation.argtypes, lib.flashcache_realisation.restype = [c_desc_p, i32, i32], i32
    lib.flashcache_workspace_bytes.argtypes, lib.flashcache_workspace_bytes.restype = [c_desc_p, i32, i32], sz
    lib.flashcache_select_workspace_bytes.argtypes = [c_desc_p]
    lib.flashcache_select_workspace_bytes.restype = sz
    lib.flashcache_prepare.argtypes, lib.flashcache_prepare.restype = [c_desc_p, i32, i32, vp, sz, vp], i32
    lib.flashcache_workspace_error.argtypes = [vp, ctypes.POINTER(i32), vp]
    lib.flashcache_workspace_error.restype = i32
    lib.flashcache_score.argtypes = [vp, vp, c_desc_p, i32, i32, vp, vp, vp, sz, vp]
    lib.flashcache_score_layer.argtypes = [vp, vp, c_desc_p, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.flashcache_score_layer.restype = i32
    lib.flashcache_score.restype = i32
    lib.flashcache_lowpass_energy.argtypes = [c_desc_p, i32, i32, vp, sz, vp, vp]
    lib.flashcache_lowpass_energy.restype = i32
    lib.flashcache_allocate.argtypes = [vp, i32, i32, i32, i32, i64, i32, i32, vp, vp, vp]
    lib.flashcache_allocate.restype = i32
    lib.flashcache_select_gather.argtypes = [vp, vp, c_desc_p, vp, vp, vp, i64, vp, vp, vp, vp, sz, vp]
    lib.flashcache_select_gather.restype = i32
    lib.flashcache_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.flashcache_decode_workspace_bytes.restype = sz
    lib.flashcache_decode_attention.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, i64,
                                                ctypes.c_float, vp, vp, sz, vp]
    lib.flashcache_decode_attention.restype = i32
    lib.flashcache_decode_static_scratch_bytes.argtypes = []
    lib.flashcache_decode_static_scratch_bytes.restype = sz
    lib.flashcache_decode_attention_static.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, i64,
                                                       ctypes.c_float, vp, vp]
    lib.flashcache_decode_attention_static.restype = i32
    lib.flashcache_decode_attention_paged.argtypes = [vp, vp, vp, vp, i32, i32, i64, i32, i32, i32, i32, i32, i32,
                                                      vp, ctypes.c_float, vp, vp, sz, vp]
    lib.flashcache_decode_attention_paged.restype = i32
    lib.flashcache_profile_enable.argtypes, lib.flashcache_profile_enable.restype = [i32], i32
    lib.flashcache_profile_read.argtypes = [i32, ctypes.c_char_p, i32, ctypes.POINTER(i32),
                                            ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.flashcache_profile_read.restype = i32
    lib.flashcache_select_gather_shared.argtypes = lib.flashcache_select_gather.argtypes
    lib.flashcache_select_gather_shared.restype = i32
    lib.flashcache_select_gather_paged.argtypes = [vp, vp, c_desc_p, vp, vp, vp, i64, i32, vp, vp, i32, i32,
                                                   i64, vp, vp, vp, sz, vp]
    lib.flashcache_select_gather_paged.restype = i32
    lib.flashcache_rotary_prepare.argtypes = [ctypes.POINTER(FcRotarySpec), ctypes.POINTER(dbl), ctypes.POINTER(FcRotaryPlan)]
    lib.flashcache_rotary.argtypes = [ctypes.POINTER(FcRotaryPlan), vp, vp, vp, ctypes.POINTER(FcHeadsDesc), vp, vp,
                                      ctypes.POINTER(FcHeadsDesc), i32, vp]
    lib.flashcache_assign_pages.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, i64, vp, vp, vp, i64, vp, vp, vp]
    lib.flashcache_mx_page_bytes.argtypes, lib.flashcache_mx_page_bytes.restype = [i32, i32], sz
    lib.flashcache_mx_store.argtypes = [vp, vp, ctypes.POINTER(FcRowsDesc), vp, i32, i64, vp, vp]
    lib.flashcache_mx_load.argtypes = [vp, vp, i32, i64, ctypes.POINTER(FcRowsDesc), vp, vp, vp]
    lib.flashcache_select_gather_mx.argtypes = [vp, vp, c_desc_p, vp, vp, vp, i64, i32, vp, vp, i32, i32, i64, vp, vp]
    lib.flashcache_mx_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.flashcache_mx_decode_workspace_bytes.restype = sz
    lib.flashcache_mx_decode_attention.argtypes = [vp, vp, vp, i32, i32, i64, i32, i32, i32, i32, i32, i32, vp,
                                                   ctypes.c_float, vp, vp, sz, vp]
    for name in ("rotary_prepare", "rotary", "assign_pages", "mx_store", "mx_load", "select_gather_mx", "mx_decode_attention"):
        getattr(lib, "flashcache_" + name).restype = i32
    lib.flashcache_status_string.argtypes, lib.flashcache_status_string.restype = [i32], ctypes.c_char_p
    return lib


_lib = _load()


def library_path() -> str:
    return _LIB_PATH


def status_string(status: int) -> str:
    return _lib.flashcache_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != FC_OK:
        raise FlashCacheError(status, where)


def _stream() -> int:
    """Handle of the current stream of the current device.  (torch.cuda.current_stream() makes a Stream
    object of it, 2.8 us each of the three times that `Compressor.run` asks; the handle itself takes 0.2.)"""
    if torch.cuda.is_initialized():
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def describe(K: torch.Tensor) -> FcKvDesc:
    """Descriptor of a [B, L, H, N, d] tensor (any strides, innermost contiguous)."""
    if K.dim() != 5:
        raise ValueError("K/V must have shape [B, L, H, N, d]")
    if K.stride(4) != 1 and K.shape[4] > 1:
        raise ValueError("the head dimension must be contiguous")
    if K.dtype == torch.float32:
        dt = FC_F32
    elif K.dtype == torch.bfloat16:
        dt = FC_BF16
    else:
        raise ValueError(f"unsupported dtype {K.dtype}")
    B, L, H, N, d = K.shape
    return FcKvDesc(B, L, H, N, d, dt, K.stride(0), K.stride(1), K.stride(2), K.stride(3))


# ---- host helpers ---------------------------------------------------------------------------
def cutoff_r(n_tokens: int, gamma: float) -> int:
    return int(_lib.flashcache_cutoff_r(n_tokens, gamma))


def total_budget(layers: int, n_tokens: int, rho: float) -> int:
    return int(_lib.flashcache_total_budget(layers, n_tokens, rho))


def resolve_path(desc: FcKvDesc, r: int, path: int = FC_PATH_AUTO) -> int:
    return int(_lib.flashcache_resolve_path(ctypes.byref(desc), r, path))


def realisation(desc: FcKvDesc, r: int, path: int = FC_PATH_AUTO) -> int:
    """What runs behind `path`: FC_PATH_BASIS, FC_PATH_STREAM or FC_PATH_RESAMPLE (0: unsupported)."""
    return int(_lib.flashcache_realisation(ctypes.byref(desc), r, path))


def workspace_bytes(desc: FcKvDesc, r: int, path: int = FC_PATH_AUTO) -> int:
    return int(_lib.flashcache_workspace_bytes(ctypes.byref(desc), r, path))


# ---- device entry points --------------------------------------------------------------------
def prepare(desc: FcKvDesc, r: int, path: int, workspace: torch.Tensor) -> None:
    _check(_lib.flashcache_prepare(ctypes.byref(desc), r, path, _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream()),
           "flashcache_prepare")


def workspace_error(workspace: torch.Tensor) -> int:
    flag = ctypes.c_int32(-1)
    _check(_lib.flashcache_workspace_error(_ptr(workspace), ctypes.byref(flag), _stream()),
           "flashcache_workspace_error")
    return flag.value


def score(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, r: int, path: int,
          scores: torch.Tensor, energy: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(_lib.flashcache_score(_ptr(K), _ptr(V), ctypes.byref(desc), r, path, _ptr(scores),
                                 _ptr(energy), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream()),
           "flashcache_score")


def score_layer(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, layer: int, total_layers: int, r: int,
                path: int, scores: torch.Tensor, energy: torch.Tensor, workspace: torch.Tensor) -> None:
    """K, V: one layer of every sequence, [B, 1, H, N, d]; scores / energy: the full
    [B, total_layers, H, N] / [B, total_layers, H, 4] arrays, of which layer `layer` is written."""
    _check(_lib.flashcache_score_layer(_ptr(K), _ptr(V), ctypes.byref(desc), layer, total_layers, r, path,
                                       _ptr(scores), _ptr(energy), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream()),
           "flashcache_score_layer")


def lowpass_energy(desc: FcKvDesc, r: int, path: int, workspace: torch.Tensor,
                   out: torch.Tensor) -> None:
    """out: float64 [B, L, H, 2]; call right after score() on the same workspace."""
    _check(_lib.flashcache_lowpass_energy(ctypes.byref(desc), r, path, _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _ptr(out),
                                          _stream()), "flashcache_lowpass_energy")


def allocate(energy: torch.Tensor, batch: int, layers: int, kv_heads: int, n_tokens: int,
             total: int, b_min: int, b_max: int, budgets: torch.Tensor,
             layer_offsets: torch.Tensor) -> None:
    _check(_lib.flashcache_allocate(_ptr(energy), batch, layers, kv_heads, n_tokens, total, b_min,
                                    b_max, _ptr(budgets), _ptr(layer_offsets), _stream()),
           "flashcache_allocate")


def select_gather(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, scores: torch.Tensor,
                  budgets: torch.Tensor, layer_offsets: torch.Tensor, rows_per_seq: int,
                  idx_out: torch.Tensor, K_out: torch.Tensor, V_out: torch.Tensor,
                  shared: bool = False) -> None:
    fn = _lib.flashcache_select_gather_shared if shared else _lib.flashcache_select_gather
    _check(fn(_ptr(K), _ptr(V), ctypes.byref(desc), _ptr(scores), _ptr(budgets), _ptr(layer_offsets),
              rows_per_seq, _ptr(idx_out), _ptr(K_out), _ptr(V_out), None, 0, _stream()),
           "flashcache_select_gather_shared" if shared else "flashcache_select_gather")


def select_gather_paged(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, scores: torch.Tensor,
                        budgets: torch.Tensor, layer_offsets: torch.Tensor, rows_per_seq: int,
                        idx_out: torch.Tensor, block_table: torch.Tensor, page_size: int,
                        K_cache: torch.Tensor, V_cache: torch.Tensor, shared: bool = False) -> None:
    """block_table int32 [B, L, H, max_pages]; K_cache/V_cache [num_pages, page_size, d]."""
    _check(_lib.flashcache_select_gather_paged(
        _ptr(K), _ptr(V), ctypes.byref(desc), _ptr(scores), _ptr(budgets), _ptr(layer_offsets),
        rows_per_seq, 1 if shared else 0, _ptr(idx_out), _ptr(block_table), page_size,
        block_table.shape[-1], K_cache.shape[0], _ptr(K_cache), _ptr(V_cache), None, 0, _stream()),
        "flashcache_select_gather_paged")


def decode_attention(Q: torch.Tensor, K_cache: torch.Tensor, V_cache: torch.Tensor, kv_heads: int,
                     budgets: torch.Tensor, layer_offsets: torch.Tensor, rows_per_seq: int,
                     scale: float, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Q [B, L, Hq, d]; K_cache/V_cache packed [B, rows_per_seq, d]; returns float32 [B, L, Hq, d]."""
    B, L, Hq, d = Q.shape
    dt = FC_BF16 if Q.dtype == torch.bfloat16 else FC_F32
    need = int(_lib.flashcache_decode_workspace_bytes(B, L, kv_heads, Hq, d))
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=Q.device)
    if out is None:
        out = torch.empty((B, L, Hq, d), dtype=torch.float32, device=Q.device)
    _check(_lib.flashcache_decode_attention(
        _ptr(Q), _ptr(K_cache), _ptr(V_cache), B, L, kv_heads, Hq, d, dt, _ptr(budgets),
        _ptr(layer_offsets), rows_per_seq, scale, _ptr(out), _ptr(workspace),
        workspace.numel(), _stream()), "flashcache_decode_attention")
    return out


def decode_static_scratch_bytes() -> int:
    return int(_lib.flashcache_decode_static_scratch_bytes())


def decode_attention_static(Q: torch.Tensor, K_cache: torch.Tensor, V_cache: torch.Tensor, kv_heads: int,
                            budgets: torch.Tensor, layer_offsets: torch.Tensor, rows_per_seq: int,
                            scale: float, out: torch.Tensor) -> torch.Tensor:
    """decode_attention without a workspace: the library's own fixed scratch array is used and the
    call allocates nothing (`out` must be given: float32 [B, L, Hq, d])."""
    B, L, Hq, d = Q.shape
    dt = FC_BF16 if Q.dtype == torch.bfloat16 else FC_F32
    _check(_lib.flashcache_decode_attention_static(
        _ptr(Q), _ptr(K_cache), _ptr(V_cache), B, L, kv_heads, Hq, d, dt, _ptr(budgets),
        _ptr(layer_offsets), rows_per_seq, scale, _ptr(out), _stream()), "flashcache_decode_attention_static")
    return out


def decode_attention_paged(Q: torch.Tensor, K_pages: torch.Tensor, V_pages: torch.Tensor, kv_heads: int,
                           budgets: torch.Tensor, block_table: torch.Tensor, scale: float,
                           out: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Q [B, L, Hq, d]; K_pages/V_pages [num_pages, page_size, d]; block_table int32
    [B, L, H, max_pages]; returns float32 [B, L, Hq, d]."""
    B, L, Hq, d = Q.shape
    num_pages, page_size = int(K_pages.shape[0]), int(K_pages.shape[1])
    max_pages = int(block_table.shape[-1])
    dt = FC_BF16 if Q.dtype == torch.bfloat16 else FC_F32
    need = int(_lib.flashcache_decode_workspace_bytes(B, L, kv_heads, Hq, d))
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=Q.device)
    if out is None:
        out = torch.empty((B, L, Hq, d), dtype=torch.float32, device=Q.device)
    _check(_lib.flashcache_decode_attention_paged(
        _ptr(Q), _ptr(K_pages), _ptr(V_pages), _ptr(block_table), page_size, max_pages, num_pages, B, L,
        kv_heads, Hq, d, dt, _ptr(budgets), scale, _ptr(out), _ptr(workspace), workspace.numel(),
        _stream()), "flashcache_decode_attention_paged")
    return out


# ---- the decode loop around a compacted cache --------------------------------------------------
def _type(dtype: torch.dtype) -> int:
    if dtype == torch.bfloat16:
        return FC_BF16
    if dtype == torch.float32:
        return FC_F32
    raise ValueError(f"unsupported dtype {dtype}")


def _dtype(t: torch.Tensor) -> int:
    return _type(t.dtype)


def _want(t: Optional[torch.Tensor], what: str, dtype: torch.dtype, shape: Tuple[int, ...], index: int) -> None:
    """A contiguous tensor of this type and shape on GPU `index`, or nothing at all."""
    if t is not None and (t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on GPU {index}")


def _here(t: torch.Tensor, what: str) -> int:
    """Index of the tensor's GPU, which has to be the current one: that is the device whose current stream the call goes to."""
    index = t.get_device()
    if index < 0 or index != torch._C._cuda_getDevice():
        raise ValueError(f"{what} must be on the current GPU")
    return index


def rotary_plan(rotary_dim: int, theta: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                factor: float = 1.0, original_tokens: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0,
                magnitude: float = 0.0, sections: Optional[Sequence[int]] = None,
                frequencies: Optional[Sequence[float]] = None) -> FcRotaryPlan:
    """What `rotary` needs (host memory; may be kept and used by any number of calls and threads).

    scaling: "none", "linear", "base" or "parts" (flashcache.h has the formulas; "parts" mixes by the turns of a pair, not by its
    number); sections: pairs that each of 2 to 4 streams of positions turns; frequencies: radians per position of each pair,
    instead of theta and the scaling (a magnitude other than 1 has to be given then)."""
    spec = FcRotarySpec(rotary_dim=rotary_dim, interleaved=1 if interleaved else 0, scaling=ROTARY_SCALINGS[scaling],
                        original_tokens=original_tokens, streams=1, theta=theta, factor=factor, beta_fast=beta_fast,
                        beta_slow=beta_slow, magnitude=magnitude)
    if sections is not None:
        if not 1 <= len(sections) <= 4:
            raise ValueError("sections: one to four streams of positions")
        spec.streams = len(sections)
        for k, n in enumerate(sections):
            spec.stream_pairs[k] = n
        if len(sections) == 1 and 2 * sections[0] != rotary_dim:
            raise ValueError("sections must share out all pairs")
    given = None
    if frequencies is not None:
        if 2 * len(frequencies) != rotary_dim:
            raise ValueError("a frequency for each pair")
        given = (ctypes.c_double * len(frequencies))(*frequencies)
    plan = FcRotaryPlan()
    _check(_lib.flashcache_rotary_prepare(ctypes.byref(spec), given, ctypes.byref(plan)), "flashcache_rotary_prepare")
    return plan


@functools.lru_cache(maxsize=1024)
def _heads_of(shape, out_shape, strides, out_strides, dtype) -> FcHeadsDesc:
    """(By what it says alone: a descriptor takes as long to make as all checks of a call; the library reads it only.)"""
    if out_shape != shape:
        raise ValueError("Q, K and their outputs must agree in shape")
    B, T, H, d = shape
    (sb, st, sh, sd), (ob, ot, oh, od) = strides, out_strides
    if (sd != 1 or od != 1) and d > 1:
        raise ValueError("the head dimension must be contiguous")
    return FcHeadsDesc(B, T, H, d, _type(dtype), 0, sb, st, sh, ob, ot, oh)


def _heads(x: torch.Tensor, out: torch.Tensor, what: str, index: int) -> FcHeadsDesc:
    if out.dtype is not x.dtype or out.get_device() != index or x.get_device() != index:
        raise ValueError(f"{what} and its output must agree in shape and dtype and be on GPU {index}")
    return _heads_of(x.shape, out.shape, x.stride(), out.stride(), x.dtype)


def rotary(plan: FcRotaryPlan, positions: torch.Tensor, Q: torch.Tensor, K: Optional[torch.Tensor] = None,
           Q_out: Optional[torch.Tensor] = None, K_out: Optional[torch.Tensor] = None,
           inverse: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rotary positions of Q [B, T, Hq, d] and K [B, T, Hk, d] (any strides, innermost contiguous); positions int32
    [B, T], or [streams, B, T].  Q_out / K_out may be Q and K themselves; without them new tensors are returned.
    inverse: the transposed map, which takes gradients of the outputs to gradients of the inputs.  The call records nothing for
    autograd: tensors that want gradients are refused unless recording is off, as in an autograd.Function's forward and backward."""
    index = _here(Q, "Q")
    if torch.is_grad_enabled() and (Q.requires_grad or K is not None and K.requires_grad or Q_out is not None and
                                    Q_out.requires_grad or K_out is not None and K_out.requires_grad):
        raise ValueError("rotary records no gradients: call it under torch.no_grad() or in an autograd.Function (backward: inverse=True)")
    if Q.dim() != 4 or (K is not None and (K.dim() != 4 or K.shape[:2] != Q.shape[:2])):
        raise ValueError("Q and K must have shape [B, T, H, d], with B and T in common")
    if plan.streams == 1 and positions.dim() == 2:
        _want(positions, "positions", torch.int32, Q.shape[:2], index)
    else:
        _want(positions, "positions", torch.int32, (plan.streams, *Q.shape[:2]), index)
    if Q_out is None:
        Q_out = torch.empty(Q.shape, dtype=Q.dtype, device=Q.device)
    qd = _heads(Q, Q_out, "Q", index)
    if K is None:
        K_ptr = Ko_ptr = kd_ref = K_out = None
    else:
        if K_out is None:
            K_out = torch.empty(K.shape, dtype=K.dtype, device=K.device)
        K_ptr, Ko_ptr, kd_ref = K.data_ptr(), K_out.data_ptr(), ctypes.byref(_heads(K, K_out, "K", index))
    _check(_lib.flashcache_rotary(ctypes.byref(plan), positions.data_ptr(), Q.data_ptr(), Q_out.data_ptr(), ctypes.byref(qd),
                                  K_ptr, Ko_ptr, kd_ref, 1 if inverse else 0, _stream()), "flashcache_rotary")
    return Q_out, K_out


def assign_pages(rows: torch.Tensor, add, page_size: int, block_table: torch.Tensor, cursor: torch.Tensor,
                 free_pages: Optional[torch.Tensor] = None, num_free: Optional[int] = None,
                 slots: Optional[torch.Tensor] = None, rows_out: Optional[torch.Tensor] = None,
                 cursor_out: Optional[torch.Tensor] = None) -> None:
    """Pages and slots for the rows that each layer adds: rows int32 [B, L] held, add int32 [B, L] or a number for all;
    block_table int32 [B, L, H, max_pages] (in/out); cursor int64 [1]; free_pages int32 [n] (None: pages 0 .. num_free - 1);
    slots int64 [B, n] (out).  rows_out / cursor_out default to `rows` and `cursor`, updated in place."""
    if block_table.dim() != 4:
        raise ValueError("block_table must have shape [B, L, H, max_pages]")
    B, L, H, most = block_table.shape
    index = _here(block_table, "block_table")
    _want(block_table, "block_table", torch.int32, (B, L, H, most), index)
    each, add_ptr = 0, None
    if isinstance(add, torch.Tensor):
        _want(add, "add", torch.int32, (B, L), index)
        add_ptr = add.data_ptr()
    else:
        each = int(add)
        if not -2 ** 31 <= each < 2 ** 31:
            raise ValueError("a number of rows has 32 bits")
    rows_out = rows if rows_out is None else rows_out
    cursor_out = cursor if cursor_out is None else cursor_out
    _want(rows, "rows", torch.int32, (B, L), index)
    _want(rows_out, "rows_out", torch.int32, (B, L), index)
    _want(cursor, "cursor", torch.int64, (1,), index)
    _want(cursor_out, "cursor_out", torch.int64, (1,), index)
    if free_pages is None and num_free is None:
        raise ValueError("either free_pages or num_free")
    if free_pages is not None:
        count = free_pages.numel()
        _want(free_pages, "free_pages", torch.int32, (count,), index)
        num_free = count if num_free is None else num_free
        if num_free > count:
            raise ValueError("num_free exceeds the list")
    per_seq = 0
    if slots is not None:
        per_seq = slots.shape[-1] if slots.dim() else 0
        _want(slots, "slots", torch.int64, (B, per_seq), index)
    _check(_lib.flashcache_assign_pages(
        rows.data_ptr(), add_ptr, each, B, L, H, page_size, most, _ptr(free_pages), num_free, cursor.data_ptr(),
        block_table.data_ptr(), _ptr(slots), per_seq, rows_out.data_ptr(), cursor_out.data_ptr(), _stream()),
        "flashcache_assign_pages")


@functools.lru_cache(maxsize=None)
def mx_page_bytes(page_size: int, head_dim: int) -> int:
    """Bytes of a page of the 4-bit cache, K and V; 0 if unsupported."""
    return int(_lib.flashcache_mx_page_bytes(page_size, head_dim))


def _mx_pages(pages: torch.Tensor, page_size: int, head_dim: int, index: int) -> int:
    nbytes = mx_page_bytes(page_size, head_dim)
    if nbytes == 0:
        raise FlashCacheError(FC_EUNSUPPORTED, "flashcache_mx_page_bytes")
    n = pages.shape[0]
    _want(pages, "pages", torch.uint8, (n, nbytes), index)
    return n


@functools.lru_cache(maxsize=1024)
def _rows_of(shape, v_shape, strides, v_strides, dtype) -> FcRowsDesc:
    if len(shape) != 3 or shape != v_shape:
        raise ValueError("K and V must have shape [B, R, d]")
    B, R, d = shape
    if strides != v_strides and any(n > 1 and s != o for n, s, o in zip(shape, strides, v_strides)):
        raise ValueError("K and V must have the same strides")
    if strides[2] != 1 and d > 1:
        raise ValueError("the head dimension must be contiguous")
    return FcRowsDesc(B, d, _type(dtype), 0, R, strides[0], strides[1])


def _mx_rows(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, index: int) -> FcRowsDesc:
    if K.dtype is not V.dtype or V.get_device() != index:
        raise ValueError("K and V must have the same dtype and device")
    desc = _rows_of(K.shape, V.shape, K.stride(), V.stride(), K.dtype)
    _want(slots, "slots", torch.int64, (desc.batch, desc.rows), index)
    return desc


def mx_store(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, pages: torch.Tensor, page_size: int) -> None:
    """Rows K, V [B, R, d] into slots int64 [B, R] (negative: left out) of pages uint8 [num_pages, mx_page_bytes]."""
    index = _here(K, "K")
    desc = _mx_rows(K, V, slots, index)
    n = _mx_pages(pages, page_size, desc.head_dim, index)
    _check(_lib.flashcache_mx_store(K.data_ptr(), V.data_ptr(), ctypes.byref(desc), slots.data_ptr(), page_size, n,
                                    pages.data_ptr(), _stream()), "flashcache_mx_store")


def mx_load(slots: torch.Tensor, pages: torch.Tensor, page_size: int, K_out: torch.Tensor, V_out: torch.Tensor) -> None:
    """Rows of the slots int64 [B, R] into K_out, V_out [B, R, d] (bf16 or fp32, both exact); zeros without a slot."""
    index = _here(K_out, "K_out")
    desc = _mx_rows(K_out, V_out, slots, index)
    n = _mx_pages(pages, page_size, desc.head_dim, index)
    _check(_lib.flashcache_mx_load(slots.data_ptr(), pages.data_ptr(), page_size, n, ctypes.byref(desc), K_out.data_ptr(),
                                   V_out.data_ptr(), _stream()), "flashcache_mx_load")


def _described(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, index: int) -> None:
    shape = (desc.batch, desc.layers, desc.kv_heads, desc.n_tokens, desc.head_dim)
    strides = (desc.stride_b, desc.stride_l, desc.stride_h, desc.stride_n, 1)
    for t in (K, V):
        given = t.stride()
        if t.shape != shape or _dtype(t) != desc.dtype or t.get_device() != index or (given != strides and any(
                n > 1 and s != o for n, s, o in zip(shape, strides, given))):
            raise ValueError("K and V must be what the descriptor describes")


def select_gather_mx(K: torch.Tensor, V: torch.Tensor, desc: FcKvDesc, scores: torch.Tensor, budgets: torch.Tensor,
                     layer_offsets: torch.Tensor, rows_per_seq: int, idx_out: torch.Tensor, block_table: torch.Tensor,
                     page_size: int, pages: torch.Tensor, shared: bool = False) -> None:
    """select_gather_paged into a 4-bit cache: pages uint8 [num_pages, mx_page_bytes]."""
    index = _here(K, "K")
    n = _mx_pages(pages, page_size, desc.head_dim, index)
    B, L, H, N = desc.batch, desc.layers, desc.kv_heads, desc.n_tokens
    _described(K, V, desc, index)
    _want(scores, "scores", torch.float32, (B, L, H, N), index)
    _want(budgets, "budgets", torch.int32, (B, L), index)
    _want(layer_offsets, "layer_offsets", torch.int64, (B, L + 1), index)
    _want(idx_out, "idx_out", torch.int32, (B, rows_per_seq), index)
    _want(block_table, "block_table", torch.int32, (B, L, H, block_table.shape[-1]), index)
    _check(_lib.flashcache_select_gather_mx(
        _ptr(K), _ptr(V), ctypes.byref(desc), _ptr(scores), _ptr(budgets), _ptr(layer_offsets), rows_per_seq,
        1 if shared else 0, _ptr(idx_out), _ptr(block_table), page_size, block_table.shape[-1], n, _ptr(pages), _stream()),
        "flashcache_select_gather_mx")


@functools.lru_cache(maxsize=256)
def _mx_decode_workspace(batch: int, layers: int, kv_heads: int, q_heads: int, head_dim: int) -> int:
    return int(_lib.flashcache_mx_decode_workspace_bytes(batch, layers, kv_heads, q_heads, head_dim))


def mx_decode_attention(Q: torch.Tensor, pages: torch.Tensor, page_size: int, kv_heads: int, rows: torch.Tensor,
                        block_table: torch.Tensor, scale: float, out: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Q [B, L, Hq, d]; pages uint8 [num_pages, mx_page_bytes]; rows int32 [B, L]; block_table int32
    [B, L, H, max_pages]; returns float32 [B, L, Hq, d].  An operator of inference: no gradients."""
    shape = Q.shape
    B, L, Hq, d = shape
    index = _here(Q, "Q")
    n = _mx_pages(pages, page_size, d, index)
    most = block_table.shape[-1]
    _want(Q, "Q", Q.dtype, shape, index)
    _want(rows, "rows", torch.int32, (B, L), index)
    _want(block_table, "block_table", torch.int32, (B, L, kv_heads, most), index)
    if workspace is None:
        workspace = torch.empty(max(_mx_decode_workspace(B, L, kv_heads, Hq, d), 16), dtype=torch.uint8, device=Q.device)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on GPU {index}")
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=Q.device)
    else:
        _want(out, "out", torch.float32, shape, index)
    _check(_lib.flashcache_mx_decode_attention(
        Q.data_ptr(), pages.data_ptr(), block_table.data_ptr(), page_size, most, n, B, L, kv_heads, Hq, d, _dtype(Q),
        rows.data_ptr(), scale, out.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream()),
        "flashcache_mx_decode_attention")
    return out


def profile_enable(on: bool) -> None:
    _check(_lib.flashcache_profile_enable(1 if on else 0), "flashcache_profile_enable")


def profile_read(max_entries: int = 32) -> dict:
    """{kernel name: (launches, total milliseconds)} recorded since profile_enable(True)."""
    stride = 64
    names = ctypes.create_string_buffer(max_entries * stride)
    launches = (ctypes.c_int32 * max_entries)()
    total_ms = (ctypes.c_float * max_entries)()
    n = ctypes.c_int32(0)
    _check(_lib.flashcache_profile_read(max_entries, names, stride, launches, total_ms,
                                        ctypes.byref(n)), "flashcache_profile_read")
    out = {}
    for k in range(min(n.value, max_entries)):
        name = names.raw[k * stride:(k + 1) * stride].split(b"\0", 1)[0].decode()
        out[name] = (int(launches[k]), float(total_ms[k]))
    return out


# ---- convenience: buffers for one shape, and the three calls in order -------------------------
class Compressor:
    """Owns the device buffers for one (shape, r, T) and enqueues score -> allocate -> select_gather.

    Pure plumbing: allocation through torch, then the three C-ABI calls on the current stream.
    """

    def __init__(self, K: torch.Tensor, r: int, total: int, path: str = "auto",
                 b_min: int = 1, b_max: Optional[int] = None, shared: bool = False):
        self.desc = describe(K)
        B, L, H, N, d = K.shape
        self.shape = (B, L, H, N, d)
        self.r, self.total = int(r), int(total)
        self.b_min, self.b_max = int(b_min), int(N if b_max is None else b_max)
        self.shared = bool(shared)
        self.path = resolve_path(self.desc, self.r, PATHS[path])
        if self.path == 0:
            raise FlashCacheError(FC_EUNSUPPORTED, "resolve_path")
        dev = K.device
        nbytes = workspace_bytes(self.desc, self.r, realisation(self.desc, self.r, self.path))
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        self.scores = torch.empty((B, L, H, N), dtype=torch.float32, device=dev)
        self.energy = torch.empty((B, L, H, 4), dtype=torch.float64, device=dev)
        self.budgets = torch.empty((B, L), dtype=torch.int32, device=dev)
        self.layer_offsets = torch.empty((B, L + 1), dtype=torch.int64, device=dev)
        self.rows_per_seq = H * self.total
        self.idx = torch.empty((B, self.rows_per_seq), dtype=torch.int32, device=dev)
        self.K_out = torch.empty((B, self.rows_per_seq, d), dtype=K.dtype, device=dev)
        self.V_out = torch.empty((B, self.rows_per_seq, d), dtype=K.dtype, device=dev)
        prepare(self.desc, self.r, self.path, self.workspace)

    def run_score(self, K, V):
        score(K, V, self.desc, self.r, self.path, self.scores, self.energy, self.workspace)

    def run_allocate(self):
        B, L, H, N, _ = self.shape
        allocate(self.energy, B, L, H, N, self.total, self.b_min, self.b_max, self.budgets,
                 self.layer_offsets)

    def run_select_gather(self, K, V):
        select_gather(K, V, self.desc, self.scores, self.budgets, self.layer_offsets,
                      self.rows_per_seq, self.idx, self.K_out, self.V_out, shared=self.shared)

    def run(self, K: torch.Tensor, V: torch.Tensor) -> None:
        self.run_score(K, V)
        self.run_allocate()
        self.run_select_gather(K, V)


class MxCache:
    """A 4-bit paged cache and its block tables: filled from a compression, then extended and attended to step by step.

    Pure plumbing, as `Compressor`: buffers through torch, calls on the current stream, nothing read back.  Of `num_pages`
    pages the first ones are taken as rows come, `max_pages` by a unit at most.  Rows without a page are counted in `rows`, but neither
    stored nor attended to; `missing()` (synchronising) says how many pages they lack.
    A step is rotary (outside), append(k, v), attend(q), and may be captured into a graph (after one eager attend, which
    makes the workspace).  Both take all layers at once; layer by layer, as a model runs, a step is assign_pages over the cache's
    tensors (all layers), then for layer l mx_store into slots[:, l*H:(l+1)*H] and mx_decode_attention over rows[:, l:l+1] and
    block_table[:, l:l+1], of which several sequences need contiguous copies.
    Calls of one cache have to follow each other: on one stream, or ordered by events."""

    def __init__(self, batch: int, layers: int, kv_heads: int, head_dim: int, page_size: int, max_pages: int,
                 num_pages: int, device="cuda"):
        nbytes = mx_page_bytes(page_size, head_dim)
        if nbytes == 0:
            raise FlashCacheError(FC_EUNSUPPORTED, "flashcache_mx_page_bytes")
        if max_pages < 1 or num_pages < 1:
            raise ValueError("a cache has at least one page, and room for one in each table")
        self.page_size, self.num_pages = int(page_size), int(num_pages)
        self.shape = (int(batch), int(layers), int(kv_heads), int(head_dim))
        self.pages = torch.empty((num_pages, nbytes), dtype=torch.uint8, device=device)
        self.block_table = torch.full((batch, layers, kv_heads, max_pages), -1, dtype=torch.int32, device=device)
        self.rows = torch.zeros((batch, layers), dtype=torch.int32, device=device)
        self.cursor = torch.zeros(1, dtype=torch.int64, device=device)
        self.slots = torch.empty((batch, layers * kv_heads), dtype=torch.int64, device=device)
        self._workspaces = {}                # by query heads; kept, since captured graphs hold their addresses
        self._empty = True

    def reset(self) -> None:
        """An empty cache again."""
        self.block_table.fill_(-1)
        self.rows.zero_()
        self.cursor.zero_()
        self._empty = True

    def fill(self, comp: Compressor, K: torch.Tensor, V: torch.Tensor) -> None:
        """The rows that `comp` (scored and allocated for this K, V) keeps, into the empty cache."""
        B, L, H, d = self.shape
        if comp.shape[:3] != (B, L, H) or comp.shape[4] != d:
            raise ValueError("the compression is of another shape")
        if not self._empty:
            raise ValueError("fill takes an empty cache: reset() first")
        _described(K, V, comp.desc, _here(K, "K"))
        if (K.data_ptr() | V.data_ptr()) % 16:
            raise ValueError("K and V must be aligned to 16 bytes")
        assign_pages(self.rows, comp.budgets, self.page_size, self.block_table, self.cursor, num_free=self.num_pages)
        self._empty = False
        try:
            select_gather_mx(K, V, comp.desc, comp.scores, comp.budgets, comp.layer_offsets, comp.rows_per_seq, comp.idx,
                             self.block_table, self.page_size, self.pages, shared=comp.shared)
        except (ValueError, FlashCacheError):    # (too many rows for one launch, for instance: nothing of them is stored)
            self.reset()
            raise

    def append(self, k: torch.Tensor, v: torch.Tensor) -> None:
        """One row more for every unit: k, v [B, L, H, d] contiguous."""
        B, L, H, d = self.shape
        if k.shape != self.shape or v.shape != self.shape:
            raise ValueError("k and v must have shape [B, L, H, d]")
        k, v = k.view(B, L * H, d), v.view(B, L * H, d)
        # (what the store would refuse, before the rows are counted)
        _mx_rows(k, v, self.slots, _here(k, "k"))
        if (k.data_ptr() | v.data_ptr()) % 16:
            raise ValueError("k and v must be aligned to 16 bytes")
        self._empty = False
        assign_pages(self.rows, 1, self.page_size, self.block_table, self.cursor, num_free=self.num_pages, slots=self.slots)
        mx_store(k, v, self.slots, self.pages, self.page_size)

    def attend(self, q: torch.Tensor, scale: float, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q [B, L, Hq, d]; float32 [B, L, Hq, d]."""
        B, L, H, d = self.shape
        if q.dim() != 4 or q.shape[:2] != (B, L) or q.shape[3] != d:
            raise ValueError("q must have shape [B, L, Hq, d]")
        heads = q.shape[2]
        workspace = self._workspaces.get(heads)
        if workspace is None:
            workspace = torch.empty(max(_mx_decode_workspace(B, L, H, heads, d), 16), dtype=torch.uint8, device=self.pages.device)
            self._workspaces[heads] = workspace
        return mx_decode_attention(q, self.pages, self.page_size, H, self.rows, self.block_table, scale, out=out,
                                   workspace=workspace)

    def missing(self) -> int:
        """Pages that the counted rows lack (those rows are not stored): beyond `num_pages` of the pool, and beyond `max_pages`
        of each unit's table, which the cursor does not count.  Reads rows and cursor back."""
        heads, most = self.block_table.shape[2:]
        pages = (self.rows.long() + (self.page_size - 1)) // self.page_size
        return max(0, int(self.cursor.item()) - self.num_pages) + heads * int((pages - most).clamp_(min=0).sum().item())
