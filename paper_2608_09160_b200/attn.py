"""Python side of include/qknorm_attn.h: rotary positions, the fused norm + rotation + cache write,
attention over a paged cache.

Argument marshalling only, as in ``binding``: tensors are used for their device pointers, shapes and
strides, every step runs in the library's kernels, a bad argument raises ``QKNormError``.  Every tensor of a call must
be on the current device.

A decode step of one layer::

    inv_freq, mscale = attn.rope_frequencies(128, theta=5e5)
    q = attn.qknorm_fwd_append(q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, 1e-6)
    out = attn.qknorm_attn_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q=1, max_kv=8192)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import binding
from .binding import QKNormError, _check, _expect, _invoke, _ptr

EXPORTS = (
    "qknorm_rope_frequencies",
    "qknorm_rope",
    "qknorm_rope_e4m3",
    "qknorm_fwd_append",
    "qknorm_attn_paged",
    "qknorm_attn_paged_workspace",
)

SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}
NORM_NONE, NORM_LAYERWISE, NORM_HEADWISE = 0, 1, 2

_vp = ctypes.c_void_p
_BF16, _F8 = torch.bfloat16, torch.float8_e4m3fn


class CRotation(ctypes.Structure):
    """qknorm_rotation"""
    _fields_ = [("positions", _vp), ("inv_freq", _vp), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("mscale", ctypes.c_float)]


class CPagedCache(ctypes.Structure):
    """qknorm_paged_cache"""
    _fields_ = [("k", _vp), ("v", _vp),
                ("k_page", ctypes.c_int64), ("k_token", ctypes.c_int64), ("k_head", ctypes.c_int64),
                ("v_page", ctypes.c_int64), ("v_token", ctypes.c_int64), ("v_head", ctypes.c_int64),
                ("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("e4m3", ctypes.c_int32),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


_ready = False


def lib() -> ctypes.CDLL:
    """The loaded library with the prototypes of qknorm_attn.h declared."""
    global _ready
    L = binding.load()
    if _ready:
        return L
    i32, i64, f32, f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double
    L.qknorm_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, ctypes.POINTER(f64), ctypes.POINTER(f32)]
    for fn in (L.qknorm_rope, L.qknorm_rope_e4m3):
        fn.argtypes = [_vp, _vp, ctypes.POINTER(CRotation), i64, i32, i32, i32, i64, i64, i32, _vp, _vp, i64, i64, _vp]
    L.qknorm_fwd_append.argtypes = [_vp, _vp, _vp, _vp, _vp, i32, f32, ctypes.POINTER(CRotation), _vp,
                                    ctypes.POINTER(CPagedCache), i64, i32, i64, i64, i64, _vp, i64, _vp]
    L.qknorm_attn_paged.argtypes = [_vp, i64, ctypes.POINTER(CPagedCache), _vp, i32, i64, _vp, _vp, i32, i64, i32, i32, i32,
                                    f32, i32, i32, _vp, i64, _vp, _vp, i64, _vp]
    L.qknorm_attn_paged_workspace.argtypes = [i32, i64, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i64)]
    for name in EXPORTS:
        getattr(L, name).restype = ctypes.c_int
    _ready = True
    return L


def rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: str = "plain", *, factor: float = 1.0,
                     original_len: float = 0.0, low: float = 1.0, high: float = 32.0, device="cuda") -> Tuple[torch.Tensor, float]:
    """qknorm_rope_frequencies: (inv_freq, mscale) -- radians per position of the rot_dim/2 pairs, a float64 tensor on
    `device`, and the factor that goes with them.  scaling: plain, linear, base, ramp (low and high in turns within
    original_len; 1 and 32 are usual) or bands (1 and 4 are usual)."""
    if scaling not in SCALINGS:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"scaling must be one of {sorted(SCALINGS)}")
    host = (ctypes.c_double * max(1, int(rot_dim) // 2))()
    mscale = ctypes.c_float(1.0)
    _check(lib().qknorm_rope_frequencies(int(rot_dim), float(theta), SCALINGS[scaling], float(factor), float(original_len),
                                         float(low), float(high), host, ctypes.byref(mscale)))
    return torch.tensor(list(host), dtype=torch.float64).to(device), float(mscale.value)


def _here(*ts) -> None:
    """Every tensor on the current device: the library launches there."""
    cur = torch.cuda.current_device()
    for t in ts:
        if t is not None and t.device.index != cur:
            raise QKNormError(-1, f"a tensor is on {t.device}, the current device is cuda:{cur}")


def _rows(t: torch.Tensor, T: int, what: str, dtype) -> int:
    """A [T, d] CUDA view of `dtype` with unit column stride; its row stride in elements (0 = contiguous)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not dtype or t.dim() != 2:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"{what}: expected a 2-D {dtype} CUDA tensor")
    (n, d), (ld, unit) = t.shape, t.stride()
    if n != T or (unit != 1 and d > 1) or (ld < d and T > 1):
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"{what}: expected {T} rows with unit column stride, got {tuple(t.shape)} "
                                                    f"with strides {tuple(t.stride())}")
    return ld if T > 1 else d


def _rotation(positions, inv_freq, T: int, interleaved: bool, mscale: float) -> Optional[CRotation]:
    if positions is None and inv_freq is None:
        return None
    _expect(positions, (T,), torch.int64, "positions")
    if inv_freq is None or inv_freq.dim() != 1:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "inv_freq: expected a 1-D float64 CUDA tensor")
    _expect(inv_freq, (inv_freq.shape[0],), torch.float64, "inv_freq")
    return CRotation(_ptr(positions), _ptr(inv_freq), 2 * inv_freq.shape[0], 1 if interleaved else 0, float(mscale))


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor, k_scale: float, v_scale: float) -> CPagedCache:
    """k_cache, v_cache [num_pages, page_size, heads, head_dim], any strides over pages, tokens and heads."""
    for t, what in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        if (not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 4 or t.dtype not in (_BF16, _F8)
                or (t.shape[3] > 1 and t.stride(3) != 1)):
            raise QKNormError(binding.QKNORM_ERR_SHAPE, f"{what}: expected a 4-D bfloat16 or float8_e4m3fn CUDA tensor "
                                                        f"[pages, page_size, heads, head_dim] with unit stride in head_dim")
    if k_cache.shape != v_cache.shape or k_cache.dtype is not v_cache.dtype:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "k_cache and v_cache differ in shape or type")
    pages, page, heads, hd = k_cache.shape
    ks, vs = k_cache.stride(), v_cache.stride()
    return CPagedCache(_ptr(k_cache), _ptr(v_cache), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], pages, page, heads, hd,
                       1 if k_cache.dtype is _F8 else 0, float(k_scale), float(v_scale))


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new tensor that belongs to the stream the call is made on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    s = torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream
    with torch.cuda.stream(s):
        return torch.empty(shape, dtype=dtype, device=device)


def qknorm_rope(q, k, positions, inv_freq, head_dim: int, out_q=None, out_k=None, *, interleaved: bool = False,
                inverse: bool = False, mscale: float = 1.0, stream=None):
    """qknorm_rope / qknorm_rope_e4m3 (chosen by the activations' dtype): rotary positions on q [T, dq] and k [T, dk]
    (either may be None; rows may be strided).  positions int64 [T]; inv_freq float64 [rot_dim/2]; rot_dim <= head_dim,
    the rest of a head passes through.  interleaved: pairs (2i, 2i+1), else (i, i + rot_dim/2).
    inverse=True turns back: the backward pass, from the gradient of the outputs to that of the inputs.
    out_* default to new tensors and may be the inputs.  Returns (out_q, out_k)."""
    L = lib()
    ref = q if q is not None else k
    if ref is None:
        raise QKNormError(binding.QKNORM_ERR_NULL, "q and k are both None")
    if ref.dim() != 2:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "q and k are 2-D: [tokens, heads * head_dim]")
    T, act = ref.shape[0], _F8 if ref.dtype is _F8 else _BF16
    _here(q, k, positions, inv_freq, out_q, out_k)
    rot = _rotation(positions, inv_freq, T, interleaved, mscale)
    if rot is None:
        raise QKNormError(binding.QKNORM_ERR_NULL, "positions and inv_freq are None")
    dq = dk = ldq = ldk = ldoq = ldok = 0
    if q is not None:
        dq, ldq = q.shape[1], _rows(q, T, "q", act)
        out_q = _empty((T, dq), act, q.device, stream) if out_q is None else out_q
        ldoq = _rows(out_q, T, "out_q", act)
        if out_q.shape[1] != dq:
            raise QKNormError(binding.QKNORM_ERR_SHAPE, "out_q: another width than q")
    if k is not None:
        dk, ldk = k.shape[1], _rows(k, T, "k", act)
        out_k = _empty((T, dk), act, k.device, stream) if out_k is None else out_k
        ldok = _rows(out_k, T, "out_k", act)
        if out_k.shape[1] != dk:
            raise QKNormError(binding.QKNORM_ERR_SHAPE, "out_k: another width than k")
    fn = L.qknorm_rope_e4m3 if act is _F8 else L.qknorm_rope
    _invoke(fn, [_ptr(q), _ptr(k), ctypes.byref(rot), T, dq, dk, int(head_dim), ldq, ldk, 1 if inverse else 0,
                 _ptr(out_q) if q is not None else None, _ptr(out_k) if k is not None else None, ldoq, ldok], stream,
            (q, k, positions, inv_freq, out_q, out_k, rot))
    return out_q, out_k


def qknorm_fwd_append(q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, eps: float, out_q=None, *,
                      headwise: bool = False, interleaved: bool = False, mscale: float = 1.0, k_scale: float = 1.0,
                      v_scale: float = 1.0, stream=None):
    """qknorm_fwd_append: norm (layerwise, or headwise; none if gamma_q and gamma_k are None), rotation (none if positions and
    inv_freq are None) and cache write in one pass.  q [T, dq] (or None), k and v [T, heads * head_dim] bf16, rows may
    be strided; slots int64 [T] (page * page_size + token; outside the pool: not written); k_cache and v_cache
    [pages, page_size, heads, head_dim] bf16 or float8_e4m3fn (holding x / scale), written in place.
    out_q defaults to a new tensor and may be q.  Returns out_q."""
    L = lib()
    cache = _cache(k_cache, v_cache, k_scale, v_scale)
    if not isinstance(k, torch.Tensor) or k.dim() != 2:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "k: expected a 2-D bfloat16 CUDA tensor")
    T, dk = k.shape[0], cache.heads * cache.head_dim
    _here(q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, out_q)
    ldk, ldv = _rows(k, T, "k", _BF16), _rows(v, T, "v", _BF16)
    if k.shape[1] != dk or v.shape[1] != dk:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"k and v: the cache holds {dk} values per token")
    _expect(slots, (T,), torch.int64, "slots")
    norm = NORM_HEADWISE if headwise else NORM_LAYERWISE
    if gamma_q is None and gamma_k is None:
        norm = NORM_NONE
    else:
        _expect(gamma_k, (dk,), _BF16, "gamma_k")
    dq = ldq = ldo = 0
    if q is not None:
        ldq = _rows(q, T, "q", _BF16)
        dq = q.shape[1]
        if norm != NORM_NONE:
            _expect(gamma_q, (dq,), _BF16, "gamma_q")
        out_q = _empty((T, dq), _BF16, q.device, stream) if out_q is None else out_q
        ldo = _rows(out_q, T, "out_q", _BF16)
        if out_q.shape[1] != dq:
            raise QKNormError(binding.QKNORM_ERR_SHAPE, "out_q: another width than q")
    rot = _rotation(positions, inv_freq, T, interleaved, mscale)
    _invoke(L.qknorm_fwd_append,
            [_ptr(q), _ptr(k), _ptr(v), _ptr(gamma_q), _ptr(gamma_k), norm, float(eps),
             ctypes.byref(rot) if rot is not None else None, _ptr(slots), ctypes.byref(cache), T, dq, ldq, ldk, ldv,
             _ptr(out_q) if q is not None else None, ldo], stream,
            (q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, out_q, rot, cache))
    return out_q


def attn_paged_workspace(num_seqs: int, tokens: int, max_q: int, max_kv: int, heads_q: int, heads_kv: int, head_dim: int,
                         window: int = 0) -> int:
    """qknorm_attn_paged_workspace: bytes a call of these sizes needs on the current device."""
    out = ctypes.c_int64(0)
    _check(lib().qknorm_attn_paged_workspace(num_seqs, tokens, max_q, max_kv, heads_q, heads_kv, head_dim, window, ctypes.byref(out)))
    return out.value


def qknorm_attn_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q: int, max_kv: int, *,
                      scale: Optional[float] = None, causal: bool = True, window: int = 0, k_scale: float = 1.0,
                      v_scale: float = 1.0, out=None, lse=None, workspace=None, stream=None):
    """qknorm_attn_paged: attention of the new tokens q [T, heads_q * head_dim] bf16 over the paged cache
    ([pages, page_size, heads, head_dim], bf16 or float8_e4m3fn).  block_table int32 [B, cols], kv_lens int32 [B],
    q_starts int32 [B+1]; max_q and max_kv bound a sequence's new tokens and keys.  scale defaults to 1/sqrt(head_dim).
    out defaults to a new tensor whose rows outside every sequence are not written; lse: fp32 [T, heads_q] to fill;
    workspace: uint8 tensor of attn_paged_workspace(...) bytes, by default a new one per call.  Returns out."""
    L = lib()
    cache = _cache(k_cache, v_cache, k_scale, v_scale)
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "q: expected a 2-D bfloat16 CUDA tensor")
    T, dq = q.shape
    _here(q, k_cache, v_cache, block_table, kv_lens, q_starts, out, lse, workspace)
    ldq = _rows(q, T, "q", _BF16)
    hd = cache.head_dim
    if dq == 0 or dq % hd != 0:
        raise QKNormError(binding.QKNORM_ERR_HEADS, f"q: {dq} columns are no whole number of heads of {hd}")
    hq = dq // hd
    if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "kv_lens: expected a 1-D int32 CUDA tensor")
    B = kv_lens.shape[0]
    _expect(kv_lens, (B,), torch.int32, "kv_lens")
    _expect(q_starts, (B + 1,), torch.int32, "q_starts")
    if (not isinstance(block_table, torch.Tensor) or not block_table.is_cuda or block_table.dtype is not torch.int32
            or block_table.dim() != 2 or block_table.shape[0] != B or (block_table.shape[1] > 1 and block_table.stride(1) != 1)):
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"block_table: expected an int32 CUDA tensor [{B}, pages per sequence]")
    cols = block_table.shape[1]
    ldt = block_table.stride(0) if B > 1 else 0
    if out is None:
        out = _empty((T, dq), _BF16, q.device, stream)
    elif out.shape != q.shape:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, "out: another shape than q")
    ldo = _rows(out, T, "out", _BF16)
    if lse is not None:
        _expect(lse, (T, hq), torch.float32, "lse")
    if workspace is None:
        need = ctypes.c_int64(0)
        _check(L.qknorm_attn_paged_workspace(B, T, int(max_q), int(max_kv), hq, cache.heads, hd, int(window), ctypes.byref(need)))
        nbytes = need.value
        workspace = _empty((nbytes,), torch.uint8, q.device, stream) if nbytes else None
    else:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise QKNormError(binding.QKNORM_ERR_SCRATCH, "workspace must be a contiguous CUDA tensor")
        nbytes = workspace.numel() * workspace.element_size()
    _invoke(L.qknorm_attn_paged,
            [_ptr(q), ldq, ctypes.byref(cache), _ptr(block_table), cols, ldt, _ptr(kv_lens), _ptr(q_starts), B, T, int(max_q),
             int(max_kv), hq, 1.0 / math.sqrt(hd) if scale is None else float(scale), 1 if causal else 0, int(window),
             _ptr(out), ldo, _ptr(lse), _ptr(workspace), nbytes], stream,
            (q, k_cache, v_cache, block_table, kv_lens, q_starts, out, lse, workspace, cache))
    return out
