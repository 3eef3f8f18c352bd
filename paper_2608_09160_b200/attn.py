"""Python side of include/qknorm_attn.h: rotary positions (along one axis or several), the fused norm + rotation + cache
write, attention over a paged cache (bf16, FP8 or 4 bits).

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
import functools
import math
import struct
from typing import Optional, Tuple

import torch

from . import binding
from .binding import QKNormError, _check, _invoke

EXPORTS = (
    "qknorm_rope_frequencies",
    "qknorm_rope",
    "qknorm_rope_e4m3",
    "qknorm_fwd_append",
    "qknorm_attn_paged",
    "qknorm_attn_paged_workspace",
    "qknorm_rope_axes",
    "qknorm_rope_axes_e4m3",
    "qknorm_fwd_append_axes",
    "qknorm_fwd_append_e2m1",
    "qknorm_attn_paged_e2m1",
    "qknorm_attn_paged_e2m1_workspace",
)

SCALINGS = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}
NORM_NONE, NORM_LAYERWISE, NORM_HEADWISE = 0, 1, 2
MAX_HEAD_DIM = 512  # QKNORM_MAX_HEAD_DIM
MAX_HEAD_DIM_E2M1 = 256  # QKNORM_MAX_HEAD_DIM_E2M1
MAX_AXES = 8  # QKNORM_MAX_AXES

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


class CRotationAxes(ctypes.Structure):
    """qknorm_rotation_axes"""
    _fields_ = [("positions", _vp), ("ld_positions", ctypes.c_int64), ("inv_freq", _vp), ("axis", _vp),
                ("num_axes", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("mscale", ctypes.c_float)]


class CPagedCacheE2m1(ctypes.Structure):
    """qknorm_paged_cache_e2m1"""
    _fields_ = ([(n, _vp) for n in ("k", "v", "k_scales", "v_scales")]
                + [(f"{side}_{axis}", ctypes.c_int64) for side in ("k", "v", "ks", "vs") for axis in ("page", "token", "head")]
                + [("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                   ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)])


# The same structs as bytes, which is what the wrappers pass: a decode step is a few microseconds long, and filling a
# ctypes structure takes two of them.
_ROTATION, _CACHE = struct.Struct("PPiif4x"), struct.Struct("PPqqqqqqqiiiiff")
_AXES, _CACHE_E2M1 = struct.Struct("PqPPiiif"), struct.Struct("PPPPqqqqqqqqqqqqqiiiff4x")
assert _ROTATION.size == ctypes.sizeof(CRotation) and _CACHE.size == ctypes.sizeof(CPagedCache)
assert _AXES.size == ctypes.sizeof(CRotationAxes) and _CACHE_E2M1.size == ctypes.sizeof(CPagedCacheE2m1)

_ready = False


def lib() -> ctypes.CDLL:
    """The loaded library with the prototypes of qknorm_attn.h declared."""
    global _ready
    L = binding.load()
    if _ready:
        return L
    i32, i64, f32, f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double
    L.qknorm_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, ctypes.POINTER(f64), ctypes.POINTER(f32)]
    for fn in (L.qknorm_rope, L.qknorm_rope_e4m3, L.qknorm_rope_axes, L.qknorm_rope_axes_e4m3):
        fn.argtypes = [_vp, _vp, _vp, i64, i32, i32, i32, i64, i64, i32, _vp, _vp, i64, i64, _vp]
    for fn in (L.qknorm_fwd_append, L.qknorm_fwd_append_axes, L.qknorm_fwd_append_e2m1):
        fn.argtypes = [_vp, _vp, _vp, _vp, _vp, i32, f32, _vp, _vp,
                       _vp, i64, i32, i64, i64, i64, _vp, i64, _vp]
    for fn in (L.qknorm_attn_paged, L.qknorm_attn_paged_e2m1):
        fn.argtypes = [_vp, i64, _vp, _vp, i32, i64, _vp, _vp, i32, i64, i32, i32, i32,
                       f32, i32, i32, _vp, i64, _vp, _vp, i64, _vp]
    for fn in (L.qknorm_attn_paged_workspace, L.qknorm_attn_paged_e2m1_workspace):
        fn.argtypes = [i32, i64, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i64)]
    for name in EXPORTS:
        getattr(L, name).restype = ctypes.c_int
    _ready = True
    return L


def _refuse(status: int, message: str):
    raise QKNormError(status, message)


_SHAPE = binding.QKNORM_ERR_SHAPE


def _int32(value, what: str) -> int:
    """An int the C ABI's int32 holds: ctypes cuts off what it does not."""
    value = int(value)
    if not -0x80000000 <= value <= 0x7fffffff:
        _refuse(_SHAPE, f"{what}: {value} does not fit 32 bits")
    return value


def rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: str = "plain", *, factor: float = 1.0,
                     original_len: float = 0.0, low: float = 1.0, high: float = 32.0, device="cuda") -> Tuple[torch.Tensor, float]:
    """qknorm_rope_frequencies: (inv_freq, mscale) -- radians per position of the rot_dim/2 pairs, a float64 tensor on
    `device`, and the factor that goes with them.  scaling: plain, linear, base, ramp (low and high in turns within
    original_len; 1 and 32 are usual) or bands (1 and 4 are usual)."""
    if scaling not in SCALINGS:
        raise QKNormError(binding.QKNORM_ERR_SHAPE, f"scaling must be one of {sorted(SCALINGS)}")
    rot_dim = _int32(rot_dim, "rot_dim")
    if rot_dim > MAX_HEAD_DIM:
        _refuse(_SHAPE, f"rot_dim: at most {MAX_HEAD_DIM}")
    host = (ctypes.c_double * max(1, rot_dim // 2))()
    mscale = ctypes.c_float(1.0)
    _check(lib().qknorm_rope_frequencies(rot_dim, float(theta), SCALINGS[scaling], float(factor), float(original_len),
                                         float(low), float(high), host, ctypes.byref(mscale)))
    return torch.tensor(list(host), dtype=torch.float64).to(device), float(mscale.value)


def _device() -> int:
    return torch._C._cuda_getDevice()


def _flat(t, shape, dtype, what: str, dev: int) -> int:
    """A contiguous tensor of that shape on the current device; its address."""
    if not isinstance(t, torch.Tensor):
        _refuse(binding.QKNORM_ERR_NULL if t is None else _SHAPE, f"{what}: expected a tensor, got {t!r}")
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse(_SHAPE, f"{what}: expected contiguous {dtype} {tuple(shape)} on cuda:{dev}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(t, T: int, what: str, dtype, dev: int, width: int = -1):
    """A [T, d] view of `dtype` with unit column stride on the current device: (address, d, row stride in elements)."""
    if not isinstance(t, torch.Tensor):
        _refuse(binding.QKNORM_ERR_NULL if t is None else _SHAPE, f"{what}: expected a tensor, got {t!r}")
    if t.dtype is dtype and t.dim() == 2 and t.get_device() == dev:
        (n, d), (ld, unit) = t.shape, t.stride()
        if T == 1:
            ld = d
        if n == T and (unit == 1 or d <= 1) and ld >= d and (width < 0 or d == width):
            return t.data_ptr(), d, ld
    _refuse(_SHAPE, f"{what}: expected {dtype} [{T}, {width if width >= 0 else 'd'}] with unit column stride on cuda:{dev}, got "
                    f"{t.dtype} {tuple(t.shape)} with strides {tuple(t.stride())} on {t.device}")


def _rotation(positions, inv_freq, T: int, interleaved: bool, mscale: float, dev: int) -> Optional[bytes]:
    if positions is None and inv_freq is None:
        return None
    if not isinstance(inv_freq, torch.Tensor) or inv_freq.dim() != 1:
        _refuse(_SHAPE, "inv_freq: expected a 1-D float64 CUDA tensor")
    n = inv_freq.shape[0]
    return _ROTATION.pack(_flat(positions, (T,), torch.int64, "positions", dev), _flat(inv_freq, (n,), torch.float64, "inv_freq", dev),
                          2 * n, 1 if interleaved else 0, mscale)


def _rotation_axes(positions, inv_freq, axis, T: int, interleaved: bool, mscale: float, dev: int) -> Optional[bytes]:
    """qknorm_rotation_axes: positions [axes, T] with axis, or [T] and axis None."""
    if axis is None:
        if positions is None and inv_freq is None:
            return None
        if not isinstance(inv_freq, torch.Tensor) or inv_freq.dim() != 1:
            _refuse(_SHAPE, "inv_freq: expected a 1-D float64 CUDA tensor")
        n = inv_freq.shape[0]
        return _AXES.pack(_flat(positions, (T,), torch.int64, "positions", dev), 0, _flat(inv_freq, (n,), torch.float64, "inv_freq", dev),
                          0, 1, 2 * n, 1 if interleaved else 0, mscale)
    if not isinstance(inv_freq, torch.Tensor) or inv_freq.dim() != 1:
        _refuse(_SHAPE, "inv_freq: expected a 1-D float64 CUDA tensor")
    if not isinstance(positions, torch.Tensor) or positions.dim() != 2 or not 1 <= positions.shape[0] <= MAX_AXES:
        _refuse(_SHAPE, f"positions: expected an int64 CUDA tensor [axes, {T}] of 1 to {MAX_AXES} axes to go with axis")
    n, axes = inv_freq.shape[0], positions.shape[0]
    ld = positions.stride(0) if axes > 1 else T
    if (positions.dtype is not torch.int64 or positions.shape[1] != T or positions.get_device() != dev
            or (T > 1 and positions.stride(1) != 1) or ld < T):
        _refuse(_SHAPE, f"positions: expected int64 [axes, {T}] with unit stride along the tokens on cuda:{dev}, got {positions.dtype} "
                        f"{tuple(positions.shape)} with strides {tuple(positions.stride())} on {positions.device}")
    return _AXES.pack(positions.data_ptr(), ld, _flat(inv_freq, (n,), torch.float64, "inv_freq", dev),
                      _flat(axis, (n,), torch.uint8, "axis", dev), axes, 2 * n, 1 if interleaved else 0, mscale)


def rope_axes(sections, *, turns: bool = False, device="cuda") -> torch.Tensor:
    """The `axis` tensor of a rotation with several axes: sections[a] pairs turn by axis a, sum(sections) = rot_dim/2.  In blocks,
    axis 0's pairs first; or (turns) dealt one to each axis in turn for as long as it has any left, from the first pair on."""
    sections = [int(n) for n in sections]
    if not 1 <= len(sections) <= MAX_AXES or min(sections) < 0:
        _refuse(_SHAPE, f"sections: expected 1 to {MAX_AXES} numbers of pairs, got {sections}")
    if turns:
        axis = [a for i in range(max(sections)) for a, n in enumerate(sections) if i < n]
    else:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    return torch.tensor(axis, dtype=torch.uint8).to(device)


def _cache(k_cache, v_cache, k_scale: float, v_scale: float, dev: int):
    """k_cache, v_cache [num_pages, page_size, heads, head_dim], any strides over pages, tokens and heads: (struct, heads,
    head_dim)."""
    if isinstance(k_cache, torch.Tensor) and isinstance(v_cache, torch.Tensor):
        dtype, shape = k_cache.dtype, k_cache.shape
        if ((dtype is _BF16 or dtype is _F8) and v_cache.dtype is dtype and len(shape) == 4 and v_cache.shape == shape
                and k_cache.get_device() == dev and v_cache.get_device() == dev):
            pages, page, heads, hd = shape
            kp, kt, kh, k1 = k_cache.stride()
            vp, vt, vh, v1 = v_cache.stride()
            if (k1 == 1 and v1 == 1) or hd == 1:
                return _CACHE.pack(k_cache.data_ptr(), v_cache.data_ptr(), kp, kt, kh, vp, vt, vh, pages, page, heads, hd,
                                   1 if dtype is _F8 else 0, k_scale, v_scale), heads, hd
    _refuse(_SHAPE, f"k_cache, v_cache: expected two bfloat16 or float8_e4m3fn tensors [pages, page_size, heads, head_dim] of one type and "
                    f"shape on cuda:{dev}, with unit stride in head_dim")


_U8, _F4 = torch.uint8, getattr(torch, "float4_e2m1fn_x2", None)  # a torch without the type has no tensors of it


def _cache_e2m1(k_cache, v_cache, k_scales, v_scales, k_scale: float, v_scale: float, dev: int):
    """k_cache, v_cache [pages, page_size, heads, head_dim/2] bytes, k_scales, v_scales [pages, page_size, heads, head_dim/16], any
    strides over pages, tokens and heads: (struct, heads, head_dim)."""
    try:
        shape, sshape, dtype, sdtype = k_cache.shape, k_scales.shape, k_cache.dtype, k_scales.dtype
        if ((dtype is _U8 or dtype is _F4) and v_cache.dtype is dtype and (sdtype is _F8 or sdtype is _U8) and v_scales.dtype is sdtype
                and v_cache.shape == shape and v_scales.shape == sshape
                and k_cache.get_device() == v_cache.get_device() == k_scales.get_device() == v_scales.get_device() == dev):
            pages, page, heads, half = shape
            kp, kt, kh, k1 = k_cache.stride()
            vp, vt, vh, v1 = v_cache.stride()
            ap, at, ah, a1 = k_scales.stride()
            bp, bt, bh, b1 = v_scales.stride()
            if (half > 0 and half % 8 == 0 and sshape == (pages, page, heads, half // 8) and k1 == 1 and v1 == 1
                    and ((a1 == 1 and b1 == 1) or half == 8)):
                return _CACHE_E2M1.pack(k_cache.data_ptr(), v_cache.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), kp, kt, kh, vp, vt, vh,
                                        ap, at, ah, bp, bt, bh, pages, page, heads, 2 * half, k_scale, v_scale), heads, 2 * half
    except (AttributeError, ValueError):  # no tensor, or not four axes
        pass
    _refuse(_SHAPE, "k_cache, v_cache, k_scales, v_scales: expected two uint8 or float4_e2m1fn_x2 tensors [pages, page_size, heads, head_dim/2] of "
                    "one type and shape and two float8_e4m3fn or uint8 tensors [pages, page_size, heads, head_dim/16], head_dim a multiple of 16, "
                    f"on cuda:{dev}, with unit stride in the last axis")


def _current(stream):
    """What `_invoke` takes: the current stream as a handle if none is given."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if stream is None else stream


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new tensor that belongs to the stream the call is made on."""
    if stream is None:  # strides given: a third less time than torch.empty
        return torch.empty_strided(shape, (shape[1], 1) if len(shape) == 2 else (1,), dtype=dtype, device=device)
    s = torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream
    with torch.cuda.stream(s):
        return torch.empty(shape, dtype=dtype, device=device)


def qknorm_rope(q, k, positions, inv_freq, head_dim: int, out_q=None, out_k=None, *, interleaved: bool = False,
                inverse: bool = False, mscale: float = 1.0, axis=None, stream=None):
    """qknorm_rope / qknorm_rope_e4m3 (chosen by the activations' dtype): rotary positions on q [T, dq] and k [T, dk]
    (either may be None; rows may be strided).  positions int64 [T]; inv_freq float64 [rot_dim/2]; rot_dim <= head_dim,
    the rest of a head passes through.  axis uint8 [rot_dim/2] (qknorm_rope_axes): positions are int64 [axes, T], and pair i turns by those
    of axis[i]; see rope_axes.  interleaved: pairs (2i, 2i+1), else (i, i + rot_dim/2).
    inverse=True turns back: the backward pass, from the gradient of the outputs to that of the inputs.
    out_* default to new tensors and may be the inputs.  Returns (out_q, out_k)."""
    L = lib()
    ref = q if q is not None else k
    if ref is None:
        _refuse(binding.QKNORM_ERR_NULL, "q and k are both None")
    if not isinstance(ref, torch.Tensor) or ref.dim() != 2:
        _refuse(_SHAPE, "q and k are 2-D tensors: [tokens, heads * head_dim]")
    T, act, dev = ref.shape[0], _F8 if ref.dtype is _F8 else _BF16, _device()
    rot = (_rotation(positions, inv_freq, T, interleaved, mscale, dev) if axis is None
           else _rotation_axes(positions, inv_freq, axis, T, interleaved, mscale, dev))
    if rot is None:
        _refuse(binding.QKNORM_ERR_NULL, "positions and inv_freq are None")
    pq = pk = poq = pok = None
    dq = dk = ldq = ldk = ldoq = ldok = 0
    if q is not None:
        pq, dq, ldq = _rows(q, T, "q", act, dev)
        if out_q is None:
            out_q = _empty((T, dq), act, q.device, stream)
            poq = out_q.data_ptr()
        else:
            poq, _, ldoq = _rows(out_q, T, "out_q", act, dev, dq)
    if k is not None:
        pk, dk, ldk = _rows(k, T, "k", act, dev)
        if out_k is None:
            out_k = _empty((T, dk), act, k.device, stream)
            pok = out_k.data_ptr()
        else:
            pok, _, ldok = _rows(out_k, T, "out_k", act, dev, dk)
    _invoke((L.qknorm_rope_e4m3 if act is _F8 else L.qknorm_rope) if axis is None else
            (L.qknorm_rope_axes_e4m3 if act is _F8 else L.qknorm_rope_axes),
            (pq, pk, rot, T, dq, dk, _int32(head_dim, "head_dim"), ldq, ldk, 1 if inverse else 0, poq, pok, ldoq, ldok), _current(stream),
            (q, k, positions, inv_freq, axis, out_q, out_k))
    return out_q, out_k


def qknorm_fwd_append(q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, eps: float, out_q=None, *,
                      headwise: bool = False, interleaved: bool = False, mscale: float = 1.0, k_scale: float = 1.0,
                      v_scale: float = 1.0, axis=None, stream=None):
    """qknorm_fwd_append: norm (layerwise, or headwise; none if gamma_q and gamma_k are None), rotation (none if positions and
    inv_freq are None) and cache write in one pass.  q [T, dq] (or None), k and v [T, heads * head_dim] bf16, rows may
    be strided; slots int64 [T] (page * page_size + token; outside the pool: not written); k_cache and v_cache
    [pages, page_size, heads, head_dim] bf16 or float8_e4m3fn (holding x / scale), written in place.  axis: as in qknorm_rope.
    out_q defaults to a new tensor and may be q.  Returns out_q."""
    L = lib()
    dev = _device()
    cache, heads, hd = _cache(k_cache, v_cache, k_scale, v_scale, dev)
    return _append(L.qknorm_fwd_append if axis is None else L.qknorm_fwd_append_axes, axis is not None, (k_cache, v_cache), cache, heads, hd, q, k, v,
                   gamma_q, gamma_k, positions, inv_freq, axis, slots, eps, out_q, headwise, interleaved, mscale, stream, dev)


def qknorm_fwd_append_e2m1(q, k, v, gamma_q, gamma_k, positions, inv_freq, slots, k_cache, v_cache, k_scales, v_scales, eps: float, out_q=None,
                           *, headwise: bool = False, interleaved: bool = False, mscale: float = 1.0, k_scale: float = 1.0,
                           v_scale: float = 1.0, axis=None, stream=None):
    """qknorm_fwd_append_e2m1: qknorm_fwd_append into a 4-bit cache, codes [pages, page_size, heads, head_dim/2] (uint8 or
    float4_e2m1fn_x2, the even element in the low four bits) and scales [pages, page_size, heads, head_dim/16] (float8_e4m3fn or
    uint8), written in place; an element reads back as code * scale * k_scale (v_scale).  Returns out_q."""
    L = lib()
    dev = _device()
    cache, heads, hd = _cache_e2m1(k_cache, v_cache, k_scales, v_scales, k_scale, v_scale, dev)
    return _append(L.qknorm_fwd_append_e2m1, True, (k_cache, v_cache, k_scales, v_scales), cache, heads, hd, q, k, v, gamma_q, gamma_k, positions,
                   inv_freq, axis, slots, eps, out_q, headwise, interleaved, mscale, stream, dev)


def _append(cfunc, several: bool, pools, cache, heads: int, hd: int, q, k, v, gamma_q, gamma_k, positions, inv_freq, axis, slots, eps, out_q,
            headwise, interleaved, mscale, stream, dev: int):
    if not isinstance(k, torch.Tensor) or k.dim() != 2:
        _refuse(_SHAPE, "k: expected a 2-D bfloat16 CUDA tensor")
    T, dk = k.shape[0], heads * hd
    pk, _, ldk = _rows(k, T, "k", _BF16, dev, dk)
    pv, _, ldv = _rows(v, T, "v", _BF16, dev, dk)
    pslots = _flat(slots, (T,), torch.int64, "slots", dev)
    norm = NORM_HEADWISE if headwise else NORM_LAYERWISE
    pgq = pgk = pq = po = None
    if gamma_q is None and gamma_k is None:
        norm = NORM_NONE
    else:
        pgk = _flat(gamma_k, (dk,), _BF16, "gamma_k", dev)
    dq = ldq = ldo = 0
    if q is not None:
        pq, dq, ldq = _rows(q, T, "q", _BF16, dev)
        if norm != NORM_NONE:
            pgq = _flat(gamma_q, (dq,), _BF16, "gamma_q", dev)
        if out_q is None:
            out_q = _empty((T, dq), _BF16, q.device, stream)
            po = out_q.data_ptr()
        else:
            po, _, ldo = _rows(out_q, T, "out_q", _BF16, dev, dq)
    rot = (_rotation_axes(positions, inv_freq, axis, T, interleaved, mscale, dev) if several
           else _rotation(positions, inv_freq, T, interleaved, mscale, dev))
    _invoke(cfunc, (pq, pk, pv, pgq, pgk, norm, eps, rot, pslots, cache, T, dq, ldq, ldk, ldv, po, ldo), _current(stream),
            (q, k, v, gamma_q, gamma_k, positions, inv_freq, axis, slots, *pools, out_q))
    return out_q


def attn_paged_workspace(num_seqs: int, tokens: int, max_q: int, max_kv: int, heads_q: int, heads_kv: int, head_dim: int,
                         window: int = 0) -> int:
    """qknorm_attn_paged_workspace: bytes a call of these sizes needs on the current device."""
    names = ("num_seqs", "max_q", "max_kv", "heads_q", "heads_kv", "head_dim", "window")
    num_seqs, max_q, max_kv, heads_q, heads_kv, head_dim, window = map(
        _int32, (num_seqs, max_q, max_kv, heads_q, heads_kv, head_dim, window), names)
    return _workspace(torch.cuda.current_device(), num_seqs, tokens, max_q, max_kv, heads_q, heads_kv, head_dim, window)


def attn_paged_e2m1_workspace(num_seqs: int, tokens: int, max_q: int, max_kv: int, heads_q: int, heads_kv: int, head_dim: int,
                              window: int = 0) -> int:
    """qknorm_attn_paged_e2m1_workspace: bytes a call of these sizes needs on the current device."""
    names = ("num_seqs", "max_q", "max_kv", "heads_q", "heads_kv", "head_dim", "window")
    num_seqs, max_q, max_kv, heads_q, heads_kv, head_dim, window = map(
        _int32, (num_seqs, max_q, max_kv, heads_q, heads_kv, head_dim, window), names)
    return _workspace_e2m1(torch.cuda.current_device(), num_seqs, tokens, max_q, max_kv, heads_q, heads_kv, head_dim, window)


@functools.lru_cache(maxsize=256)
def _workspace(device: int, *sizes: int) -> int:
    out = ctypes.c_int64(0)
    _check(lib().qknorm_attn_paged_workspace(*sizes, ctypes.byref(out)))
    return out.value


@functools.lru_cache(maxsize=256)
def _workspace_e2m1(device: int, *sizes: int) -> int:
    out = ctypes.c_int64(0)
    _check(lib().qknorm_attn_paged_e2m1_workspace(*sizes, ctypes.byref(out)))
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
    dev = _device()
    cache, heads, hd = _cache(k_cache, v_cache, k_scale, v_scale, dev)
    return _attend(L.qknorm_attn_paged, _workspace, (k_cache, v_cache), cache, heads, hd, q, block_table, kv_lens, q_starts, max_q, max_kv, scale,
                   causal, window, out, lse, workspace, stream, dev)


def qknorm_attn_paged_e2m1(q, k_cache, v_cache, k_scales, v_scales, block_table, kv_lens, q_starts, max_q: int, max_kv: int, *,
                           scale: Optional[float] = None, causal: bool = True, window: int = 0, k_scale: float = 1.0,
                           v_scale: float = 1.0, out=None, lse=None, workspace=None, stream=None):
    """qknorm_attn_paged_e2m1: qknorm_attn_paged over a 4-bit cache (codes and scales as in qknorm_fwd_append_e2m1).
    workspace: uint8 tensor of attn_paged_e2m1_workspace(...) bytes, by default a new one per call.  Returns out."""
    L = lib()
    dev = _device()
    cache, heads, hd = _cache_e2m1(k_cache, v_cache, k_scales, v_scales, k_scale, v_scale, dev)
    return _attend(L.qknorm_attn_paged_e2m1, _workspace_e2m1, (k_cache, v_cache, k_scales, v_scales), cache, heads, hd, q, block_table, kv_lens,
                   q_starts, max_q, max_kv, scale, causal, window, out, lse, workspace, stream, dev)


def _attend(cfunc, bytes_of, pools, cache, heads: int, hd: int, q, block_table, kv_lens, q_starts, max_q, max_kv, scale, causal, window, out, lse,
            workspace, stream, dev: int):
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        _refuse(_SHAPE, "q: expected a 2-D bfloat16 CUDA tensor")
    T = q.shape[0]
    pq, dq, ldq = _rows(q, T, "q", _BF16, dev)
    if dq == 0 or dq % hd != 0:
        _refuse(binding.QKNORM_ERR_HEADS, f"q: {dq} columns are no whole number of heads of {hd}")
    hq, max_q, max_kv, window = dq // hd, _int32(max_q, "max_q"), _int32(max_kv, "max_kv"), _int32(window, "window")
    if not isinstance(kv_lens, torch.Tensor) or kv_lens.dim() != 1:
        _refuse(_SHAPE, "kv_lens: expected a 1-D int32 CUDA tensor")
    B = kv_lens.shape[0]
    plens = _flat(kv_lens, (B,), torch.int32, "kv_lens", dev)
    pstarts = _flat(q_starts, (B + 1,), torch.int32, "q_starts", dev)
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        _refuse(_SHAPE, f"block_table: expected an int32 CUDA tensor [{B}, pages per sequence]")
    ptable, cols, ldt = _rows(block_table, B, "block_table", torch.int32, dev)
    if out is None:
        out = _empty((T, dq), _BF16, q.device, stream)
        po, ldo = out.data_ptr(), 0
    else:
        po, _, ldo = _rows(out, T, "out", _BF16, dev, dq)
    plse = None if lse is None else _flat(lse, (T, hq), torch.float32, "lse", dev)
    if workspace is None:
        nbytes = bytes_of(dev, B, T, max_q, max_kv, hq, heads, hd, window)
        workspace = _empty((nbytes,), torch.uint8, q.device, stream) if nbytes else None
    else:
        if not workspace.is_contiguous() or workspace.get_device() != dev:
            _refuse(binding.QKNORM_ERR_SCRATCH, f"workspace: expected a contiguous tensor on cuda:{dev}")
        nbytes = workspace.numel() * workspace.element_size()
    _invoke(cfunc,
            (pq, ldq, cache, ptable, cols, ldt, plens, pstarts, B, T, max_q, max_kv, hq, 1.0 / math.sqrt(hd) if scale is None else scale,
             1 if causal else 0, window, po, ldo, plse, workspace.data_ptr() if workspace is not None else None, nbytes),
            _current(stream), (q, *pools, block_table, kv_lens, q_starts, out, lse, workspace))
    return out
