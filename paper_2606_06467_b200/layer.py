"""Binding of the calls around a layer's cache (`include/clsa_layer.h`): the same names and argument orders, tensors in place of
pointers. Checks of dtypes, shapes, strides, sizes and devices that C cannot make happen here (an address in place of a tensor is
taken as it is); everything else is marshalling. As in cache8.py, the usual call goes through the native module `_marshal`.
"""
from __future__ import annotations

import ctypes

from . import _P, _check, _i64, _lib, _ptr, _sz, _vp, cache8, clsa_params
from .cache8 import _C, _D, _N, _dense, _describes, _device, _device_of, _fits, _heads, _stream8, _want, _workspace

CLSA_MAX_AXES = 4

_torch = None  # the torch module, from the first call on
_marshal = cache8._marshal  # the native module, or None

EXPORTS_LAYER = ("clsa_dense_workspace_bytes", "clsa_dense_attn", "clsa_dense_attn8", "clsa_add_norm", "clsa_norm_rope_axes")


class clsa_rows(ctypes.Structure):
    """Mirror of `clsa_rows` in include/clsa_layer.h."""

    _fields_ = [("data", _vp), ("stride", _i64)]


class clsa_add_norm_spec(ctypes.Structure):
    """Mirror of `clsa_add_norm_spec` in include/clsa_layer.h."""

    _device = None  # where the tensor behind it lies, if it was made of one

    _fields_ = [("dim", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", _vp), ("scale_group", ctypes.c_int32)]


class clsa_rope_axes(ctypes.Structure):
    """Mirror of `clsa_rope_axes` in include/clsa_layer.h."""

    _pairs = None  # pairs that it was made for

    _fields_ = [("num_axes", ctypes.c_int32), ("axis_of_pair", ctypes.c_uint8 * 128)]


_R = ctypes.POINTER(clsa_rows)
_lib.clsa_dense_workspace_bytes.argtypes = [_P, ctypes.POINTER(_sz)]
_lib.clsa_dense_attn.argtypes = [_P, ctypes.c_int32, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.clsa_dense_attn8.argtypes = [_P, _C, ctypes.c_int32, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.clsa_add_norm.argtypes = [ctypes.POINTER(clsa_add_norm_spec), ctypes.c_int32, _R, _R, _R, _R, _R, _R, _vp]
_lib.clsa_norm_rope_axes.argtypes = [_N, ctypes.POINTER(clsa_rope_axes), ctypes.c_int32, _vp, _i64, _D, _D, _D, _D, _vp]
for _name in EXPORTS_LAYER:
    getattr(_lib, _name).restype = ctypes.c_int


def _load_torch():
    torch = cache8._torch or cache8._load_torch()
    if _marshal is not None:
        where = [ctypes.cast(getattr(_lib, n), _vp).value for n in ("clsa_dense_attn", "clsa_dense_attn8", "clsa_add_norm", "clsa_norm_rope_axes")]
        _marshal.setup_layer(*where, torch.float8_e4m3fn, torch.float8_e8m0fnu, clsa_add_norm_spec, clsa_rope_axes)
    global _torch
    _torch = torch
    return torch


def clsa_dense_workspace_bytes(p: clsa_params) -> int:
    n = _sz(0)
    _check(_lib.clsa_dense_workspace_bytes(ctypes.byref(p), ctypes.byref(n)), "clsa_dense_workspace_bytes")
    return int(n.value)


def _holds(p, device):
    """Refuse params whose K and V, if they are tensors still, are not bf16 on the device or hold less than the params name."""
    for what, t, now in (("k_cache", p._kv[0], p.k_cache), ("v_cache", p._kv[1], p.v_cache)) if p._kv else ():
        if t is None or t[0] != now:
            continue
        _, dtype, reach, where = t
        need = (p.num_cache_rows - 1) * p.kv_token_stride + (p.num_kv_heads - 1) * p.kv_head_stride + p.head_dim
        if dtype != "torch.bfloat16" or where != device or reach < need:
            raise ValueError(f"{what}: bf16 values on the current CUDA device for {p.num_cache_rows} rows of {p.num_kv_heads} heads of {p.head_dim} at "
                             f"strides {p.kv_token_stride} and {p.kv_head_stride} are wanted")


def _dense_call(name, call, p, window, q, out, lse, workspace, workspace_bytes, stream, made):
    torch = _torch
    dev, bf16, heads = _device(torch), torch.bfloat16, p.num_seqs * p.q_per_seq * p.num_q_heads
    _describes(p, dev)
    ws, nbytes = _workspace(workspace, workspace_bytes, made, dev)
    if not -(1 << 31) <= window < 1 << 31:
        raise ValueError(f"window: a 32-bit number is wanted, got {window}")
    status = call(int(window), _dense(q, "q", bf16, dev, heads * p.head_dim), _dense(out, "out", bf16, dev, heads * p.head_dim, output=True),
                  _dense(lse, "lse", torch.float32, dev, heads, output=True), ws, nbytes, _stream8(stream, dev))
    if status:
        _check(status, name)


def clsa_dense_attn(p, window, q, out, lse, workspace, workspace_bytes=None, stream=None) -> None:
    """Attention of the T newest tokens of every sequence over all of its rows of p's bf16 caches (window 0) or the last `window` of each
    token. q, out [B, T, Hq, D] bf16, lse [B, T, Hq] fp32 or None."""
    torch = _torch or _load_torch()
    status = _marshal.dense(p, window, q, out, lse, workspace, workspace_bytes, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_dense_attn") if status else None
    _holds(p, _device(torch))
    _dense_call("clsa_dense_attn", lambda *a: _lib.clsa_dense_attn(ctypes.byref(p), *a), p, window, q, out, lse, workspace, workspace_bytes,
                stream, ())


def clsa_dense_attn8(p, c, window, q, out, lse, workspace, workspace_bytes=None, stream=None) -> None:
    """clsa_dense_attn over an 8-bit K and V cache."""
    _torch or _load_torch()
    status = _marshal.dense8(p, c, window, q, out, lse, workspace, workspace_bytes, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_dense_attn8") if status else None
    _fits(p, c, True, False)
    _dense_call("clsa_dense_attn8", lambda *a: _lib.clsa_dense_attn8(ctypes.byref(p), ctypes.byref(c), *a), p, window, q, out, lse, workspace,
                workspace_bytes, stream, (c,))


def make_add_norm(*, dim, eps=1e-6, weight=None, scale_group=0) -> clsa_add_norm_spec:
    """Fill a clsa_add_norm_spec, which keeps the tensor alive."""
    import torch

    if weight is not None and not isinstance(weight, int):
        _want(weight.dtype == torch.bfloat16 and weight.is_contiguous() and weight.numel() == dim, f"weight: {dim} contiguous values of bf16 are wanted")
    spec = clsa_add_norm_spec(dim, eps, _ptr(weight), scale_group)
    spec._tensors = (weight,)
    spec._device = _device_of(*spec._tensors)
    return spec


def _matrix(t, what, dtypes, device, rows, length):
    """The clsa_rows of a matrix [.., length] whose rows are evenly spaced, and its number of rows."""
    if t is None:
        return None, rows
    shape, stride = t.shape, t.stride()
    even = len(shape) >= 1 and shape[-1] == length and (stride[-1] == 1 or length == 1)
    n, step = 1, None
    for size, s in zip(reversed(shape[:-1]), reversed(stride[:-1])):  # from the innermost axis of rows outwards
        if size == 1:
            continue
        if step is None:
            step = s
        elif s != n * step and 0 not in shape:  # (of no rows at all nothing is spaced)
            even = False
        n *= size
    if not even or t.dtype not in dtypes or t.get_device() != device:
        raise ValueError(f"{what}: rows of {length} dense values of {'/'.join(str(d) for d in dtypes)}, evenly spaced, on the current CUDA device are wanted; "
                         f"got {t.dtype} {tuple(shape)} on {t.device}, strides {stride}")
    if rows is not None and n != rows:
        raise ValueError(f"{what}: {rows} rows are wanted, got {tuple(shape)}")
    return clsa_rows(t.data_ptr(), length if step is None else step), n


def clsa_add_norm(spec, x, residual, sum_out, y_out, codes_out=None, scales_out=None, stream=None) -> None:
    """s = x + residual and its RMS norm: x, residual, sum_out, y_out [.., dim] bf16, codes_out [.., dim] (float8_e4m3fn or uint8),
    scales_out [.., dim / scale_group] (float8_e8m0fnu or uint8). residual, sum_out, and y_out or both of the last may be None."""
    torch = _torch or _load_torch()
    status = _marshal.add_norm(spec, x, residual, sum_out, y_out, codes_out, scales_out, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_add_norm") if status else None
    dev, bf16 = _device(torch), (torch.bfloat16,)
    if spec._device not in (None, dev):
        raise ValueError("the tensors of clsa_add_norm_spec are not on the current CUDA device")
    if (codes_out is None) != (scales_out is None) or (codes_out is None and y_out is None):
        raise ValueError("y_out, codes_out with scales_out, or all three are wanted")
    if codes_out is not None and spec.scale_group < 1:
        raise ValueError("codes_out: a spec with a scale_group is wanted")
    a, n = _matrix(x, "x", bf16, dev, None, spec.dim)
    rest = [_matrix(t, what, bf16, dev, n, spec.dim)[0] for t, what in ((residual, "residual"), (sum_out, "sum_out"), (y_out, "y_out"))]
    rest.append(_matrix(codes_out, "codes_out", (torch.uint8, torch.float8_e4m3fn), dev, n, spec.dim)[0])
    rest.append(_matrix(scales_out, "scales_out", (torch.uint8, torch.float8_e8m0fnu), dev, n, spec.dim // max(spec.scale_group, 1))[0])
    status = _lib.clsa_add_norm(ctypes.byref(spec), n, ctypes.byref(a), *(None if r is None else ctypes.byref(r) for r in rest), _stream8(stream, dev))
    if status:
        _check(status, "clsa_add_norm")


def make_rope_axes(axis_of_pair, num_axes=None) -> clsa_rope_axes:
    """Fill a clsa_rope_axes from the axis of each pair."""
    axis_of_pair = [int(x) for x in axis_of_pair]
    _want(0 < len(axis_of_pair) <= 128 and min(axis_of_pair) >= 0, "axis_of_pair: 1 to 128 axes are wanted")
    num_axes = max(axis_of_pair) + 1 if num_axes is None else num_axes
    _want(max(axis_of_pair) < num_axes <= CLSA_MAX_AXES, f"num_axes: up to {CLSA_MAX_AXES}, more than the largest axis, is wanted")
    axes = clsa_rope_axes(num_axes)
    axes.axis_of_pair[:len(axis_of_pair)] = axis_of_pair
    axes._pairs = len(axis_of_pair)
    return axes


def clsa_norm_rope_axes(spec, axes, positions, q, q_out, k=None, k_out=None, stream=None) -> None:
    """clsa_norm_rope with positions [num_axes, tokens] (int32, dense rows; or [tokens], one position for every axis)."""
    torch = _torch or _load_torch()
    status = _marshal.norm_rope_axes(spec, axes, positions, q, q_out, k, k_out, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_norm_rope_axes") if status else None
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (q is None and k is None):
        raise ValueError("q with q_out, k with k_out, or both are wanted")
    dev, bf16, dim = _device(torch), torch.bfloat16, spec.head_dim
    a = b = c = d = n = None
    if q is not None:
        a, n, h = _heads(q, "q", dev, bf16, n, None, dim)
        b, _, _ = _heads(q_out, "q_out", dev, bf16, n, h, dim)
    if k is not None:
        c, n, h = _heads(k, "k", dev, bf16, n, None, dim)
        d, _, _ = _heads(k_out, "k_out", dev, bf16, n, h, dim)
    if axes._pairs is not None and axes._pairs * 2 != spec.rot_dim:
        raise ValueError(f"axes: {spec.rot_dim // 2} pairs are wanted, got {axes._pairs}")
    if positions.dtype != torch.int32 or positions.get_device() != dev or positions.shape[-1:] != (n,) or positions.dim() > 2 or (
            positions.stride(-1) != 1 and n > 1) or (positions.dim() == 2 and (positions.shape[0] != axes.num_axes or 0 < positions.stride(0) < n)):
        raise ValueError(f"positions: int32 [{axes.num_axes}, {n}] or [{n}] with dense rows on the current CUDA device is wanted; got {positions.dtype} "
                         f"{tuple(positions.shape)} on {positions.device}, strides {positions.stride()}")
    if spec._device not in (None, dev):
        raise ValueError("the tensors of clsa_norm_rope_spec are not on the current CUDA device")
    step = positions.stride(0) if positions.dim() == 2 and axes.num_axes > 1 else 0
    status = _lib.clsa_norm_rope_axes(ctypes.byref(spec), ctypes.byref(axes), n, positions.data_ptr(), step, a, b, c, d, _stream8(stream, dev))
    if status:
        _check(status, "clsa_norm_rope_axes")
