"""Binding of the 8-bit cache calls (`include/clsa_cache8.h`): the same names and argument orders, tensors in place of
pointers. Checks of dtypes, shapes, strides and devices that C cannot make happen here; everything else is marshalling.
"""
from __future__ import annotations

import ctypes

from . import (_H, _P, _check, _i64, _lib, _nbytes, _ptr, _stream, _sz, _vp, clsa_params)

CLSA_DEV_BAD_SCALE_BLOCK = 64

EXPORTS_CACHE8 = ("clsa_norm_rope", "clsa_cache8_workspace_bytes", "clsa_cache8_append", "clsa_index_scores8",
                  "clsa_sparse_attn8")


class clsa_heads(ctypes.Structure):
    """Mirror of `clsa_heads` in include/clsa_cache8.h."""

    _fields_ = [("data", _vp), ("num_heads", ctypes.c_int32), ("token_stride", _i64), ("head_stride", _i64)]


class clsa_norm_rope_spec(ctypes.Structure):
    """Mirror of `clsa_norm_rope_spec` in include/clsa_cache8.h."""

    _fields_ = [("head_dim", ctypes.c_int32), ("norm", ctypes.c_int32), ("eps", ctypes.c_float),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("rot_scale", ctypes.c_float),
                ("inv_freq", _vp), ("q_weight", _vp), ("k_weight", _vp)]


class clsa_cache8(ctypes.Structure):
    """Mirror of `clsa_cache8` in include/clsa_cache8.h."""

    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("kv_token_stride", _i64),
                ("kv_head_stride", _i64), ("scale_head_stride", _i64), ("idx_k", _vp), ("idx_k_scale", _vp),
                ("idx_token_stride", _i64), ("scale_block", ctypes.c_int32)]


_C = ctypes.POINTER(clsa_cache8)
_N = ctypes.POINTER(clsa_norm_rope_spec)
_D = ctypes.POINTER(clsa_heads)
_lib.clsa_norm_rope.argtypes = [_N, ctypes.c_int32, _vp, _D, _D, _D, _D, _vp]
_lib.clsa_cache8_workspace_bytes.argtypes = [_P, _C, ctypes.POINTER(_sz)]
_lib.clsa_cache8_append.argtypes = [_P, _C, _N, _D, _D, _D, _vp, _sz, _vp]
_lib.clsa_index_scores8.argtypes = [_P, _C, _vp, _vp, _i64, _vp, _sz, _vp]
_lib.clsa_sparse_attn8.argtypes = [_P, _C, _vp, _vp, _vp, _vp, _vp, _H, _vp, _sz, _vp]
for _name in EXPORTS_CACHE8:
    getattr(_lib, _name).restype = ctypes.c_int


def _want(ok, message):
    if not ok:
        raise ValueError(message)


def _here(t, what, dtype=None):
    """A tensor of the current CUDA device (where the call's kernels run) and of the dtype, if one is asked for. Device
    addresses pass as they are."""
    if not isinstance(t, int):
        import torch

        _want(t.is_cuda and t.get_device() == torch.cuda.current_device(), f"{what}: a tensor of the current CUDA device is wanted")
        _want(dtype is None or t.dtype == dtype, f"{what}: dtype {dtype} is wanted, got {t.dtype}")
    return t


def _dense(t, what, dtype, where=_here):
    """The same for a buffer that is addressed as one dense array (None passes)."""
    if t is None or isinstance(t, int):
        return
    if where is not None:
        where(t, what, dtype)
    _want(t.dtype == dtype and t.is_contiguous(), f"{what}: contiguous values of {dtype} are wanted")


def _bytes_like(t, what, names):
    import torch

    _want(t.dtype in (torch.uint8,) + tuple(getattr(torch, n) for n in names), f"{what}: uint8 or {'/'.join(names)} is wanted, got {t.dtype}")


def make_norm_rope(*, head_dim=128, norm=1, eps=1e-6, rot_dim=0, interleaved=0, rot_scale=1.0, inv_freq=None, q_weight=None,
                   k_weight=None) -> clsa_norm_rope_spec:
    """Fill a clsa_norm_rope_spec, which keeps the tensors alive."""
    import torch

    for t, what, dtype, n in ((inv_freq, "inv_freq", torch.float32, rot_dim // 2), (q_weight, "q_weight", torch.bfloat16, head_dim),
                              (k_weight, "k_weight", torch.bfloat16, head_dim)):
        if t is not None and not isinstance(t, int):
            _want(t.dtype == dtype and t.is_contiguous() and t.numel() == n, f"{what}: {n} contiguous values of {dtype} are wanted")
    spec = clsa_norm_rope_spec(head_dim, int(norm), eps, rot_dim, int(interleaved), rot_scale, _ptr(inv_freq), _ptr(q_weight),
                               _ptr(k_weight))
    spec._tensors = (inv_freq, q_weight, k_weight)
    return spec


def make_cache8(*, k=None, v=None, k_scale=None, v_scale=None, idx_k=None, idx_k_scale=None, scale_block=64) -> clsa_cache8:
    """Describe an 8-bit cache: k, v [rows, Hkv, D] (float8_e4m3fn or uint8, one layout), k_scale, v_scale [Hkv, blocks]
    (float8_e8m0fnu or uint8), idx_k [rows, d_idx], idx_k_scale [blocks]. The struct keeps the tensors alive."""
    c = clsa_cache8()
    c._tensors = (k, v, k_scale, v_scale, idx_k, idx_k_scale)
    c.scale_block = scale_block
    if k is not None or v is not None:
        for t, what in ((k, "k"), (v, "v")):
            _want(t is not None and t.dim() == 3 and t.stride(2) == 1, f"{what}: [rows, heads, dim] with dense rows is wanted")
            _bytes_like(t, what, ("float8_e4m3fn",))
        _want(k.shape == v.shape and k.stride() == v.stride(), "k and v: one shape and one layout are wanted")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _want(t is not None and t.dim() == 2 and t.stride(1) == 1 and t.shape[0] == k.shape[1]
                  and t.shape[1] * scale_block >= k.shape[0], f"{what}: [heads, blocks] bytes for every row is wanted")
            _bytes_like(t, what, ("float8_e8m0fnu",))
        _want(k_scale.stride(0) == v_scale.stride(0) or k.shape[1] == 1, "k_scale and v_scale: one layout is wanted")
        c.k, c.v, c.k_scale, c.v_scale = _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale)
        c.kv_token_stride, c.kv_head_stride = k.stride(0), k.stride(1)
        c.scale_head_stride = max(k_scale.stride(0), k_scale.shape[1])
    if idx_k is not None:
        _want(idx_k.dim() == 2 and idx_k.stride(1) == 1, "idx_k: [rows, d_idx] with dense rows is wanted")
        _bytes_like(idx_k, "idx_k", ("float8_e4m3fn",))
        _want(idx_k_scale is not None and idx_k_scale.dim() == 1 and idx_k_scale.is_contiguous()
              and idx_k_scale.numel() * scale_block >= idx_k.shape[0], "idx_k_scale: [blocks] bytes for every row is wanted")
        _bytes_like(idx_k_scale, "idx_k_scale", ("float8_e8m0fnu",))
        c.idx_k, c.idx_k_scale, c.idx_token_stride = _ptr(idx_k), _ptr(idx_k_scale), idx_k.stride(0)
    return c


def _heads(t, what, tokens=None, flat=None):
    """clsa_heads of a bf16 tensor [tokens, heads, D] or [B, T, heads, D] (or [.., D] with flat=1: one head)."""
    import torch

    _here(t, what, torch.bfloat16)
    if flat:
        t = t.unsqueeze(-2)
    _want(t.dim() in (3, 4) and t.stride(-1) == 1, f"{what}: [tokens, heads, dim] or [B, T, heads, dim] with dense heads is wanted")
    if t.dim() == 4:
        B, T = t.shape[0], t.shape[1]
        token = t.stride(0) if T == 1 else t.stride(1)
        _want(T == 1 or B == 1 or t.stride(0) == T * t.stride(1), f"{what}: the tokens of all sequences must be evenly spaced")
        n = B * T
    else:
        n, token = t.shape[0], t.stride(0)
    _want(tokens is None or n == tokens, f"{what}: {tokens} tokens are wanted, got {n}")
    return clsa_heads(t.data_ptr(), t.shape[-2], token, t.stride(-2) if t.shape[-2] > 1 else max(t.stride(-2), t.shape[-1])), t


def _ref(x):
    return None if x is None else ctypes.byref(x)


def clsa_norm_rope(spec, positions, q, q_out, k=None, k_out=None, stream=None) -> None:
    """Norm and rotation of the heads of q and k ([tokens, heads, D] or [B, T, heads, D], bf16, any token and head strides)
    into q_out and k_out, which may be q and k themselves. positions: int32, one per token (negative: skipped), or None."""
    import torch

    _want((q is None) == (q_out is None) and (k is None) == (k_out is None) and (q is not None or k is not None),
          "q with q_out, k with k_out, or both are wanted")
    _dense(positions, "positions", torch.int32)
    n = None if positions is None else positions.numel()
    made = []
    for t, o, what in ((q, q_out, "q"), (k, k_out, "k")):
        if t is None:
            made += [None, None]
            continue
        a, ta = _heads(t, what, n)
        n = ta.shape[0] if ta.dim() == 3 else ta.shape[0] * ta.shape[1]
        b, tb = _heads(o, what + "_out", n)
        _want(ta.shape[-2:] == tb.shape[-2:] and ta.shape[-1] == spec.head_dim, f"{what}: heads of head_dim, as many in as out, are wanted")
        made += [a, b]
    _check(_lib.clsa_norm_rope(ctypes.byref(spec), n, _ptr(positions), *map(_ref, made), _stream(stream)), "clsa_norm_rope")


def clsa_cache8_workspace_bytes(p: clsa_params, c: clsa_cache8) -> int:
    n = _sz(0)
    _check(_lib.clsa_cache8_workspace_bytes(ctypes.byref(p), ctypes.byref(c), ctypes.byref(n)), "clsa_cache8_workspace_bytes")
    return int(n.value)


def clsa_cache8_append(p, c, spec, k_new, v_new, idx_k_new, workspace, workspace_bytes=None, stream=None) -> None:
    """The newest T tokens of every sequence into the 8-bit caches: k_new, v_new [B, T, Hkv, D], idx_k_new [B, T, d_idx]
    (bf16; None leaves K and V, or K_idx, out). spec: the norm and rotation of K's rows (or None)."""
    n = p.num_seqs * p.q_per_seq
    k = v = i = None
    if k_new is not None or v_new is not None:
        _want(k_new is not None and v_new is not None, "k_new and v_new: both or neither are wanted")
        (k, tk), (v, tv) = _heads(k_new, "k_new", n), _heads(v_new, "v_new", n)
        _want(tk.shape[-2:] == tv.shape[-2:] == (p.num_kv_heads, p.head_dim), "k_new, v_new: [num_kv_heads, head_dim] per token is wanted")
    if idx_k_new is not None:
        i, ti = _heads(idx_k_new, "idx_k_new", n, flat=1)
        _want(ti.shape[-1] == p.idx_dim, "idx_k_new: idx_dim elements per token are wanted")
    _check(_lib.clsa_cache8_append(ctypes.byref(p), ctypes.byref(c), _ref(spec), _ref(k), _ref(v), _ref(i), _ptr(workspace),
                                   _nbytes(workspace, workspace_bytes), _stream(stream)), "clsa_cache8_append")


def clsa_index_scores8(p, c, q_idx, scores, score_stride, workspace, workspace_bytes=None, stream=None) -> None:
    """clsa_index_scores over an 8-bit indexer-key cache."""
    import torch

    _dense(q_idx, "q_idx", torch.bfloat16)
    _here(scores, "scores", torch.float32)
    _check(_lib.clsa_index_scores8(ctypes.byref(p), ctypes.byref(c), _ptr(q_idx), _ptr(scores), score_stride, _ptr(workspace),
                                   _nbytes(workspace, workspace_bytes), _stream(stream)), "clsa_index_scores8")


def clsa_sparse_attn8(p, c, q, idx, count, out, lse, hints, workspace, workspace_bytes=None, stream=None) -> None:
    """clsa_sparse_attn_hinted over an 8-bit K and V cache (hints: None or a clsa_attn_hints with shared_gpu 0)."""
    import torch

    _dense(q, "q", torch.bfloat16)
    _dense(idx, "idx", torch.int32)
    _dense(count, "count", torch.int32)
    _dense(out, "out", torch.bfloat16, None)  # outputs may lie in pinned host memory
    _dense(lse, "lse", torch.float32, None)
    _check(_lib.clsa_sparse_attn8(ctypes.byref(p), ctypes.byref(c), _ptr(q), _ptr(idx), _ptr(count), _ptr(out), _ptr(lse),
                                  _ref(hints), _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream)),
           "clsa_sparse_attn8")
