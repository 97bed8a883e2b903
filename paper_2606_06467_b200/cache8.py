"""Binding of the 8-bit cache calls (`include/clsa_cache8.h`): the same names and argument orders, tensors in place of
pointers. Checks of dtypes, shapes, strides, sizes and devices that C cannot make happen here (an address in place of a tensor is
taken as it is); everything else is marshalling. The
usual call goes through the native module `_marshal` (csrc/marshal.c), which makes the same checks without the interpreter and
hands back what it does not take as it is; without the module every call takes the way below.
"""
from __future__ import annotations

import ctypes
import struct

from . import _H, _P, _check, _i64, _lib, _ptr, _stream, _sz, _vp, clsa_attn_hints, clsa_params

CLSA_DEV_BAD_SCALE_BLOCK = 64

EXPORTS_CACHE8 = ("clsa_norm_rope", "clsa_cache8_workspace_bytes", "clsa_cache8_append", "clsa_index_scores8",
                  "clsa_sparse_attn8")


class clsa_heads(ctypes.Structure):
    """Mirror of `clsa_heads` in include/clsa_cache8.h."""

    _fields_ = [("data", _vp), ("num_heads", ctypes.c_int32), ("token_stride", _i64), ("head_stride", _i64)]


class clsa_norm_rope_spec(ctypes.Structure):
    """Mirror of `clsa_norm_rope_spec` in include/clsa_cache8.h."""

    _device = None  # where the tensors behind it lie, if it was made of tensors

    _fields_ = [("head_dim", ctypes.c_int32), ("norm", ctypes.c_int32), ("eps", ctypes.c_float),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("rot_scale", ctypes.c_float),
                ("inv_freq", _vp), ("q_weight", _vp), ("k_weight", _vp)]


class clsa_cache8(ctypes.Structure):
    """Mirror of `clsa_cache8` in include/clsa_cache8.h."""

    _device = None  # where the tensors behind it lie, if it was made of tensors
    _extent = None  # and what they hold: rows, heads and dimension of K and V, rows and dimension of K_idx (0: there are none), and
    # the addresses of K and K_idx that this is true of

    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("kv_token_stride", _i64),
                ("kv_head_stride", _i64), ("scale_head_stride", _i64), ("idx_k", _vp), ("idx_k_scale", _vp),
                ("idx_token_stride", _i64), ("scale_block", ctypes.c_int32)]


_C = ctypes.POINTER(clsa_cache8)
_N = ctypes.POINTER(clsa_norm_rope_spec)
_D = _vp  # clsa_heads by its bytes (or a reference)
_lib.clsa_norm_rope.argtypes = [_N, ctypes.c_int32, _vp, _D, _D, _D, _D, _vp]
_lib.clsa_cache8_workspace_bytes.argtypes = [_P, _C, ctypes.POINTER(_sz)]
_lib.clsa_cache8_append.argtypes = [_P, _C, _N, _D, _D, _D, _vp, _sz, _vp]
_lib.clsa_index_scores8.argtypes = [_P, _C, _vp, _vp, _i64, _vp, _sz, _vp]
_lib.clsa_sparse_attn8.argtypes = [_P, _C, _vp, _vp, _vp, _vp, _vp, _H, _vp, _sz, _vp]
for _name in EXPORTS_CACHE8:
    getattr(_lib, _name).restype = ctypes.c_int


_pack_heads = struct.Struct("@Piqq").pack  # clsa_heads


def _want(ok, message):
    if not ok:
        raise ValueError(message)


def _dense(t, what, dtype, device, need, rows=False, output=False):
    """Address of a buffer on the current device that is addressed as one dense array of `need` or more values of `dtype` (None and
    device addresses pass). rows: its rows alone are dense. output: it may also lie in pinned host memory."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype != dtype or not (t.is_contiguous() or (rows and t.stride(-1) == 1)) or (
            t.get_device() != device and not (output and t.get_device() < 0 and t.is_pinned())):
        raise ValueError(f"{what}: contiguous values of {dtype} on the current CUDA device are wanted, got {t.dtype} on {t.device}, "
                         f"strides {t.stride()}")
    has = 1 + sum((n - 1) * step for n, step in zip(t.shape, t.stride())) if t.numel() else 0
    if has < need:
        raise ValueError(f"{what}: {need} values are wanted, got {has} (shape {tuple(t.shape)})")
    return t.data_ptr()


def _fits(p, c, kv, idx):
    """Refuse params that name more of a cache than its tensors hold."""
    if c._extent is None:
        return
    rows, heads, dim, idx_rows, idx_dim, k, idx_k = c._extent
    if kv and heads and c.k == k and (p.num_cache_rows > rows or p.num_kv_heads > heads or p.head_dim > dim):
        raise ValueError(f"the params name {p.num_cache_rows} rows of {p.num_kv_heads} heads of {p.head_dim}, K and V hold {rows} of {heads} of {dim}")
    if idx and idx_dim and c.idx_k == idx_k and (p.num_cache_rows > idx_rows or p.idx_dim > idx_dim):
        raise ValueError(f"the params name {p.num_cache_rows} rows of {p.idx_dim}, K_idx holds {idx_rows} of {idx_dim}")


def _describes(p, device):
    """Refuse params made of tensors that describe fewer sequences than they name or lie elsewhere (what has been given another address
    since is not looked at)."""
    if p._made is None:
        return
    for what, made, now in zip(("seq_start", "seq_len", "block_table"), p._made, (p.seq_start, p.seq_len, p.block_table)):
        if made is None or made[0] != now or what == "seq_start" and p.block_table:
            continue
        if made[1] < p.num_seqs or made[2] not in (None, device):
            kind = {"seq_start": "int64", "seq_len": "int32"}.get(what, f"int32 [.., {p.max_blocks_per_seq}]")
            raise ValueError(f"{what}: contiguous {kind} values for {p.num_seqs} sequences on the current CUDA device are wanted")


def _workspace(ws, ws_bytes, made, device):
    """Address and size of a workspace, behind a check that it and what the structs in `made` point to are on the device."""
    for s in made:
        if s is not None and s._device not in (None, device):
            raise ValueError(f"the tensors of {type(s).__name__} are not on the current CUDA device")
    if ws is None or isinstance(ws, int):
        return ws, ws_bytes
    if ws.get_device() != device:
        raise ValueError(f"workspace: a tensor on the current CUDA device is wanted, got {ws.device}")
    has = ws.numel() * ws.element_size()
    if ws_bytes is not None and ws_bytes > has:
        raise ValueError(f"workspace: a tensor of {ws_bytes} bytes is wanted, got {has}")
    return ws.data_ptr(), has if ws_bytes is None else ws_bytes


def _device_of(*tensors):
    """The one device of the tensors (-1: host memory), None if there are none (addresses do not count)."""
    found = {t.get_device() for t in tensors if t is not None and not isinstance(t, int)}
    _want(len(found) <= 1, "tensors on one device are wanted")
    return found.pop() if found else None


_torch = None  # the torch module, from the first call on (importing this package does not import it)
try:
    from . import _marshal
except ImportError:
    _marshal = None


def _load_torch():
    global _torch
    import torch

    if _marshal is not None:
        where = [ctypes.cast(getattr(_lib, n), _vp).value for n in ("clsa_norm_rope", "clsa_cache8_append", "clsa_index_scores8", "clsa_sparse_attn8")]
        _marshal.setup(*where, torch.Tensor, torch.bfloat16, torch.int32, torch.float32, torch.uint8, torch._C._cuda_getDevice,
                       torch._C._cuda_getCurrentRawStream, clsa_params, clsa_cache8, clsa_norm_rope_spec, clsa_attn_hints)
    _torch = torch
    return torch


def _device(torch):
    """The current CUDA device's number, where the calls' kernels run; None before anything is on a GPU."""
    return torch._C._cuda_getDevice() if torch.cuda.is_initialized() else None


def _stream8(stream, device):
    """The stream to launch on: the current one's handle without the object around it, or the caller's."""
    if stream is None and device is not None:
        return _torch._C._cuda_getCurrentRawStream(device)
    return _stream(stream)


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
    spec._device = _device_of(*spec._tensors)
    return spec


def make_cache8(*, k=None, v=None, k_scale=None, v_scale=None, idx_k=None, idx_k_scale=None, scale_block=64) -> clsa_cache8:
    """Describe an 8-bit cache: k, v [rows, Hkv, D] (float8_e4m3fn or uint8, one layout), k_scale, v_scale [Hkv, blocks]
    (float8_e8m0fnu or uint8), idx_k [rows, d_idx], idx_k_scale [blocks]. The struct keeps the tensors alive."""
    c = clsa_cache8()
    c._tensors = (k, v, k_scale, v_scale, idx_k, idx_k_scale)
    c._device = _device_of(*c._tensors)
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
        one = k.shape[1] == 1  # nothing lies between heads then
        _want(one or k_scale.stride(0) == v_scale.stride(0), "k_scale and v_scale: one layout is wanted")
        _want(one or min(k_scale.stride(0), v_scale.stride(0)) >= max(k_scale.shape[1], v_scale.shape[1]), "k_scale and v_scale: every head's own bytes are wanted")
        c.k, c.v, c.k_scale, c.v_scale = _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale)
        c.kv_token_stride, c.kv_head_stride = k.stride(0), k.stride(1)
        c.scale_head_stride = k_scale.shape[1] if one else k_scale.stride(0)
    if idx_k is not None:
        _want(idx_k.dim() == 2 and idx_k.stride(1) == 1, "idx_k: [rows, d_idx] with dense rows is wanted")
        _bytes_like(idx_k, "idx_k", ("float8_e4m3fn",))
        _want(idx_k_scale is not None and idx_k_scale.dim() == 1 and idx_k_scale.is_contiguous()
              and idx_k_scale.numel() * scale_block >= idx_k.shape[0], "idx_k_scale: [blocks] bytes for every row is wanted")
        _bytes_like(idx_k_scale, "idx_k_scale", ("float8_e8m0fnu",))
        c.idx_k, c.idx_k_scale, c.idx_token_stride = _ptr(idx_k), _ptr(idx_k_scale), idx_k.stride(0)
    c._extent = (*((0, 0, 0) if k is None else k.shape), *((0, 0) if idx_k is None else idx_k.shape), c.k or 0, c.idx_k or 0)
    return c


def _heads(t, what, device, bf16, tokens, heads, dim, flat=False):
    """The clsa_heads bytes of a bf16 tensor [tokens, heads, dim] or [B, T, heads, dim] ([.., dim] with flat: one head), its
    number of tokens and of heads. tokens, heads: what they have to be, or None."""
    shape, stride = t.shape, t.stride()
    if flat:
        shape, stride = (*shape[:-1], 1, shape[-1]), (*stride[:-1], dim, stride[-1])
    try:
        if len(shape) == 3:
            n, h, d = shape
            token, head, one = stride
            even = True
        else:
            B, T, h, d = shape
            token, s1, head, one = stride
            n = B * T
            even = T == 1 or B == 1 or n == 0 or token == T * s1
            if T > 1:
                token = s1
    except ValueError:
        even = False
    if not even or d != dim or one != 1 or t.dtype is not bf16 or t.get_device() != device:
        raise ValueError(f"{what}: a bf16 tensor [tokens, heads, {dim}] or [B, T, heads, {dim}] on the current CUDA device, with dense heads and "
                         f"evenly spaced tokens, is wanted; got {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")
    if tokens != n and tokens is not None or heads != h and heads is not None:
        raise ValueError(f"{what}: {tokens} tokens of {heads} heads are wanted, got {tuple(t.shape)}")
    return _pack_heads(t.data_ptr(), h, token, head if h > 1 else dim), n, h


def clsa_norm_rope(spec, positions, q, q_out, k=None, k_out=None, stream=None) -> None:
    """Norm and rotation of the heads of q and k ([tokens, heads, D] or [B, T, heads, D], bf16, any token and head strides)
    into q_out and k_out, which may be q and k themselves. positions: int32, one per token (negative: skipped), or None."""
    torch = _torch or _load_torch()
    status = _marshal.norm_rope(spec, positions, q, q_out, k, k_out, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_norm_rope") if status else None
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (q is None and k is None):
        raise ValueError("q with q_out, k with k_out, or both are wanted")
    dev, bf16, dim = _device(torch), torch.bfloat16, spec.head_dim
    n = None if positions is None else positions.numel()
    a = b = c = d = None
    if q is not None:
        a, n, h = _heads(q, "q", dev, bf16, n, None, dim)
        b, _, _ = _heads(q_out, "q_out", dev, bf16, n, h, dim)
    if k is not None:
        c, n, h = _heads(k, "k", dev, bf16, n, None, dim)
        d, _, _ = _heads(k_out, "k_out", dev, bf16, n, h, dim)
    if spec._device not in (None, dev):
        raise ValueError("the tensors of clsa_norm_rope_spec are not on the current CUDA device")
    status = _lib.clsa_norm_rope(ctypes.byref(spec), n, _dense(positions, "positions", torch.int32, dev, n), a, b, c, d, _stream8(stream, dev))
    if status:
        _check(status, "clsa_norm_rope")


def clsa_cache8_workspace_bytes(p: clsa_params, c: clsa_cache8) -> int:
    n = _sz(0)
    _check(_lib.clsa_cache8_workspace_bytes(ctypes.byref(p), ctypes.byref(c), ctypes.byref(n)), "clsa_cache8_workspace_bytes")
    return int(n.value)


def clsa_cache8_append(p, c, spec, k_new, v_new, idx_k_new, workspace, workspace_bytes=None, stream=None) -> None:
    """The newest T tokens of every sequence into the 8-bit caches: k_new, v_new [B, T, Hkv, D], idx_k_new [B, T, d_idx]
    (bf16; None leaves K and V, or K_idx, out). spec: the norm and rotation of K's rows (or None)."""
    torch = _torch or _load_torch()
    status = _marshal.append(p, c, spec, k_new, v_new, idx_k_new, workspace, workspace_bytes, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_cache8_append") if status else None
    if (k_new is None) != (v_new is None) or (k_new is None and idx_k_new is None):
        raise ValueError("k_new with v_new, idx_k_new, or all three are wanted")
    dev, bf16, n = _device(torch), torch.bfloat16, p.num_seqs * p.q_per_seq
    k = v = i = None
    _describes(p, dev)
    _fits(p, c, k_new is not None, idx_k_new is not None)
    if k_new is not None:
        k, _, _ = _heads(k_new, "k_new", dev, bf16, n, p.num_kv_heads, p.head_dim)
        v, _, _ = _heads(v_new, "v_new", dev, bf16, n, p.num_kv_heads, p.head_dim)
    if idx_k_new is not None:
        i, _, _ = _heads(idx_k_new, "idx_k_new", dev, bf16, n, 1, p.idx_dim, True)
    ws, nbytes = _workspace(workspace, workspace_bytes, (c, spec), dev)
    status = _lib.clsa_cache8_append(ctypes.byref(p), ctypes.byref(c), None if spec is None else ctypes.byref(spec), k, v, i, ws, nbytes,
                                     _stream8(stream, dev))
    if status:
        _check(status, "clsa_cache8_append")


def clsa_index_scores8(p, c, q_idx, scores, score_stride, workspace, workspace_bytes=None, stream=None) -> None:
    """clsa_index_scores over an 8-bit indexer-key cache."""
    torch = _torch or _load_torch()
    status = _marshal.scores(p, c, q_idx, scores, score_stride, workspace, workspace_bytes, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_index_scores8") if status else None
    dev, n = _device(torch), p.num_seqs * p.q_per_seq
    _describes(p, dev)
    _fits(p, c, False, True)
    ws, nbytes = _workspace(workspace, workspace_bytes, (c,), dev)
    status = _lib.clsa_index_scores8(ctypes.byref(p), ctypes.byref(c), _dense(q_idx, "q_idx", torch.bfloat16, dev, n * p.idx_dim),
                                     _dense(scores, "scores", torch.float32, dev, (n - 1) * score_stride + p.max_seq_len, rows=True), score_stride,
                                     ws, nbytes, _stream8(stream, dev))
    if status:
        _check(status, "clsa_index_scores8")


def clsa_sparse_attn8(p, c, q, idx, count, out, lse, hints, workspace, workspace_bytes=None, stream=None) -> None:
    """clsa_sparse_attn_hinted over an 8-bit K and V cache (hints: None or a clsa_attn_hints with shared_gpu 0)."""
    torch = _torch or _load_torch()
    status = _marshal.attn(p, c, q, idx, count, out, lse, hints, workspace, workspace_bytes, stream) if _marshal else None
    if status is not None:
        return _check(status, "clsa_sparse_attn8") if status else None
    dev, i32, bf16, n = _device(torch), torch.int32, torch.bfloat16, p.num_seqs * p.q_per_seq
    heads = n * p.num_q_heads
    _describes(p, dev)
    _fits(p, c, True, False)
    ws, nbytes = _workspace(workspace, workspace_bytes, (c,), dev)
    status = _lib.clsa_sparse_attn8(ctypes.byref(p), ctypes.byref(c), _dense(q, "q", bf16, dev, heads * p.head_dim),
                                    _dense(idx, "idx", i32, dev, n * p.top_k), _dense(count, "count", i32, dev, n),
                                    _dense(out, "out", bf16, dev, heads * p.head_dim, output=True), _dense(lse, "lse", torch.float32, dev, heads, output=True),
                                    None if hints is None else ctypes.byref(hints), ws, nbytes, _stream8(stream, dev))
    if status:
        _check(status, "clsa_sparse_attn8")
