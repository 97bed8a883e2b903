"""Host-side checks of the calls around a layer's cache that need no GPU: symbols, struct layouts, what the C side refuses, what the binding
refuses in both of its marshallings (with stand-ins for tensors and for the library's entry points)."""
import ctypes
import os
import re
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
from test_cache8_edges_host import BF16, F32, I32, U8, Tensor

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "clsa_layer.h")
BAD, UNS, WS = 1, 2, 3


@pytest.fixture(scope="module")
def clsa():
    sys.path.insert(0, ROOT)
    import __graft_entry__ as entry

    entry._load_build_module().build()
    import paper_2606_06467_b200 as mod

    return mod


def test_symbols(clsa):
    names = set(re.findall(r"CLSA_API\s+[\w\s\*]+?\b(clsa_\w+)\s*\(", open(HEADER).read()))
    assert names == set(clsa.EXPORTS_LAYER)
    for n in names:
        assert hasattr(ctypes.CDLL(clsa.LIB_PATH), n), n


@pytest.mark.parametrize("name", ["clsa_rows", "clsa_add_norm_spec", "clsa_rope_axes"])
def test_struct_layouts_match_the_header(clsa, tmp_path, name):
    cls = getattr(clsa, name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "clsa_layer.h"\nint main(void){printf("%zu", sizeof(' + name + "));\n"
                   + "".join(f'printf(" %zu", offsetof({name}, {f}));\n' for f, _ in cls._fields_) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    nums = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert nums == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]


def _params(clsa, **kw):
    base = dict(num_seqs=2, num_q_heads=32, num_kv_heads=8, head_dim=128, idx_dim=128, top_k=64, max_seq_len=1024, sm_scale=0.088,
                seq_start=0x1000, seq_len=0x2000, num_cache_rows=2048, k_cache=0x10000, v_cache=0x20000)
    base.update(kw)
    return clsa.make_params(**base)


def _cache(clsa, **kw):
    c = clsa.clsa_cache8(0x10000, 0x20000, 0x30000, 0x40000, 1024, 128, 64, 0x50000, 0x60000, 128, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


_PARAMS = [
    (dict(num_seqs=0), BAD), (dict(q_per_seq=0), BAD), (dict(num_q_heads=30), BAD), (dict(causal=2), BAD), (dict(sm_scale=0.0), BAD),
    (dict(sm_scale=-1.0), BAD), (dict(sm_scale=float("nan")), BAD), (dict(max_seq_len=0), BAD), (dict(q_per_seq=8, max_seq_len=7, causal=1), BAD),
    (dict(max_seq_len=0x7fffffff), UNS), (dict(num_seqs=1 << 26, max_seq_len=1024), UNS), (dict(num_cache_rows=0), BAD), (dict(num_cache_rows=1 << 31), BAD),
    (dict(head_dim=64), UNS), (dict(head_dim=256), UNS), (dict(q_per_seq=33), UNS), (dict(num_q_heads=34, num_kv_heads=2), UNS),
    (dict(num_q_heads=2048, num_kv_heads=2048), BAD),
]
_ROWS = [
    (dict(seq_len=None), BAD), (dict(seq_start=None), BAD), (dict(seq_len=0x2002), BAD), (dict(seq_start=0x1004), BAD),
    (dict(block_table=0x3000, block_size=24, max_blocks_per_seq=64), BAD), (dict(block_table=0x3000, block_size=8, max_blocks_per_seq=128), BAD),
    (dict(block_table=0x3002, block_size=64, max_blocks_per_seq=16), BAD), (dict(block_table=0x3000, block_size=64, max_blocks_per_seq=8), BAD),
]


@pytest.mark.parametrize("kw,want", _PARAMS + _ROWS, ids=[str(k) for k, _ in _PARAMS + _ROWS])
def test_bad_params_are_refused(clsa, kw, want):
    P, raw = ctypes.byref, clsa.raw()
    p, c = _params(clsa, **kw), _cache(clsa)
    assert raw.clsa_dense_attn(P(p), 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == want
    assert raw.clsa_dense_attn8(P(p), P(c), 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == want
    n = ctypes.c_size_t(0)
    if (kw, want) in _PARAMS and not kw.get("causal"):
        assert raw.clsa_dense_workspace_bytes(P(p), P(n)) == want


def test_windows_want_their_queries_in_the_cache(clsa):
    P, raw = ctypes.byref, clsa.raw()
    p = _params(clsa, q_per_seq=8, max_seq_len=7)
    assert raw.clsa_dense_attn(P(p), 16, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == BAD
    assert raw.clsa_dense_attn(P(_params(clsa)), -1, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == BAD


def test_bad_caches_and_buffers_are_refused(clsa):
    P, raw = ctypes.byref, clsa.raw()
    p, c = _params(clsa), _cache(clsa)
    for kw, want in ((dict(k_cache=None), BAD), (dict(v_cache=None), BAD), (dict(k_cache=0x10008), BAD), (dict(v_cache=0x20002), BAD),
                     (dict(kv_token_stride=64), BAD), (dict(kv_token_stride=1028), BAD), (dict(kv_head_stride=64), BAD),
                     (dict(kv_head_stride=132), BAD), (dict(kv_token_stride=1 << 38), UNS)):
        q = _params(clsa, **kw)
        assert raw.clsa_dense_attn(P(q), 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == want, kw
    for kw, want in ((dict(scale_block=48), BAD), (dict(k=None), BAD), (dict(v=0x20008), BAD), (dict(k_scale=None), BAD), (dict(kv_token_stride=1032), BAD),
                     (dict(kv_head_stride=64), BAD), (dict(scale_head_stride=31), BAD), (dict(kv_token_stride=1 << 26), UNS)):
        assert raw.clsa_dense_attn8(P(p), P(_cache(clsa, **kw)), 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == want, kw
    assert raw.clsa_dense_attn8(P(p), None, 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == BAD
    assert raw.clsa_dense_attn(None, 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == BAD
    small = _params(clsa, block_table=0x3000, block_size=32, max_blocks_per_seq=64)
    assert raw.clsa_dense_attn8(P(small), P(c), 0, 0x50000, 0x80000, None, 0x100000, 1 << 30, None) == BAD  # a page smaller than a scale block
    for args in ((None, 0x80000, None), (0x50008, 0x80000, None), (0x50000, None, None), (0x50000, 0x80004, None), (0x50000, 0x80000, 0x90002)):
        assert raw.clsa_dense_attn(P(p), 0, *args, 0x100000, 1 << 30, None) == BAD, args
        assert raw.clsa_dense_attn8(P(p), P(c), 0, *args, 0x100000, 1 << 30, None) == BAD, args
    for ws in (None, 0x100010):
        assert raw.clsa_dense_attn(P(p), 0, 0x50000, 0x80000, None, ws, 1 << 30, None) == WS
    assert raw.clsa_dense_workspace_bytes(P(p), None) == BAD


def _rows(clsa, data=0x100000, stride=2560):
    return clsa.clsa_rows(data, stride)


def test_bad_add_norm_calls_are_refused(clsa):
    P, raw = ctypes.byref, clsa.raw()
    spec = clsa.clsa_add_norm_spec(2560, 1e-6, 0x7000, 32)
    x, r, s, y = (_rows(clsa, 0x100000 * k) for k in (1, 2, 3, 4))
    c, e = _rows(clsa, 0x500000), _rows(clsa, 0x600001, 80)
    call = lambda n=4, sp=spec, x=x, r=r, s=s, y=y, c=c, e=e: raw.clsa_add_norm(  # noqa: E731
        P(sp) if sp else None, n, *(P(t) if t else None for t in (x, r, s, y, c, e)), None)
    assert call(n=0) == clsa.CLSA_OK and call(n=0, x=_rows(clsa, None, 0)) == clsa.CLSA_OK  # no rows: nothing to do, no addresses
    assert call(n=-1) == BAD and call(n=(1 << 30) + 1) == BAD and call(sp=None) == BAD and call(x=None) == BAD
    for kw, want in ((dict(dim=0), BAD), (dict(dim=2568), UNS), (dict(dim=16400), UNS), (dict(eps=-1.0), BAD), (dict(eps=float("inf")), BAD),
                     (dict(weight=0x7008), BAD), (dict(scale_group=-32), BAD), (dict(scale_group=48), UNS), (dict(scale_group=16), UNS), (dict(scale_group=0), BAD)):
        t = clsa.clsa_add_norm_spec(2560, 1e-6, 0x7000, 32)
        for k, v in kw.items():
            setattr(t, k, v)
        assert call(sp=t) == want, kw
    assert call(sp=clsa.clsa_add_norm_spec(2576, 1e-6, None, 32)) == BAD  # groups that do not divide the row
    assert call(c=None) == BAD and call(e=None) == BAD and call(y=None, c=None, e=None) == BAD
    for name in ("x", "r", "s", "y", "c"):
        for bad in (_rows(clsa, None), _rows(clsa, 0x900008), _rows(clsa, 0x900000, 2564), _rows(clsa, 0x900000, 1280), _rows(clsa, 0x900000, -2560)):
            assert call(**{name: bad}) == BAD, name
    for name in ("s", "y", "c"):
        assert call(**{name: _rows(clsa, 0x900000, 0)}) == BAD  # rows on one another
    assert call(e=_rows(clsa, 0x600000, 79)) == BAD and call(e=_rows(clsa, None, 80)) == BAD
    assert call(s=y) == BAD  # two outputs in one place
    assert call(s=_rows(clsa, 0x100000, 5120)) == BAD and call(y=_rows(clsa, 0x200000, 5120)) == BAD  # in place with another stride


def test_bad_axes_are_refused(clsa):
    P, raw = ctypes.byref, clsa.raw()
    spec = clsa.clsa_norm_rope_spec(128, 1, 1e-6, 128, 0, 1.0, 0x7000, 0x8000, 0x9000)
    h = clsa.clsa_heads(0x100000, 8, 1024, 128)
    good = clsa.make_rope_axes([i % 3 for i in range(64)])
    call = lambda sp=spec, ax=good, n=4, pos=0x1000, step=4, a=h, b=h: raw.clsa_norm_rope_axes(  # noqa: E731
        P(sp), P(ax) if ax else None, n, pos, step, P(a), P(b), None, None, None)
    assert call(n=0, pos=None) == clsa.CLSA_OK
    assert call(ax=None) == BAD and call(pos=None) == BAD and call(pos=0x1002) == BAD and call(step=3) == BAD and call(step=-4) == BAD and call(n=-1) == BAD
    for axes, n in (([0] * 64, 0), ([0] * 64, 5), ([0] * 63 + [3], 3)):
        t = clsa.clsa_rope_axes(n)
        t.axis_of_pair[:64] = axes
        assert call(ax=t) == BAD
    t = clsa.clsa_norm_rope_spec(128, 1, 1e-6, 0, 0, 1.0, None, 0x8000, 0x9000)
    assert call(sp=t) == BAD  # nothing to turn
    t = clsa.clsa_norm_rope_spec(128, 1, 1e-6, 24, 0, 1.0, 0x7000, 0x8000, 0x9000)
    assert call(sp=t) == UNS
    assert call(b=clsa.clsa_heads(0x200000, 4, 1024, 128)) == BAD
    for bad in ([], [0] * 129, [0, -1], [4]):
        with pytest.raises(ValueError):
            clsa.make_rope_axes(bad)
    with pytest.raises(ValueError):
        clsa.make_rope_axes([0, 2], num_axes=2)


@pytest.fixture(params=["native", "python"])
def binding(clsa, request, monkeypatch):
    """The package with entry points that record their calls in place of the library's, and Tensor in place of torch's."""
    from paper_2606_06467_b200 import cache8, layer

    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    layer._load_torch()
    monkeypatch.setattr(layer, "_lib", Lib())
    monkeypatch.setattr(layer, "_device", lambda torch: 0)
    monkeypatch.setattr(layer, "_stream8", lambda stream, device: 0)
    if request.param == "python":
        monkeypatch.setattr(layer, "_marshal", None)
        yield clsa, calls
        return
    if layer._marshal is None:
        pytest.skip("built without Python.h")
    kinds = {"clsa_dense_attn": 8, "clsa_dense_attn8": 9, "clsa_add_norm": 9, "clsa_norm_rope_axes": 10}  # (any number of integers will do)
    keep = [ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p] * n)(lambda *a, name=name: calls.append("native " + name) or 0) for name, n in kinds.items()]
    addresses = [ctypes.cast(f, ctypes.c_void_p).value for f in keep]
    layer._marshal.setup(*addresses, Tensor, BF16, I32, F32, U8, lambda: 0, lambda d: 0, clsa.clsa_params, clsa.clsa_cache8, clsa.clsa_norm_rope_spec,
                         clsa.clsa_attn_hints)
    layer._marshal.setup_layer(*addresses, torch.float8_e4m3fn, torch.float8_e8m0fnu, clsa.clsa_add_norm_spec, clsa.clsa_rope_axes)
    yield clsa, calls
    monkeypatch.undo()
    cache8._load_torch()
    layer._load_torch()


def _taken(calls, name):
    got = list(calls)
    calls.clear()
    return got in ([name], ["native " + name])


def test_the_binding_compares_dense_calls_with_the_params(binding):
    clsa, calls = binding
    p = _params(clsa, q_per_seq=3)
    p._kv = ((0x10000, "torch.bfloat16", 2048 * 1024, 0), (0x20000, "torch.bfloat16", 2048 * 1024, 0))
    q, out, lse, ws = Tensor((2, 3, 32, 128), BF16), Tensor((2, 3, 32, 128), BF16), Tensor((2, 3, 32), F32), Tensor((1 << 20,), U8)
    cache = clsa.make_cache8(k=torch.zeros(2048, 8, 128, dtype=U8), v=torch.zeros(2048, 8, 128, dtype=U8), k_scale=torch.zeros(8, 32, dtype=U8),
                             v_scale=torch.zeros(8, 32, dtype=U8), scale_block=64)
    cache._device = 0
    for call, name in ((lambda *a, **k: clsa.clsa_dense_attn(p, *a, **k), "clsa_dense_attn"), (lambda *a, **k: clsa.clsa_dense_attn8(p, cache, *a, **k), "clsa_dense_attn8")):
        call(0, q, out, lse, ws)
        assert _taken(calls, name)
        call(512, q, out, None, ws, 1 << 20)
        assert _taken(calls, name)
        for bad in ((0, Tensor((2, 3, 32, 128), F32), out, lse, ws), (0, Tensor((2, 2, 32, 128), BF16), out, lse, ws), (0, q, Tensor((2, 3, 32, 64), BF16), lse, ws),
                    (0, q, out, Tensor((2, 3, 31), F32), ws), (0, q, out, Tensor((2, 3, 32), I32), ws), (0, Tensor((2, 3, 32, 128), BF16, device=1), out, lse, ws),
                    (0, q, out, lse, Tensor((1 << 20,), U8, device=1)), (0, Tensor((2, 3, 32, 128), BF16, (24576, 8192, 256, 1)), out, lse, ws),
                    (0, q, out, lse, ws, 1 << 21)):
            with pytest.raises(ValueError):
                call(*bad)
            assert not calls, bad
    for kv in ((0x10000, "torch.bfloat16", 2048 * 1024 - 1, 0), (0x10000, "torch.float16", 2048 * 1024, 0), (0x10000, "torch.bfloat16", 2048 * 1024, 1)):
        p._kv = (kv, None)
        with pytest.raises(ValueError):
            clsa.clsa_dense_attn(p, 0, q, out, lse, ws)
        assert not calls
    p.k_cache = 0x30000  # given another address since: not looked at
    clsa.clsa_dense_attn(p, 0, q, out, lse, ws)
    assert _taken(calls, "clsa_dense_attn")
    cache._extent = (1024, *cache._extent[1:])
    with pytest.raises(ValueError):
        clsa.clsa_dense_attn8(p, cache, 0, q, out, lse, ws)
    p._made = (None, (p.seq_len, 1, 0), None)  # lengths of one sequence
    with pytest.raises(ValueError):
        clsa.clsa_dense_attn(p, 0, q, out, lse, ws)


def test_the_binding_refuses_windows_beyond_32_bits(binding):
    clsa, calls = binding
    p = _params(clsa)
    p._kv = None
    q, out, ws = Tensor((2, 1, 32, 128), BF16), Tensor((2, 1, 32, 128), BF16), Tensor((1 << 20,), U8)
    clsa.clsa_dense_attn(p, 0x7fffffff, q, out, None, ws)
    assert _taken(calls, "clsa_dense_attn")
    for window in (1 << 31, (1 << 32) + 5, -(1 << 32) + 5, -(1 << 31) - 1):  # as 32 bits some of these would be other windows
        with pytest.raises(ValueError):
            clsa.clsa_dense_attn(p, window, q, out, None, ws)
        assert not calls, window


def test_the_binding_takes_rows_of_any_even_spacing(binding):
    clsa, calls = binding
    spec = clsa.make_add_norm(dim=256, scale_group=32)
    x, r = Tensor((10, 256), BF16), Tensor((10, 256), BF16, (320, 1))
    c, e = Tensor((10, 256), U8), Tensor((10, 8), U8, (9, 1))
    for args in ((x, r, x, Tensor((10, 256), BF16), None, None), (x, None, None, x, c, e), (Tensor((2, 5, 256), BF16, (1600, 320, 1)), r, None, None, c, e),
                 (x, Tensor((10, 256), BF16, (0, 1)), None, None, Tensor((10, 256), torch.float8_e4m3fn), Tensor((10, 8), torch.float8_e8m0fnu)),
                 (Tensor((0, 256), BF16), None, None, Tensor((0, 256), BF16), None, None), (Tensor((1, 10, 256), BF16), r, None, None, c, e)):
        clsa.clsa_add_norm(spec, *args)
        assert _taken(calls, "clsa_add_norm"), args
    for args in ((x, r, x, None, None, None), (x, r, None, None, c, None), (x, Tensor((9, 256), BF16), None, x, None, None), (x, r, None, x, c, Tensor((10, 7), U8)),
                 (Tensor((10, 256), F32), r, None, x, None, None), (x, Tensor((10, 256), BF16, (256, 2)), None, x, None, None), (x, r, None, None, Tensor((10, 256), BF16), e),
                 (Tensor((2, 5, 256), BF16, (1500, 320, 1)), r, None, x, None, None), (x, r, None, Tensor((10, 256), BF16, device=1), None, None),
                 (x, r, Tensor((10, 128), BF16), x, None, None)):
        with pytest.raises(ValueError):
            clsa.clsa_add_norm(spec, *args)
        assert not calls, args
    with pytest.raises(ValueError):  # codes without a group
        clsa.clsa_add_norm(clsa.make_add_norm(dim=256), x, r, None, None, c, e)
    far = clsa.make_add_norm(dim=256)
    far._device = 1
    with pytest.raises(ValueError):
        clsa.clsa_add_norm(far, x, r, None, x)


def test_the_binding_takes_positions_per_axis_or_shared(binding):
    clsa, calls = binding
    spec = clsa.make_norm_rope(head_dim=128, rot_dim=128)
    ax = clsa.make_rope_axes([i % 3 for i in range(64)])
    q, k = Tensor((7, 8, 128), BF16), Tensor((7, 2, 128), BF16)
    for pos in (Tensor((3, 7), I32), Tensor((3, 7), I32, (100, 1)), Tensor((3, 7), I32, (0, 1)), Tensor((7,), I32)):
        clsa.clsa_norm_rope_axes(spec, ax, pos, q, q, k, k)
        assert _taken(calls, "clsa_norm_rope_axes")
    for pos in (Tensor((2, 7), I32), Tensor((3, 8), I32), Tensor((3, 7), F32), Tensor((3, 7), I32, (1, 3)), Tensor((3, 7), I32, (5, 1)), Tensor((3, 7), I32, device=1)):
        with pytest.raises(ValueError):
            clsa.clsa_norm_rope_axes(spec, ax, pos, q, q, k, k)
        assert not calls, pos
    for args in ((None, None, None, None), (q, None, k, k), (q, q, k, q), (q, q, Tensor((6, 2, 128), BF16), k)):
        with pytest.raises(ValueError):
            clsa.clsa_norm_rope_axes(spec, ax, Tensor((3, 7), I32), *args)
        assert not calls
    with pytest.raises(ValueError):  # axes of another number of pairs
        clsa.clsa_norm_rope_axes(spec, clsa.make_rope_axes([0] * 32, num_axes=3), Tensor((3, 7), I32), q, q)


def test_the_native_module_hands_back_what_it_does_not_take(clsa):
    from paper_2606_06467_b200 import layer

    if layer._marshal is None:
        pytest.skip("built without Python.h")
    layer._load_torch()
    m, p = layer._marshal, _params(clsa)
    t, ws = torch.zeros(2, 1, 32, 128, dtype=BF16), torch.zeros(4096, dtype=U8)
    for args in ((p, 0, t, t, None, ws, None, None), (p, "x", t, t, None, ws, None, None), (p, 1 << 70, t, t, None, ws, None, None), (p, 0, 1, 2, None, 3, 4, 5), ()):
        assert m.dense(*args) is None
    for args in ((p, p, 0, t, t, None, ws, None, None), (p, None, 0, t, t, None, ws, None, None), ()):
        assert m.dense8(*args) is None
    spec = clsa.make_add_norm(dim=128)
    for args in ((spec, t, t, None, t, None, None, None), (p, t, t, None, t, None, None, 0), (spec, None, t, None, t, None, None, 0), (spec, 1, 2, 3, 4, 5, 6, 7), ()):
        assert m.add_norm(*args) is None
    rope, ax = clsa.make_norm_rope(rot_dim=128), clsa.make_rope_axes([0] * 64)
    for args in ((rope, ax, t, t, t, None, None, None), (ax, rope, t, t, t, None, None, 0), (rope, ax, None, t, t, None, None, 0), (rope, ax, 0x1000, 1, 2, 3, 4, 0), ()):
        assert m.norm_rope_axes(*args) is None
