"""Host-side checks of the 8-bit cache calls that need no GPU: symbols, struct layouts, refusals, and the reference itself."""
import ctypes
import os
import re
import subprocess
import sys

import numpy as np
import pytest

import _cache8_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "clsa_cache8.h")


@pytest.fixture(scope="module")
def clsa():
    sys.path.insert(0, ROOT)
    import __graft_entry__ as entry

    entry._load_build_module().build()
    import paper_2606_06467_b200 as mod

    return mod


def test_symbols(clsa):
    names = set(re.findall(r"CLSA_API\s+[\w\s\*]+?\b(clsa_\w+)\s*\(", open(HEADER).read()))
    assert names == set(clsa.EXPORTS_CACHE8)
    for n in names:
        assert hasattr(ctypes.CDLL(clsa.LIB_PATH), n), n


@pytest.mark.parametrize("name", ["clsa_heads", "clsa_norm_rope_spec", "clsa_cache8"])
def test_struct_layouts_match_the_header(clsa, tmp_path, name):
    cls = getattr(clsa, name)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "clsa_cache8.h"\nint main(void){printf("%zu", sizeof(' + name + "));\n"
                   + "".join(f'printf(" %zu", offsetof({name}, {f}));\n' for f, _ in cls._fields_) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    nums = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert nums == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]


def _params(clsa, **kw):
    base = dict(num_seqs=2, num_q_heads=32, num_kv_heads=8, head_dim=128, idx_dim=128, top_k=64, max_seq_len=1024, sm_scale=0.088,
                seq_start=0x1000, seq_len=0x2000, num_cache_rows=2048)
    base.update(kw)
    return clsa.make_params(**base)


def _cache(clsa, **kw):
    c = clsa.clsa_cache8(0x10000, 0x20000, 0x30000, 0x40000, 1024, 128, 64, 0x50000, 0x60000, 128, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _spec(clsa, **kw):
    s = clsa.clsa_norm_rope_spec(128, 1, 1e-6, 128, 0, 1.0, 0x7000, 0x8000, 0x9000)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _heads(clsa, data=0x100000, num=8, token=1024, head=128):
    return clsa.clsa_heads(data, num, token, head)


BAD, UNS, WS = 1, 2, 3
_PARAMS = [
    (dict(num_seqs=0), BAD), (dict(q_per_seq=0), BAD), (dict(num_q_heads=30), BAD), (dict(causal=2), BAD), (dict(sm_scale=0.0), BAD),
    (dict(sm_scale=float("inf")), BAD), (dict(max_seq_len=0), BAD), (dict(max_seq_len=0x7fffffff), UNS), (dict(num_seqs=1 << 29, max_seq_len=256), UNS), (dict(num_cache_rows=0), BAD), (dict(num_cache_rows=1 << 31), BAD),
    (dict(head_dim=64), UNS), (dict(idx_dim=96), UNS), (dict(num_q_heads=34, num_kv_heads=2), UNS), (dict(seq_len=None), BAD),
    (dict(seq_start=None), BAD), (dict(seq_len=0x2002), BAD), (dict(block_table=0x3000, block_size=24, max_blocks_per_seq=64), BAD),
    (dict(block_table=0x3000, block_size=64, max_blocks_per_seq=8), BAD),
    (dict(block_table=0x3000, block_size=32, max_blocks_per_seq=64), BAD),  # a page smaller than a scale block
]


@pytest.mark.parametrize("kw,want", _PARAMS, ids=[str(k) for k, _ in _PARAMS])
def test_bad_params_are_refused(clsa, kw, want):
    P, raw = ctypes.byref, clsa.raw()
    p, c, h, i = _params(clsa, **kw), _cache(clsa), _heads(clsa), _heads(clsa, num=1)
    assert raw.clsa_cache8_append(P(p), P(c), None, P(h), P(h), P(i), 0x100000, 1 << 30, None) == want
    assert raw.clsa_index_scores8(P(p), P(c), 0x50000, 0x40000, 1024, 0x100000, 1 << 30, None) == want
    assert raw.clsa_sparse_attn8(P(p), P(c), 0x50000, 0x60000, 0x70000, 0x80000, None, None, 0x100000, 1 << 30, None) == want
    assert raw.clsa_sparse_attn8(None, P(c), 0x50000, 0x60000, 0x70000, 0x80000, None, None, 0x100000, 1 << 30, None) == BAD


_CACHES = [
    (dict(scale_block=0), BAD, "kvi"), (dict(scale_block=48), BAD, "kvi"), (dict(scale_block=256), BAD, "kvi"),
    (dict(k=None), BAD, "kv"), (dict(v=0x20008), BAD, "kv"), (dict(k_scale=None), BAD, "kv"), (dict(v_scale=None), BAD, "kv"),
    (dict(kv_token_stride=1032), BAD, "kv"), (dict(kv_head_stride=64), BAD, "kv"), (dict(scale_head_stride=31), BAD, "kv"),
    (dict(kv_token_stride=1 << 26), UNS, "kv"), (dict(idx_k=None), BAD, "i"), (dict(idx_k=0x50008), BAD, "i"),
    (dict(idx_k_scale=None), BAD, "i"), (dict(idx_token_stride=64), BAD, "i"), (dict(idx_token_stride=136), BAD, "i"),
]


@pytest.mark.parametrize("kw,want,users", _CACHES, ids=[str(k) for k, _, _ in _CACHES])
def test_bad_caches_are_refused(clsa, kw, want, users):
    P, raw = ctypes.byref, clsa.raw()
    p, c, h, i = _params(clsa), _cache(clsa, **kw), _heads(clsa), _heads(clsa, num=1)
    if "k" in users:
        assert raw.clsa_cache8_append(P(p), P(c), None, P(h), P(h), None, 0x100000, 1 << 30, None) == want
        assert raw.clsa_sparse_attn8(P(p), P(c), 0x50000, 0x60000, 0x70000, 0x80000, None, None, 0x100000, 1 << 30, None) == want
    if "i" in users:
        assert raw.clsa_cache8_append(P(p), P(c), None, None, None, P(i), 0x100000, 1 << 30, None) == want
        assert raw.clsa_index_scores8(P(p), P(c), 0x50000, 0x40000, 1024, 0x100000, 1 << 30, None) == want
    n = ctypes.c_size_t(0)
    if "scale_block" in kw:
        assert raw.clsa_cache8_workspace_bytes(P(p), P(c), P(n)) == want


def test_bad_calls_are_refused(clsa):
    P, raw = ctypes.byref, clsa.raw()
    p, c, h, i = _params(clsa), _cache(clsa), _heads(clsa), _heads(clsa, num=1)
    ws, wsb = 0x100000, 1 << 30
    n = ctypes.c_size_t(0)
    assert raw.clsa_cache8_workspace_bytes(P(p), P(c), None) == BAD and raw.clsa_cache8_workspace_bytes(P(p), None, P(n)) == BAD
    ap = raw.clsa_cache8_append
    assert ap(P(p), None, None, P(h), P(h), P(i), ws, wsb, None) == BAD
    assert ap(P(p), P(c), None, P(h), None, P(i), ws, wsb, None) == BAD
    assert ap(P(p), P(c), None, None, None, None, ws, wsb, None) == BAD
    assert ap(P(p), P(c), None, P(_heads(clsa, num=4)), P(h), None, ws, wsb, None) == BAD
    assert ap(P(p), P(c), None, P(h), P(h), P(_heads(clsa, num=2)), ws, wsb, None) == BAD
    for bad in (dict(data=None), dict(data=0x100008), dict(token=1028), dict(head=100), dict(head=64), dict(token=-8)):
        assert ap(P(p), P(c), None, P(_heads(clsa, **bad)), P(h), None, ws, wsb, None) == BAD, bad
        assert ap(P(p), P(c), None, P(h), P(_heads(clsa, **bad)), None, ws, wsb, None) == BAD, bad
    assert ap(P(p), P(c), P(_spec(clsa, head_dim=64, rot_dim=64)), P(h), P(h), None, ws, wsb, None) == BAD
    assert ap(P(p), P(c), P(_spec(clsa, rot_dim=8)), P(h), P(h), None, ws, wsb, None) == UNS
    assert ap(P(p), P(c), None, P(h), P(h), P(i), None, wsb, None) == WS
    assert ap(P(p), P(c), None, P(h), P(h), P(i), ws + 16, wsb, None) == WS
    assert ap(P(p), P(c), None, P(h), P(h), P(i), ws, 128, None) == WS
    sc = raw.clsa_index_scores8
    assert sc(P(p), P(c), None, 0x40000, 1024, ws, wsb, None) == BAD
    assert sc(P(p), P(c), 0x50008, 0x40000, 1024, ws, wsb, None) == BAD
    assert sc(P(p), P(c), 0x50000, 0x40002, 1024, ws, wsb, None) == BAD
    assert sc(P(p), P(c), 0x50000, 0x40000, 1000, ws, wsb, None) == BAD
    assert sc(P(p), P(c), 0x50000, 0x40000, 1024, None, wsb, None) == WS
    big = _params(clsa, num_seqs=1 << 16, q_per_seq=64, max_seq_len=1 << 17)
    assert sc(P(big), P(c), 0x50000, 0x40000, 1 << 17, ws, wsb, None) == UNS  # expanded keys past 32-bit rows
    at = raw.clsa_sparse_attn8
    good = [0x50000, 0x60000, 0x70000, 0x80000, None]
    for k, v in ((0, None), (0, 0x50008), (1, None), (1, 0x60002), (2, None), (3, None), (3, 0x80004), (4, 0x90001)):
        args = list(good)
        args[k] = v
        assert at(P(p), P(c), *args, None, ws, wsb, None) == BAD, (k, v)
    for hint, want in ((clsa.make_hints(reverse=2), BAD), (clsa.make_hints(keep_rows=-1), BAD), (clsa.make_hints(only_q_pending=3), BAD),
                       (clsa.make_hints(shared_gpu=5), BAD), (clsa.make_hints(shared_gpu=1), UNS), (clsa.make_hints(shared_gpu=4), UNS)):
        assert at(P(p), P(c), *good, P(hint), ws, wsb, None) == want
    assert at(P(p), P(c), *good, None, None, wsb, None) == WS and at(P(p), P(c), *good, None, ws + 8, wsb, None) == WS


def test_bad_norm_rope_calls_are_refused(clsa):
    P, raw = ctypes.byref, clsa.raw()
    h, s = _heads(clsa), _spec(clsa)
    nr = raw.clsa_norm_rope
    assert nr(P(s), 0, 0x1000, P(h), P(h), None, None, None) == clsa.CLSA_OK  # no tokens: nothing to do
    assert nr(None, 4, 0x1000, P(h), P(h), None, None, None) == BAD
    for kw, want in ((dict(norm=2), BAD), (dict(interleaved=-1), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD),
                     (dict(rot_dim=-16), BAD), (dict(rot_dim=144), BAD), (dict(rot_dim=24), UNS), (dict(inv_freq=None), BAD),
                     (dict(rot_scale=float("inf")), BAD), (dict(q_weight=0x8008), BAD), (dict(k_weight=0x9002), BAD),
                     (dict(head_dim=0, rot_dim=0), BAD), (dict(head_dim=96, rot_dim=96), UNS)):
        assert nr(P(_spec(clsa, **kw)), 4, 0x1000, P(h), P(h), None, None, None) == want, kw
    assert nr(P(s), -1, 0x1000, P(h), P(h), None, None, None) == BAD
    assert nr(P(s), 4, None, P(h), P(h), None, None, None) == BAD and nr(P(s), 4, 0x1001, P(h), P(h), None, None, None) == BAD
    assert nr(P(s), 4, 0x1000, None, None, None, None, None) == BAD and nr(P(s), 4, 0x1000, P(h), None, None, None, None) == BAD
    assert nr(P(s), 4, 0x1000, P(h), P(h), None, P(h), None) == BAD
    assert nr(P(s), 4, 0x1000, P(h), P(_heads(clsa, num=7)), None, None, None) == BAD
    assert nr(P(s), 4, 0x1000, P(h), P(_heads(clsa, token=2048)), None, None, None) == BAD  # in place with another layout
    assert nr(P(s), 4, 0x1000, P(h), P(_heads(clsa, data=0x200000, token=0)), None, None, None) == BAD  # tokens on one another
    for bad in (dict(data=None), dict(data=0x100004), dict(token=1025), dict(head=4), dict(num=0), dict(num=2000)):
        assert nr(P(s), 4, 0x1000, P(_heads(clsa, **bad)), P(_heads(clsa, **bad)), None, None, None) == BAD, bad


def test_binding_refuses_wrong_tensors(clsa):
    torch = pytest.importorskip("torch")
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    k, s, i, si = u8(128, 2, 128), u8(2, 2), u8(128, 64), u8(2)
    c = clsa.make_cache8(k=k, v=k.clone(), k_scale=s, v_scale=s, idx_k=i, idx_k_scale=si, scale_block=64)
    assert (c.kv_token_stride, c.kv_head_stride, c.scale_head_stride, c.idx_token_stride) == (256, 128, 2, 64)
    for bad in (dict(k=k.float()), dict(v=None), dict(v=u8(128, 1, 128)), dict(k_scale=u8(2, 1)), dict(v_scale=u8(1, 2)),
                dict(idx_k=u8(128, 64).int()), dict(idx_k_scale=u8(1)), dict(idx_k_scale=None)):
        with pytest.raises(ValueError):
            clsa.make_cache8(**{**dict(k=k, v=k, k_scale=s, v_scale=s, idx_k=i, idx_k_scale=si, scale_block=64), **bad})
    with pytest.raises(ValueError):
        clsa.make_norm_rope(head_dim=128, rot_dim=64, inv_freq=torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        clsa.make_norm_rope(head_dim=128, q_weight=torch.zeros(64, dtype=torch.bfloat16))
    spec = clsa.make_norm_rope(head_dim=128)
    q = torch.zeros(2, 3, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # host tensors
        clsa.clsa_norm_rope(spec, None, q, q)
    with pytest.raises(ValueError):
        clsa.clsa_norm_rope(spec, None, q, None)
    p = _params(clsa, num_kv_heads=2, num_q_heads=2)
    ws = torch.zeros(256, dtype=torch.uint8)
    b = torch.bfloat16
    for call in (lambda: clsa.clsa_cache8_append(p, c, None, None, None, torch.zeros(2, 1, 128, dtype=b), ws),
                 lambda: clsa.clsa_cache8_append(p, c, None, None, torch.zeros(2, 1, 2, 128, dtype=b), None, ws),
                 lambda: clsa.clsa_index_scores8(p, c, torch.zeros(2, 1, 128, dtype=b), torch.zeros(2, 1, 1024), 1024, ws),
                 lambda: clsa.clsa_sparse_attn8(p, c, torch.zeros(2, 1, 2, 128, dtype=b), torch.zeros(2, 1, 64, dtype=torch.int32),
                                                torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1, 2, 128, dtype=b), None, None, ws)):
        with pytest.raises(ValueError):  # host tensors, host workspaces, host caches
            call()


def test_reference_codes_round_to_nearest_even():
    torch = pytest.importorskip("torch")
    x = np.random.default_rng(0).normal(size=20000) * 10.0 ** np.random.default_rng(1).uniform(-4, 2.4, 20000)
    x = np.concatenate([x.clip(-448, 448), ref.E4M3[:127], -ref.E4M3[:127], ref._MID, -ref._MID])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    x = x.astype(np.float32).astype(np.float64)
    np.testing.assert_array_equal(ref.encode(x), want)
    assert list(ref.encode(np.array([np.inf, -np.inf, 1e9, np.nan]))) == [126, 254, 126, 127]
    for amax, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (224.1, 0), (0.0, -100), (1e-40, -100), (3e38, 120), (1.75, -8), (1.0, -8)):
        assert ref.need_exponent(amax) == e, amax


def test_native_marshalling_hands_back_what_it_does_not_take(clsa):
    """Host tensors, addresses, wrong counts and foreign objects: the native module returns None and raises nothing."""
    torch = pytest.importorskip("torch")
    from paper_2606_06467_b200 import cache8

    if cache8._marshal is None:
        pytest.skip("built without Python.h")
    cache8._load_torch()
    m, p, c = cache8._marshal, _params(clsa), _cache(clsa)
    spec = clsa.make_norm_rope()
    t = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    ws = torch.zeros(4096, dtype=torch.uint8)
    for args in ((spec, None, t, t, None, None, None), (spec, None, None, None, None, None, None), (p, None, t, t, None, None, 0),
                 (spec, None, 5, 5, None, None, 0), (None, None, t, t, None, None, 0), (), (object(),) * 7):
        assert m.norm_rope(*args) is None
    for args in ((p, c, None, t, t, None, ws, None, None), (c, p, None, t, t, None, ws, None, None), (p, c, None, None, None, None, ws, None, 0), ()):
        assert m.append(*args) is None
    for args in ((p, c, 0x1000, 0x2000, 1024, 0x3000, 4096, 0), (p, c, t, t, "x", ws, None, None), (p, c, t, t, 1 << 70, ws, None, None), ()):
        assert m.scores(*args) is None
    for args in ((p, c, 1, 2, 3, 4, None, None, 5, 6, 7), (p, c, t, t, t, t, None, 3, ws, -1, object()), ()):
        assert m.attn(*args) is None
