"""Host-side checks of the 8-bit cache calls without a GPU: empty batches, layouts of scales, sizes of buffers against the params,
in the Python marshalling and in the native one (which gets stand-ins for tensors and for the library's entry points)."""
import ctypes
import os
import sys

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, I32, F32, U8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8


@pytest.fixture(scope="module")
def clsa():
    sys.path.insert(0, ROOT)
    import __graft_entry__ as entry

    entry._load_build_module().build()
    import paper_2606_06467_b200 as mod

    return mod


def test_an_empty_batch_is_a_call_that_does_nothing(clsa):
    """No tokens, as empty tensors give them: no address of positions or heads, strides of any kind."""
    P, raw = ctypes.byref, clsa.raw()
    spec = clsa.clsa_norm_rope_spec(128, 1, 1e-6, 128, 0, 1.0, 0x7000, None, None)
    a, b = clsa.clsa_heads(None, 8, 1536, 128), clsa.clsa_heads(None, 8, 1024, 128)
    assert raw.clsa_norm_rope(P(spec), 0, None, P(a), P(b), None, None, None) == clsa.CLSA_OK
    assert raw.clsa_norm_rope(P(spec), 0, None, None, None, P(a), P(b), None) == clsa.CLSA_OK
    assert raw.clsa_norm_rope(P(spec), 0, None, P(a), None, None, None, None) == 1  # what is wrong without tokens is still wrong
    assert raw.clsa_norm_rope(P(spec), 4, None, P(a), P(b), None, None, None) == 1


def test_scale_strides_are_the_tensors_own(clsa):
    u8 = lambda *s: torch.zeros(s, dtype=U8)  # noqa: E731
    k = u8(128, 4, 128)
    with pytest.raises(ValueError):  # one row of scales for all heads
        clsa.make_cache8(k=k, v=k, k_scale=u8(1, 2).expand(4, 2), v_scale=u8(1, 2).expand(4, 2), scale_block=64)
    with pytest.raises(ValueError):  # overlapping rows
        s = u8(16).as_strided((4, 2), (1, 1))
        clsa.make_cache8(k=k, v=k, k_scale=s, v_scale=s, scale_block=64)
    wide = u8(4, 9)[:, :2]
    assert clsa.make_cache8(k=k, v=k, k_scale=wide, v_scale=wide, scale_block=64).scale_head_stride == 9
    one = u8(128, 1, 128)
    for s in (u8(1, 2), u8(2).expand(1, 2), u8(2, 2)[:1]):  # one head: no distance between heads
        assert clsa.make_cache8(k=one, v=one, k_scale=s, v_scale=s, scale_block=64).scale_head_stride >= 2


class Tensor:
    """What the marshalling asks of a tensor."""

    def __init__(self, shape, dtype, stride=None, device=0):
        self.shape, self.dtype, self.device = tuple(shape), dtype, device
        dense = [1] * len(shape)
        for i in reversed(range(len(shape) - 1)):
            dense[i] = dense[i + 1] * max(shape[i + 1], 1)
        self._dense, self._stride = tuple(dense), tuple(stride or dense)

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def element_size(self):
        return {BF16: 2, U8: 1}.get(self.dtype, 4)

    def is_contiguous(self):
        return self._stride == self._dense

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 0x100000 if self.numel() else 0


@pytest.fixture(params=["native", "python"])
def binding(clsa, request, monkeypatch):
    """The package with entry points that record their calls in place of the library's, and Tensor in place of torch's."""
    from paper_2606_06467_b200 import cache8

    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    cache8._load_torch()
    monkeypatch.setattr(cache8, "_lib", Lib())
    monkeypatch.setattr(cache8, "_device", lambda torch: 0)
    monkeypatch.setattr(cache8, "_stream8", lambda stream, device: 0)
    if request.param == "python":
        monkeypatch.setattr(cache8, "_marshal", None)
        yield clsa, calls
        return
    if cache8._marshal is None:
        pytest.skip("built without Python.h")
    # any number of integer arguments will do: the recorder looks at none
    kinds = {"clsa_norm_rope": 8, "clsa_cache8_append": 9, "clsa_index_scores8": 8, "clsa_sparse_attn8": 11}
    keep = [ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p] * n)(lambda *a, name=name: calls.append("native " + name) or 0) for name, n in kinds.items()]
    cache8._marshal.setup(*[ctypes.cast(f, ctypes.c_void_p).value for f in keep], Tensor, BF16, I32, F32, U8, lambda: 0, lambda d: 0, clsa.clsa_params,
                          clsa.clsa_cache8, clsa.clsa_norm_rope_spec, clsa.clsa_attn_hints)
    yield clsa, calls
    monkeypatch.undo()
    cache8._load_torch()


def _cache(clsa, rows=2048, heads=8, idx_dim=128):
    u8 = lambda *s: torch.zeros(s, dtype=U8)  # noqa: E731
    c = clsa.make_cache8(k=u8(rows, heads, 128), v=u8(rows, heads, 128), k_scale=u8(heads, rows // 64), v_scale=u8(heads, rows // 64),
                         idx_k=u8(rows, idx_dim), idx_k_scale=u8(rows // 64), scale_block=64)
    c._device = 0
    return c


def _params(clsa, **kw):
    base = dict(num_seqs=2, q_per_seq=3, num_q_heads=32, num_kv_heads=8, head_dim=128, idx_dim=128, top_k=64, max_seq_len=1000, sm_scale=0.088,
                seq_start=0x1000, seq_len=0x2000, num_cache_rows=2048)
    base.update(kw)
    return clsa.make_params(**base)


def _taken(calls, name):
    """One call was made, by the native module where that is the one under test."""
    got = list(calls)
    calls.clear()
    return got in ([name], ["native " + name])


def test_buffers_are_measured_against_the_params(binding):
    clsa, calls = binding
    p, c, ws = _params(clsa), _cache(clsa), Tensor((4096,), U8)
    good = dict(q=Tensor((2, 3, 32, 128), BF16), idx=Tensor((2, 3, 64), I32), count=Tensor((2, 3), I32), out=Tensor((2, 3, 32, 128), BF16),
                lse=Tensor((2, 3, 32), F32))
    attn = lambda n=None, **kw: clsa.clsa_sparse_attn8(p, c, *[{**good, **kw}[x] for x in ("q", "idx", "count", "out", "lse")], None, ws, n)  # noqa: E731
    for ok in ({}, dict(lse=None), dict(q=Tensor((7, 32, 128), BF16)), dict(n=4096), dict(n=256), dict(idx=Tensor((6 * 64,), I32))):
        attn(**ok)
        assert _taken(calls, "clsa_sparse_attn8"), ok
    for bad in (dict(q=Tensor((2, 3, 31, 128), BF16)), dict(idx=Tensor((6, 63), I32)), dict(count=Tensor((5,), I32)), dict(out=Tensor((5, 32, 128), BF16)),
                dict(lse=Tensor((6, 31), F32)), dict(n=4097)):
        with pytest.raises(ValueError):
            attn(**bad)
    scores = lambda q, s, n: clsa.clsa_index_scores8(p, c, q, s, n, ws)  # noqa: E731
    q = Tensor((2, 3, 128), BF16)
    for s, n in ((Tensor((2, 3, 1040), F32), 1040), (Tensor((2, 3, 1000), F32, (3096, 1032, 1)), 1032), (Tensor((5 * 1040 + 1000,), F32), 1040)):
        scores(q, s, n)
        assert _taken(calls, "clsa_index_scores8")
    for q_, s, n in ((Tensor((5, 128), BF16), Tensor((2, 3, 1040), F32), 1040), (q, Tensor((2, 3, 1000), F32), 1040), (q, Tensor((5 * 1040 + 999,), F32), 1040),
                     (q, Tensor((2, 3, 999), F32, (3096, 1032, 1)), 1032), (q, Tensor((5, 1040), F32), 1040)):
        with pytest.raises(ValueError):
            scores(q_, s, n)
    assert not calls


def test_caches_are_measured_against_the_params(binding):
    clsa, calls = binding
    ws, p = Tensor((4096,), U8), _params(clsa)

    def each(p, c):
        q, s = Tensor((2, 3, p.num_q_heads, 128), BF16), Tensor((2, 3, 1040), F32)
        new, idx = Tensor((2, 3, p.num_kv_heads, 128), BF16), Tensor((2, 3, p.idx_dim), BF16)
        return dict(kv=[lambda: clsa.clsa_cache8_append(p, c, None, new, new, None, ws),
                        lambda: clsa.clsa_sparse_attn8(p, c, q, Tensor((6, 64), I32), Tensor((6,), I32), q, None, None, ws)],
                    idx=[lambda: clsa.clsa_cache8_append(p, c, None, None, None, idx, ws), lambda: clsa.clsa_index_scores8(p, c, idx, s, 1040, ws)])

    def refused(p, c, which):
        for call in which:
            with pytest.raises(ValueError):
                call()
        assert not calls

    for c in (_cache(clsa), _cache(clsa, rows=4096), _cache(clsa, heads=9)):
        for call in sum(each(p, c).values(), []):
            call()
            assert len(calls) == 1
            calls.clear()
    for c in (_cache(clsa, rows=2048 - 64),):
        refused(p, c, each(p, c)["kv"] + each(p, c)["idx"])
    c = _cache(clsa, heads=7)
    refused(p, c, each(p, c)["kv"])
    c = _cache(clsa, idx_dim=64)
    refused(p, c, each(p, c)["idx"])
    c = _cache(clsa, rows=64)  # another buffer's address since: nothing is known of it
    c.k, c.idx_k = 0x10000, 0x50000
    c.scale_head_stride = 64
    for call in sum(each(p, c).values(), []):
        call()
        assert len(calls) == 1
        calls.clear()
    # a cache described by addresses has no sizes to compare
    c = clsa.clsa_cache8(0x10000, 0x20000, 0x30000, 0x40000, 1024, 128, 64, 0x50000, 0x60000, 128, 64)
    for call in sum(each(p, c).values(), []):
        call()
        assert len(calls) == 1
        calls.clear()


def test_empty_tensors_are_taken(binding):
    clsa, calls = binding
    spec = clsa.make_norm_rope(head_dim=128, norm=1, rot_dim=0)
    for shape in ((0, 8, 128), (0, 4, 8, 128), (3, 0, 8, 128)):
        q = Tensor(shape, BF16)
        clsa.clsa_norm_rope(spec, Tensor((0,), I32), q, q)
        assert _taken(calls, "clsa_norm_rope"), shape
        clsa.clsa_norm_rope(spec, Tensor((0,), I32), None, None, q, q)
        assert _taken(calls, "clsa_norm_rope"), shape


def test_the_params_own_tensors_are_measured(binding):
    """seq_start, seq_len and the block table: types, layouts, how many sequences they describe, where they lie."""
    clsa, calls = binding
    ws, c = Tensor((4096,), U8), clsa.clsa_cache8(0x10000, 0x20000, 0x30000, 0x40000, 1024, 128, 64, 0x50000, 0x60000, 128, 64)
    heads, idx, s = Tensor((2, 3, 8, 128), BF16), Tensor((2, 3, 128), BF16), Tensor((2, 3, 1040), F32)
    q = Tensor((2, 3, 32, 128), BF16)
    each = (lambda p: clsa.clsa_cache8_append(p, c, None, heads, heads, idx, ws), lambda p: clsa.clsa_index_scores8(p, c, idx, s, 1040, ws),
            lambda p: clsa.clsa_sparse_attn8(p, c, q, Tensor((6, 64), I32), Tensor((6,), I32), q, None, None, ws))
    zeros = lambda *shape, dtype=I32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    here = lambda p: setattr(p, "_made", tuple(m and (*m[:2], 0) for m in p._made)) or p  # noqa: E731  (host tensors as if on device 0)
    start, length, table = zeros(2, dtype=torch.int64), zeros(2), zeros(2, 16)
    paged = dict(block_size=64, max_seq_len=1000)
    good = [dict(seq_start=start, seq_len=length), dict(seq_start=zeros(9, dtype=torch.int64), seq_len=zeros(2, 1)), dict(seq_len=length, seq_start=0x1000),
            dict(seq_start=None, seq_len=length, block_table=table, **paged),
            dict(seq_start=None, seq_len=length, block_table=zeros(2, 20)[:, :16], max_blocks_per_seq=20, **paged),
            dict(seq_start=zeros(1), seq_len=length, block_table=table, **paged)]  # with pages the starts are not read
    for kw in good:
        for call in each:
            call(here(_params(clsa, **kw)))
            assert len(calls) == 1, kw
            calls.clear()
    bad = [dict(seq_len=zeros(2, dtype=torch.int64)), dict(seq_len=zeros(1)), dict(seq_len=zeros(2, 2)[:, 0]), dict(seq_start=zeros(2)),
           dict(seq_start=zeros(1, dtype=torch.int64)), dict(block_table=zeros(1, 16), **paged), dict(block_table=zeros(2, 16, dtype=torch.int64), **paged),
           dict(block_table=zeros(2, 20)[:, :16], **paged)]
    for kw in bad:
        for call in each:
            with pytest.raises(ValueError):
                call(here(_params(clsa, **kw)))
    for call in each:
        with pytest.raises(ValueError):
            call(_params(clsa, seq_len=length))  # host memory
    p = _params(clsa, seq_len=zeros(1))
    p.seq_len = 0x2000  # another buffer since
    each[0](p)
    assert len(calls) == 1
