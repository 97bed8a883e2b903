"""The 8-bit cache calls on the GPU against their definitions in 64 bits (tests/_cache8_ref.py has the tolerances)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import __graft_entry__ as entry

entry._load_build_module().build()

import _cache8_ref as ref
import paper_2606_06467_b200 as clsa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def f64(t):
    return t.detach().cpu().double().numpy() if t.dtype != BF16 else t.detach().float().cpu().double().numpy()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


# ------------------------------------------------------------------------------------------------------------ norm_rope
def check_norm_rope(q, q_out, pos, spec_kw, weight, before):
    """q_out against the definition; rows of negative positions unchanged."""
    freq = spec_kw.get("inv_freq")
    p = np.zeros(q.shape[0]) if pos is None else pos.cpu().numpy()
    z, mag = ref.norm_rope(f64(q), p, None if weight is None else f64(weight), spec_kw["norm"], np.float32(1e-6).astype(np.float64),
                           None if freq is None else freq.cpu().numpy(), spec_kw["interleaved"], spec_kw.get("rot_scale", 1.0))
    got, live = f64(q_out), p >= 0
    err = np.abs(got - z) - (2.0 ** -8 * np.abs(z) + 2.0 ** -19 * mag)
    assert (err[live] <= 0).all(), float(err[live].max())
    np.testing.assert_array_equal(got[~live], f64(before)[~live])


@pytest.mark.parametrize("tokens,hq,hk,D,rot,inter,layout", [
    (1, 1, 0, 64, 64, 0, "dense"), (1, 8, 1, 128, 128, 0, "dense"), (16, 32, 8, 128, 128, 0, "fused"), (37, 20, 4, 128, 64, 1, "fused"),
    (5, 0, 3, 256, 256, 0, "dense"), (3, 16, 16, 256, 32, 1, "fused"), (130, 2, 2, 64, 16, 0, "fused"), (7, 40, 5, 128, 0, 0, "dense"),
    (700, 32, 8, 128, 128, 0, "heads first"), (900, 3, 1, 128, 96, 1, "fused"), (1300, 33, 7, 64, 48, 0, "dense")])
@pytest.mark.parametrize("norm", [1, 0])
def test_norm_rope(tokens, hq, hk, D, rot, inter, layout, norm):
    g = gen(tokens + D + rot)

    def make(h):
        if h == 0:
            return None
        if layout == "heads first":
            return randn(g, h, tokens, D, scale=3.0).transpose(0, 1)
        return randn(g, tokens, h + 3, D, scale=3.0)[:, 1:1 + h] if layout == "fused" else randn(g, tokens, h, D, scale=3.0)

    q, k = make(hq), make(hk)
    pos = torch.randint(0, 131072, (tokens,), generator=g, device=DEV, dtype=torch.int32)
    if tokens > 2:
        pos[1] = -1
        pos[2] = 2 ** 31 - 1
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV) if rot else None
    kw = dict(norm=norm, interleaved=inter, inv_freq=freq)
    wq, wk = randn(g, D), (None if tokens % 2 else randn(g, D))
    spec = clsa.make_norm_rope(head_dim=D, eps=1e-6, rot_dim=rot, q_weight=wq, k_weight=wk, **kw)
    outs = [None if t is None else torch.full((tokens, t.shape[1] + 2, D), 7.0, dtype=BF16, device=DEV)[:, 1:-1] for t in (q, k)]
    before = [None if o is None else o.clone() for o in outs]
    clsa.clsa_norm_rope(spec, pos, q, outs[0], k, outs[1])
    for t, o, w, b in ((q, outs[0], wq, before[0]), (k, outs[1], wk, before[1])):
        if t is not None:
            check_norm_rope(t, o, pos, kw, w if norm else None, b)
            assert (o._base[:, 0] == 7).all() and (o._base[:, -1] == 7).all()  # nothing beside the heads is written
    # in place, bit for bit the same
    for t, o in ((q, outs[0]), (k, outs[1])):
        if t is not None:
            own = t.clone(memory_format=torch.preserve_format)
            clsa.clsa_norm_rope(spec, pos, *((own, own) if t is q else (None, None, own, own)))
            live = (pos >= 0)
            assert torch.equal(own[live], o[live]) and torch.equal(own[~live], t[~live])


def test_norm_rope_special_values_and_shapes():
    g = gen(3)
    spec = clsa.make_norm_rope(head_dim=128, norm=0, rot_dim=64, inv_freq=torch.ones(32, device=DEV), rot_scale=1.5)
    q = randn(g, 6, 2, 4, 128)  # [B, T, heads, D]
    out = torch.empty_like(q)
    pos = torch.arange(12, device=DEV, dtype=torch.int32)
    clsa.clsa_norm_rope(spec, pos, q, out)
    check_norm_rope(q.flatten(0, 1), out.flatten(0, 1), pos, dict(norm=0, interleaved=0, inv_freq=torch.ones(32), rot_scale=1.5), None, out.flatten(0, 1))
    # infinities and NaN stay in their pair; dimensions behind the rotated ones pass through
    q[0, 0, 0, 70] = float("inf")
    q[0, 0, 1, 3] = float("nan")
    clsa.clsa_norm_rope(spec, pos, q, out)
    assert torch.isinf(out[0, 0, 0, 70]) and torch.isfinite(out[0, 0, 0, :70]).all() and torch.isfinite(out[0, 0, 0, 71:]).all()
    bad = torch.isnan(out[0, 0, 1]).nonzero().flatten().tolist()
    assert bad == [3, 35]
    # one row read for every token (an expanded tensor)
    one = randn(g, 1, 4, 128).expand(5, 4, 128)
    o5 = torch.empty((5, 4, 128), dtype=BF16, device=DEV)
    clsa.clsa_norm_rope(spec, torch.full((5,), 9, dtype=torch.int32, device=DEV), one, o5)
    assert (o5 == o5[:1]).all()
    # a zero row under a norm stays zero
    nspec = clsa.make_norm_rope(head_dim=128, norm=1, rot_dim=0)
    z = torch.zeros((2, 1, 128), dtype=BF16, device=DEV)
    clsa.clsa_norm_rope(nspec, None, z, z)
    assert (z == 0).all()
    with pytest.raises(ValueError):
        clsa.clsa_norm_rope(spec, pos[:5], q, out)
    with pytest.raises(ValueError):
        clsa.clsa_norm_rope(spec, pos, q, out.float())


# ------------------------------------------------------------------------------------------------------------ the cache
class Cache:
    """A pool with sequences placed contiguously (seq_start a multiple of the block) or in scattered pages, filled with random
    codes and scales; a row-major copy on the host."""

    def __init__(self, lens, T, hkv, d_idx, block, page, seed, capacity=None, fill=True, exps=(119, 122), pad_strides=False):
        g = gen(seed)
        B = len(lens)
        cap = capacity or max(lens)
        if page:
            per = -(-cap // page)
            self.rows = (B * per + 1) * page
            self.table = (torch.randperm(B * per, generator=g, device=DEV) + 1).to(torch.int32).view(B, per)
            self.start = None
        else:
            room = -(-cap // block) * block
            self.rows = B * room + block
            self.start = block + room * torch.arange(B, device=DEV, dtype=torch.int64)
            self.table = None
        self.B, self.T, self.hkv, self.d_idx, self.block, self.page = B, T, hkv, d_idx, block, page
        self.lens = list(lens)
        self.max_len = cap
        self.seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
        nb = self.rows // block

        def codes(*shape):
            if not fill:
                return torch.zeros(shape, dtype=torch.uint8, device=DEV)
            return (torch.randn(shape, generator=g, device=DEV) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

        def exp(*shape):
            return torch.randint(exps[0], exps[1], shape, generator=g, device=DEV, dtype=torch.uint8)

        if pad_strides:  # rows with unused bytes between heads and tokens
            wide = codes(self.rows, hkv + 1, 2, 144)
            self.k, self.v = wide[:, :hkv, 0, :128], wide[:, :hkv, 1, :128]
            self.idx = codes(self.rows, d_idx + 32)[:, :d_idx]
            sc = exp(hkv, 2, nb + 3)
            self.ks, self.vs = sc[:, 0, :nb], sc[:, 1, :nb]
        else:
            self.k, self.v, self.idx = codes(self.rows, hkv, 128), codes(self.rows, hkv, 128), codes(self.rows, d_idx)
            self.ks, self.vs = exp(hkv, nb), exp(hkv, nb)
        self.isc = exp(nb)
        self.cache = clsa.make_cache8(k=self.k, v=self.v, k_scale=self.ks, v_scale=self.vs, idx_k=self.idx, idx_k_scale=self.isc, scale_block=block)

    def params(self, hq=None, top_k=1, causal=0, **kw):
        base = dict(num_seqs=self.B, q_per_seq=self.T, num_q_heads=hq or self.hkv, num_kv_heads=self.hkv, idx_dim=self.d_idx, top_k=top_k,
                    causal=causal, max_seq_len=self.max_len, sm_scale=128 ** -0.5, seq_start=self.start, seq_len=self.seq_len,
                    num_cache_rows=self.rows, block_table=self.table, block_size=self.page)
        base.update(kw)
        self.p = clsa.make_params(**base)
        self.ws = torch.zeros(clsa.clsa_cache8_workspace_bytes(self.p, self.cache), dtype=torch.uint8, device=DEV)
        return self.p

    def row(self, b, s):
        if self.page:
            t = self.table[b].cpu().numpy()
            return t[np.asarray(s) // self.page].astype(np.int64) * self.page + np.asarray(s) % self.page
        return int(self.start[b]) + np.asarray(s)

    def host(self):
        """(codes, scales) of K, V and K_idx as numpy copies, heads explicit."""
        c = lambda t: t.cpu().numpy().copy()  # noqa: E731
        return [(c(self.k), c(self.ks)), (c(self.v), c(self.vs)), (c(self.idx)[:, None], c(self.isc)[None])]

    def status(self):
        return clsa.clsa_device_status(self.ws)


# ------------------------------------------------------------------------------------------------------------ append
def run_append(c, seed, spec_kw=None, weight=None, fused=False, special=False, scale=1.0):
    g = gen(seed)
    if fused:
        new = randn(g, c.B, c.T, 2 * c.hkv + 3, 128, scale=scale)
        k, v = new[:, :, 1:1 + c.hkv], new[:, :, 2 + c.hkv:2 + 2 * c.hkv]
    else:
        k, v = randn(g, c.B, c.T, c.hkv, 128, scale=scale), randn(g, c.B, c.T, c.hkv, 128, scale=scale)
    i = randn(g, c.B, c.T, c.d_idx, scale=scale)
    if special:
        v[0, 0, 0, 5], v[0, -1, 0, 7], i[-1, 0, 1], i[-1, -1, 2] = float("inf"), float("nan"), float("-inf"), 2.0 ** 100
        v[-1, :, -1] = 0
    spec = None
    if spec_kw is not None:
        spec = clsa.make_norm_rope(head_dim=128, eps=1e-6, k_weight=weight, rot_dim=0 if spec_kw["inv_freq"] is None else
                                   2 * spec_kw["inv_freq"].numel(), **spec_kw)
    before = c.host()
    clsa.clsa_cache8_append(c.p, c.cache, spec, k, v, i, c.ws)
    after = c.host()
    for which, new in ((0, k), (1, v), (2, i[:, :, None])):
        (code, sc), (got, gsc) = before[which], after[which]
        for b in range(c.B):
            n = c.lens[b]
            pos = np.arange(n - c.T, n)
            if which == 0 and spec is not None:
                x, mag = ref.norm_rope(f64(new[b]), pos, None if weight is None else f64(weight), spec_kw["norm"], np.float32(1e-6).astype(np.float64),
                                       None if spec_kw["inv_freq"] is None else spec_kw["inv_freq"].cpu().numpy(), spec_kw["interleaved"])
            else:
                x, mag = f64(new[b]), None
            done = ref.append(code, sc, lambda s, b=b: int(c.row(b, s)), n, x, c.block)
            rows = c.row(b, pos)
            if mag is not None:  # behind a norm: the nearest code up to the fp32 chain's error
                for (home, h), e in done.items():
                    mine = np.array([s for s in range(c.T) if home <= rows[s] < home + c.block])
                    err = np.abs(ref.E4M3[got[rows[mine], h]] * 2.0 ** e - x[mine, h])
                    assert (err <= ref.half_step(x[mine, h], e) + 2.0 ** -19 * mag[mine, h]).all()
                    code[rows[mine], h] = got[rows[mine], h]
        np.testing.assert_array_equal(gsc, sc)
        np.testing.assert_array_equal(got, code)  # new, re-coded and untouched rows alike
    assert c.status() == 0


@pytest.mark.parametrize("lens,T,hkv,d_idx,block,page", [
    ([1], 1, 1, 64, 16, 0), ([1, 17, 64, 65], 1, 8, 128, 64, 0), ([33, 40], 33, 4, 64, 16, 16), ([16, 32, 48], 16, 2, 128, 16, 32),
    ([200, 131, 129], 129, 1, 128, 128, 0), ([77, 300], 70, 3, 64, 32, 64), ([500, 333], 260, 8, 128, 64, 64), ([1000], 1000, 5, 64, 128, 128),
    (list(range(40, 110)), 2, 2, 64, 32, 0)])
@pytest.mark.parametrize("kind", ["plain", "special", "strided"])
def test_append(lens, T, hkv, d_idx, block, page, kind):
    c = Cache(lens, T, hkv, d_idx, block, page, seed=T + block, pad_strides=kind == "strided", capacity=max(lens) + 3)
    c.params()
    run_append(c, 1, fused=kind == "strided", special=kind == "special", scale=1.0 if kind == "plain" else 40.0)


@pytest.mark.parametrize("rot,inter,norm", [(128, 0, 1), (64, 1, 1), (0, 0, 1), (32, 0, 0)])
@pytest.mark.parametrize("lens,T,block,page", [([9, 130, 65], 1, 64, 0), ([300, 220], 200, 128, 128), ([4097], 55, 16, 16)])
def test_append_with_norm_and_rotation(lens, T, block, page, rot, inter, norm):
    c = Cache(lens, T, 4, 128, block, page, seed=rot + T)
    c.params()
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV) if rot else None
    run_append(c, 2, dict(norm=norm, interleaved=inter, inv_freq=freq), randn(gen(4), 128) if norm else None, fused=True)


@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("rot,inter", [(128, 0), (112, 0), (128, 1)])
def test_append_several_heads_per_block(block, rot, inter):
    """Enough scale blocks for several heads per block of threads, a head count that they do not divide, rows on both sides of a
    block's ends, older rows in the first blocks: whole-head rotations and others."""
    c = Cache([1600, 1513, 2000], 1500, 7, 64, block, 0, seed=block)
    c.params()
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(DEV)
    run_append(c, 6, dict(norm=1, interleaved=inter, inv_freq=freq), randn(gen(4), 128), fused=True)


def test_append_token_by_token_grows_its_blocks():
    """A sequence fed one token at a time, magnitudes rising and falling by powers of ten: every step equal to the reference
    that carries the state, re-coded rows included."""
    c = Cache([1, 5], 1, 2, 64, 16, 16, seed=9, capacity=64)
    for step in range(40):
        c.lens = [1 + step, 5 + step]
        c.seq_len.copy_(torch.tensor(c.lens, dtype=torch.int32))
        c.params()
        run_append(c, 100 + step, scale=10.0 ** (step % 7 - 3))


def test_append_one_side_only_and_refused_sequences():
    c = Cache([20, 30], 2, 2, 64, 16, 0, seed=5)
    c.params()
    k, i = randn(gen(1), 2, 2, 2, 128), randn(gen(2), 2, 2, 64)
    b = c.host()
    clsa.clsa_cache8_append(c.p, c.cache, None, None, None, i, c.ws)
    a = c.host()
    assert all((x == y).all() for w in (0, 1) for x, y in zip(a[w], b[w])) and not (a[2][0] == b[2][0]).all()
    b = c.host()
    clsa.clsa_cache8_append(c.p, c.cache, None, k, k, None, c.ws)
    a = c.host()
    assert all((x == y).all() for x, y in zip(a[2], b[2])) and not (a[0][0] == b[0][0]).all()
    # a bad length, a start off the scale blocks, rows beyond the extent: skipped and flagged, the other sequence appended
    for change, bit in ((lambda: c.seq_len.__setitem__(0, 1), clsa.CLSA_DEV_BAD_SEQLEN), (lambda: c.seq_len.__setitem__(0, 31), clsa.CLSA_DEV_BAD_SEQLEN),
                        (lambda: c.start.__setitem__(0, 24), clsa.CLSA_DEV_BAD_SCALE_BLOCK), (lambda: c.start.__setitem__(0, -32), clsa.CLSA_DEV_BAD_INDEX),
                        (lambda: c.start.__setitem__(0, c.rows - 16), clsa.CLSA_DEV_BAD_INDEX), (lambda: c.start.__setitem__(0, 1 << 40), clsa.CLSA_DEV_BAD_INDEX)):
        change()
        b = c.host()
        clsa.clsa_cache8_append(c.p, c.cache, None, k * 3, k, i, c.ws)
        a = c.host()
        assert c.status() == bit
        rows1 = c.row(1, np.arange(16, 30))
        keep = np.ones(c.rows, bool)
        keep[rows1] = False
        assert all((a[w][0][keep] == b[w][0][keep]).all() for w in range(3))
        clsa.clsa_clear_status(c.ws)
        c.seq_len.copy_(torch.tensor([20, 30], dtype=torch.int32))
        c.start.copy_(16 + 32 * torch.arange(2))


def test_append_bad_pages_are_skipped_and_flagged():
    c = Cache([40, 40], 20, 2, 64, 16, 16, seed=6)
    c.params()
    c.table[0, 1] = -3
    c.table[0, 2] = c.rows // 16
    k, i = randn(gen(1), 2, 20, 2, 128), randn(gen(2), 2, 20, 64)
    b = c.host()
    clsa.clsa_cache8_append(c.p, c.cache, None, k, k, i, c.ws)
    a = c.host()
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    keep = np.ones(c.rows, bool)
    keep[c.row(1, np.arange(16, 40))] = False
    assert all((a[w][0][keep] == b[w][0][keep]).all() for w in range(3))


# ------------------------------------------------------------------------------------------------------------ index scores
def check_scores(c, q, got, causal):
    code, sc = c.host()[2]
    vals = ref.values(code, sc, c.block)[:, 0]
    for b in range(c.B):
        n = c.lens[b]
        want, mag = ref.scores(f64(q[b]), vals[c.row(b, np.arange(n))])
        for t in range(c.T):
            v = n - c.T + t + 1 if causal else n
            g = got[b, t].cpu().double().numpy()
            assert (np.abs(g[:v] - want[t, :v]) <= 2.0 ** -16 * mag[t, :v] + 2.0 ** -149).all(), (b, t)
            assert np.isnan(g[v:]).all(), "scores past the visible prefix must not be written"


def run_scores(c, q, causal):
    stride = c.max_len + 5 if c.T <= 32 else (c.max_len + 63) // 64 * 64
    s = torch.full((c.B, c.T, stride), float("nan"), device=DEV)
    clsa.clsa_index_scores8(c.p, c.cache, q, s, stride, c.ws)
    return s


@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17, 32, 33, 130])
@pytest.mark.parametrize("d_idx,block,page,causal", [(128, 64, 0, 0), (64, 16, 16, 1), (128, 16, 64, 1), (64, 128, 128, 0), (128, 128, 0, 1)])
def test_index_scores(T, d_idx, block, page, causal):
    lens = [T, T + 1, 517 + T, 300]
    lens = [max(x, T) for x in lens]
    c = Cache(lens, T, 1, d_idx, block, page, seed=T + d_idx, pad_strides=page == 64)
    c.params(causal=causal)
    q = randn(gen(T), c.B, T, d_idx)
    check_scores(c, q, run_scores(c, q, causal), causal)
    assert c.status() == 0


def test_index_scores_ranges_of_queries_and_scales():
    """Queries from 2^-100 to 2^80, a zero query, elements 2^-20 of the row's largest; scale bytes over the whole range; bytes
    outside it read as the nearest allowed one."""
    c = Cache([200, 200, 200, 200], 2, 1, 128, 16, 0, seed=1, exps=(100, 150))
    c.params()
    q = randn(gen(5), 4, 2, 128)
    q[0, 0] *= 2.0 ** -100
    q[1, 0] *= 2.0 ** 80
    q[2, 0] = 0
    q[3, 0, ::2] *= 2.0 ** -20
    c.isc[3:9] = torch.tensor([0, 26, 27, 200, 30, 100], dtype=torch.uint8)
    check_scores(c, q, run_scores(c, q, 0), 0)


def test_index_scores_equal_keys_score_equally_and_bad_rows_are_flagged():
    c = Cache([700, 90], 1, 1, 128, 16, 16, seed=2)
    c.params()
    q = randn(gen(1), 2, 1, 128)
    rows = c.row(0, np.arange(700))
    c.idx[rows] = c.idx[rows[0]].clone()
    c.isc[rows // 16] = 120
    s = run_scores(c, q, 0)
    assert (s[0, 0, :700] == s[0, 0, 0]).all()
    c.table[0, 2] = -1
    c.table[0, 5] = 1 << 20
    s = run_scores(c, q, 0)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    assert (s[0, 0, 32:48] == 0).all() and (s[0, 0, 80:96] == 0).all() and (s[0, 0, 48:80] == s[0, 0, 0]).all()
    clsa.clsa_clear_status(c.ws)
    c.seq_len[1] = 701
    run_scores(c, q, 0)
    assert c.status() & clsa.CLSA_DEV_BAD_SEQLEN


def test_index_scores_bad_rows_of_a_chunk():
    c = Cache([300], 40, 1, 64, 16, 16, seed=2)
    c.params(causal=1)
    c.table[0, 1] = 1 << 22
    q = randn(gen(1), 1, 40, 64)
    s = run_scores(c, q, 1)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX and (s[0, :, 16:32] == 0).all() and torch.isfinite(s[0, 0, :261]).all()
    clsa.clsa_clear_status(c.ws)
    c.seq_len[0] = 39
    run_scores(c, q, 1)
    assert c.status() == clsa.CLSA_DEV_BAD_SEQLEN


@pytest.mark.parametrize("T", [1, 40])
def test_index_scores_of_a_sequence_off_the_scale_blocks_are_flagged(T):
    c = Cache([300, 300], T, 1, 64, 32, 0, seed=2)
    c.params(causal=1)
    c.start[0] += 16
    q = randn(gen(1), 2, T, 64)
    s = run_scores(c, q, 1)
    assert c.status() == clsa.CLSA_DEV_BAD_SCALE_BLOCK
    code, sc = c.host()[2]
    want, mag = ref.scores(f64(q[1]), ref.values(code, sc, 32)[c.row(1, np.arange(300)), 0])
    assert (np.abs(s[1, 0, :301 - T].cpu().double().numpy() - want[0, :301 - T]) <= 2.0 ** -16 * mag[0, :301 - T]).all()


# ------------------------------------------------------------------------------------------------------------ attention
def make_index(c, top_k, causal, seed, order="ascending", counts=None):
    r = np.random.default_rng(seed)
    idx, cnt = np.full((c.B, c.T, top_k), -1, np.int32), np.zeros((c.B, c.T), np.int32)
    for b in range(c.B):
        for t in range(c.T):
            v = c.lens[b] - c.T + t + 1 if causal else c.lens[b]
            m = min(top_k, v) if counts is None else min(counts[(b * c.T + t) % len(counts)], v, top_k)
            pick = r.permutation(v)[:m]
            idx[b, t, :m] = np.sort(pick) if order == "ascending" else pick
            cnt[b, t] = m
    return torch.from_numpy(idx).to(DEV), torch.from_numpy(cnt).to(DEV)


def check_attn(c, hq, q, idx, cnt, out, lse, sm_scale=128 ** -0.5, sample=None):
    (kc, ks), (vc, vs), _ = c.host()
    kv, vv = ref.values(kc, ks, c.block), ref.values(vc, vs, c.block)
    ih, ch = idx.cpu().numpy(), cnt.cpu().numpy()
    pairs = [(b, t) for b in range(c.B) for t in range(c.T)]
    for b, t in pairs if sample is None else [pairs[i] for i in np.random.default_rng(0).permutation(len(pairs))[:sample]]:
        rows = c.row(b, ih[b, t, :ch[b, t]])
        f = 2.0 ** (np.clip(vs[:, np.asarray(rows) // c.block].astype(np.float64), 27, 247).T - 127)
        o, l, tol, ltol = ref.attention(f64(q[b, t]), kv[rows], vv[rows], f, sm_scale)
        got = f64(out[b, t])
        assert (np.abs(got - o) <= tol).all(), (b, t, float((np.abs(got - o) - tol).max()))
        if lse is not None:
            gl = lse[b, t].cpu().double().numpy()
            if ch[b, t] == 0:
                assert np.isneginf(gl).all() and (got == 0).all()
            else:
                assert (np.abs(gl - l) <= ltol).all(), (b, t)


def run_attn(c, q, idx, cnt, hints=None, lse=True):
    out = torch.full(q.shape, float("nan"), dtype=BF16, device=DEV)
    l = torch.full(q.shape[:3], float("nan"), device=DEV) if lse else None
    clsa.clsa_sparse_attn8(c.p, c.cache, q, idx, cnt, out, l, hints, c.ws)
    return out, l


@pytest.mark.parametrize("hq,hkv", [(8, 1), (32, 8), (20, 4), (16, 1), (4, 4), (14, 2), (9, 1), (3, 3), (26, 2)])
@pytest.mark.parametrize("lens,T,top_k,block,page,causal", [
    ([1], 1, 1, 16, 0, 0), ([700, 31, 1, 257], 1, 256, 64, 0, 0), ([300, 40], 3, 37, 16, 16, 1), ([900] * 19, 1, 333, 128, 128, 0),
    ([90, 150], 40, 100, 32, 64, 1)])
def test_sparse_attn(hq, hkv, lens, T, top_k, block, page, causal):
    c = Cache(lens, T, hkv, 64, block, page, seed=hq + T, pad_strides=page == 64)
    c.params(hq=hq, top_k=top_k, causal=causal)
    q = randn(gen(1), c.B, T, hq, 128)
    idx, cnt = make_index(c, top_k, causal, 1, order="any" if T == 3 else "ascending")
    out, lse = run_attn(c, q, idx, cnt)
    check_attn(c, hq, q, idx, cnt, out, lse, sample=12)
    assert c.status() == 0
    again, lse2 = run_attn(c, q, idx, cnt)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert torch.equal(run_attn(c, q, idx, cnt, lse=False)[0], out)


def test_sparse_attn_long_rows_and_hints():
    """Rows that many warps and several blocks share, whole rows per warp, hints, and launches of different shapes on one
    workspace one after another."""
    big = Cache([5000, 4000, 2500], 1, 2, 64, 64, 64, seed=3)
    big.params(hq=8, top_k=2048)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device=DEV)
    shapes = [(big, 8, 2048, 0)]
    for T, hq, hkv, k in ((1, 16, 1, 1500), (70, 8, 4, 90), (300, 4, 2, 17)):
        c = Cache([1600] * 2, T, hkv, 64, 16, 0, seed=T)
        c.params(hq=hq, top_k=k, causal=int(T > 1))
        shapes.append((c, hq, k, int(T > 1)))
    for rnd in range(2):
        for c, hq, k, causal in shapes:
            c.ws = ws
            q = randn(gen(hq), c.B, c.T, hq, 128)
            idx, cnt = make_index(c, k, causal, 4, counts=[k, k - 1, 0, 1, k // 2])
            out, lse = run_attn(c, q, idx, cnt)
            check_attn(c, hq, q, idx, cnt, out, lse, sample=10)
            for h in (dict(reverse=1), dict(keep_rows=1), dict(only_q_pending=1), dict(reverse=1, keep_rows=1, only_q_pending=1)):
                torch.cuda.synchronize()
                o2, l2 = run_attn(c, q, idx, cnt, clsa.make_hints(**h))
                check_attn(c, hq, q, idx, cnt, o2, l2, sample=4)
            assert clsa.clsa_device_status(ws) == 0
    counters = ws[256:256 + 148 * 64].view(torch.int32)
    assert (counters == 0).all()


@pytest.mark.parametrize("T,hq,hkv,top_k,lens", [
    (223, 32, 8, 64, [700]),         # one whole unit per warp, and one that two warps share, in some blocks
    (148, 32, 8, 300, [500]),        # eight units per block, all shared by its twelve warps
    (190, 64, 8, 512, [800]),        # eight query heads per group
    (111, 128, 8, 256, [400]),       # sixteen: eight warps per block, six units of a block
    (130, 16, 8, 33, [300, 131]),    # a unit of two stages
    (52, 40, 8, 700, [900]),         # more units than blocks, too few for whole units: units that blocks share
    (401, 32, 8, 2048, [401]),       # short causal rows under a large budget: most stages are empty
])
def test_sparse_attn_ways_of_dealing_the_stages(T, hq, hkv, top_k, lens):
    """Chunks on either side of the rules that deal units to blocks and warps, walked both ways; every row is written."""
    c = Cache(lens, T, hkv, 64, 16, 16 if T % 2 else 0, seed=T)
    c.params(hq=hq, top_k=top_k, causal=1)
    q = randn(gen(T), c.B, T, hq, 128)
    idx, cnt = make_index(c, top_k, 1, 2, counts=[top_k, 0, top_k - 1, 1, top_k])
    out, lse = run_attn(c, q, idx, cnt)
    assert not out.isnan().any() and not lse.isnan().any()
    check_attn(c, hq, q, idx, cnt, out, lse, sample=40)
    again, lse2 = run_attn(c, q, idx, cnt)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    o2, l2 = run_attn(c, q, idx, cnt, clsa.make_hints(reverse=1, keep_rows=1))
    check_attn(c, hq, q, idx, cnt, o2, l2, sample=40)
    # an output row depends on its own query only: one query's rows changed leave all others bit-identical
    q2 = q.clone()
    q2[0, T // 2] = randn(gen(5), hq, 128)
    o3, l3 = run_attn(c, q2, idx, cnt)
    keep = torch.ones(c.B, T, dtype=torch.bool, device=DEV)
    keep[0, T // 2] = False
    assert torch.equal(o3[keep], out[keep]) and torch.equal(l3[keep], lse[keep])
    assert c.status() == 0
    assert (c.ws[256:256 + 148 * 64].view(torch.int32) == 0).all()


def test_sparse_attn_scales_far_apart():
    """Blocks whose V (and K) scales differ by many powers of two, a dominant logit on a block of tiny values, saturated codes."""
    c = Cache([512, 512], 1, 2, 64, 16, 0, seed=8)
    c.params(hq=8, top_k=512)
    r = np.random.default_rng(0)
    c.vs.copy_(torch.from_numpy(r.integers(27, 187, c.vs.shape).astype(np.uint8)))
    c.ks.copy_(torch.from_numpy(r.integers(90, 121, c.ks.shape).astype(np.uint8)))
    q = randn(gen(2), 2, 1, 8, 128)
    q[1] *= 2.0 ** -30
    idx, cnt = make_index(c, 512, 0, 1)
    out, lse = run_attn(c, q, idx, cnt)
    check_attn(c, 8, q, idx, cnt, out, lse)
    c.vs.fill_(27)  # every value tiny
    out, lse = run_attn(c, q, idx, cnt)
    check_attn(c, 8, q, idx, cnt, out, lse)
    c.vs.fill_(120)
    c.ks.fill_(119)
    c.k.view(torch.float8_e4m3fn)[int(c.start[0]) + 3].copy_((q[0, 0, :2].float() * 200).clamp(-448, 448).to(torch.float8_e4m3fn))  # one token takes all
    q *= 20
    out, lse = run_attn(c, q, idx, cnt)
    check_attn(c, 8, q, idx, cnt, out, lse)


def test_sparse_attn_reads_only_what_is_selected():
    """NaN codes everywhere else: unselected rows, index entries past the count, pad tokens of the last stage."""
    c = Cache([300, 300], 2, 2, 64, 16, 16, seed=8)
    c.params(hq=4, top_k=50, causal=1)
    idx, cnt = make_index(c, 50, 1, 3, counts=[50, 3, 0, 17])
    k0, v0 = c.k.clone(), c.v.clone()
    sel = np.concatenate([c.row(b, idx[b, t, :int(cnt[b, t])].cpu().numpy()) for b in range(2) for t in range(2)])
    c.k.fill_(127)
    c.v.fill_(127)
    c.k[sel], c.v[sel] = k0[sel], v0[sel]
    idx[idx == -1] = 12345
    q = randn(gen(2), 2, 2, 4, 128)
    out, lse = run_attn(c, q, idx, cnt)
    check_attn(c, 4, q, idx, cnt, out, lse)
    assert c.status() == 0
    c.v[sel[0], 0, 9] = 127  # a NaN that is selected reaches its dimension of its heads, and nothing else
    out, _ = run_attn(c, q, idx, cnt)
    assert torch.isnan(out[0, 0, :2, 9]).all() and int(torch.isnan(out[0, 0]).sum()) == 2


def test_sparse_attn_bad_entries_are_skipped_and_flagged():
    c = Cache([100, 120, 90], 1, 2, 64, 16, 16, seed=8)
    c.params(hq=8, top_k=40)
    idx, cnt = make_index(c, 40, 0, 3)
    q = randn(gen(2), 3, 1, 8, 128)
    bad = idx.clone()
    bad[0, 0, 5], bad[0, 0, 17], bad[1, 0, 39] = -4, 100, 2 ** 31 - 1
    out, lse = run_attn(c, q, bad, cnt)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    good = [np.delete(idx[0, 0].cpu().numpy(), [5, 17]), idx[1, 0, :39].cpu().numpy(), idx[2, 0].cpu().numpy()]
    i2, c2 = torch.full_like(idx, -1), torch.tensor([[38], [39], [40]], dtype=torch.int32, device=DEV)
    for b in range(3):
        i2[b, 0, :len(good[b])] = torch.from_numpy(good[b])
    check_attn(c, 8, q, i2, c2, out, lse)
    clsa.clsa_clear_status(c.ws)
    c.table[2, 1] = 1 << 21  # a page beyond the pool: its tokens are left out
    out, lse = run_attn(c, q, idx, cnt)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    keep = idx[2, 0].cpu().numpy()
    keep = keep[keep // 16 != 1]
    i2, c2 = idx.clone(), cnt.clone()
    i2[2, 0, :len(keep)], c2[2, 0] = torch.from_numpy(keep), len(keep)
    check_attn(c, 8, q, i2, c2, out, lse)
    clsa.clsa_clear_status(c.ws)
    c.seq_len[0], c.seq_len[1] = 0, 121
    cnt[2, 0] = 41
    c.table[2, 1] = 1
    out, lse = run_attn(c, q, idx, cnt)
    assert c.status() == clsa.CLSA_DEV_BAD_SEQLEN | clsa.CLSA_DEV_BAD_COUNT
    assert (out[:2] == 0).all() and torch.isneginf(lse[:2]).all() and torch.isfinite(out[2]).all()


def test_far_rows_of_a_large_cache():
    """Rows whose byte offsets exceed 32 bits, appended, scored and attended to."""
    rows, hkv = 5_000_000, 8
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB of device memory")
    block, B, T = 64, 2, 3
    nb = rows // block
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)  # noqa: E731
    k, v, i, ks, vs, isc = u8(rows, hkv, 128), u8(rows, hkv, 128), u8(rows, 128), u8(hkv, nb), u8(hkv, nb), u8(nb)
    cache = clsa.make_cache8(k=k, v=v, k_scale=ks, v_scale=vs, idx_k=i, idx_k_scale=isc, scale_block=block)
    start = torch.tensor([rows - 128, 0], dtype=torch.int64, device=DEV)
    n = torch.tensor([100, 100], dtype=torch.int32, device=DEV)
    g = gen(0)
    nk, nv, ni = (torch.cat([t, t]) for t in (randn(g, 1, 100, hkv, 128), randn(g, 1, 100, hkv, 128), randn(g, 1, 100, 128)))
    mk = lambda T, **kw: clsa.make_params(num_seqs=B, q_per_seq=T, num_q_heads=32, num_kv_heads=hkv, idx_dim=128, top_k=64, max_seq_len=128,  # noqa: E731
                                          sm_scale=0.1, seq_start=start, seq_len=n, num_cache_rows=rows, **kw)
    p = mk(100)
    ws = u8(64 << 20)
    clsa.clsa_cache8_append(p, cache, None, nk, nv, ni, ws)
    for t in (k, v, i):
        assert torch.equal(t[rows - 128:rows - 28], t[:100]) and int(t[:100].count_nonzero()) > t[:100].numel() * 0.9
    p = mk(T)
    qi, q = randn(g, 1, T, 128).expand(2, T, 128).contiguous(), randn(g, 1, T, 32, 128).expand(2, T, 32, 128).contiguous()
    s = torch.zeros((B, T, 128), device=DEV)
    clsa.clsa_index_scores8(p, cache, qi, s, 128, ws)
    assert torch.equal(s[0], s[1]) and float(s.abs().max()) > 1
    idx, cnt = torch.empty((B, T, 64), dtype=torch.int32, device=DEV), torch.empty((B, T), dtype=torch.int32, device=DEV)
    clsa.clsa_topk(p, s, 128, idx, cnt, ws)
    out = torch.empty((B, T, 32, 128), dtype=BF16, device=DEV)
    clsa.clsa_sparse_attn8(p, cache, q, idx, cnt, out, None, None, ws)
    # (the two sequences' rows are split over the warps at different places: equal up to rounding)
    assert clsa.clsa_device_status(ws) == 0 and torch.allclose(out[0].float(), out[1].float(), rtol=2.0 ** -6, atol=2.0 ** -8) and float(out.abs().max()) > 0.1


# ------------------------------------------------------------------------------------------------------------ together
def chain(c, spec, hid, ws, stream=None):
    """One step as a model runs it: new rows appended, queries normed and turned, scores, TopK, one layer's attention."""
    p = c.p
    clsa.clsa_cache8_append(p, c.cache, spec, hid["k"], hid["v"], hid["i"], ws, stream=stream)
    clsa.clsa_index_scores8(p, c.cache, hid["qi"], hid["scores"], hid["scores"].shape[-1], ws, stream=stream)
    clsa.clsa_topk(p, hid["scores"], hid["scores"].shape[-1], hid["idx"], hid["cnt"], ws, stream=stream)
    clsa.clsa_norm_rope(spec, hid["pos"], hid["q"], hid["qn"], stream=stream)
    clsa.clsa_sparse_attn8(p, c.cache, hid["qn"], hid["idx"], hid["cnt"], hid["out"], hid["lse"], clsa.make_hints(keep_rows=1, only_q_pending=1),
                           ws, stream=stream)


def make_hidden(c, hq, top_k, seed):
    g = gen(seed)
    d = dict(k=randn(g, c.B, c.T, c.hkv, 128), v=randn(g, c.B, c.T, c.hkv, 128), i=randn(g, c.B, c.T, c.d_idx), qi=randn(g, c.B, c.T, c.d_idx),
             q=randn(g, c.B, c.T, hq, 128))
    d["scores"] = torch.empty((c.B, c.T, (c.max_len + 63) // 64 * 64), device=DEV)
    d["idx"] = torch.empty((c.B, c.T, top_k), dtype=torch.int32, device=DEV)
    d["cnt"] = torch.empty((c.B, c.T), dtype=torch.int32, device=DEV)
    d["qn"], d["out"] = torch.empty_like(d["q"]), torch.empty_like(d["q"])
    d["lse"] = torch.empty((c.B, c.T, hq), device=DEV)
    d["pos"] = torch.cat([torch.arange(n - c.T, n, device=DEV, dtype=torch.int32) for n in c.lens])
    return d


@pytest.mark.parametrize("lens,T,page", [([2000, 77, 1300], 1, 64), ([900, 640], 5, 0), ([700], 50, 64)])
def test_a_step_of_all_operators(lens, T, page):
    hq, top_k = 8, 128
    c = Cache(lens, T, 2, 128, 64, page, seed=4)
    c.params(hq=hq, top_k=top_k, causal=int(T > 1))
    freq = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float().to(DEV)
    w = randn(gen(7), 128)
    spec = clsa.make_norm_rope(head_dim=128, norm=1, rot_dim=128, inv_freq=freq, q_weight=w, k_weight=w)
    d = make_hidden(c, hq, top_k, 5)
    chain(c, spec, d, c.ws)
    assert c.status() == 0
    check_norm_rope(d["q"].flatten(0, 1), d["qn"].flatten(0, 1), d["pos"], dict(norm=1, interleaved=0, inv_freq=freq), w, d["qn"].flatten(0, 1))
    d["scores"] = d["scores"].clone()
    code, sc = c.host()[2]
    vals = ref.values(code, sc, 64)[:, 0]
    for b in range(c.B):
        s, mag = ref.scores(f64(d["qi"][b]), vals[c.row(b, np.arange(c.lens[b]))])
        for t in range(T):
            v = c.lens[b] - T + t + 1 if T > 1 else c.lens[b]
            got = d["scores"][b, t, :v].cpu().double().numpy()
            assert (np.abs(got - s[t, :v]) <= 2.0 ** -16 * mag[t, :v]).all()
            m = min(top_k, v)
            assert int(d["cnt"][b, t]) == m
            want = np.sort(np.lexsort((np.arange(v), -got))[:m])
            np.testing.assert_array_equal(d["idx"][b, t, :m].cpu().numpy(), want)
    check_attn(c, hq, d["qn"], d["idx"], d["cnt"], d["out"], d["lse"], sample=20)


def test_two_captured_graphs_and_another_stream():
    """The step captured twice (two shapes, one workspace), replayed in turn and on new inputs, equal to eager calls; eager calls
    on a stream of their own."""
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().to(DEV)
    spec = clsa.make_norm_rope(head_dim=128, norm=1, rot_dim=64, interleaved=1, inv_freq=freq)
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=DEV)
    cs, ds, graphs = [], [], []
    for lens, T, hq in (([1500, 900], 1, 8), ([400, 333, 80], 4, 20)):
        c = Cache(lens, T, 2 if hq == 8 else 4, 64, 16, 16, seed=T)
        c.params(hq=hq, top_k=200, causal=int(T > 1))
        d = make_hidden(c, hq, 200, T)
        chain(c, spec, d, ws)  # warm-up
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            chain(c, spec, d, ws)
        cs.append(c), ds.append(d), graphs.append(gr)
    for rnd in range(3):
        for c, d, gr in zip(cs, ds, graphs):
            for n in ("k", "v", "i", "qi", "q"):
                d[n].copy_(randn(gen(100 * rnd + len(n)), *d[n].shape))
            start = [t.clone() for t in (c.k, c.v, c.idx, c.ks, c.vs, c.isc)]
            d["out"].fill_(float("nan"))
            gr.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in (d["out"], d["lse"], d["idx"], d["qn"], c.k, c.ks)]
            for t, s in zip((c.k, c.v, c.idx, c.ks, c.vs, c.isc), start):
                t.copy_(s)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            chain(c, spec, d, ws, stream=side if rnd else None)
            torch.cuda.synchronize()
            for a, b in zip(got, (d["out"], d["lse"], d["idx"], d["qn"], c.k, c.ks)):
                assert torch.equal(a, b)
    assert clsa.clsa_device_status(ws) == 0


def test_outputs_in_pinned_host_memory():
    c = Cache([300], 1, 2, 64, 16, 0, seed=4)
    c.params(hq=8, top_k=64)
    q = randn(gen(2), 1, 1, 8, 128)
    idx, cnt = make_index(c, 64, 0, 3)
    want, _ = run_attn(c, q, idx, cnt)
    host = torch.empty((1, 1, 8, 128), dtype=BF16).pin_memory()
    clsa.clsa_sparse_attn8(c.p, c.cache, q, idx, cnt, host, None, None, c.ws)
    torch.cuda.synchronize()
    assert torch.equal(host, want.cpu())


def test_the_native_marshalling_and_the_python_one_agree(monkeypatch):
    """The usual calls are taken by the native module; without it, and with layouts that only one of them takes, nothing differs."""
    from paper_2606_06467_b200 import cache8

    assert cache8._marshal is not None
    spec = clsa.make_norm_rope(head_dim=128, norm=1, q_weight=randn(gen(1), 128), k_weight=randn(gen(2), 128))
    taken, results = [], []
    for native in (True, False):
        if native:
            class Watch:
                def __getattr__(self, name):
                    def call(*a):
                        taken.append((name, getattr(real, name)(*a)))
                        return taken[-1][1]
                    return call
            real = cache8._marshal
            monkeypatch.setattr(cache8, "_marshal", Watch())
        else:
            monkeypatch.setattr(cache8, "_marshal", None)
        for T, lens in ((1, [300, 70]), (3, [300, 70])):
            c = Cache(lens, T, 2, 128, 64, 0, seed=8)
            c.params(hq=8, top_k=64, causal=int(T > 1))
            d = make_hidden(c, 8, 64, 9)
            # (the first of three tokens sees 68 keys of the shorter sequence; what lies behind is not written)
            # heads first: [B, T, H, D] as a view of [B, H, T, D], and of a fused projection
            d["q"] = d["q"].transpose(1, 2).contiguous().transpose(1, 2) if T == 1 else d["q"]
            fused = torch.cat([d["k"], d["v"]], 2)
            d["k"], d["v"] = fused[:, :, :2], fused[:, :, 2:]
            chain(c, spec, d, c.ws)
            # the fallback's own layouts and its addresses
            clsa.clsa_norm_rope(spec, None, d["q"].flatten(0, 1)[:1], d["qn"].flatten(0, 1)[:1])
            out = torch.empty_like(d["out"])
            clsa.clsa_sparse_attn8(c.p, c.cache, d["qn"], d["idx"].data_ptr(), d["cnt"], out, None, None, c.ws)
            torch.cuda.synchronize()
            assert c.status() == 0
            results.append([t.clone() for t in (d["qn"], d["scores"][:, :, :68], d["idx"], d["out"], d["lse"], out, c.k, c.ks, c.idx)])
        for wrong in (lambda: clsa.clsa_norm_rope(spec, d["pos"].long(), d["q"], d["qn"]),
                      lambda: clsa.clsa_norm_rope(spec, d["pos"][1:], d["q"], d["qn"]),
                      lambda: clsa.clsa_norm_rope(spec, d["pos"], d["q"].float(), d["qn"]),
                      lambda: clsa.clsa_norm_rope(spec, d["pos"], d["q"], None),
                      lambda: clsa.clsa_norm_rope(spec, d["pos"], d["q"], d["qn"][:, :, :4]),
                      lambda: clsa.clsa_cache8_append(c.p, c.cache, None, d["k"][:, :, :1], d["v"], None, c.ws),
                      lambda: clsa.clsa_cache8_append(c.p, c.cache, None, d["k"], None, None, c.ws),
                      lambda: clsa.clsa_index_scores8(c.p, c.cache, d["qi"].half(), d["scores"], d["scores"].shape[-1], c.ws),
                      lambda: clsa.clsa_index_scores8(c.p, c.cache, d["qi"], d["scores"], d["scores"].shape[-1], c.ws.cpu()),
                      lambda: clsa.clsa_sparse_attn8(c.p, c.cache, d["qn"], d["idx"].transpose(0, 1), d["cnt"], d["out"], None, None, c.ws)):
            with pytest.raises(ValueError):
                wrong()
        with pytest.raises(clsa.ClsaError):  # the C side's refusals
            clsa.clsa_sparse_attn8(c.p, c.cache, d["qn"], d["idx"], d["cnt"], d["out"], None, None, c.ws, 16)
    n = len(results) // 2
    for a, b in zip(results[:n], results[n:]):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
    usual = [name for name, status in taken if status == 0]
    assert set(usual) == {"norm_rope", "append", "scores", "attn"} and len(usual) >= 10
