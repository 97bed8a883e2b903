"""The 8-bit cache calls at the ends of what their header allows: starts far from zero or outside the row space, scales and
queries at both ends of their exponents, logits of any size, many sequences, long rows, empty batches, buffers of the wrong
size. Definitions and tolerances are those of tests/_cache8_ref.py where a test does not derive its own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import _cache8_ref as ref
import paper_2606_06467_b200 as clsa
from test_gpu_cache8 import BF16, DEV, Cache, check_attn, check_scores, f64, gen, make_index, randn, run_attn, run_scores

pytestmark = pytest.mark.gpu


def test_index_scores_of_a_far_start_under_a_loose_length_bound():
    """A start that together with max_seq_len passes 2^31: its own rows are scored, with their own scales."""
    rows, block, bound = 131072, 64, 0x7fff0000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB of device memory")
    g = gen(1)
    idx = (torch.randn((rows, 64), generator=g, device=DEV) * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    isc = torch.randint(110, 130, (rows // block,), generator=g, device=DEV, dtype=torch.uint8)
    cache = clsa.make_cache8(idx_k=idx, idx_k_scale=isc, scale_block=block)
    start, n = rows - 256, 200
    at, length = torch.tensor([start], dtype=torch.int64, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    p = clsa.make_params(num_seqs=1, num_q_heads=1, num_kv_heads=1, idx_dim=64, top_k=1, max_seq_len=bound, sm_scale=0.1,
                         seq_start=at, seq_len=length, num_cache_rows=rows)
    ws = torch.zeros(clsa.clsa_cache8_workspace_bytes(p, cache), dtype=torch.uint8, device=DEV)
    q = randn(g, 1, 1, 64)
    s = torch.empty((1, 1, bound), device=DEV)
    clsa.clsa_index_scores8(p, cache, q, s, bound, ws)
    vals = ref.values(idx.cpu().numpy()[:, None], isc.cpu().numpy()[None], block)[start:start + n, 0]
    want, mag = ref.scores(f64(q[0]), vals)
    assert (np.abs(s[0, 0, :n].cpu().double().numpy() - want[0]) <= 2.0 ** -16 * mag[0]).all()
    assert clsa.clsa_device_status(ws) == 0


@pytest.mark.parametrize("T", [1, 2, 40])
@pytest.mark.parametrize("d_idx", [64, 128])
@pytest.mark.parametrize("first", [-16, -48, -80])
def test_index_scores_of_rows_outside_the_row_space(T, d_idx, first):
    """A sequence that begins before row 0 and one that ends behind the last row: the rows that exist are scored, the others are
    rows of zeros, and both are flagged; without pages."""
    c = Cache([150, 150, 150], T, 1, d_idx, 16, 0, seed=T + d_idx)
    c.params()
    c.start[0], c.start[1] = first, c.rows - 16 * 5
    q = randn(gen(T), 3, T, d_idx)
    s = run_scores(c, q, 0)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    code, sc = c.host()[2]
    vals = ref.values(code, sc, 16)[:, 0]
    for b in range(3):
        rows = c.row(b, np.arange(150))
        there = (rows >= 0) & (rows < c.rows)
        want, mag = ref.scores(f64(q[b]), np.where(there[:, None], vals[np.clip(rows, 0, c.rows - 1)], 0.0))
        assert (np.abs(s[b, :, :150].cpu().double().numpy() - want) <= 2.0 ** -16 * mag).all(), b


def test_sparse_attn_of_rows_outside_the_row_space():
    """The same starts for attention: entries whose rows do not exist are left out and flagged."""
    c = Cache([150, 150, 150], 1, 2, 64, 16, 0, seed=3)
    c.params(hq=8, top_k=60)
    c.start[0], c.start[1] = -48, c.rows - 80
    q = randn(gen(2), 3, 1, 8, 128)
    idx, cnt = make_index(c, 60, 0, 1)
    out, lse = run_attn(c, q, idx, cnt)
    assert c.status() == clsa.CLSA_DEV_BAD_INDEX
    i2, c2 = torch.full_like(idx, -1), cnt.clone()
    for b in range(3):
        mine = idx[b, 0, :int(cnt[b, 0])].cpu().numpy()
        rows = c.row(b, mine)
        mine = mine[(rows >= 0) & (rows < c.rows)]
        i2[b, 0, :len(mine)], c2[b, 0] = torch.from_numpy(mine), len(mine)
    assert int(c2[0, 0]) < 60 and int(c2[1, 0]) < 60 and int(c2[2, 0]) == 60
    check_attn(c, 8, q, i2, c2, out, lse)


@pytest.mark.parametrize("T", [2, 40])
def test_index_scores_at_both_ends_of_the_exponents(T):
    """Largest scales under small queries, smallest scales under large ones: the scores are ordinary numbers."""
    c = Cache([200] * 4, T, 1, 128, 16, 0, seed=6)
    c.params()
    q = randn(gen(5), 4, T, 128)
    for b, (s, lo, hi) in enumerate(((-100, 244, 248), (120, 27, 30), (-20, 247, 248), (60, 27, 40))):
        q[b] *= 2.0 ** s
        at = int(c.start[b]) // 16
        c.isc[at:at + 13] = torch.randint(lo, hi, (13,), generator=gen(b), device=DEV, dtype=torch.uint8)
    assert int((c.idx.view(torch.float8_e4m3fn).float().abs() >= 256).sum()) > 100  # values of 2^128 and more among them
    s = run_scores(c, q, 0)
    assert torch.isfinite(s[:, :, :200]).all()
    check_scores(c, q, s, 0)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (8, 1), (16, 1)])
@pytest.mark.parametrize("power,lo,hi", [(-116, 240, 248), (97, 27, 35), (-116, 27, 248)])
def test_sparse_attn_at_both_ends_of_the_exponents(hq, hkv, power, lo, hi):
    """K scales at the ends of their range under queries that make ordinary logits of them."""
    c = Cache([300, 200], 1, hkv, 64, 16, 0, seed=hq)
    c.params(hq=hq, top_k=128, sm_scale=2.0 ** -10)
    c.ks.copy_(torch.randint(lo, hi, c.ks.shape, generator=gen(1), device=DEV, dtype=torch.uint8))
    q = (torch.randn((2, 1, hq, 128), generator=gen(2), device=DEV) * 2.0 ** power).to(BF16)
    q[1, 0, 1] = 0
    idx, cnt = make_index(c, 128, 0, 1)
    out, lse = run_attn(c, q, idx, cnt)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    check_attn(c, hq, q, idx, cnt, out, lse, sm_scale=2.0 ** -10)


@pytest.mark.parametrize("heads,top_k", [(2, 300), (1, 2048)])
@pytest.mark.parametrize("power", [0, 8, 16, 24, 60, 100])
def test_sparse_attn_one_token_takes_all(power, heads, top_k):
    """Logits of any size, one far above the rest: the output is that token's V row however large the logits are. (One weight
    is left: it and its sum differ by the weight's f16 rounding and the exponential's and the products' fp32 ones, 2^-10 at most,
    then one bf16 rounding.)"""
    c = Cache([2500, 2500], 1, heads, 64, 16, 0, seed=8, exps=(100, 140))
    c.params(hq=heads, top_k=top_k)
    c.ks.fill_(124)
    q = randn(gen(2), 2, 1, heads, 128) * 4
    idx, cnt = make_index(c, top_k, 0, 1)
    kf = c.k.view(torch.float8_e4m3fn)
    best = []
    for b in range(2):
        s = int(idx[b, 0, (77, 200)[b]])
        row = int(c.row(b, s))
        kf[row].copy_((q[b, 0].float() * 40).clamp(-448, 448).to(torch.float8_e4m3fn))
        best.append(row)
    q *= 2.0 ** power
    out, lse = run_attn(c, q, idx, cnt)
    (kc, ks), (vc, vs), _ = c.host()
    kv, vv = ref.values(kc, ks, 16), ref.values(vc, vs, 16)
    for b in range(2):
        rows = c.row(b, idx[b, 0, :top_k].cpu().numpy())
        for h in range(heads):
            x = kv[rows, h] @ f64(q[b, 0, h]) * 128 ** -0.5
            mag = 2.0 ** -16 * (np.abs(kv[rows, h]) @ np.abs(f64(q[b, 0, h]))).max() * 128 ** -0.5
            order = np.argsort(x)
            assert rows[order[-1]] == best[b] and x[order[-1]] - x[order[-2]] > 170 + 2 * mag  # 2^40 of V's scales and 2^-40 of weight are left
            v = vv[best[b], h]
            got = f64(out[b, 0, h])
            assert (np.abs(got - v) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(v) + 2.0 ** -149).all(), (b, h, float(np.nanmax(np.abs(got / np.where(v == 0, 1, v) - 1))))
            assert abs(float(lse[b, 0, h]) - x[order[-1]]) <= mag + 2.0 ** -20 * (abs(x[order[-1]]) + 128)


def test_sparse_attn_logits_far_below_zero():
    """A selected token whose logit lies far below -1e30 still is the one that there is."""
    c = Cache([64], 1, 1, 64, 16, 0, seed=8)
    c.params(hq=1, top_k=1)
    q = randn(gen(2), 1, 1, 1, 128) * 2.0 ** 100
    row = int(c.row(0, 9))
    c.k.view(torch.float8_e4m3fn)[row].copy_((q[0, 0].float() * -(2.0 ** -94)).clamp(-448, 448).to(torch.float8_e4m3fn))
    idx, cnt = torch.full((1, 1, 1), 9, dtype=torch.int32, device=DEV), torch.ones((1, 1), dtype=torch.int32, device=DEV)
    out, lse = run_attn(c, q, idx, cnt)
    assert float(lse) < -1e30
    check_attn(c, 1, q, idx, cnt, out, None)
    (kc, ks), (vc, vs), _ = c.host()
    v = ref.values(vc, vs, 16)[row, 0]
    assert (np.abs(f64(out[0, 0, 0]) - v) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(v)).all()


def test_queries_that_are_not_finite():
    """An infinity or a NaN in a query row shows in that row's results and in no others."""
    c = Cache([200, 200], 2, 2, 128, 16, 0, seed=5)
    c.params(hq=8, top_k=64)
    c.idx[(c.idx & 127) == 0] = 1  # no zero codes: an infinity times zero is a NaN
    qi = randn(gen(1), 2, 2, 128)
    clean = run_scores(c, qi, 0)
    qi[0, 0, 5], qi[1, 1, 9] = float("inf"), float("nan")
    s = run_scores(c, qi, 0)
    code, _ = c.host()[2]
    sign = np.where(code[c.row(0, np.arange(200)), 0, 5] & 128, -np.inf, np.inf)
    np.testing.assert_array_equal(s[0, 0, :200].cpu().numpy(), sign)
    assert torch.isnan(s[1, 1, :200]).all()
    assert torch.equal(s[0, 1, :200], clean[0, 1, :200]) and torch.equal(s[1, 0, :200], clean[1, 0, :200])
    q = randn(gen(2), 2, 2, 8, 128)
    idx, cnt = make_index(c, 64, 0, 1)
    clean, lse0 = run_attn(c, q, idx, cnt)
    q[0, 1, 3, 7], q[1, 0, 6, 100] = float("nan"), float("inf")
    out, lse = run_attn(c, q, idx, cnt)
    hit = torch.zeros((2, 2, 8), dtype=torch.bool, device=DEV)
    hit[0, 1, 3] = hit[1, 0, 6] = True
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[0, 1, 3])
    unit = hit.view(2, 2, 2, 4).any(-1, keepdim=True).expand(2, 2, 2, 4).reshape(2, 2, 8)  # heads that share a KV head share references
    assert torch.equal(out[~unit], clean[~unit]) and torch.equal(lse[~unit], lse0[~unit])
    q[hit] = 0
    out[hit], lse[hit] = run_attn(c, q, idx, cnt)[0][hit], run_attn(c, q, idx, cnt)[1][hit]
    check_attn(c, 8, q, idx, cnt, out, lse)


def test_index_scores_of_more_sequences_than_lengths_fit_in_shared_memory():
    lens = [1 + (7 * b) % 40 for b in range(2100)]
    c = Cache(lens, 1, 1, 64, 16, 0, seed=1, capacity=48)
    c.params()
    q = randn(gen(1), 2100, 1, 64)
    s = run_scores(c, q, 0)
    assert c.status() == 0
    code, sc = c.host()[2]
    vals = ref.values(code, sc, 16)[:, 0]
    got, qh, start = s[:, 0].cpu().double().numpy(), f64(q[:, 0]), c.start.cpu().numpy()
    for b in range(2100):
        want, mag = ref.scores(qh[b:b + 1], vals[start[b]:start[b] + lens[b]])
        assert (np.abs(got[b, :lens[b]] - want[0]) <= 2.0 ** -16 * mag[0]).all() and np.isnan(got[b, lens[b]:]).all(), b
    for change, bit in ((lambda: c.seq_len.__setitem__(2077, 49), clsa.CLSA_DEV_BAD_SEQLEN), (lambda: c.start.__setitem__(2099, 24), clsa.CLSA_DEV_BAD_SCALE_BLOCK)):
        change()
        again = run_scores(c, q, 0)
        assert c.status() == bit
        bad = 2077 if bit == clsa.CLSA_DEV_BAD_SEQLEN else 2099
        keep = [b for b in range(2100) if b != bad]
        assert torch.equal(again[keep].nan_to_num(7.0), s[keep].nan_to_num(7.0)) and torch.isnan(again[bad]).all()
        clsa.clsa_clear_status(c.ws)
        c.seq_len[2077] = lens[2077]


@pytest.mark.parametrize("hq", [4, 16])
def test_sparse_attn_of_a_row_over_more_than_32_blocks(hq):
    """One KV head's 27000 selected rows: the blocks' partials are joined in two rounds."""
    c = Cache([30000], 1, 1, 64, 64, 64, seed=2)
    c.params(hq=hq, top_k=27000)
    q = randn(gen(1), 1, 1, hq, 128)
    for counts in ([27000], [13001], [1]):
        idx, cnt = make_index(c, 27000, 0, 3, counts=counts)
        out, lse = run_attn(c, q, idx, cnt)
        check_attn(c, hq, q, idx, cnt, out, lse)
        o2, l2 = run_attn(c, q, idx, cnt, clsa.make_hints(reverse=1))
        check_attn(c, hq, q, idx, cnt, o2, l2)
    assert c.status() == 0


@pytest.mark.parametrize("extra", [1, 4, 5])
def test_index_scores_of_a_chunk_with_odd_strides(extra):
    """More than 32 query tokens, rows of scores that are not 32-byte aligned."""
    c = Cache([517, 300], 40, 1, 128, 64, 64, seed=4)
    c.params(causal=1)
    q = randn(gen(1), 2, 40, 128)
    stride = 520 + extra
    s = torch.full((2, 40, stride), float("nan"), device=DEV)
    clsa.clsa_index_scores8(c.p, c.cache, q, s, stride, c.ws)
    check_scores(c, q, s, 1)
    assert c.status() == 0


@pytest.mark.parametrize("T", [1, 300])
def test_append_of_indexer_keys_alone_leaves_k_and_v(T):
    c = Cache([300 + 7 * b for b in range(40)], T, 4, 64, 16, 16, seed=2)
    c.params()
    i = randn(gen(1), c.B, T, 64)
    before = c.host()
    clsa.clsa_cache8_append(c.p, c.cache, None, None, None, i, c.ws)
    after = c.host()
    for w in (0, 1):
        assert all((x == y).all() for x, y in zip(before[w], after[w]))
    code, sc = before[2]
    for b in range(c.B):
        ref.append(code, sc, lambda s, b=b: int(c.row(b, s)), c.lens[b], f64(i[b])[:, None], 16)
    np.testing.assert_array_equal(after[2][0], code)
    np.testing.assert_array_equal(after[2][1], sc)


@pytest.mark.parametrize("rot,inter", [(128, 0), (64, 0), (128, 1)])
@pytest.mark.parametrize("T,norm", [(1, 0), (1, 1), (70, 0), (70, 1)])
def test_append_with_a_scaled_rotation(rot, inter, T, norm):
    c = Cache([200, 131], T, 3, 64, 64, 0, seed=T)
    c.params()
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(DEV)
    spec = clsa.make_norm_rope(head_dim=128, norm=norm, eps=1e-6, rot_dim=rot, interleaved=inter, inv_freq=freq, rot_scale=1.375)
    k, v = randn(gen(1), 2, T, 3, 128), randn(gen(2), 2, T, 3, 128)
    code, sc = c.host()[0]
    clsa.clsa_cache8_append(c.p, c.cache, spec, k, v, None, c.ws)
    got, gsc = c.host()[0]
    for b in range(2):
        pos = np.arange(c.lens[b] - T, c.lens[b])
        x, mag = ref.norm_rope(f64(k[b]), pos, None, norm, np.float32(1e-6).astype(np.float64), freq.cpu().numpy(), inter, 1.375)
        done = ref.append(code, sc, lambda s, b=b: int(c.row(b, s)), c.lens[b], x, 64)
        rows = c.row(b, pos)
        for (home, h), e in done.items():
            mine = np.array([s for s in range(T) if home <= rows[s] < home + 64])
            err = np.abs(ref.E4M3[got[rows[mine], h]] * 2.0 ** e - x[mine, h])
            assert (err <= ref.half_step(x[mine, h], e) + 2.0 ** -19 * mag[mine, h]).all()
    np.testing.assert_array_equal(gsc, sc)


def test_empty_batches_do_nothing():
    freq = torch.ones(64, device=DEV)
    spec = clsa.make_norm_rope(head_dim=128, norm=1, rot_dim=128, inv_freq=freq)
    pos = torch.empty(0, dtype=torch.int32, device=DEV)
    for shape in ((0, 8, 128), (0, 4, 8, 128), (3, 0, 8, 128)):
        q = torch.empty(shape, dtype=BF16, device=DEV)
        clsa.clsa_norm_rope(spec, pos, q, q)
        clsa.clsa_norm_rope(spec, pos, torch.empty((*shape[:-2], 12, 128), dtype=BF16, device=DEV)[..., 2:10, :], q)  # another layout
        clsa.clsa_norm_rope(spec, pos, None, None, q, torch.empty_like(q))


@pytest.mark.parametrize("native", [True, False])
def test_buffers_that_are_too_small_are_refused(native, monkeypatch):
    from paper_2606_06467_b200 import cache8

    if native:
        assert cache8._marshal is not None
    else:
        monkeypatch.setattr(cache8, "_marshal", None)
    c = Cache([100, 90], 3, 2, 64, 16, 0, seed=1)
    c.params(hq=8, top_k=40)
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
    i32, f32, W = torch.int32, torch.float32, 128
    good = dict(q=z(2, 3, 8, 128), idx=z(2, 3, 40, dtype=i32), count=z(2, 3, dtype=i32), out=z(2, 3, 8, 128), lse=z(2, 3, 8, dtype=f32))
    attn = lambda p=c.p, cache=c.cache, ws=c.ws, n=None, **kw: clsa.clsa_sparse_attn8(  # noqa: E731
        p, cache, *[{**good, **kw}[x] for x in ("q", "idx", "count", "out", "lse")], None, ws, n)
    attn()
    for kw in (dict(q=z(2, 3, 7, 128)), dict(idx=z(2, 3, 39, dtype=i32)), dict(count=z(5, dtype=i32)), dict(out=z(2, 2, 8, 128)), dict(lse=z(47, dtype=f32)),
               dict(n=c.ws.numel() + 1)):
        with pytest.raises(ValueError):
            attn(**kw)
    qi, s = z(2, 3, 64), z(2, 3, W, dtype=f32)
    clsa.clsa_index_scores8(c.p, c.cache, qi, s, W, c.ws)
    clsa.clsa_index_scores8(c.p, c.cache, qi, s[:, :, :100], W, c.ws)  # a view of rows W apart
    for args in ((z(2, 2, 64), s, W), (qi, s, W + 30), (qi, z(2, 3, 99, dtype=f32), 100), (qi, s[:, :2], W)):
        with pytest.raises(ValueError):
            clsa.clsa_index_scores8(c.p, c.cache, *args, c.ws)
    # a cache of fewer rows, heads or dimensions than the params name
    new, ni = z(2, 3, 2, 128), z(2, 3, 64)
    clsa.clsa_cache8_append(c.p, c.cache, None, new, new, ni, c.ws)
    for kw in (dict(num_cache_rows=c.rows + 1), dict(num_kv_heads=4), dict(idx_dim=128)):
        p = c.params(hq=8, top_k=40, **kw)
        with pytest.raises(ValueError):
            clsa.clsa_cache8_append(p, c.cache, None, z(2, 3, p.num_kv_heads, 128), z(2, 3, p.num_kv_heads, 128), z(2, 3, p.idx_dim), c.ws)
        with pytest.raises(ValueError):
            attn(p=p) if "idx_dim" not in kw else clsa.clsa_index_scores8(p, c.cache, z(2, 3, 128), s, W, c.ws)
    assert c.status() == 0
