"""clsa_dense_attn and clsa_dense_attn8 on a GPU against the definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import __graft_entry__ as entry

entry._load_build_module().build()

import _layer_ref as ref
import paper_2606_06467_b200 as clsa

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SM = 128 ** -0.5


class Problem:
    """Sequences of the given lengths in a cache whose other rows are poison (NaN, or the NaN code)."""

    def __init__(self, lens, hq, hkv, T=1, eight=False, page=0, block=16, causal=0, window=0, layout="rows", seed=0, max_len=None, shift=0,
                 poison=True, first_row=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.g, self.T, self.hq, self.hkv, self.eight, self.page, self.block = g, T, hq, hkv, eight, page, block
        self.causal, self.window, self.lens = causal, window, list(lens)
        B = len(self.lens)
        longest = max(max(self.lens), 1)
        unit = max(page, block, 16)
        room = -(-longest // unit) * unit
        spare = 3 * unit  # rows of nobody
        self.rows = first_row + B * room + spare
        self.start = self.table = None
        if page:
            pages = self.rows // page
            order = torch.randperm(B * (room // page), generator=g, device=DEV).to(torch.int32) + first_row // page
            self.table = order.view(B, room // page).contiguous()
            self.rows = pages * page
        else:
            self.start = torch.tensor([first_row + b * room + shift for b in range(B)], dtype=torch.int64, device=DEV)
        self.seq_len = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        dtype = torch.uint8 if eight else torch.bfloat16
        shape = (self.rows, hkv, 128)

        def cache():
            if layout == "rows":
                return torch.empty(shape, dtype=dtype, device=DEV)
            if layout == "fused":  # a slice of wider rows
                return torch.empty((self.rows, 2 * hkv + 1, 128), dtype=dtype, device=DEV)[:, 1:hkv + 1]
            return torch.empty((hkv, self.rows, 128), dtype=dtype, device=DEV).transpose(0, 1)  # heads outermost

        self.k, self.v = cache(), cache()
        if first_row == 0:
            for t in (self.k, self.v):
                t.copy_(torch.full((1,), 0x7f if eight else math.nan, device=DEV).to(dtype).expand(shape))
        for b, n in enumerate(self.lens):
            if n > 0:
                r = self.row_of(b, torch.arange(n, device=DEV))
                for t in (self.k, self.v):
                    x = torch.randn((n, hkv, 128), generator=g, device=DEV)
                    t[r] = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if eight else x.to(torch.bfloat16)
        if eight:
            blocks = -(-self.rows // block)
            self.ks = torch.randint(118, 122, (hkv, blocks), generator=g, device=DEV, dtype=torch.uint8)
            self.vs = torch.randint(116, 124, (hkv, blocks), generator=g, device=DEV, dtype=torch.uint8)
        self.q = torch.randn((B, T, hq, 128), generator=g, device=DEV).to(torch.bfloat16)
        self.out = torch.full((B, T, hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((B, T, hq), 7.0, dtype=torch.float32, device=DEV)
        self.max_len = max_len or max(longest, T)
        self.table_ = self.table
        self.make()

    def make(self):
        own = {} if self.eight else dict(k_cache=self.k, v_cache=self.v)
        self.p = clsa.make_params(num_seqs=len(self.lens), q_per_seq=self.T, num_q_heads=self.hq, num_kv_heads=self.hkv, idx_dim=128, top_k=1,
                                  causal=self.causal, max_seq_len=self.max_len, sm_scale=SM, seq_start=self.start, seq_len=self.seq_len,
                                  num_cache_rows=self.rows, block_table=self.table_, block_size=self.page, **own)
        self.cache = clsa.make_cache8(k=self.k, v=self.v, k_scale=self.ks, v_scale=self.vs, scale_block=self.block) if self.eight else None
        self.ws = torch.zeros(clsa.clsa_dense_workspace_bytes(self.p), dtype=torch.uint8, device=DEV)
        self.ws[256 + 16 * 1024:] = 0xff  # scratch needs no clearing

    def row_of(self, b, pos):
        if self.table is None:
            return self.start[b] + pos
        return self.table[b].long()[pos // self.page] * self.page + pos % self.page

    def run(self, q=None, out=None, lse="own", ws=None, stream=None):
        a = (self.window, self.q if q is None else q, self.out if out is None else out, self.lse if lse == "own" else lse,
             self.ws if ws is None else ws)
        if self.eight:
            clsa.clsa_dense_attn8(self.p, self.cache, *a, stream=stream)
        else:
            clsa.clsa_dense_attn(self.p, *a, stream=stream)

    def want(self, lens=None, exists=None):
        table = ref.e4m3_table(DEV) if self.eight else None

        def side(t, scale, b, n):
            r = self.row_of(b, torch.arange(n, device=DEV))
            ok = torch.ones(n, dtype=torch.bool, device=DEV) if exists is None else exists(b, n)
            r = torch.where(ok, r, 0)
            if not self.eight:
                return t[r].double(), ok, None
            f = torch.exp2(scale[:, r // self.block].double() - 127).T
            return table[t[r].long()] * f[..., None], ok, f

        lens = self.lens if lens is None else lens
        cols = self.T * (self.hq // self.hkv)
        eps = 2.0 ** -11 if self.eight else 2.0 ** -16 if cols <= 32 else 2.0 ** -8
        k_of = lambda b: side(self.k, getattr(self, "ks", None), b, int(lens[b]))[:2]  # noqa: E731
        v_of = lambda b: side(self.v, getattr(self, "vs", None), b, int(lens[b]))[::2]  # noqa: E731
        return ref.dense(self.q, k_of, v_of, lens, self.T, self.hq // self.hkv, SM, self.causal, self.window, eps)

    def check(self, status=0, **kw):
        self.run()
        torch.cuda.synchronize()
        assert clsa.clsa_device_status(self.ws) == status
        out, lse, tol, ltol = self.want(**kw)
        ref.check_close(self.lse, lse, ltol, "lse")
        ref.check_close(self.out, out, tol, "out")


HEADS = [(8, 1), (32, 8), (20, 4), (16, 1), (4, 4), (14, 2), (40, 5), (1, 1), (48, 3), (64, 16)]


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_one_token_over_ragged_lengths(heads, eight):
    Problem([1, 0, 15, 16, 17, 333, 1, 2050], *heads, eight=eight, seed=1).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,heads", [(2, (8, 1)), (2, (32, 8)), (3, (20, 4)), (5, (4, 4)), (8, (32, 8)), (7, (14, 2)), (16, (16, 1)), (32, (8, 8)), (32, (16, 1)), (4, (40, 5)), (9, (8, 2))], ids=str)
@pytest.mark.parametrize("causal", [0, 1])
def test_several_tokens(T, heads, causal, eight):
    Problem([T, 700, T + 1, 64, 131], *heads, T=T, causal=causal, eight=eight, page=16 if T % 2 else 64, block=16, seed=T).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 512, 5000])
@pytest.mark.parametrize("T,causal", [(1, 0), (1, 1), (4, 1), (4, 0)])
def test_windows(window, T, causal, eight):
    Problem([T, 17, 600, 1025, 40], 20, 4, T=T, causal=causal, window=window, eight=eight, page=32, block=32, seed=window).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["fused", "heads"])
@pytest.mark.parametrize("page,block", [(0, 128), (128, 64), (4096, 16)])
def test_strides_and_pages(layout, page, block, eight):
    Problem([900, 4100, 31], 12, 2, layout=layout, page=page, block=block, eight=eight, seed=3).check()


@pytest.mark.parametrize("shift", [1, 5, 8, 63])
def test_sequences_that_start_anywhere(shift):
    Problem([100, 1000, 1], 8, 2, shift=shift, block=64, seed=shift).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_non_causal_queries_outside_the_cache(eight):
    """Cross attention: fewer cached states than queries, none at all included."""
    Problem([3, 0, 1, 40], 8, 2, T=8, eight=eight, seed=5).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("count,T", [(700, 1), (300, 3)])
def test_many_sequences(count, T, eight):
    Problem([T + (7 * i) % 61 for i in range(count)], 8, 2, T=T, causal=1, eight=eight, page=16, seed=6).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[40000], [9000, 30000, 5], [16384] * 4])
def test_long_sequences_split_over_blocks(lens, eight):
    Problem(lens, 16, 4, eight=eight, page=64, block=64, seed=7).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("T,heads", [(1, (32, 8)), (1, (8, 1)), (3, (20, 4)), (8, (32, 8)), (16, (16, 2)), (32, (16, 1))], ids=str)
@pytest.mark.parametrize("lens", [[1], [600, 0, 17], [0, 0, 0, 5000], [33] * 24, "24", "129", "300"], ids=str)
def test_stretches_of_the_list(lens, T, heads, eight):
    """Where sequences may be long (and are not) the work is cut into stretches, a unit's ends counted: of single granules, of units' ends only."""
    if isinstance(lens, str):
        g = torch.Generator()
        g.manual_seed(int(lens))
        lens = [0 if n < 60 else n for n in torch.randint(0, 700, (int(lens),), generator=g).tolist()]
    Problem(lens, *heads, T=T, eight=eight, max_len=1 << 20, seed=len(lens)).check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("T,heads", [(1, (32, 8)), (4, (20, 4)), (8, (16, 2))], ids=str)
def test_stretches_of_paged_sequences(page, T, heads, eight):
    w = Problem([900, 8, 1300, 77, 513, 16, 31], *heads, T=T, eight=eight, page=page, causal=1)
    pad = torch.full((7, (1 << 20) // page - w.table.shape[1]), -1, dtype=torch.int32, device=DEV)  # pages that no length reaches
    w.table_ = torch.cat([w.table, pad], 1).contiguous()
    w.max_len = 1 << 20
    w.make()
    w.check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_numbers_that_are_not_finite_stay_where_they_are_seen(eight):
    """V (and K) of the newest tokens not finite: the queries in front of them do not see them."""
    for T, heads, window in ((4, (8, 2), 0), (8, (32, 8), 0), (3, (5, 1), 6), (8, (8, 8), 4)):
        p = Problem([70, 50, 161], *heads, T=T, causal=1, window=window, eight=eight, seed=8)
        for b in range(3):
            n = p.lens[b]
            last = p.row_of(b, torch.tensor([n - 1, n - 2], device=DEV))
            bad = torch.tensor([0x7f, 0xff], dtype=torch.uint8, device=DEV) if eight else torch.tensor([math.inf, math.nan], device=DEV, dtype=torch.bfloat16)
            p.v[last[0], 0, 3:9] = bad[0]
            p.v[last[1], -1, 100] = bad[1]
            if window:  # .. and of a token that the first query's window alone reaches
                old = p.row_of(b, torch.tensor([n - T - window + 1], device=DEV))
                p.v[old[0], 0, 60] = bad[1]
        p.run()
        torch.cuda.synchronize()
        out, lse, tol, ltol = p.want()
        assert torch.isnan(out).any() or torch.isinf(out).any()
        ref.check_close(p.lse, lse, ltol, "lse")
        got = p.out.double()
        strange = ~torch.isfinite(out)
        assert torch.equal(~torch.isfinite(got), strange)
        ref.check_close(torch.where(strange, 0.0, got), torch.where(strange, 0.0, out), torch.where(strange, 0.0, tol), "out")


def test_logits_that_are_not_finite():
    """A key whose logit is -inf has weight 0; a query whose keys all are yields zeros; +inf and NaN give NaN."""
    p = Problem([40, 1, 20, 20], 2, 2, seed=9)
    p.q[:] = 1.0
    p.k[p.row_of(0, torch.tensor([7], device=DEV))] = -math.inf
    p.k[p.row_of(1, torch.tensor([0], device=DEV))] = -math.inf
    p.k[p.row_of(2, torch.tensor([3], device=DEV))] = math.inf
    p.k[p.row_of(3, torch.tensor([3], device=DEV)), 0, 5] = math.nan
    p.run()
    out, lse, tol, ltol = p.want()
    assert (p.out[1] == 0).all() and (p.lse[1] == -math.inf).all()
    assert torch.isnan(p.out[2]).all() and torch.isnan(p.out[3, :, 0]).all()
    ref.check_close(p.out[0], out[0], tol[0], "out")
    ref.check_close(p.out[3, :, 1], out[3, :, 1], tol[3, :, 1], "out")


@pytest.mark.parametrize("size", [1e-3, 30.0, 1e4])
def test_logits_of_any_size(size):
    p = Problem([500, 77], 16, 4, seed=10)
    p.q.copy_((p.q.float() * size).to(torch.bfloat16))
    p.check()


def test_logits_that_grow_and_fall():
    """The reference moves many times, and then never again."""
    for flip in (False, True):
        p = Problem([3000], 8, 2, seed=11)
        r = p.row_of(0, torch.arange(3000, device=DEV))
        ramp = torch.linspace(-20, 20, 3000, device=DEV)
        p.k[r] = (p.q[0, 0, ::4].float()[None] * (ramp.flip(0) if flip else ramp)[:, None, None] / 10).to(torch.bfloat16)
        p.check()


def test_scales_far_apart():
    """8-bit blocks of exponents at both ends beside one another: neither the denominators nor the numerators underflow."""
    p = Problem([200, 64], 8, 2, eight=True, seed=12)
    p.vs[:, ::2] = 27
    p.vs[:, 1::2] = 100
    p.ks[:, ::3] = 40
    p.check()
    p.vs[:] = 27
    p.check()


@pytest.mark.parametrize("heads", [(8, 1), (20, 4), (8, 8)], ids=str)
@pytest.mark.parametrize("offset,gap,page", [(0, 0, 0), (1, 2, 0), (2, 1, 16), (3, 4, 16), (3, 0, 64), (1, 3, 32)])
def test_scale_bytes_at_any_address(offset, gap, page, heads):
    """Heads' scale bytes at every place of a 4-byte word, the last head's last one at the end of its memory."""
    w = Problem([1, 17, 333, 2049, 640], *heads, T=2, eight=True, page=page, block=16, seed=offset + 5)
    for name in ("ks", "vs"):
        of = getattr(w, name)
        stride = of.shape[1] + gap
        room = torch.full((offset + (heads[1] - 1) * stride + of.shape[1],), 255, dtype=torch.uint8, device=DEV)
        there = room.as_strided(of.shape, (stride, 1), offset)
        there.copy_(of)
        setattr(w, name, there)
    w.make()
    w.check()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_bad_pages_and_rows(eight):
    p = Problem([200, 90, 33], 8, 2, T=2, causal=1, eight=eight, page=16, seed=13)
    p.table_ = p.table.clone()
    p.table_[0, 3], p.table_[0, 12], p.table_[1, 0], p.table_[2, 2] = -1, p.rows // 16, -(2 ** 31), 2 ** 31 - 1
    p.make()

    def exists(b, n):
        page = torch.arange(n, device=DEV) // 16
        t = p.table_[b].long()[page]
        return (t >= 0) & (t < p.rows // 16)

    p.check(status=clsa.CLSA_DEV_BAD_INDEX, exists=exists)
    # a bad page behind the sequence, or in front of its window, is nobody's business
    p.table_ = p.table.clone()
    p.window = 20
    p.table_[0, 3] = -1
    p.table_[2, 3:] = -1
    p.make()
    p.check()


def test_rows_outside_the_row_space():
    p = Problem([100, 60], 8, 2, seed=14)
    p.start[1] = p.rows - 37  # its last rows do not exist
    p.k[p.rows - 37:], p.v[p.rows - 37:] = 0.5, 0.25
    exists = lambda b, n: p.start[b] + torch.arange(n, device=DEV) < p.rows  # noqa: E731
    p.row_of = lambda b, pos: (p.start[b] + pos).clamp(max=p.rows - 1)
    p.check(status=clsa.CLSA_DEV_BAD_INDEX, exists=exists)
    p.start[1] = -9  # nor do its first
    p.k[:60], p.v[:60] = p.k[200:260].nan_to_num(0.25), p.v[200:260].nan_to_num(0.5)
    clsa.clsa_clear_status(p.ws)
    p.row_of = lambda b, pos: (p.start[b] + pos).clamp(min=0)
    p.start[0] = 128
    p.k[128:228], p.v[128:228] = 0.125, 0.5
    p.check(status=clsa.CLSA_DEV_BAD_INDEX, exists=lambda b, n: p.start[b] + torch.arange(n, device=DEV) >= 0)
    for far in (1 << 40, -(1 << 40), (1 << 31) + 3):
        p.start[1] = far
        clsa.clsa_clear_status(p.ws)
        p.row_of = lambda b, pos: (p.start[b] + pos).clamp(0, p.rows - 1)
        p.check(status=clsa.CLSA_DEV_BAD_INDEX, exists=lambda b, n: torch.full((n,), b == 0, device=DEV))


def test_bad_lengths_and_starts():
    p = Problem([50, 60, 70, 80], 8, 2, T=2, causal=1, seed=15, max_len=80)
    p.seq_len[:3] = torch.tensor([1, 81, -5], dtype=torch.int32)
    p.check(status=clsa.CLSA_DEV_BAD_SEQLEN, lens=[0, 0, 0, 80])
    p = Problem([50, 60], 8, 2, eight=True, seed=16)
    p.start[0] += 1
    p.check(status=clsa.CLSA_DEV_BAD_SCALE_BLOCK, lens=[0, 60])


def test_rows_beyond_4_gib():
    for eight in (False, True):
        first = (1 << 32) // (1024 if eight else 2048) + 4096
        p = Problem([1000, 77], 32, 8, eight=eight, page=64, block=64, first_row=first, seed=17)
        p.check()
        del p
        torch.cuda.empty_cache()


def test_equal_to_sparse_attention_over_everything():
    p = Problem([900, 1500], 32, 8, seed=18)
    p.run()
    full = clsa.make_params(num_seqs=2, num_q_heads=32, num_kv_heads=8, idx_dim=128, top_k=1536, max_seq_len=1536, sm_scale=SM, seq_start=p.start,
                            seq_len=p.seq_len, k_cache=p.k, v_cache=p.v, num_cache_rows=p.rows)
    idx = torch.arange(1536, dtype=torch.int32, device=DEV).repeat(2, 1, 1)
    count = p.seq_len.view(2, 1).clone()
    ws = torch.zeros(clsa.clsa_workspace_bytes(full), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(p.out), torch.empty_like(p.lse)
    clsa.clsa_sparse_attn(full, p.q, idx, count, out, lse, ws)
    _, _, tol, ltol = p.want()
    assert ((p.out.double() - out.double()).abs() <= 2 * tol + 2.0 ** -7 * out.double().abs().amax()).all()
    assert ((p.lse - lse).abs() <= 2.0 ** -7).all()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_two_parts_of_a_context_join(eight):
    """By their log-sum-exps: the whole is what its two halves give together."""
    p = Problem([640], 8, 2, eight=eight, seed=19)
    p.run()
    whole, lse = p.out.double(), p.lse.double()
    parts = []
    for lo, n in ((0, 256), (256, 384)):
        p.start[0] += lo
        p.seq_len[0] = n
        p.run()
        parts.append((p.out.double(), p.lse.double()))
        p.start[0] -= lo
    both = torch.logaddexp(parts[0][1], parts[1][1])
    joined = sum(o * torch.exp(l - both)[..., None] for o, l in parts)
    assert (both - lse).abs().max() < 1e-4
    assert ((joined - whole).abs() <= 3 * 2.0 ** -8 * (whole.abs() + sum(o.abs() for o, _ in parts)) + 1e-6).all()


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
def test_streams_graphs_and_repeats(eight):
    p = Problem([3000, 20, 511], 20, 4, T=2, causal=1, eight=eight, page=16, seed=20)
    p.run()
    first, lse = p.out.clone(), p.lse.clone()
    for _ in range(3):
        p.out.fill_(0)
        p.run()
        assert torch.equal(first.view(torch.int16), p.out.view(torch.int16)) and torch.equal(lse, p.lse)
    p.run(lse=None)
    # another stream, with a workspace of its own, beside this one
    other, out2, ws2 = torch.cuda.Stream(), torch.zeros_like(p.out), torch.zeros_like(p.ws)
    other.wait_stream(torch.cuda.current_stream())
    lse2 = torch.zeros_like(p.lse)
    for _ in range(5):
        p.run()
        p.run(out=out2, lse=lse2, ws=ws2, stream=other)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), out2.view(torch.int16)) and torch.equal(lse, lse2)
    # captured twice on one workspace, replayed with other lengths in between
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
        p.run(out=out2, lse=lse2)
    out2.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), out2.view(torch.int16)) and torch.equal(lse, p.lse)
    p.seq_len.copy_(torch.tensor([2, 20, 300], dtype=torch.int32))
    p.lens = [2, 20, 300]
    graph.replay()
    torch.cuda.synchronize()
    out, l, tol, ltol = p.want()
    ref.check_close(out2, out, tol, "out")
    ref.check_close(lse2, l, ltol, "lse")
    assert clsa.clsa_device_status(p.ws) == 0


def test_outputs_in_pinned_host_memory():
    p = Problem([900, 40], 8, 2, seed=21)
    p.run()
    out, lse = torch.zeros(p.out.shape, dtype=torch.bfloat16).pin_memory(), torch.zeros(p.lse.shape).pin_memory()
    p.run(out=out, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), p.out.cpu().view(torch.int16)) and torch.equal(lse, p.lse.cpu())
