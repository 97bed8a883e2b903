"""The 8-bit cache operators as cases with inputs, a plain form, a 64-bit definition and the library's own calls.

Four operators that belong together: per-head norms and rotation of queries and keys (`clsa_norm_rope`), the append of new
rows to a cache of e4m3 codes with a power-of-two scale per block of tokens and head (`clsa_cache8_append`), index scores over
such a cache (`clsa_index_scores8`) and sparse attention over its selected rows (`clsa_sparse_attn8`).

`listed()` and `draw()` give cases, `prepare()` the tensors a serving program has in hand, `run()` one pass (plain torch, or
the library's calls where `own` is true), `exact()` the same outputs in 64 bits, `work()` the bytes and operations of a pass.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
EXP_MIN, EXP_MAX = -100, 120  # exponents a scale may take


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # the new token of each of 16 sequences: one decode step's queries and keys, half-split rotation, far positions
        dict(name="norm_rope decode 16", op="norm_rope", tokens=16, hq=32, hk=8, head_dim=128, rot=128, interleaved=False,
             fused=True, padded=0, max_pos=131072),
        # an odd number of packed tokens with padded rows between them, the 20/4 head layout, half of each head rotated
        dict(name="norm_rope ragged 777", op="norm_rope", tokens=777, hq=20, hk=4, head_dim=128, rot=64, interleaved=True,
             fused=True, padded=9, max_pos=32768),
        # a prefill chunk of 4096 tokens
        dict(name="norm_rope chunk 4096", op="norm_rope", tokens=4096, hq=32, hk=8, head_dim=128, rot=128, interleaved=False,
             fused=True, padded=0, max_pos=135168),
        # the append of a decode step: one token in each of 16 sequences, K normed and rotated in the same pass
        dict(name="append decode 16", op="append", seqs=16, q_per_seq=1, hkv=8, idx_dim=128, scale_block=64, page=0,
             before_min=100, before=1000, norm=True, rot=128),
        # the last 4096 tokens of a long prompt into a paged cache
        dict(name="append chunk 4096", op="append", seqs=1, q_per_seq=4096, hkv=8, idx_dim=128, scale_block=64, page=64,
             before_min=4137, before=4137, norm=True, rot=128),
        # odd chunks that begin and end inside blocks, four KV heads, keys taken as they are (no rotation)
        dict(name="append odd 333", op="append", seqs=7, q_per_seq=333, hkv=4, idx_dim=64, scale_block=16, page=0,
             before_min=0, before=219, norm=False, rot=0),
        # the headline decode step's scan: 16 sequences of 131072 indexer keys
        dict(name="scores decode 128K", op="scores", seqs=16, q_per_seq=1, ctx=131072, ctx_min=131072, idx_dim=128,
             scale_block=64, page=0, causal=False),
        # four drafted tokens per sequence, ragged lengths in a paged cache, narrow indexer keys
        dict(name="scores draft ragged", op="scores", seqs=24, q_per_seq=4, ctx=32768, ctx_min=1024, idx_dim=64,
             scale_block=16, page=64, causal=True),
        # a prefill chunk's scores
        dict(name="scores chunk 1024", op="scores", seqs=1, q_per_seq=1024, ctx=33792, ctx_min=33792, idx_dim=128,
             scale_block=64, page=0, causal=True),
        # the smallest decode: one sequence, one KV head
        dict(name="attn tiny", op="attn", seqs=1, q_per_seq=1, ctx=4096, ctx_min=4096, hq=8, hkv=1, top_k=256,
             scale_block=64, page=0, causal=False, empty=0),
        # one layer of the headline decode step
        dict(name="attn decode 128K", op="attn", seqs=16, q_per_seq=1, ctx=131072, ctx_min=131072, hq=32, hkv=8,
             top_k=2048, scale_block=64, page=0, causal=False, empty=0),
        # one layer of a prefill chunk over a paged cache, every query with its own selection, three of them with none
        dict(name="attn chunk 512", op="attn", seqs=1, q_per_seq=512, ctx=33280, ctx_min=33280, hq=32, hkv=8, top_k=2048,
             scale_block=64, page=64, causal=True, empty=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "append", "scores", "attn"])
    hq, hkv = rng.choice([(8, 1), (32, 8), (20, 4), (16, 1), (4, 4), (14, 2)])
    block = rng.choice([16, 32, 64, 128])
    page = rng.choice([0, block, 2 * block])
    if op == "norm_rope":
        dim = rng.choice([64, 128, 128, 256])
        tokens = _log_int(rng, 1, 4096)
        return dict(op=op, tokens=tokens, hq=hq, hk=hkv, head_dim=dim, rot=rng.choice([0, 32, dim // 2, dim]),
                    interleaved=rng.random() < 0.5, fused=rng.random() < 0.5, padded=min(tokens - 1, rng.randrange(5)),
                    max_pos=_log_int(rng, 64, 1 << 20))
    if op == "append":
        seqs = _log_int(rng, 1, 64)
        before = _log_int(rng, 1, 2000)
        norm = rng.random() < 0.6
        return dict(op=op, seqs=seqs, q_per_seq=_log_int(rng, 1, max(1, 4096 // seqs)), hkv=hkv,
                    idx_dim=rng.choice([64, 128]), scale_block=block, page=page, before_min=rng.randrange(before + 1),
                    before=before, norm=norm, rot=rng.choice([0, 64, 128]) if norm else 0)
    if op == "scores":
        seqs = _log_int(rng, 1, 32)
        t = rng.choice([1, 1, 1, 2, 5, 8, 17, 40])
        ctx = _log_int(rng, 64, (1 << 21) // seqs // (1 if t == 1 else 8))
        return dict(op=op, seqs=seqs, q_per_seq=t, ctx=ctx, ctx_min=rng.randrange(min(t, ctx), ctx + 1),
                    idx_dim=rng.choice([64, 128]), scale_block=block, page=page, causal=t > 1 and rng.random() < 0.8)
    t = rng.choice([1, 1, 1, 2, 6, 31])
    seqs = _log_int(rng, 1, 64 // t)
    top_k = _log_int(rng, 1, 2048)
    ctx = _log_int(rng, 64, 32768)
    return dict(op=op, seqs=seqs, q_per_seq=t, ctx=ctx, ctx_min=rng.randrange(min(t, ctx), ctx + 1), hq=hq, hkv=hkv,
                top_k=top_k, scale_block=block, page=page, causal=t > 1 and rng.random() < 0.8,
                empty=rng.randrange(min(3, seqs * t)))


def _lengths(count, lo, hi):
    """Lengths spread over lo..hi, the same for every seed."""
    if count == 1:
        return [hi]
    return [lo + (hi - lo) * (b * 5 % count) // (count - 1) for b in range(count)]


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _device():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


def _random_codes(gen, shape, dev):
    """e4m3 codes of normal values whose maxima come near the format's largest."""
    count = math.prod(shape)
    table = (torch.randn(1 << 16, generator=gen, device=dev) * 100).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    table = table.view(torch.uint8)
    out = torch.empty(count, dtype=torch.uint8, device=dev)
    step = 1 << 26
    for at in range(0, count, step):
        m = min(step, count - at)
        out[at:at + m] = table[torch.randint(0, 1 << 16, (m,), generator=gen, device=dev, dtype=torch.int32)]
    return out.view(shape)


def _place(lens, capacity, block, page, gen, dev):
    """Where sequences of up to `capacity` rows lie: starts, or a table of scattered pages; and the rows of the pool."""
    B = len(lens)
    if page:
        per_seq = -(-capacity // page)
        table = torch.randperm(B * per_seq, generator=gen, device=dev).to(torch.int32).view(B, per_seq)
        return dict(seq_start=None, block_table=table, rows=B * per_seq * page)
    unit = max(block, 64)
    room = -(-capacity // unit) * unit
    start = torch.arange(B, device=dev, dtype=torch.int64) * room
    return dict(seq_start=start, block_table=None, rows=B * room)


def _normal(gen, shape, dev, scale=1.0):
    return (torch.randn(shape, generator=gen, device=dev) * scale).to(torch.bfloat16)


def _frequencies(rot, dev):
    if rot == 0:
        return None
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(dev)


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s = dict(case=dict(case))
    if case["op"] == "norm_rope":
        n, hq, hk, d = case["tokens"], case["hq"], case["hk"], case["head_dim"]
        if case["fused"]:  # queries and keys as slices of one projection's output rows
            rows = _normal(gen, (n, hq + 2 * hk, d), dev, 2.0)
            s["q"], s["k"] = rows[:, :hq], rows[:, hq:hq + hk]
        else:
            s["q"], s["k"] = _normal(gen, (n, hq, d), dev, 2.0), _normal(gen, (n, hk, d), dev, 0.5)
        pos = torch.randint(0, case["max_pos"], (n,), generator=gen, device=dev, dtype=torch.int32)
        if case["padded"]:
            pos[torch.randperm(n, generator=gen, device=dev)[:case["padded"]]] = -1
        s["positions"] = pos
        s["inv_freq"] = _frequencies(case["rot"], dev)
        s["q_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16)
        s["k_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16)
        s["q_out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=dev)
        s["k_out"] = torch.zeros((n, hk, d), dtype=torch.bfloat16, device=dev)
        return s

    B, T, block = case["seqs"], case["q_per_seq"], case["scale_block"]
    if case["op"] == "append":
        lens = [b + T for b in _lengths(B, case["before_min"], case["before"])]
    else:
        lens = _lengths(B, case["ctx_min"], case["ctx"])
    s["max_len"] = max(lens)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s |= _place(lens, max(lens), block, case["page"], gen, dev)
    rows, blocks = s["rows"], s["rows"] // block
    if case["op"] in ("append", "attn"):
        hkv = case["hkv"]
        s["k8"] = _random_codes(gen, (rows, hkv, 128), dev)
        s["v8"] = _random_codes(gen, (rows, hkv, 128), dev)
        s["k_scale"] = torch.randint(119, 122, (hkv, blocks), generator=gen, device=dev, dtype=torch.uint8)
        s["v_scale"] = torch.randint(118, 122, (hkv, blocks), generator=gen, device=dev, dtype=torch.uint8)
    if case["op"] in ("append", "scores"):
        s["idx8"] = _random_codes(gen, (rows, case["idx_dim"]), dev)
        s["idx_scale"] = torch.randint(119, 122, (blocks,), generator=gen, device=dev, dtype=torch.uint8)
    if case["op"] == "append":
        new = _normal(gen, (B, T, 2 * hkv, 128), dev)  # keys and values of one projection's output rows
        s["k_new"], s["v_new"] = new[:, :, :hkv], new[:, :, hkv:]
        s["idx_new"] = _normal(gen, (B, T, case["idx_dim"]), dev)
        s["inv_freq"] = _frequencies(case["rot"], dev)
        s["k_weight"] = (1 + 0.1 * torch.randn(128, generator=gen, device=dev)).to(torch.bfloat16)
    elif case["op"] == "scores":
        s["q_idx"] = _normal(gen, (B, T, case["idx_dim"]), dev)
        s["stride"] = -(-max(lens) // 64) * 64
        s["scores"] = torch.zeros((B, T, s["stride"]), dtype=torch.float32, device=dev)
    else:
        hq, k = case["hq"], case["top_k"]
        s["q"] = _normal(gen, (B, T, hq, 128), dev)
        visible = _visible(s)
        count = visible.clamp(max=k)
        count.view(-1)[:case["empty"]] = 0
        # distinct ascending positions, one in each of `count` equal parts of what the query sees
        slot = torch.arange(k, device=dev, dtype=torch.float64)
        u = torch.rand((B, T, k), generator=gen, device=dev, dtype=torch.float64)
        idx = ((slot + u) * (visible / count.clamp(min=1))[..., None]).floor().to(torch.int64)
        idx = torch.minimum(idx, visible[..., None] - 1)
        s["idx"] = torch.where(slot < count[..., None], idx, -1).to(torch.int32)
        s["count"] = count.to(torch.int32)
        s["out"] = torch.zeros((B, T, hq, 128), dtype=torch.bfloat16, device=dev)
        s["lse"] = torch.zeros((B, T, hq), dtype=torch.float32, device=dev)
    return s


def _visible(s):
    """[B][T] tokens that each query sees."""
    c, T = s["case"], s["case"]["q_per_seq"]
    n = s["seq_len"].to(torch.int64)[:, None]
    t = torch.arange(T, device=n.device)[None]
    return n - T + t + 1 if c["causal"] else n.expand(-1, T)


def _rows_of(s, pos):
    """Cache rows of positions [B, ...] (in range)."""
    B = pos.shape[0]
    shape = (B,) + (1,) * (pos.dim() - 1)
    if s["block_table"] is None:
        return s["seq_start"].view(shape) + pos
    page = s["case"]["page"]
    seq = torch.arange(B, device=pos.device).view(shape).expand_as(pos)
    return s["block_table"].to(torch.int64)[seq, pos // page] * page + pos % page


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _norm_rotate(x, pos, weight, norm, inv_freq, interleaved):
    """x [..., heads, D] fp32, pos [...]: RMS norm of each head, then the rotation of its first dimensions."""
    if norm:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    if inv_freq is None:
        return x
    angle = pos.double()[..., None] * inv_freq.double()
    cos, sin = angle.cos().float()[..., None, :], angle.sin().float()[..., None, :]
    half = inv_freq.numel()
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_norm_rope(s):
    c = s["case"]
    live = (s["positions"] >= 0)[:, None, None]
    for x, w, out in ((s["q"], s["q_weight"], s["q_out"]), (s["k"], s["k_weight"], s["k_out"])):
        y = _norm_rotate(x.float(), s["positions"], w, True, s["inv_freq"], c["interleaved"])
        out.copy_(torch.where(live, y.to(torch.bfloat16), out))
    return s["q_out"], s["k_out"]


def _append_plain_one(s, new, codes, scale):
    """new [B, T, H, D] fp32 into codes [rows, H, D] and scale [H, blocks] (bytes)."""
    B, T, H, D = new.shape
    block = s["case"]["scale_block"]
    n = s["seq_len"].to(torch.int64)
    first = n - T
    pos = first[:, None] + torch.arange(T, device=n.device)
    row = _rows_of(s, pos)
    # exponent that each new row needs, and the largest of each block
    mag = new.abs()
    amax = torch.where(mag <= 3.4028234663852886e38, mag, torch.zeros_like(mag)).amax(-1)
    mant, exp = torch.frexp(amax)  # amax = mant * 2^exp, mant in [0.5, 1)
    need = torch.where(amax > 0, exp - 9 + (mant > 0.875), torch.full_like(exp, EXP_MIN)).clamp(EXP_MIN, EXP_MAX)
    local = pos // block - (first // block)[:, None]
    spans = (T - 1) // block + 2
    at = local[..., None].expand(B, T, H)
    e = torch.full((B, spans, H), EXP_MIN, dtype=torch.int32, device=new.device)
    e.scatter_reduce_(1, at, need.to(torch.int32), "amax")
    # the first block may hold older rows: its exponent does not shrink, and they are coded anew where it grows
    begin = first // block * block
    begin_row = _rows_of(s, begin[:, None])[:, 0]
    old_e = scale[:, begin_row // block].to(torch.int32).t() - 127
    older = (first > begin)[:, None]
    e[:, 0] = torch.where(older, torch.maximum(e[:, 0], old_e), e[:, 0])
    inside = torch.arange(block - 1, device=n.device)
    is_old = begin[:, None] + inside < first[:, None]
    old_row = begin_row[:, None] + inside
    shift = torch.exp2((old_e - e[:, 0]).clamp(min=-60).float())[:, None, :, None]
    value = codes[old_row].view(torch.float8_e4m3fn).float() * shift
    codes[old_row[is_old]] = value[is_old].to(torch.float8_e4m3fn).view(torch.uint8)
    # the new rows
    mine = torch.gather(e, 1, at)
    x = new * torch.exp2(-mine.float())[..., None]
    codes[row.flatten()] = x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8).flatten(0, 1)
    head = torch.arange(H, device=n.device)
    scale[head, (row // block)[..., None]] = (mine + 127).to(torch.uint8)


def _plain_append(s):
    c = s["case"]
    pos = (s["seq_len"].to(torch.int64) - c["q_per_seq"])[:, None] + torch.arange(c["q_per_seq"], device=s["seq_len"].device)
    k = s["k_new"].float()
    if c["norm"]:
        k = _norm_rotate(k, pos, s["k_weight"], True, s["inv_freq"], False)
    _append_plain_one(s, k, s["k8"], s["k_scale"])
    _append_plain_one(s, s["v_new"].float(), s["v8"], s["v_scale"])
    _append_plain_one(s, s["idx_new"].float()[:, :, None], s["idx8"][:, None], s["idx_scale"][None])


def _plain_scores(s):
    c = s["case"]
    B, block = c["seqs"], c["scale_block"]
    n, width = s["max_len"], s["stride"]
    pos = torch.arange(n, device=s["seq_len"].device)[None].expand(B, n)
    row = _rows_of(s, torch.minimum(pos, s["seq_len"].to(torch.int64)[:, None] - 1))
    keys = s["idx8"][row].view(torch.float8_e4m3fn).float()
    scale = torch.exp2(s["idx_scale"][row // block].float() - 127)
    got = torch.matmul(s["q_idx"].float(), keys.transpose(1, 2)) * scale[:, None]
    seen = torch.arange(n, device=row.device) < _visible(s)[..., None]
    s["scores"][..., :n] = torch.where(seen, got, s["scores"][..., :n])
    return s["scores"]


def _plain_attn(s):
    c = s["case"]
    hq, hkv, block = c["hq"], c["hkv"], c["scale_block"]
    live = torch.arange(c["top_k"], device=s["idx"].device) < s["count"][..., None]
    row = _rows_of(s, torch.where(live, s["idx"], 0).to(torch.int64))
    k = s["k8"][row].view(torch.float8_e4m3fn).float()
    v = s["v8"][row].view(torch.float8_e4m3fn).float()
    ks = torch.exp2(s["k_scale"][:, row // block].float() - 127)  # [Hkv, B, T, k]
    vs = torch.exp2(s["v_scale"][:, row // block].float() - 127)
    q = s["q"].float().unflatten(2, (hkv, hq // hkv))
    x = torch.einsum("btgmd,btkgd->btgmk", q, k) * ks.permute(1, 2, 0, 3)[:, :, :, None] / math.sqrt(128.0)
    x = x.masked_fill(~live[:, :, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    w = w * vs.permute(1, 2, 0, 3)[:, :, :, None]
    out = torch.einsum("btgmk,btkgd->btgmd", w, v) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(out.flatten(2, 3).to(torch.bfloat16))
    s["lse"].copy_((torch.log(total) + top)[..., 0].flatten(2, 3))
    return s["out"], s["lse"]


# ---------------------------------------------------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------------------------------------------------
def _plan(s):
    """What a serving program makes once for its buffers: the params struct, the cache's description, a workspace."""
    import paper_2606_06467_b200 as clsa

    c = s["case"]
    if c["op"] == "norm_rope":
        return clsa, clsa.make_norm_rope(head_dim=c["head_dim"], norm=1, eps=1e-6, rot_dim=c["rot"],
                                         interleaved=int(c["interleaved"]), inv_freq=s["inv_freq"],
                                         q_weight=s["q_weight"], k_weight=s["k_weight"])
    p = clsa.make_params(num_seqs=c["seqs"], q_per_seq=c["q_per_seq"], num_q_heads=c.get("hq", c.get("hkv", 1)),
                         num_kv_heads=c.get("hkv", 1), idx_dim=c.get("idx_dim", 128), top_k=c.get("top_k", 1),
                         causal=int(c.get("causal", False)), max_seq_len=s["max_len"], sm_scale=1 / math.sqrt(128.0),
                         seq_start=s["seq_start"], seq_len=s["seq_len"], num_cache_rows=s["rows"],
                         block_table=s["block_table"], block_size=c["page"])
    cache = clsa.make_cache8(k=s.get("k8"), v=s.get("v8"), k_scale=s.get("k_scale"), v_scale=s.get("v_scale"),
                             idx_k=s.get("idx8"), idx_k_scale=s.get("idx_scale"), scale_block=c["scale_block"])
    ws = torch.zeros(clsa.clsa_cache8_workspace_bytes(p, cache), dtype=torch.uint8, device=s["seq_len"].device)
    spec = None
    if c.get("norm"):
        spec = clsa.make_norm_rope(head_dim=128, norm=1, eps=1e-6, rot_dim=c["rot"], interleaved=0,
                                   inv_freq=s["inv_freq"], k_weight=s["k_weight"])
    return clsa, p, cache, ws, spec


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    op = s["case"]["op"]
    if op == "norm_rope":
        clsa, spec = s["plan"]
        clsa.clsa_norm_rope(spec, s["positions"], s["q"], s["q_out"], s["k"], s["k_out"])
        return
    clsa, p, cache, ws, spec = s["plan"]
    if op == "append":
        clsa.clsa_cache8_append(p, cache, spec, s["k_new"], s["v_new"], s["idx_new"], ws)
    elif op == "scores":
        clsa.clsa_index_scores8(p, cache, s["q_idx"], s["scores"], s["stride"], ws)
    else:
        clsa.clsa_sparse_attn8(p, cache, s["q"], s["idx"], s["count"], s["out"], s["lse"], None, ws)


def run(state):
    op = state["case"]["op"]
    if own:
        _own(state)
    else:
        {"norm_rope": _plain_norm_rope, "append": _plain_append, "scores": _plain_scores, "attn": _plain_attn}[op](state)
    if op == "norm_rope":
        return state["q_out"], state["k_out"]
    if op == "append":  # codes and scales as the values that they stand for
        return tuple(state[n].view(torch.float8_e4m3fn) for n in ("k8", "v8", "idx8")) + tuple(
            state[n].view(torch.float8_e8m0fnu) for n in ("k_scale", "v_scale", "idx_scale"))
    return state["scores"] if op == "scores" else (state["out"], state["lse"])


# ---------------------------------------------------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm_rope":
        n, d, heads = case["tokens"] - case["padded"], case["head_dim"], case["hq"] + case["hk"]
        return dict(bytes=n * (4 + heads * d * 4) + case["rot"] * 2 + 4 * d, flops=n * heads * d * 6)
    B, T, block = case["seqs"], case["q_per_seq"], case["scale_block"]
    if case["op"] == "append":
        width = 2 * case["hkv"] * 128 + case["idx_dim"]
        return dict(bytes=B * T * width * 3 + B * (-(-T // block)) * (2 * case["hkv"] + 1), flops=B * T * width * 4)
    lens = _lengths(B, case["ctx_min"], case["ctx"])
    if case["op"] == "scores":
        d = case["idx_dim"]
        seen = sum(T * n - (T * (T - 1) // 2 if case["causal"] else 0) for n in lens)
        return dict(bytes=sum(n * d + -(-n // block) for n in lens) + B * T * d * 2 + 4 * seen, flops=2 * seen * d)
    hq, hkv, k = case["hq"], case["hkv"], case["top_k"]
    taken = [[min(k, n - T + t + 1 if case["causal"] else n) if b * T + t >= case["empty"] else 0 for t in range(T)]
             for b, n in enumerate(lens)]
    distinct = sum(min(n, sum(row)) for n, row in zip(lens, taken))
    total = sum(sum(row) for row in taken)
    return dict(bytes=distinct * hkv * 256 + total * 4 + B * T * (4 + hq * (512 + 4)), flops=4 * total * hq * 128)


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _decode_table(dev):
    """The 256 e4m3 values from their bits: sign, four exponent bits (bias 7), three mantissa bits."""
    values = []
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        mag = math.nan if code & 127 == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        values.append(-mag if code & 128 else mag)
    return torch.tensor(values, dtype=torch.float64, device=dev)


def _exact_head(x, pos, weight, inv_freq, interleaved):
    """x [tokens, heads, D]: the definition, one rotation pair at a time."""
    x = x.double()
    y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * weight.double()
    if inv_freq is None:
        return y
    z = y.clone()
    pairs = inv_freq.numel()
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        angle = (pos.double() * float(inv_freq[i]))[:, None]
        z[..., a] = y[..., a] * torch.cos(angle) - y[..., b] * torch.sin(angle)
        z[..., b] = y[..., a] * torch.sin(angle) + y[..., b] * torch.cos(angle)
    return z


def _exact_row(s, b, pos):
    """Cache rows of the positions `pos` of sequence b."""
    page = s["case"]["page"]
    if page:
        return s["block_table"][b].long()[pos // page] * page + pos % page
    return s["seq_start"][b] + pos


def _exact_append(s, new, codes, scale, table):
    """The values that the codes stand for before their rounding, and the scales (new [B, T, H, D] in 64 bits)."""
    block = s["case"]["scale_block"]
    B, T, H, D = new.shape
    value = table[codes.long()].view(codes.shape[0], H, D)
    factor = torch.exp2(scale.double() - 127)
    for b in range(B):
        n = int(s["seq_len"][b])
        at = n - T
        while at < n:
            begin, end = at // block * block, min(n, (at // block + 1) * block)
            rows = _exact_row(s, b, torch.arange(begin, end, device=new.device))
            fresh = new[b, at - (n - T):end - (n - T)]
            amax = fresh.abs().amax((0, 2))
            e = torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(EXP_MIN, EXP_MAX)
            e = torch.where(amax > E4M3_MAX * torch.exp2(e), e + 1, e)
            e = torch.where(amax <= E4M3_MAX * torch.exp2(e - 1), e - 1, e).clamp(EXP_MIN, EXP_MAX)
            home = int(rows[0]) // block
            if at > begin:
                before = torch.log2(factor[:, home])
                e = torch.maximum(e, before)
                value[rows[:at - begin]] *= torch.exp2(before - e)[None, :, None]
            value[rows[at - begin:]] = fresh / torch.exp2(e)[None, :, None]
            factor[:, home] = torch.exp2(e)
            at = end
    return value, factor


def exact(case, seed):
    s = prepare(case, seed)
    dev = _device()
    if case["op"] == "norm_rope":
        got = []
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            y = _exact_head(x, s["positions"], w, s["inv_freq"], case["interleaved"])
            y[s["positions"] < 0] = 0.0
            got.append(y)
        return tuple(got)
    table = _decode_table(dev)
    B, T, block = case["seqs"], case["q_per_seq"], case["scale_block"]
    if case["op"] == "append":
        if B * (T // block + 2) > 4000:
            return None
        k = s["k_new"].double()
        if case["norm"]:
            pos = torch.cat([torch.arange(int(n) - T, int(n), device=dev) for n in s["seq_len"]])
            k = _exact_head(s["k_new"].flatten(0, 1), pos, s["k_weight"], s["inv_freq"], False).view(k.shape)
        k8, ks = _exact_append(s, k, s["k8"], s["k_scale"], table)
        v8, vs = _exact_append(s, s["v_new"].double(), s["v8"], s["v_scale"], table)
        i8, ic = _exact_append(s, s["idx_new"].double()[:, :, None], s["idx8"], s["idx_scale"][None], table)
        return k8, v8, i8[:, 0], ks, vs, ic[0]
    if case["op"] == "scores":
        out = torch.zeros((B, T, s["stride"]), dtype=torch.float64, device=dev)
        for b in range(B):
            n = int(s["seq_len"][b])
            rows = _exact_row(s, b, torch.arange(n, device=dev))
            keys = table[s["idx8"][rows].long()] * torch.exp2(s["idx_scale"][rows // block].double() - 127)[:, None]
            got = s["q_idx"][b].double() @ keys.T
            if case["causal"]:
                got = torch.tril(got, n - T)
            out[b, :, :n] = got
        return out
    hq, hkv = case["hq"], case["hkv"]
    out = torch.zeros((B, T, hq, 128), dtype=torch.float64, device=dev)
    lse = torch.full((B, T, hq), -math.inf, dtype=torch.float64, device=dev)
    for b in range(B):
        for t in range(T):
            m = int(s["count"][b, t])
            if m == 0:
                continue
            rows = _exact_row(s, b, s["idx"][b, t, :m].long())
            k = table[s["k8"][rows].long()] * torch.exp2(s["k_scale"][:, rows // block].double() - 127).T[..., None]
            v = table[s["v8"][rows].long()] * torch.exp2(s["v_scale"][:, rows // block].double() - 127).T[..., None]
            k, v = (x.repeat_interleave(hq // hkv, 1).transpose(0, 1) for x in (k, v))
            logits = (k @ s["q"][b, t].double()[..., None])[..., 0] / 128 ** 0.5
            lse[b, t] = torch.logsumexp(logits, -1)
            out[b, t] = (torch.softmax(logits, -1)[:, None] @ v)[:, 0]
    return out, lse
