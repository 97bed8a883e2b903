"""The operators around a layer's attention as cases with inputs, a plain form, a 64-bit definition and the library's own calls.

Four operators that a decoder layer runs one after another: the residual's addition with an RMS norm and an 8-bit output
(`clsa_add_norm`), the heads' norms with a rotation over several position axes (`clsa_norm_rope_axes`), and the attention of the
newest tokens over a whole cache or its last tokens, bf16 (`clsa_dense_attn`) or 8-bit (`clsa_dense_attn8`).

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
        # the smallest decode: one short sequence, one KV head
        dict(name="dense tiny 777", op="dense", bits=16, seqs=1, q_per_seq=1, ctx=777, ctx_min=777, hq=8, hkv=1, window=0,
             page=0, scale_block=64, causal=False),
        # one dense layer of a decode step over 16 sequences of 32768 tokens
        dict(name="dense decode 32K", op="dense", bits=16, seqs=16, q_per_seq=1, ctx=32768, ctx_min=32768, hq=32, hkv=8,
             window=0, page=0, scale_block=64, causal=False),
        # one sliding-window layer (512 tokens, 20/4 heads) of a decode step over 64 paged sequences, some shorter than the window
        dict(name="dense window 512", op="dense", bits=16, seqs=64, q_per_seq=1, ctx=8192, ctx_min=300, hq=20, hkv=4,
             window=512, page=64, scale_block=64, causal=True),
        # four drafted tokens per sequence, ragged lengths, small pages
        dict(name="dense draft ragged", op="dense", bits=16, seqs=24, q_per_seq=4, ctx=32768, ctx_min=1001, hq=32, hkv=8,
             window=0, page=16, scale_block=16, causal=True),
        # one sequence over an 8-bit cache, one KV head
        dict(name="dense8 tiny 4096", op="dense", bits=8, seqs=1, q_per_seq=1, ctx=4096, ctx_min=4096, hq=8, hkv=1, window=0,
             page=0, scale_block=64, causal=False),
        # the 16 sequences of above over an 8-bit cache
        dict(name="dense8 decode 32K", op="dense", bits=8, seqs=16, q_per_seq=1, ctx=32768, ctx_min=32768, hq=32, hkv=8,
             window=0, page=0, scale_block=64, causal=False),
        # three drafted tokens, ragged lengths, pages and scale blocks of 16 rows
        dict(name="dense8 draft ragged", op="dense", bits=8, seqs=24, q_per_seq=3, ctx=32768, ctx_min=1001, hq=20, hkv=4,
             window=0, page=16, scale_block=16, causal=True),
        # a decode step's 16 new tokens: hidden size 2560, 8-bit output with a scale per 32 values
        dict(name="add_norm decode 16", op="add_norm", rows=16, dim=2560, group=32, bf16=False),
        # an odd number of packed tokens, both outputs, a scale per row
        dict(name="add_norm ragged 777", op="add_norm", rows=777, dim=4096, group=4096, bf16=True),
        # a prefill chunk of 8192 tokens
        dict(name="add_norm chunk 8192", op="add_norm", rows=8192, dim=5120, group=128, bf16=False),
        # a decode step's queries and keys behind a prompt with images: pairs of 128 dimensions in three runs of axes
        dict(name="axes decode 16", op="axes", tokens=16, hq=32, hk=8, head_dim=128, rot=128, interleaved=False, cycle=False,
             fused=True, padded=0, max_pos=131072),
        # a video's prefill chunk: axes of the pairs in turn, some padded rows
        dict(name="axes chunk 4096", op="axes", tokens=4096, hq=32, hk=8, head_dim=128, rot=128, interleaved=False, cycle=True,
             fused=True, padded=7, max_pos=32768),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dense", "dense", "add_norm", "axes"])
    if op == "add_norm":
        dim = rng.choice([64, 128, 896, 1536, 2560, 4096, 5120, 8192])
        group = rng.choice([0, 32, 64, 128, dim])
        if group and dim % group:
            group = 32
        return dict(op=op, rows=_log_int(rng, 1, 8192 * 5120 // max(dim, 5120)), dim=dim, group=group,
                    bf16=group == 0 or rng.random() < 0.4)
    hq, hkv = rng.choice([(8, 1), (32, 8), (20, 4), (16, 1), (4, 4), (14, 2), (40, 5)])
    if op == "axes":
        dim = rng.choice([64, 128, 128, 256])
        tokens = _log_int(rng, 1, 4096 * 128 // max(dim, 128))
        return dict(op=op, tokens=tokens, hq=hq, hk=hkv, head_dim=dim, rot=rng.choice([32, dim // 2, dim]),
                    interleaved=rng.random() < 0.3, cycle=rng.random() < 0.5, fused=rng.random() < 0.5,
                    padded=min(tokens - 1, rng.randrange(5)), max_pos=_log_int(rng, 64, 1 << 20))
    t = rng.choice([1, 1, 1, 2, 3, 5, 8, 16])
    columns = t * (hq // hkv)
    seqs = _log_int(rng, 1, 64)
    ctx = _log_int(rng, max(16, t), max(64, min(65536, (1 << 22) // (seqs * hkv * max(1, columns // 32)))))
    causal = t > 1 and rng.random() < 0.8
    block = rng.choice([16, 32, 64, 128])
    return dict(op=op, bits=rng.choice([16, 8]), seqs=seqs, q_per_seq=t, ctx=ctx, ctx_min=rng.randrange(t, ctx + 1), hq=hq,
                hkv=hkv, window=rng.choice([0, 0, _log_int(rng, 1, 4096)]), page=rng.choice([0, block, 2 * block]),
                scale_block=block, causal=causal)


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


def _normal(gen, shape, dev, scale=1.0):
    return (torch.randn(shape, generator=gen, device=dev) * scale).to(torch.bfloat16)


def _big_normal(gen, shape, dev):
    """bf16 normal values, drawn in that type (a large cache's fp32 ones would take long)."""
    return torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16)


def _random_codes(gen, shape, dev):
    """e4m3 codes of normal values whose maxima come near the format's largest."""
    count = math.prod(shape)
    table = (torch.randn(1 << 16, generator=gen, device=dev) * 100).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    table = table.view(torch.uint8)
    out = torch.empty(count, dtype=torch.uint8, device=dev)
    step = 1 << 27
    for at in range(0, count, step):
        m = min(step, count - at)
        out[at:at + m] = table[torch.randint(0, 1 << 16, (m,), generator=gen, device=dev, dtype=torch.int32)]
    return out.view(shape)


def prepare(case, seed):
    dev = _device()
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s = dict(case=dict(case))
    if case["op"] == "add_norm":
        n, d, group = case["rows"], case["dim"], case["group"]
        s["x"] = _normal(gen, (n, d), dev, 0.5)          # an attention's or an MLP's output
        s["residual"] = _normal(gen, (n, d), dev, 3.0)   # the stream that it is added to
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16)
        s["sum"] = torch.zeros((n, d), dtype=torch.bfloat16, device=dev)
        s["y"] = torch.zeros((n, d), dtype=torch.bfloat16, device=dev) if case["bf16"] else None
        s["codes"] = torch.zeros((n, d), dtype=torch.uint8, device=dev) if group else None
        s["scales"] = torch.zeros((n, d // group), dtype=torch.uint8, device=dev) if group else None
        return s
    if case["op"] == "axes":
        n, hq, hk, d = case["tokens"], case["hq"], case["hk"], case["head_dim"]
        if case["fused"]:  # queries and keys as slices of one projection's output rows
            rows = _normal(gen, (n, hq + 2 * hk, d), dev, 2.0)
            s["q"], s["k"] = rows[:, :hq], rows[:, hq:hq + hk]
        else:
            s["q"], s["k"] = _normal(gen, (n, hq, d), dev, 2.0), _normal(gen, (n, hk, d), dev, 0.5)
        # time counts through the sequence, height and width from a frame's place in it
        time = torch.randint(0, case["max_pos"], (n,), generator=gen, device=dev, dtype=torch.int32)
        place = torch.randint(0, 96, (2, n), generator=gen, device=dev, dtype=torch.int32)
        s["positions"] = torch.cat((time[None], time[None] + place))
        if case["padded"]:
            s["positions"][:, torch.randperm(n, generator=gen, device=dev)[:case["padded"]]] = -1
        rot = case["rot"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(dev)
        s["axis"] = _axis_of_pair(case)
        s["axis_index"] = torch.tensor(s["axis"], device=dev)
        s["q_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16)
        s["k_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16)
        s["q_out"] = torch.zeros((n, hq, d), dtype=torch.bfloat16, device=dev)
        s["k_out"] = torch.zeros((n, hk, d), dtype=torch.bfloat16, device=dev)
        return s

    B, T, hq, hkv, page, block = (case[n] for n in ("seqs", "q_per_seq", "hq", "hkv", "page", "scale_block"))
    lens = _lengths(B, case["ctx_min"], case["ctx"])
    s["max_len"] = max(lens)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["seq_start"] = s["block_table"] = None
    if page:  # scattered pages
        per_seq = -(-max(lens) // page)
        s["block_table"] = torch.randperm(B * per_seq, generator=gen, device=dev).to(torch.int32).view(B, per_seq)
        rows = B * per_seq * page
    else:
        room = -(-max(lens) // 128) * 128
        s["seq_start"] = torch.arange(B, device=dev, dtype=torch.int64) * room
        rows = B * room
    s["rows"] = rows
    if case["bits"] == 16:
        s["k"], s["v"] = _big_normal(gen, (rows, hkv, 128), dev), _big_normal(gen, (rows, hkv, 128), dev)
    else:
        s["k"], s["v"] = _random_codes(gen, (rows, hkv, 128), dev), _random_codes(gen, (rows, hkv, 128), dev)
        s["k_scale"] = torch.randint(119, 122, (hkv, rows // block), generator=gen, device=dev, dtype=torch.uint8)
        s["v_scale"] = torch.randint(118, 122, (hkv, rows // block), generator=gen, device=dev, dtype=torch.uint8)
    s["q"] = _normal(gen, (B, T, hq, 128), dev)
    s["out"] = torch.zeros((B, T, hq, 128), dtype=torch.bfloat16, device=dev)
    s["lse"] = torch.zeros((B, T, hq), dtype=torch.float32, device=dev)
    return s


def _axis_of_pair(case):
    """The position axis that turns each pair: in turn, or in three runs (a quarter, and two of three eighths)."""
    pairs = case["rot"] // 2
    if case["cycle"]:
        return [i % 3 for i in range(pairs)]
    return [0 if i < pairs // 4 else 1 if i < pairs // 4 + pairs * 3 // 8 else 2 for i in range(pairs)]


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_add_norm(s):
    c = s["case"]
    total = s["x"].float() + s["residual"].float()
    s["sum"].copy_(total.to(torch.bfloat16))
    y = total * torch.rsqrt(total.square().mean(-1, keepdim=True) + 1e-6) * s["weight"].float()
    if c["bf16"]:
        s["y"].copy_(y.to(torch.bfloat16))
    if c["group"]:
        part = y.unflatten(-1, (-1, c["group"]))
        mant, exp = torch.frexp(part.abs().amax(-1))  # mant * 2^exp, mant in [0.5, 1)
        e = torch.where(mant > 0, exp - 9 + (mant > 0.875), torch.full_like(exp, EXP_MIN)).clamp(EXP_MIN, EXP_MAX)
        code = (part * torch.exp2(-e.float())[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s["codes"].copy_(code.view(torch.uint8).flatten(-2))
        s["scales"].copy_((e + 127).to(torch.uint8))


def _plain_axes(s):
    c = s["case"]
    live = (s["positions"][0] >= 0)[:, None, None]
    half = s["inv_freq"].numel()
    angle = s["positions"][s["axis_index"]].t().double() * s["inv_freq"].double()  # [tokens, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for x, w, out in ((s["q"], s["q_weight"], s["q_out"]), (s["k"], s["k_weight"], s["k_out"])):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        if c["interleaved"]:
            a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :half], y[..., half:2 * half]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        y = torch.cat((turned, y[..., 2 * half:]), -1)
        out.copy_(torch.where(live, y.to(torch.bfloat16), out))


def _span(c, longest):
    """Positions that some query of a sequence may see: all of them, or those of the last query's window and the T - 1 before it."""
    return min(longest, c["window"] + c["q_per_seq"] - 1) if c["window"] else longest


def _plain_dense(s):
    c = s["case"]
    B, T, hq, hkv = c["seqs"], c["q_per_seq"], c["hq"], c["hkv"]
    dev, n = s["seq_len"].device, s["seq_len"].to(torch.int64)[:, None]
    width = _span(c, s["max_len"])
    pos = torch.arange(width, device=dev)[None] + (n - width if c["window"] else torch.zeros_like(n))  # [B, width]
    safe = torch.minimum(pos.clamp(min=0), (n - 1).clamp(min=0))
    if s["block_table"] is None:
        row = s["seq_start"][:, None] + safe
    else:
        row = torch.gather(s["block_table"].to(torch.int64), 1, safe // c["page"]) * c["page"] + safe % c["page"]
    at = n - T + torch.arange(T, device=dev)  # the queries' own positions [B, T]
    seen = (pos >= 0)[:, None] & (pos[:, None] < (at[..., None] + 1 if c["causal"] else n[..., None]))
    if c["window"]:
        seen = seen & (pos[:, None] > at[..., None] - c["window"])
    seen = seen[:, None, :, None]  # [B, 1, T, 1, width]
    k, v = s["k"][row], s["v"][row]
    if c["bits"] == 8:
        block = row // c["scale_block"]
        k = k.view(torch.float8_e4m3fn).float() * torch.exp2(s["k_scale"][:, block].float() - 127).permute(1, 2, 0)[..., None]
        v = v.view(torch.float8_e4m3fn).float() * torch.exp2(s["v_scale"][:, block].float() - 127).permute(1, 2, 0)[..., None]
    group = hq // hkv
    q = s["q"].float().view(B, T, hkv, group, 128).permute(0, 2, 1, 3, 4).reshape(B, hkv, T * group, 128)
    x = torch.matmul(q, k.float().permute(0, 2, 3, 1)).view(B, hkv, T, group, width) / math.sqrt(128.0)
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    w = w / torch.where(total > 0, total, 1.0)
    out = torch.matmul(w.view(B, hkv, T * group, width), v.float().permute(0, 2, 1, 3)).view(B, hkv, T, group, 128)
    s["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(B, T, hq, 128).to(torch.bfloat16))
    s["lse"].copy_((torch.log(total) + top)[..., 0].permute(0, 2, 1, 3).reshape(B, T, hq))


# ---------------------------------------------------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------------------------------------------------
def _plan(s):
    """What a serving program makes once for its buffers: specs, the params struct, the cache's description, a workspace."""
    import paper_2606_06467_b200 as clsa

    c = s["case"]
    if c["op"] == "add_norm":
        return clsa, clsa.make_add_norm(dim=c["dim"], eps=1e-6, weight=s["weight"], scale_group=c["group"])
    if c["op"] == "axes":
        spec = clsa.make_norm_rope(head_dim=c["head_dim"], norm=1, eps=1e-6, rot_dim=c["rot"], interleaved=int(c["interleaved"]),
                                   inv_freq=s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"])
        return clsa, spec, clsa.make_rope_axes(s["axis"], num_axes=3)
    own_cache = dict(k_cache=s["k"], v_cache=s["v"]) if c["bits"] == 16 else {}
    p = clsa.make_params(num_seqs=c["seqs"], q_per_seq=c["q_per_seq"], num_q_heads=c["hq"], num_kv_heads=c["hkv"], idx_dim=128,
                         top_k=1, causal=int(c["causal"]), max_seq_len=s["max_len"], sm_scale=1 / math.sqrt(128.0),
                         seq_start=s["seq_start"], seq_len=s["seq_len"], num_cache_rows=s["rows"], block_table=s["block_table"],
                         block_size=c["page"], **own_cache)
    cache = None
    if c["bits"] == 8:
        cache = clsa.make_cache8(k=s["k"], v=s["v"], k_scale=s["k_scale"], v_scale=s["v_scale"], scale_block=c["scale_block"])
    ws = torch.zeros(clsa.clsa_dense_workspace_bytes(p), dtype=torch.uint8, device=s["seq_len"].device)
    return clsa, p, cache, ws


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    c = s["case"]
    if c["op"] == "add_norm":
        clsa, spec = s["plan"]
        clsa.clsa_add_norm(spec, s["x"], s["residual"], s["sum"], s["y"], s["codes"], s["scales"])
    elif c["op"] == "axes":
        clsa, spec, axes = s["plan"]
        clsa.clsa_norm_rope_axes(spec, axes, s["positions"], s["q"], s["q_out"], s["k"], s["k_out"])
    else:
        clsa, p, cache, ws = s["plan"]
        if cache is None:
            clsa.clsa_dense_attn(p, c["window"], s["q"], s["out"], s["lse"], ws)
        else:
            clsa.clsa_dense_attn8(p, cache, c["window"], s["q"], s["out"], s["lse"], ws)


def run(state):
    op = state["case"]["op"]
    if own:
        _own(state)
    else:
        {"add_norm": _plain_add_norm, "axes": _plain_axes, "dense": _plain_dense}[op](state)
    if op == "axes":
        return state["q_out"], state["k_out"]
    if op == "dense":
        return state["out"], state["lse"]
    got = dict(sum=state["sum"])
    if state["y"] is not None:
        got["y"] = state["y"]
    if state["codes"] is not None:  # codes and scales as the values that they stand for
        got["codes"] = state["codes"].view(torch.float8_e4m3fn)
        got["scales"] = state["scales"].view(torch.float8_e8m0fnu)
    return got


# ---------------------------------------------------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "add_norm":
        n, d, group = case["rows"], case["dim"], case["group"]
        each = 6 + (2 if case["bf16"] else 0) + (1 if group else 0)
        return dict(bytes=n * d * each + (n * (d // group) if group else 0) + 2 * d, flops=n * d * (7 if group else 5))
    if case["op"] == "axes":
        n, d, heads = case["tokens"] - case["padded"], case["head_dim"], case["hq"] + case["hk"]
        return dict(bytes=n * (12 + heads * d * 4) + case["rot"] * 2 + 4 * d, flops=n * heads * d * 6)
    B, T, hq, hkv, window = (case[k] for k in ("seqs", "q_per_seq", "hq", "hkv", "window"))
    lens = _lengths(B, case["ctx_min"], case["ctx"])
    rows = sum(_span(case, n) for n in lens)
    seen = 0
    for n in lens:
        for t in range(T):
            end = n - T + t + 1 if case["causal"] else n
            seen += end - (max(0, n - T + t + 1 - window) if window else 0)
    each = 512 if case["bits"] == 16 else 256
    scales = 0 if case["bits"] == 16 else sum(-(-_span(case, n) // case["scale_block"]) for n in lens) * 2 * hkv
    return dict(bytes=rows * hkv * each + scales + B * T * hq * (256 + 256 + 4), flops=4 * seen * hq * 128)


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


def _exact_add_norm(s, case):
    total = s["x"].double() + s["residual"].double()
    y = total / (total.pow(2).sum(-1, keepdim=True) / case["dim"] + 1e-6).sqrt() * s["weight"].double()
    got = dict(sum=total)
    if case["bf16"]:
        got["y"] = y
    if case["group"]:  # the values that the codes stand for before their rounding
        part = y.view(case["rows"], -1, case["group"])
        top = part.abs().amax(-1)
        e = torch.ceil(torch.log2(top / E4M3_MAX)).clamp(EXP_MIN, EXP_MAX)
        e = torch.where(top > E4M3_MAX * torch.exp2(e), e + 1, e)
        e = torch.where(top <= E4M3_MAX * torch.exp2(e - 1), e - 1, e).clamp(EXP_MIN, EXP_MAX)
        got["codes"] = (part / torch.exp2(e)[..., None]).view(case["rows"], case["dim"])
        got["scales"] = torch.exp2(e)
    return got


def _exact_axes(s, case):
    got = []
    pairs = case["rot"] // 2
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        x = x.double()
        y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6).sqrt() * w.double()
        z = y.clone()
        for i in range(pairs):  # one rotation pair at a time
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + pairs)
            angle = (s["positions"][s["axis"][i]].double() * float(s["inv_freq"][i]))[:, None]
            z[..., a] = y[..., a] * torch.cos(angle) - y[..., b] * torch.sin(angle)
            z[..., b] = y[..., a] * torch.sin(angle) + y[..., b] * torch.cos(angle)
        z[s["positions"][0] < 0] = 0.0
        got.append(z)
    return tuple(got)


def exact(case, seed):
    s = prepare(case, seed)
    dev = _device()
    if case["op"] == "add_norm":
        return _exact_add_norm(s, case)
    if case["op"] == "axes":
        return _exact_axes(s, case)
    table = _decode_table(dev)
    B, T, hq, hkv, page = (case[k] for k in ("seqs", "q_per_seq", "hq", "hkv", "page"))
    out = torch.zeros((B, T, hq, 128), dtype=torch.float64, device=dev)
    lse = torch.full((B, T, hq), -math.inf, dtype=torch.float64, device=dev)
    for b in range(B):
        n = int(s["seq_len"][b])
        for t in range(T):
            here = n - T + t
            end = here + 1 if case["causal"] else n
            begin = max(0, here + 1 - case["window"]) if case["window"] else 0
            if end <= begin:
                continue
            pos = torch.arange(begin, end, device=dev)
            rows = s["block_table"][b].long()[pos // page] * page + pos % page if page else s["seq_start"][b] + pos
            if case["bits"] == 16:
                k, v = s["k"][rows].double(), s["v"][rows].double()
            else:
                block = rows // case["scale_block"]
                k = table[s["k"][rows].long()] * torch.exp2(s["k_scale"][:, block].double() - 127).T[..., None]
                v = table[s["v"][rows].long()] * torch.exp2(s["v_scale"][:, block].double() - 127).T[..., None]
            q = s["q"][b, t].double().view(hkv, hq // hkv, 128)
            logits = torch.einsum("gmd,sgd->gms", q, k) / 128 ** 0.5
            lse[b, t] = torch.logsumexp(logits, -1).view(hq)
            out[b, t] = torch.einsum("gms,sgd->gmd", torch.softmax(logits, -1), v).reshape(hq, 128)
    return out, lse
