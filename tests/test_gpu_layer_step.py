"""The calls around a layer's cache one after another, as a decoder runs them: addition and norm, projection and append, rotation over
three axes, attention over the window and over everything, over bf16 and over 8-bit caches; eager, captured and replayed."""
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


@pytest.mark.parametrize("T,hq,hkv", [(1, 20, 4), (3, 32, 8)])
def test_a_layers_step(T, hq, hkv):
    B, dm, page, ctx = 5, 512, 64, 700
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    n16 = lambda *s, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(torch.bfloat16)  # noqa: E731
    lens = [T, 64, 129, 500, ctx]
    per = -(-ctx // page)
    rows = B * per * page
    table = torch.randperm(B * per, generator=g, device=DEV).to(torch.int32).view(B, per)
    seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    k, v, idx_k = n16(rows, hkv, 128), n16(rows, hkv, 128), n16(rows, 128)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)  # noqa: E731
    c = clsa.make_cache8(k=u8(rows, hkv, 128), v=u8(rows, hkv, 128), k_scale=u8(hkv, rows // 64), v_scale=u8(hkv, rows // 64), idx_k=u8(rows, 128),
                         idx_k_scale=u8(rows // 64), scale_block=64)
    make = lambda t, **kw: clsa.make_params(num_seqs=B, q_per_seq=t, num_q_heads=hq, num_kv_heads=hkv, idx_dim=128, top_k=64, causal=1, max_seq_len=ctx,  # noqa: E731
                                            sm_scale=SM, num_cache_rows=rows, block_table=table, block_size=page, k_cache=k, v_cache=v, idx_k_cache=idx_k, **kw)
    p = make(T, seq_len=seq_len)
    ws = torch.zeros(max(clsa.clsa_dense_workspace_bytes(p), clsa.clsa_cache8_workspace_bytes(p, c)), dtype=torch.uint8, device=DEV)
    ws_project = torch.zeros(clsa.clsa_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    # the 8-bit cache's older rows
    for b, n in enumerate(lens):
        if n > T:
            pos = torch.arange(n - T, device=DEV)
            r = table[b].long()[pos // page] * page + pos % page
            old = clsa.make_params(num_seqs=1, q_per_seq=n - T, num_q_heads=hq, num_kv_heads=hkv, idx_dim=128, top_k=1, causal=1, max_seq_len=n - T, sm_scale=SM,
                                   seq_len=torch.tensor([n - T], dtype=torch.int32, device=DEV), num_cache_rows=rows, block_table=table[b:b + 1], block_size=page)
            clsa.clsa_cache8_append(old, c, None, k[r][None].contiguous(), v[r][None].contiguous(), None, ws)
            torch.cuda.synchronize()
    x, stream_in = n16(B, T, dm), n16(B, T, dm, scale=2.0)
    weight = (1 + 0.1 * torch.randn(dm, generator=g, device=DEV)).to(torch.bfloat16)
    add = clsa.make_add_norm(dim=dm, weight=weight, scale_group=32)
    w_idx, w_ik, w_k, w_v, w_q = (n16(o, dm, scale=dm ** -0.5) for o in (128, 128, hkv * 128, hkv * 128, hq * 128))
    freq = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float().to(DEV)
    spec = clsa.make_norm_rope(head_dim=128, rot_dim=128, inv_freq=freq)
    axes = clsa.make_rope_axes([i % 3 for i in range(64)])
    pos = torch.randint(0, 5000, (3, B * T), generator=g, device=DEV, dtype=torch.int32)
    stream, h = torch.empty_like(x), torch.empty_like(x)
    codes, scales = u8(B, T, dm), u8(B, T, dm // 32)
    q_idx = torch.empty((B, T, 128), dtype=torch.bfloat16, device=DEV)
    q, q_turned = (torch.empty((B, T, hq, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    outs = [torch.empty_like(q) for _ in range(4)]
    lses = [torch.empty((B, T, hq), device=DEV) for _ in range(4)]
    k_new, v_new = (torch.empty((B, T, hkv, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step():
        clsa.clsa_add_norm(add, x, stream_in, stream, h, codes, scales)
        clsa.clsa_project_append(p, dm, h, w_idx, w_ik, w_k, w_v, q_idx, idx_k, k, v, ws_project)
        torch.matmul(h.view(-1, dm), w_q.t(), out=q.view(B * T, hq * 128))
        clsa.clsa_norm_rope_axes(spec, axes, pos, q, q_turned)
        for i, window in enumerate((0, 100)):
            clsa.clsa_dense_attn(p, window, q_turned, outs[i], lses[i], ws)
        torch.matmul(h.view(-1, dm), w_k.t(), out=k_new.view(B * T, hkv * 128))
        torch.matmul(h.view(-1, dm), w_v.t(), out=v_new.view(B * T, hkv * 128))
        clsa.clsa_cache8_append(p, c, None, k_new, v_new, None, ws)
        for i, window in enumerate((0, 100)):
            clsa.clsa_dense_attn8(p, c, window, q_turned, outs[2 + i], lses[2 + i], ws)

    step()
    torch.cuda.synchronize()
    assert clsa.clsa_device_status(ws) == 0 and clsa.clsa_device_status(ws_project) == 0
    total = x.double() + stream_in.double()
    normed = total * (total.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.double()
    ref.check_close(stream, total, 2.0 ** -8 * total.abs(), "stream")
    ref.check_close(h, normed, (2.0 ** -8 + 2.0 ** -19) * normed.abs(), "h")
    table8 = ref.e4m3_table(DEV)
    kept = c._tensors
    for i, (window, eight) in enumerate(((0, False), (100, False), (0, True), (100, True))):
        def side(t, scale, b):
            at = torch.arange(lens[b], device=DEV)
            r = table[b].long()[at // page] * page + at % page
            ok = torch.ones(lens[b], dtype=torch.bool, device=DEV)
            if not eight:
                return t[r].double(), ok, None
            f = torch.exp2(scale[:, r // 64].double() - 127).T
            return table8[t[r].long()] * f[..., None], ok, f
        K, V = (kept[0], kept[1]) if eight else (k, v)
        eps = 2.0 ** -11 if eight else 2.0 ** -16
        out, lse, tol, ltol = ref.dense(q_turned, lambda b: side(K, kept[2], b)[:2], lambda b: side(V, kept[3], b)[::2], lens, T, hq // hkv, SM, 1, window, eps)
        ref.check_close(outs[i], out, tol, f"out {i}")
        ref.check_close(lses[i], lse, ltol, f"lse {i}")
    # the same step captured and replayed: the same results, bit for bit
    kept_out = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    side_stream = torch.cuda.Stream()
    side_stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side_stream):
        step()  # (the matrix products' own workspaces)
    torch.cuda.current_stream().wait_stream(side_stream)
    with torch.cuda.graph(graph):
        step()
    for o in outs:
        o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(kept_out, outs):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert clsa.clsa_device_status(ws) == 0
