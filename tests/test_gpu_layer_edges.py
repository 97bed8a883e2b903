"""Calls around a layer's cache at the edges of what their header allows, on a GPU against the definitions in 64 bits."""
import math
import os

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import __graft_entry__ as entry

entry._load_build_module().build()

import _layer_ref as ref
import paper_2606_06467_b200 as clsa
from test_gpu_dense_attn import SM, Problem
from test_gpu_layer_norms import check_add_norm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("gap,exponent", [(20.0, 0), (23.4, 0), (24.5, 0), (25.1, 0), (28.0, 0), (31.0, 0), (15.0, 10)])
@pytest.mark.parametrize("T,heads", [(1, (32, 8)), (3, (20, 4)), (16, (8, 2))], ids=str)
def test_a_flat_tail_behind_large_weights(T, heads, gap, exponent):
    """One row of every 32 has 2^gap times the others' weight and a V of zeros: the outputs are the others' alone. exponent: of the V scale in
    those rows' blocks."""
    p = Problem([2048, 333], *heads, T=T, eight=True, block=16, seed=3)
    p.q.fill_(gap * math.log(2.0) / (SM * 128))
    p.ks.fill_(127)
    p.vs.fill_(127)
    for b, n in enumerate(p.lens):
        r = p.row_of(b, torch.arange(n, device=DEV))
        strong = torch.arange(n, device=DEV) % 32 == 5
        p.k[r] = torch.where(strong, 0x38, 0).to(torch.uint8)[:, None, None].expand(n, heads[1], 128)  # 1 and 0
        p.v[r] = torch.where(strong, 0, 0x38).to(torch.uint8)[:, None, None].expand(n, heads[1], 128)  # 0 and 1
        p.vs[:, r[strong] // 16] = 127 + exponent
    p.run()
    torch.cuda.synchronize()
    assert clsa.clsa_device_status(p.ws) == 0
    out, lse, _, ltol = p.want()
    ref.check_close(p.lse, lse, ltol, "lse")
    # Logits are off by eps, all weights' sum with them, a weight by 2^-11 and by 2^-25 of f16's steps, of which the largest weight is at least 2^11:
    # 2^-36 max(p 2^ev) of every code. The largest p is 1 / (32's number) at most.
    x = gap * math.log(2.0) * 1.01
    eps, tol = 2.0 ** -16 * x + 2.0 ** -22 * (2 * x + 16), torch.zeros_like(out)
    for b, n in enumerate(p.lens):
        steps = 2.0 ** -22 * (n / 16 + 64)
        largest = 2.0 ** exponent / len(range(5, n, 32))
        tol[b] = (2.0 ** -8 + 2.0 ** -11 + 4 * eps + 2 * steps) * out[b].abs() + 2.0 ** -36 * largest * n
    ref.check_close(p.out, out, tol, "out")


@pytest.mark.parametrize("dim,group", [(256, 32), (512, 512), (2560, 0), (2560, 2560), (8192, 128)])
def test_add_norm_in_place_over_many_rows(dim, group):
    """Blocks that stay and fetch rows ahead of those that they overwrite; a row that all share; arguments side by side in one buffer."""
    rows = 4099
    g = torch.Generator(device=DEV)
    g.manual_seed(dim + group)
    new = lambda: torch.randn((rows, dim), generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    x, r, weight = new(), new() * 3, (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)
    spec = clsa.make_add_norm(dim=dim, eps=1e-5, weight=weight, scale_group=group)
    outs = lambda: (torch.full((rows, dim), 0x55, dtype=torch.uint8, device=DEV), torch.full((rows, dim // group), 0x55, dtype=torch.uint8, device=DEV)) if group else (None, None)  # noqa: E731
    s, y = torch.empty_like(x), torch.empty_like(x)
    codes, scales = outs()
    clsa.clsa_add_norm(spec, x, r, s, y, codes, scales)
    check_add_norm(spec, x, r, weight, 1e-5, s, y, codes, scales, group)

    def same(a, b):
        assert (a is None and b is None) or torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))

    for into_s, into_y in (("x", "r"), ("r", "x"), ("x", None), (None, "r"), ("r", "own")):
        t = dict(x=x.clone(), r=r.clone(), own=torch.empty_like(x))
        c2, e2 = outs()
        if into_y is None and not group:
            into_y = "own"
        clsa.clsa_add_norm(spec, t["x"], t["r"], t.get(into_s), t.get(into_y), c2, e2)
        if into_s:
            same(t[into_s], s)
        if into_y:
            same(t[into_y], y)
        same(c2, codes), same(e2, scales)
    t = x.clone()
    clsa.clsa_add_norm(spec, t, t, t, y, None, None) if not group else clsa.clsa_add_norm(spec, t, t, t, y, *outs())
    check_add_norm(spec, x, x, weight, 1e-5, t, y, None, None, group)
    shared, t = r[17:18].clone().expand(rows, dim), x.clone()
    clsa.clsa_add_norm(spec, t, shared, t, y, *outs())
    check_add_norm(spec, x, shared, weight, 1e-5, t, y, None, None, group)
    wide = torch.zeros((rows, 5 * dim), dtype=torch.bfloat16, device=DEV)
    part = [wide[:, k * dim:(k + 1) * dim] for k in range(5)]
    part[0].copy_(x), part[2].copy_(r)
    tail = part[4].view(torch.uint8)
    clsa.clsa_add_norm(spec, part[0], part[2], part[1], part[3], *((tail[:, :dim], tail[:, dim:dim + dim // group]) if group else (None, None)))
    want = dict(zip(range(4), (x, s, r, None)))
    for k in (0, 1, 2):
        same(part[k], want[k])
    check_add_norm(spec, x, r, weight, 1e-5, part[1], part[3], *((tail[:, :dim], tail[:, dim:dim + dim // group]) if group else (None, None)), group)
    assert group == 0 or (tail[:, dim + dim // group:] == 0).all()


def test_the_readme_runs():
    """The documented calls around a layer as they stand there, and their attention's results."""
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    block = text[text.index("### Around a layer"):].split("```python\n")[1].split("```")[0]
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    n16 = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    w = Problem([700, 33], 32, 8, causal=1, window=512, seed=31)
    w8 = Problem([700, 33], 32, 8, causal=1, eight=True, block=64, seed=32)
    assert w.rows <= w8.rows
    names = dict(clsa=clsa, torch=torch, B=2, T=1, n=700, rows=w.rows, seq_start=w.start, seq_len=w.seq_len, k_cache=w.k, v_cache=w.v, q=w.q, out=w.out,
                 lse=w.lse, cache=w8.cache, inv_freq=torch.rand(64, generator=g, device=DEV), w_norm=n16(2560), wq=n16(128), wk=n16(128), x=n16(2, 1, 2560),
                 residual=n16(2, 1, 2560), x_sum=n16(2, 1, 2560), codes=torch.zeros(2, 1, 2560, dtype=torch.uint8, device=DEV),
                 scales=torch.zeros(2, 1, 80, dtype=torch.uint8, device=DEV), positions=torch.tensor([[699, 32], [5, 6], [7, 8]], dtype=torch.int32, device=DEV),
                 k=n16(2, 1, 8, 128))
    first = block.index("clsa.clsa_dense_attn8(")
    exec(block[:first], names)
    torch.cuda.synchronize()
    out, lse, tol, ltol = w.want()
    ref.check_close(w.lse, lse, ltol, "lse")
    ref.check_close(w.out, out, tol, "out")
    w8.start, w8.q = w.start, w.q  # (the other cache's rows are where this one's are)
    exec(block[first:], names)
    out, lse, tol, ltol = w8.want()
    ref.check_close(w.out, out, tol, "out over codes")


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("scale", [1e-9, 1e-20, 1e-44])
def test_tiny_scales_and_queries(eight, scale):
    """Logits of next to nothing: the mean of what is seen. (A factor that falls to 0 would make NaN of the logits, -inf, of what is not seen.)"""
    p = Problem([100, 17, 1], 8, 2, T=2, causal=0, eight=eight, seed=33)
    p.q.zero_()
    p.p.sm_scale = scale
    p.check()
    p.q.fill_(2.0 ** -100)
    p.run()
    p.q.zero_()  # (the reference's: its scale is another)
    out, lse, tol, ltol = p.want()
    ref.check_close(p.lse, lse, ltol, "lse")
    ref.check_close(p.out, out, tol, "out")


@pytest.mark.parametrize("eight", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("power", [-100, -30, 30, 100])
def test_scales_and_queries_that_make_up_for_one_another(eight, power):
    p = Problem([300, 77], 16, 4, eight=eight, seed=34)
    if eight:
        p.check()
    q = p.q.clone()
    p.q.copy_((q.float() * 2.0 ** power).to(torch.bfloat16))
    p.p.sm_scale = SM * 2.0 ** -power
    p.run()
    p.q.copy_(q)
    out, lse, tol, ltol = p.want()
    ref.check_close(p.lse, lse, ltol, "lse")
    ref.check_close(p.out, out, tol, "out")


@pytest.mark.parametrize("rows,dim,group", [(15, 512, 32), (3000, 1536, 128), (700, 4096, 4096)])
def test_norm_codes_captured_and_replayed(rows, dim, group):
    """Every output of the eager call, and of replays with other inputs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    new = lambda: torch.randn((rows, dim), generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    x, r, s, y = new(), new(), new(), new()
    weight = (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)
    codes, scales = torch.zeros((rows, dim), dtype=torch.uint8, device=DEV), torch.zeros((rows, dim // group), dtype=torch.uint8, device=DEV)
    spec = clsa.make_add_norm(dim=dim, eps=1e-5, weight=weight, scale_group=group)
    call = lambda: clsa.clsa_add_norm(spec, x, r, s, y, codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu))  # noqa: E731
    call()
    check_add_norm(spec, x, r, weight, 1e-5, s, y, codes, scales, group)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for size in (1.0, 100.0):
        x.copy_(new() * size)
        r.copy_(new())
        for t in (s, y, codes, scales):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_add_norm(spec, x, r, weight, 1e-5, s, y, codes, scales, group)
