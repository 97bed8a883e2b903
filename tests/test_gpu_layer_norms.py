"""clsa_add_norm and clsa_norm_rope_axes on a GPU against their definitions in 64 bits."""
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


def _rows(g, n, d, scale=1.0, extra=0):
    t = (torch.randn((n, d + extra), generator=g, device=DEV) * scale).to(torch.bfloat16)
    return t[:, :d]


def check_add_norm(spec, x, residual, weight, eps, s, y, codes, scales, group):
    total = x.double() + (0 if residual is None else residual.double())
    want = total * (total.square().mean(-1, keepdim=True) + eps).rsqrt() * (1.0 if weight is None else weight.double())
    if s is not None:
        ref.check_close(s, total, 2.0 ** -8 * total.abs(), "sum")
    if y is not None:
        ref.check_close(y, want, (2.0 ** -8 + 2.0 ** -19) * want.abs(), "y")
    if codes is not None:
        part = want.unflatten(-1, (-1, group))
        e = scales.view(torch.uint8).double() - 127
        best = ref.exponents(part)
        near = (ref.exponents(part * (1 + 2.0 ** -19)) != best) | (ref.exponents(part * (1 - 2.0 ** -19)) != best)
        assert ((e == best) | (near & ((e - best).abs() == 1))).all(), "scales"
        got = ref.e4m3_table(DEV)[codes.view(torch.uint8).long()].unflatten(-1, (-1, group))
        exact = part / torch.exp2(e)[..., None]
        clipped = exact.clamp(-448, 448)
        # half a step: 2^-4 of the value, or half of 2^-9 where codes are subnormal
        tol = torch.maximum(2.0 ** -4 * clipped.abs(), torch.full_like(clipped, 2.0 ** -10)) + 2.0 ** -19 * clipped.abs()
        ref.check_close(got, clipped, tol, "codes")


@pytest.mark.parametrize("dim,group", [(16, 0), (16, 16), (32, 32), (64, 32), (128, 128), (144, 144), (160, 32), (896, 64), (2560, 32), (2560, 2560), (4096, 128),
                                       (4112, 0), (5120, 128), (8192, 8192), (8208, 8208), (16384, 64), (16384, 16384), (16352, 32)])
@pytest.mark.parametrize("rows", [1, 2, 37, 700])
def test_add_norm(rows, dim, group):
    g = torch.Generator(device=DEV)
    g.manual_seed(rows * dim + group)
    weight = (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)
    for k, (with_residual, with_weight, with_sum, with_y, extra) in enumerate([(1, 1, 1, 1, 0), (0, 1, 1, 1, 8), (1, 0, 0, 0, 64), (1, 1, 1, 0, 16)]):
        x = _rows(g, rows, dim, extra=extra)
        r = _rows(g, rows, dim, 3.0, extra=extra * 2) if with_residual else None
        with_y = with_y or not group
        s = _rows(g, rows, dim, extra=extra) if with_sum else None
        y = _rows(g, rows, dim, extra=extra) if with_y else None
        codes = torch.full((rows, dim + 2 * extra), 0x55, dtype=torch.uint8, device=DEV) if group else None
        scales = torch.full((rows, dim // group + extra + 3), 0x55, dtype=torch.uint8, device=DEV) if group else None
        spec = clsa.make_add_norm(dim=dim, eps=1e-5, weight=weight if with_weight else None, scale_group=group)
        clsa.clsa_add_norm(spec, x, r, s, y, None if codes is None else codes[:, :dim], None if scales is None else scales[:, :dim // group])
        check_add_norm(spec, x, r, weight if with_weight else None, 1e-5, s, y, None if codes is None else codes[:, :dim],
                       None if scales is None else scales[:, :dim // group], group)
        if group:  # nothing beside the rows is written
            assert (codes[:, dim:] == 0x55).all() and (scales[:, dim // group:] == 0x55).all()


@pytest.mark.parametrize("dim,group", [(64, 64), (128, 32), (512, 64), (768, 0), (768, 128), (896, 896), (1536, 64), (2304, 32)])
def test_blocks_that_take_many_short_rows(dim, group):
    g = torch.Generator(device=DEV)
    g.manual_seed(dim + group)
    rows = 19003
    x, r, weight = _rows(g, rows, dim), _rows(g, rows, dim, 3.0), (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(torch.bfloat16)
    s, y = torch.empty_like(x), torch.empty_like(x)
    codes = torch.empty((rows, dim), dtype=torch.uint8, device=DEV) if group else None
    scales = torch.empty((rows, dim // group), dtype=torch.uint8, device=DEV) if group else None
    spec = clsa.make_add_norm(dim=dim, eps=1e-5, weight=weight, scale_group=group)
    clsa.clsa_add_norm(spec, x, r, s, y, codes, scales)
    check_add_norm(spec, x, r, weight, 1e-5, s, y, codes, scales, group)


def test_add_norm_in_place_and_shared_rows():
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, r = _rows(g, 300, 2560), _rows(g, 300, 2560, 2.0)
    spec = clsa.make_add_norm(dim=2560)
    s, y = torch.empty_like(x), torch.empty_like(x)
    clsa.clsa_add_norm(spec, x, r, s, y)
    x2, r2 = x.clone(), r.clone()
    clsa.clsa_add_norm(spec, x2, r2, r2, x2)  # the sum into the residual, the norm into x
    assert torch.equal(r2, s) and torch.equal(x2, y)
    shared = r[:1].expand(300, 2560)  # one row that all share
    clsa.clsa_add_norm(spec, x, shared, s, y)
    check_add_norm(spec, x, shared, None, 1e-6, s, y, None, None, 0)
    grid = x.view(3, 100, 2560)
    clsa.clsa_add_norm(spec, grid, shared.view(3, 100, 2560), s.view(3, 100, 2560), y.view(3, 100, 2560))
    check_add_norm(spec, x, shared, None, 1e-6, s, y, None, None, 0)
    clsa.clsa_add_norm(spec, x[:0], None, None, y[:0])  # nothing to do
    torch.cuda.synchronize()


@pytest.mark.parametrize("group", [32, 128, 256])
def test_add_norm_special_rows(group):
    """Rows of zeros, of tiny and large magnitudes, of single spikes; infinities and NaN stay in their row."""
    dim = 256
    x = torch.zeros((10, dim), dtype=torch.bfloat16, device=DEV)
    x[1] = 1e-30
    x[2] = 1e15
    x[3, 5] = 3.0
    x[4, ::2] = -1.0
    x[5, 7] = math.inf
    x[6, 200] = math.nan
    x[7] = 448.0
    x[8] = torch.linspace(-1, 1, dim).to(torch.bfloat16)
    s, y = torch.empty_like(x), torch.empty_like(x)
    weight = torch.ones(dim, dtype=torch.bfloat16, device=DEV)
    weight[3:9] = 2.0 ** 60
    codes, scales = torch.empty((10, dim), dtype=torch.uint8, device=DEV), torch.empty((10, dim // group), dtype=torch.uint8, device=DEV)
    spec = clsa.make_add_norm(dim=dim, eps=1e-6, weight=weight, scale_group=group)
    clsa.clsa_add_norm(spec, x, torch.zeros_like(x), s, y, codes, scales)
    plain = [i for i in range(10) if i not in (5, 6)]
    check_add_norm(spec, x[plain], None, weight, 1e-6, s[plain], y[plain], codes[plain], scales[plain], group)
    assert (scales[0] == 27).all() and (codes[0] == 0).all()
    # an infinity: the norm is 0 and it times 0 is NaN; a NaN: the whole row
    assert torch.isnan(y[5, 7]) and (y[5, :7] == 0).all() and (y[5, 8:] == 0).all() and (codes[5, 7] & 0x7f) == 0x7f
    assert torch.isnan(y[6]).all() and ((codes[6] & 0x7f) == 0x7f).all()


def _rope(n, hq, hk, d, rot, interleaved, axes, num_axes, seed, layout="dense"):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if layout == "fused":
        rows = torch.randn((n, hq + 2 * hk, d), generator=g, device=DEV).to(torch.bfloat16)
        q, k = rows[:, :hq], rows[:, hq:hq + hk]
    else:
        q, k = (torch.randn((n, h, d), generator=g, device=DEV).to(torch.bfloat16) for h in (hq, hk))
    pos = torch.randint(-500, 200000, (num_axes, n), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = pos[0].abs()
    freq = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().to(DEV)
    wq, wk = ((1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))
    return q, k, pos, freq, wq, wk


def _want_rope(x, w, pos, freq, axes, interleaved, norm):
    y = x.double()
    if norm:
        y = y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w.double()
    z, tol = y.clone(), torch.zeros_like(y)
    pairs = freq.numel()
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        angle = (pos[axes[i]].double() * float(freq[i]))[:, None]
        z[..., a] = y[..., a] * torch.cos(angle) - y[..., b] * torch.sin(angle)
        z[..., b] = y[..., b] * torch.cos(angle) + y[..., a] * torch.sin(angle)
        tol[..., a] = tol[..., b] = y[..., a].abs() + y[..., b].abs()
    tol[..., 2 * pairs:] = y[..., 2 * pairs:].abs()
    return z, 2.0 ** -8 * z.abs() + 2.0 ** -19 * tol


@pytest.mark.parametrize("n", [1, 16, 333, 2500])
@pytest.mark.parametrize("d,rot,interleaved", [(64, 64, 0), (128, 128, 0), (128, 64, 0), (128, 128, 1), (256, 256, 0), (256, 32, 1), (128, 96, 0), (128, 48, 1)])
@pytest.mark.parametrize("num_axes,hq,hk,layout", [(3, 32, 8, "fused"), (2, 5, 1, "dense"), (4, 20, 4, "dense"), (1, 8, 2, "fused")])
def test_axes(n, d, rot, interleaved, num_axes, hq, hk, layout):
    pairs = rot // 2
    for axes in ([i % num_axes for i in range(pairs)], [min(num_axes - 1, i * num_axes // pairs) for i in range(pairs)]):
        q, k, pos, freq, wq, wk = _rope(n, hq, hk, d, rot, interleaved, axes, num_axes, n + d, layout)
        skipped = torch.zeros(n, dtype=torch.bool, device=DEV)
        if n > 3:
            skipped[[1, n - 2]] = True
            pos[0, skipped] = -7
        spec = clsa.make_norm_rope(head_dim=d, norm=1, rot_dim=rot, interleaved=interleaved, inv_freq=freq, q_weight=wq, k_weight=wk)
        ax = clsa.make_rope_axes(axes, num_axes=num_axes)
        qo, ko = torch.full((n, hq, d), 9.0, dtype=torch.bfloat16, device=DEV), torch.full((n, hk, d), 9.0, dtype=torch.bfloat16, device=DEV)
        clsa.clsa_norm_rope_axes(spec, ax, pos, q, qo, k, ko)
        for x, w, got in ((q, wq, qo), (k, wk, ko)):
            z, tol = _want_rope(x, w, pos, freq, axes, interleaved, True)
            assert (got[skipped] == 9.0).all()
            ref.check_close(got[~skipped], z[~skipped], tol[~skipped], "heads")


def test_axes_of_one_position_are_the_plain_rotation():
    """Equal positions on all axes, given three times or once: clsa_norm_rope's results bit for bit; in place; [B, T, heads, D]."""
    n, d = 200, 128
    axes = [i % 3 for i in range(64)]
    q, k, pos, freq, wq, wk = _rope(n, 20, 4, d, d, 0, axes, 3, 5)
    pos[1] = pos[2] = pos[0]
    spec = clsa.make_norm_rope(head_dim=d, rot_dim=d, inv_freq=freq, q_weight=wq, k_weight=wk)
    ax = clsa.make_rope_axes(axes)
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    clsa.clsa_norm_rope(spec, pos[0].contiguous(), q, want_q, k, want_k)
    for given in (pos, pos[0].contiguous(), pos[0][None].expand(3, n)):
        a, b = torch.empty_like(q), torch.empty_like(k)
        clsa.clsa_norm_rope_axes(spec, ax, given, q, a, k, b)
        assert torch.equal(a, want_q) and torch.equal(b, want_k)
    wide = torch.zeros((3, n + 100), dtype=torch.int32, device=DEV)  # rows further apart than they are long
    wide[:, :n] = pos
    a = q.clone().view(10, 20, 20, d)
    clsa.clsa_norm_rope_axes(spec, ax, wide[:, :n], a, a)
    assert torch.equal(a.view_as(q), want_q)
    clsa.clsa_norm_rope_axes(spec, ax, pos[:, :0], q[:0], a[:0, 0], None, None)
    torch.cuda.synchronize()
