"""Calls around a layer's cache at the edges of what their header allows, on a GPU against the definitions in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import __graft_entry__ as entry

entry._load_build_module().build()

import _layer_ref as ref
import paper_2606_06467_b200 as clsa
from test_gpu_dense_attn import SM, Problem

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
