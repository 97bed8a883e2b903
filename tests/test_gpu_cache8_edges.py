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
