"""Host-side checks of the calls around a layer's cache at the edges of what their header allows; no GPU."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
from test_cache8_edges_host import BF16, U8, Tensor
from test_layer_host import binding, clsa  # noqa: F401 (fixtures)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_06467_b200", "csrc")


def test_notes_of_units_that_nobody_wrote_name_no_records(tmp_path):
    """Whatever scratch holds where a launch gave up, the joining kernel reads records of existing stretches or none."""
    src, exe = tmp_path / "units.cpp", tmp_path / "units"
    src.write_text("""
#include <initializer_list>
#include <stdint.h>
#include <stdio.h>
#include "dense_units.h"
using namespace clsa;
int main() {
  const int odd[] = {INT32_MIN, INT32_MIN + 1, -2, -1, 0, 1, 2, 3, 17, 18, 147, 148, 149, 295, 296, 297, 0x7f7f7f7f, INT32_MAX - 1, INT32_MAX};
  for (int spans : {1, 18, 148}) {
    for (int begin : odd)
      for (int last : odd) {
        const Noted n = noted_unit(begin, last, spans);
        const long first = begin >= 0 ? begin / 2 : -1;
        const bool possible = first >= 0 && first <= last && last < spans;
        if (n != (!possible ? Noted::kNever : first < last ? Noted::kCut : Noted::kWhole)) return printf("%d %d %d\\n", begin, last, spans), 1;
      }
    for (int first = 0; first < spans; ++first)
      for (int last = first; last < spans; ++last)
        for (int aside = 0; aside < 2; ++aside)
          if (noted_unit(2 * first + aside, last, spans) != (first < last ? Noted::kCut : Noted::kWhole)) return 2;
  }
  return 0;
}
""")
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0


def test_add_norm_refuses_outputs_that_share_memory(clsa):
    raw, P = clsa.raw(), ctypes.byref
    base = dict(x=(0x1000000, 256), residual=(0x2000000, 256), sum_out=(0x3000000, 256), y_out=(0x4000000, 256), codes_out=(0x5000000, 256),
                scales_out=(0x6000000, 8))

    def call(n=100, weight=0x7000000, **kw):
        args = [clsa.clsa_rows(*v) if v else None for v in {**base, **kw}.values()]
        return raw.clsa_add_norm(P(clsa.clsa_add_norm_spec(256, 1e-6, weight, 32)), n, *(P(a) if a else None for a in args), None)

    bad = [
        dict(codes_out=base["x"]), dict(codes_out=base["residual"]), dict(codes_out=base["sum_out"]), dict(codes_out=base["y_out"]),
        dict(codes_out=(0x1000000, 512)), dict(codes_out=(0x1000000 + 51200 - 16, 512)), dict(codes_out=(0x1000000 - 99 * 256 - 16, 256)),  # x: 51200 bytes
        dict(scales_out=base["x"]), dict(scales_out=(0x5000000, 256)), dict(scales_out=(0x5000000 + 99 * 256 + 255, 8)), dict(scales_out=(0x4000000 - 799, 8)),
        dict(sum_out=(0x1000000 + 16, 256)), dict(y_out=(0x2000000 - 512, 256)), dict(y_out=(0x3000000 + 512, 256)),  # a row, or some elements, further on
        dict(sum_out=(0x1000000 + 256, 512), x=(0x1000000, 512)), dict(y_out=(0x1000000, 512)),  # half of each row; in place with another distance
        dict(x=(0x3000000, 0)), dict(residual=(0x4000000 + 99 * 512, 0)),  # a shared row that is one of an output's
        dict(weight=0x3000000 + 512), dict(weight=0x5000000 + 16), dict(weight=0x6000000 + 16),
        dict(sum_out=base["x"], residual=(0x1000000 + 512, 256)),  # in place over rows that the residual has too
        dict(n=1, codes_out=base["x"]), dict(n=1, scales_out=(0x5000000 + 255, 8)), dict(n=1, sum_out=(0x1000000 + 496, 256)),
        dict(codes_out=(0x3000000 + 1024, 256)), dict(n=1 << 30, x=(0x1000000, 1 << 60), sum_out=(0x1000000 + 16, 1 << 60)),
    ]
    for kw in bad:
        assert call(**kw) == 1, kw


def test_the_readme_makes_params_that_the_dense_calls_take(clsa):
    """The documented calls around a layer, with stand-ins for what they launch: the params are complete (0; 4 where there is no device)."""
    text = open(os.path.join(ROOT, "README.md")).read()
    block = text[text.index("### Around a layer"):].split("```python\n")[1].split("```")[0]
    made = []

    class Stand:
        def __getattr__(self, name):
            if name.startswith("make_"):
                return getattr(clsa, name)
            if name == "clsa_dense_workspace_bytes":
                return lambda p: made.append(p) or 1024
            return lambda *a: made.extend(x for x in a if isinstance(x, clsa.clsa_params)) or 0

    kv = lambda: torch.zeros(256, 8, 128, dtype=torch.bfloat16)  # noqa: E731
    names = dict(clsa=Stand(), torch=torch, B=2, T=1, n=100, rows=256, seq_start=torch.tensor([0, 128]), seq_len=torch.tensor([100, 7], dtype=torch.int32),
                 k_cache=kv(), v_cache=kv(), inv_freq=torch.zeros(64), w_norm=torch.zeros(2560, dtype=torch.bfloat16), wq=torch.zeros(128, dtype=torch.bfloat16),
                 wk=torch.zeros(128, dtype=torch.bfloat16), **{k: None for k in "x residual x_sum codes scales positions q k out lse cache".split()})
    exec(block.replace('device="cuda"', 'device="cpu"'), names)
    assert len(made) == 3
    n = ctypes.c_size_t(0)
    for p in made:
        assert clsa.raw().clsa_dense_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) in (0, 4)


@pytest.mark.parametrize("shape", [(0, 256), (2, 0, 256), (0, 5, 256), (3, 0, 2, 256), (2, 2, 0, 256)])
def test_the_binding_takes_batches_without_rows(binding, shape):  # noqa: F811
    clsa, calls = binding
    spec = clsa.make_add_norm(dim=256, scale_group=32)
    t, c, e = Tensor(shape, BF16), Tensor(shape, U8), Tensor((*shape[:-1], 8), U8)
    for args in ((t, None, None, t, None, None), (t, t, t, None, c, e)):
        clsa.clsa_add_norm(spec, *args)
        assert calls in (["clsa_add_norm"], ["native clsa_add_norm"])
        calls.clear()
