"""Host-side checks of the calls around a layer's cache at the edges of what their header allows; no GPU."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
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
