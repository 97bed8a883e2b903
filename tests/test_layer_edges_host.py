"""Host-side checks of the calls around a layer's cache at the edges of what their header allows; no GPU."""
import os
import subprocess

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
