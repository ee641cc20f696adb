"""The layouts that the cases of test_gpu_rotate_many.py take, by the library's own rules on the host (CPU: no kernel is run)."""
import os
import shutil
import subprocess

import pytest

import test_gpu_rotate_many as many
from paper_2406_05317_amd import build as lib_build

TEXT = """#include "rows_rotate.hip"
#include "pages_append.hip"
#include <cstdio>
int lococo::cu_count() { return 256; }
using namespace lococo;
int main() {
  char what;
  int tokens, hq, hkv, d, banks;
  while (std::scanf(" %c %d %d %d %d %d", &what, &tokens, &hq, &hkv, &d, &banks) == 6) {
    RotateView rv{};
    rv.heads[0] = hq;
    rv.heads[1] = hkv;
    rv.ws[0] = rv.ws[1] = banks ? d : 0;
    rv.d = d;
    PagesView pg{};
    pg.Hq = hq;
    pg.Hkv = hkv;
    pg.d = d;
    if (what == 'f') {
      const RotatePlan p = rotate_plan(rv, tokens);
      std::printf("%d %d %lld\\n", 1 << p.sh.lt, p.sh.hb, (long long)p.groups);
    } else if (what == 'a') {
      const AppendPlan p = append_plan(pg, tokens);
      std::printf("%d %d %lld\\n", 1 << p.sh.lt, p.sh.hb, (long long)p.groups);
    } else {
      const BackPlan p = back_plan(rv, tokens);
      std::printf("%d %d %d\\n", 1 << p.sh.lt, p.tiles, p.chunks);
    }
  }
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_layouts_of_many_rows(tmp_path):
    (tmp_path / "plans.hip").write_text(TEXT)
    r = subprocess.run(["hipcc", "-x", "hip", *lib_build.FLAGS, "-I", lib_build.CSRC, str(tmp_path / "plans.hip"), "-o", str(tmp_path / "plans")],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    cases = [("f", c) for c in many.FORWARDS] + [("a", c) for c in many.APPENDS] + [("b", c) for c in many.BACKWARDS]
    asked = "".join(f"{k} {c[0] * c[1]} {c[2]} {c[3]} {c[4]} {int(c[8] == 'heads')}\n" for k, c in cases)
    out = subprocess.run([str(tmp_path / "plans")], input=asked, capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and len(out.stdout.splitlines()) == len(cases)
    for (k, c), line in zip(cases, out.stdout.splitlines()):
        positions, x, groups = map(int, line.split())
        tokens, d = c[0] * c[1], c[4]
        lanes = 1
        while 8 * lanes < d:
            lanes *= 2
        assert positions == 256 // lanes, (k, c)                        # positions side by side, a last tile that is not full
        assert tokens % positions, (k, c)
        if k == "b":
            tiles = -(-tokens // positions)
            assert x > 1 and tiles % x, (k, c, line)                    # tiles in turn, fewer for the last workgroup
        else:
            assert x < max(c[2], c[3]) and max(c[2], c[3]) % x, (k, c)  # heads in turn, and a second block of them
