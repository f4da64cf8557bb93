"""Which rows the columns of an attention workgroup's tiles read (CPU): those of other workgroups never, whatever columns are left over.
Results may be written over the queries, and another workgroup may have written its own by then."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_13319_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
FLAGS = ["-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]

PROGRAM = r"""
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include "device_attend.h"
using namespace pipesd;

#define CHECK(x) do { if (!(x)) { printf("%s: group %d, %d rows, %d tiles, column %d of group %d\n", #x, group, rows, tiles, c, g); exit(1); } } while (0)

int main() {
  long idle = 0;
  for (int group = 1; group <= 256; ++group)
    for (int rows : {1, 2, 3, 5, 6, 7, 11, 16, 17, 64, 100, 256, 2047, 2048})
      for (int tiles : {1, 2, 4, 8}) {
        const int all = group * rows, per = 16 * tiles, row_off = 1000, kvh = 3;
        for (int g = 0; g * per < all; ++g)
          for (int c = 0; c < per; ++c)
            for (float rinv : {nextafterf(1.f / group, 0.f), 1.f / group, nextafterf(1.f / group, 2.f)}) {  // (the reciprocal is off by an ulp at most)
              const TileRow t = tile_row(g * per + c, group, rinv, rows, row_off, kvh);
              const int row = t.row - row_off, head = t.head - kvh * group, at = row * group + head;
              CHECK(row >= 0 && row < rows && head >= 0 && head < group);
              CHECK(t.live == (g * per + c < all));
              CHECK(at >= g * per && at < g * per + per);
              if (t.live) CHECK(at == g * per + c);
              else ++idle;
            }
      }
  printf("%ld\n", idle);
  return 0;
}
"""


def test_columns_read_rows_of_their_own_workgroup(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    (tmp_path / "rows.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "-O2", *FLAGS, "-I", CSRC, str(tmp_path / "rows.hip"), "-o", str(tmp_path / "rows")], check=True, capture_output=True)
    done = subprocess.run([str(tmp_path / "rows")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
    assert int(done.stdout) > 10000
