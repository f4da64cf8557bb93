"""What the 4-bit cache allocates at its creation is enough for every pass that the interface says it is for: up to 16 clients of up to
32 rows, at whatever lengths.  On the host, over many ragged passes; and on the device, where such a pass takes no memory."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2605_13319_amd import nav
from tests.test_gpu_kv4 import shape_of

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13319_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "kv4.h"
using namespace pipesd;
int main() {
  unsigned seed = 5;
  auto rnd = [&](long n) { seed = seed * 1664525u + 1013904223u; return (long)((seed >> 8) % (unsigned long)n); };
  const int heads[][2] = {{32, 8}, {40, 40}, {128, 16}, {8, 2}, {256, 1}, {4, 4}, {24, 8}, {1, 1}, {7, 1}, {64, 8}};
  std::vector<Kv4Launch> out;
  double closest = 0;
  for (auto& h : heads)
    for (int hd : {64, 128})
      for (int dtype : {PIPESD_F32, PIPESD_BF16})
        for (int n_cu : {256, 304, 64, 1})
          for (int t = 0; t < 1500; ++t) {
            const int clients = 1 + (int)rnd(16), most_rows = 1 + (int)rnd(32), most_len = 33 + (int)rnd(1l << (1 + rnd(20)));
            const Kv4PlanNeeds most = kv4_plan_most(clients, most_rows, most_len, dtype, hd, h[0], h[1], n_cu);
            const int mode = (int)rnd(4), n = rnd(2) ? clients : 1 + (int)rnd(clients), same = 1 + (int)rnd(most_rows), len = 1 + (int)rnd(most_len);
            std::vector<Kv4Client> cl;
            for (int i = 0; i < n; ++i) {
              const int rows = mode & 1 ? same : 1 + (int)rnd(most_rows);
              cl.push_back(Kv4Client{i, rows, 0, std::max(rows, mode & 2 ? len : i == 0 ? most_len : 1 + (int)rnd(most_len))});
            }
            const Kv4PlanNeeds need = kv4_plan(cl.data(), n, dtype, hd, h[0], h[1], n_cu, out);
            if (need.part_tiles > most.part_tiles || need.counters > most.counters) {
              printf("%zu of %zu tiles, %zu of %zu counters: heads %d/%d x %d, dtype %d, %d CUs;", need.part_tiles, most.part_tiles, need.counters, most.counters,
                     h[0], h[1], hd, dtype, n_cu);
              for (auto& c : cl) printf(" %d rows of %d tokens,", c.n_rows, c.len);
              printf("\n");
              return 1;
            }
            if (most.part_tiles) closest = std::max(closest, need.part_tiles / (double)most.part_tiles);
          }
  printf("%f\n", closest);
  return 0;
}
"""


def test_no_pass_takes_more_than_the_most(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    (tmp_path / "most.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", CSRC,
                    str(tmp_path / "most.hip"), "-o", str(tmp_path / "most")], check=True, capture_output=True)
    r = subprocess.run([str(tmp_path / "most")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert float(r.stdout) > 0.5  # (and it is not many times what is needed)


# heads, clients, rows of each, tokens of each
CASES = [((32, 8, 128), [32] * 5, [32000] * 5), ((32, 8, 128), [32] * 11, [8192] * 11), ((32, 8, 128), [32] * 13, [32000] * 13),
         ((128, 16, 64), [32, 31, 30, 32] * 4, [16000, 9000, 12000, 3] * 4), ((4, 4, 64), [3] * 16, [9000] * 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("heads,rows,before", CASES)
def test_a_pass_takes_no_memory(heads, rows, before):
    n = len(rows)
    kv = nav.KV4Cache(shape_of(*heads), 16, sum(-(-(b + r) // 16) for b, r in zip(before, rows)))
    kv.extend(list(range(n)), before)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    kv.extend(list(range(n)), rows)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
