"""The plan of a pass over the 4-bit cache, on the host: every client's rows and tokens are covered once by workgroups whose
partial rows and counters lie apart, splits are as few as the joins take, and which kernel passes are given to, those of
tests/test_gpu_kv4_many.py among them.  And the compiled kernels: no result of the matrix cores is read early."""
import os
import re
import shutil
import subprocess

import pytest

from tests import isa_lint
from tests.test_gpu_kv4_many import CASES

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13319_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
#include "kv4.h"
using namespace pipesd;
static std::vector<Kv4Launch> out;
static int fail(const char* what, int nq, int nkv, int hd, int dtype, const std::vector<Kv4Client>& cl) {
  printf("%s: heads %d/%d x %d, dtype %d;", what, nq, nkv, hd, dtype);
  for (auto& c : cl) printf(" %d rows of %d tokens,", c.n_rows, c.len);
  printf("\n");
  return 1;
}
static int check(int nq, int nkv, int hd, int dtype, int n_cu, const std::vector<Kv4Client>& cl) {
  const Kv4PlanNeeds need = kv4_plan(cl.data(), (int)cl.size(), dtype, hd, nq, nkv, n_cu, out);
  std::vector<int> seen(cl.size(), 0);
  size_t part = 0, count = 0;
  for (const Kv4Launch& l : out) {
    if (l.c.n < 1 || l.c.n > kKv4ClientsPerLaunch || l.c.span < 1) return fail("launch", nq, nkv, hd, dtype, cl);
    int item = 0;
    for (int j = 0; j < kKv4ClientsPerLaunch; ++j) {
      if (l.c.first[j] != item) return fail("items", nq, nkv, hd, dtype, cl);
      if (j >= l.c.n) continue;
      size_t i = 0;
      while (i < cl.size() && !(cl[i].seq == l.c.seq[j])) ++i;
      if (i == cl.size() || seen[i]++) return fail("client", nq, nkv, hd, dtype, cl);
      const Kv4Client& c = cl[i];
      const long tiles = ((long)(nq / nkv) * c.n_rows + 15) / 16;
      if (l.c.len[j] != c.len || l.c.n_rows[j] != c.n_rows || l.c.row_off[j] != c.row_off) return fail("numbers", nq, nkv, hd, dtype, cl);
      if ((long)l.c.groups[j] * l.tiles < tiles || (long)(l.c.groups[j] - 1) * l.tiles >= tiles) return fail("groups", nq, nkv, hd, dtype, cl);
      const long n = l.c.nsplit[j], span = l.c.span;
      if (n < 1 || n > kKv4MaxSplits || n * span + kKv4SplitSlack < c.len || (n - 1) * span >= c.len) return fail("splits", nq, nkv, hd, dtype, cl);
      if (n > 1) {
        if ((size_t)l.c.part_off[j] != part) return fail("partials", nq, nkv, hd, dtype, cl);
        part += (size_t)nkv * l.c.groups[j] * n * l.tiles;
      }
      if ((size_t)l.c.count_off[j] != count) return fail("counters", nq, nkv, hd, dtype, cl);
      count += (size_t)nkv * l.c.groups[j];
      item += l.c.groups[j] * n;
      if (l.wide ? l.tiles != kKv4WideTiles : l.tiles != 1 && (l.tiles != 2 || dtype == PIPESD_F32)) return fail("tiles", nq, nkv, hd, dtype, cl);
    }
    if (l.c.items != item || item > 65535) return fail("number of items", nq, nkv, hd, dtype, cl);
  }
  for (size_t i = 0; i < cl.size(); ++i)
    if (seen[i] != (cl[i].n_rows > 0)) return fail("a client missing", nq, nkv, hd, dtype, cl);
  if (part != need.part_tiles || count != need.counters) return fail("needs", nq, nkv, hd, dtype, cl);
  return 0;
}
int main(int argc, char** argv) {
  if (!strcmp(argv[1], "kind")) {  // nq nkv hd dtype n_cu (len rows)...: per client, tiles of a workgroup and splits
    const int nq = atoi(argv[2]), nkv = atoi(argv[3]), hd = atoi(argv[4]), dtype = atoi(argv[5]), n_cu = atoi(argv[6]);
    std::vector<Kv4Client> cl;
    int row = 0;
    for (int i = 7; i + 1 < argc; i += 2) {
      cl.push_back(Kv4Client{(int)cl.size(), atoi(argv[i + 1]), row, atoi(argv[i])});
      row += atoi(argv[i + 1]);
    }
    if (check(nq, nkv, hd, dtype, n_cu, cl)) return 1;
    for (size_t i = 0; i < cl.size(); ++i)
      for (const Kv4Launch& l : out)
        for (int j = 0; j < l.c.n; ++j)
          if (l.c.seq[j] == (int)i) printf("%d %d\n", l.tiles, l.c.nsplit[j]);
    return 0;
  }
  unsigned seed = 99;
  auto rnd = [&](long n) { seed = seed * 1664525u + 1013904223u; return (long)((seed >> 8) % (unsigned long)n); };
  const int heads[][2] = {{1, 1}, {8, 2}, {32, 8}, {40, 40}, {7, 1}, {256, 1}, {64, 8}};
  long kinds[3] = {0, 0, 0};
  for (int t = 0; t < 20000; ++t) {
    const int* h = heads[rnd(7)];
    const int hd = rnd(2) ? 64 : 128, dtype = rnd(3) ? PIPESD_BF16 : PIPESD_F32, n_cu = rnd(4) ? 256 : 1 + (int)rnd(304);
    const int n = rnd(3) ? 1 + (int)rnd(5) : 1 + (int)rnd(70);
    std::vector<Kv4Client> cl;
    int row = 0;
    for (int i = 0; i < n; ++i) {
      const int rows = rnd(12) == 0 ? 0 : rnd(3) ? 1 + (int)rnd(32) : 1 + (int)rnd(kKv4MaxRows);
      const int len = rows + (int)(rnd(4) ? rnd(1 << (1 + rnd(14))) : rnd(1 << 24));
      cl.push_back(Kv4Client{i, rows, row, len});
      row += rows;
    }
    if (check(h[0], h[1], hd, dtype, n_cu, cl)) return 1;
    for (const Kv4Launch& l : out) kinds[l.wide ? 2 : l.tiles - 1]++;
  }
  for (int dtype : {PIPESD_F32, PIPESD_BF16}) {  // more workgroups than a grid has in y
    std::vector<Kv4Client> cl;
    for (int i = 0; i < 256; ++i) cl.push_back(Kv4Client{i, kKv4MaxRows, i * kKv4MaxRows, kKv4MaxRows + 1000 * i});
    if (check(256, 1, 64, dtype, 256, cl)) return 1;
    for (Kv4Client& c : cl) c.n_rows = 130, c.len = 700;
    if (check(256, 1, 128, dtype, 256, cl)) return 1;
  }
  printf("%ld %ld %ld\n", kinds[0], kinds[1], kinds[2]);
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", CSRC,
                    str(d / "plan.hip"), "-o", str(d / "plan")], check=True, capture_output=True)
    return lambda *args: subprocess.run([str(d / "plan"), *map(str, args)], check=True, capture_output=True, text=True).stdout


def kinds(plan, heads, dtype, before, rows):
    text = plan("kind", *heads, 0 if dtype == "f32" else 1, 256, *[x for b, r in zip(before, rows) for x in (b + r, r)])
    return [tuple(map(int, line.split())) for line in text.splitlines()]


def test_passes_are_covered_once(plan):
    one, two, many = map(int, plan("sweep").split())
    assert min(one, two, many) > 500


@pytest.mark.parametrize("name", CASES)
def test_the_cases_of_many_tiles_are_that(plan, name):
    heads, dtype, before, rows = CASES[name]
    got = kinds(plan, heads, dtype, before, rows)
    assert [tiles == 8 for tiles, _ in got] == [r > 3 for r in rows]
    if name == "long":
        assert got[0][1] > 32
    if name == "prompt":
        assert got[0][1] == 1


def test_what_passes_are_given_to(plan):
    """(tiles of a workgroup, splits) where both sides have been measured: the faster one."""
    assert kinds(plan, (32, 8, 128), "bf16", [2040] * 4, [8] * 4) == [(1, 8)] * 4  # 11.7 us
    assert {t for t, _ in kinds(plan, (32, 8, 128), "bf16", [4096] * 32, [8] * 32)} == {2}  # 41; 48 with one
    assert {t for t, _ in kinds(plan, (32, 8, 128), "bf16", [8192] * 32, [4] * 32)} == {1}  # 57; 73 with two
    assert kinds(plan, (32, 8, 128), "bf16", [4096], [64])[0][0] == 1  # 16; 26 with eight
    assert kinds(plan, (32, 8, 128), "bf16", [65536], [64])[0][0] == 8  # 98; 115 with two
    assert kinds(plan, (32, 8, 128), "bf16", [6144], [2048]) == [(8, 1)]  # 265; 349 with two
    assert kinds(plan, (32, 8, 64), "bf16", [6144], [2048]) == [(8, 1)]  # 182; 225 with two
    assert kinds(plan, (32, 8, 128), "f32", [2048], [2048])[0][0] == 8  # 210; 248 with one
    assert kinds(plan, (32, 8, 128), "bf16", [600], [1]) == [(1, 1)]  # (no split below 768 tokens)


def test_no_early_read_of_matrix_core_results(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    out = tmp_path / "attn.s"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-S",
                    "--cuda-device-only", "-o", str(out), os.path.join(CSRC, "kernels_kv4_attn.hip")], check=True, capture_output=True)
    text = out.read_text()
    assert len(re.findall(r"^_ZN6pipesd22kv4_attend_many_kernel\w+:", text, re.M)) == 4 and "v_mfma_f32_32x32x16_bf16" in text
    assert isa_lint.check_mfma(str(out)) == 0
