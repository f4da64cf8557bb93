"""How a pass over the paged cache is divided: every client's rows and tokens once, within the scratch that creation provides, and the kinds
of workgroups that have been measured to be the fastest (CPU).  And the listing of its kernels: no product is read early."""
import os
import re
import shutil
import subprocess

import pytest

from tests import isa_lint

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_13319_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
FLAGS = ["-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <random>
#include <vector>

#include "pages.h"
using namespace pipesd;

#define CHECK(x) do { if (!(x)) { printf("%s: %d rows %d clients\n", #x, cl[0].n_rows, (int)cl.size()); exit(1); } } while (0)
static long kinds[9];

static void check(int nq, int nkv, int hd, int dtype, int n_cu, const std::vector<PagesClient>& cl) {
  std::vector<PagesLaunch> out;
  const PagesNeeds need = pages_plan(cl.data(), (int)cl.size(), dtype, hd, nq, nkv, n_cu, out);
  std::vector<int> seen(cl.size(), 0);
  size_t parts = 0, counters = 0;
  for (const PagesLaunch& l : out) {
    CHECK(l.tiles == 1 || l.tiles == 2 || (dtype == PIPESD_BF16 && (l.tiles == 4 || l.tiles == 8)));
    CHECK(l.c.n >= 1 && l.c.n <= kPagesPerLaunch && l.c.items >= 1 && l.c.items <= kPagesMaxItems);
    CHECK(l.c.span > 0 && l.c.span % kPagesStep == 0);
    int item = 0;
    ++kinds[l.tiles];
    for (int j = 0; j < l.c.n; ++j) {
      CHECK(l.c.first[j] == item);
      const int groups = l.c.groups[j], ns = l.c.nsplit[j], rows = l.c.n_rows[j] * (nq / nkv);
      item += groups * ns;
      int which = -1;
      for (size_t i = 0; i < cl.size(); ++i)
        if (cl[i].n_rows > 0 && cl[i].row_off == l.c.row_off[j]) which = (int)i;
      CHECK(which >= 0 && !seen[which]++);
      CHECK(l.c.len[j] == cl[which].len && l.c.n_rows[j] == cl[which].n_rows && l.c.table_off[j] == cl[which].table_off);
      CHECK(groups * 16 * l.tiles >= rows && (groups - 1) * 16 * l.tiles < rows);
      // the splits but the last are whole, and none is empty
      CHECK(ns >= 1 && ns <= kPagesMaxSplits && (int64_t)(ns - 1) * l.c.span < cl[which].len);
      CHECK(ns == 1 || (int64_t)ns * l.c.span + kPagesSplitSlack >= cl[which].len);
      CHECK((size_t)l.c.count_off[j] == counters);
      counters += (size_t)nkv * groups;
      if (ns > 1) {
        CHECK((size_t)l.c.part_off[j] == parts);
        parts += (size_t)nkv * groups * ns * l.tiles;
        CHECK(!(l.tiles > 2 && !l.c.apart));
      }
    }
    for (int j = l.c.n; j < kPagesPerLaunch; ++j) CHECK(l.c.first[j] == l.c.items);
    CHECK(item == l.c.items);
    if (l.c.apart) {
      PagesJoin join;
      const int wgs = pages_join_plan(l.c, l.tiles * 16, hd, &join), per = (1024 / hd) >> join.log_shares;
      CHECK(wgs >= 1 && wgs <= 65535 && join.log_shares >= 0 && per >= 1);  // (a grid's in y)
      for (int j = 0; j < kPagesPerLaunch; ++j) {
        const int next = j + 1 < kPagesPerLaunch ? join.first[j + 1] : wgs;
        CHECK(next - join.first[j] == (j < l.c.n && l.c.nsplit[j] > 1 ? l.c.groups[j] * (l.tiles * 16 / per) : 0));
      }
    }
  }
  for (size_t i = 0; i < cl.size(); ++i) CHECK(seen[i] == (cl[i].n_rows > 0));
  CHECK(need.part_tiles == parts && need.counters == counters);
  int64_t len = 0;
  int rows = 0, n = 0;
  for (const PagesClient& c : cl) len = std::max<int64_t>(len, c.len), rows = std::max(rows, c.n_rows), n += c.n_rows > 0;
  const PagesNeeds most = pages_plan_most(n, rows, len, dtype, hd, nq, nkv, n_cu);
  CHECK(need.part_tiles <= most.part_tiles && need.counters <= most.counters);
}

int main(int argc, char** argv) {
  if (!strcmp(argv[1], "kind")) {  // kind nq nkv hd dtype len rows ..
    std::vector<PagesClient> cl;
    int row = 0;
    for (int i = 6; i + 1 < argc; i += 2) {
      cl.push_back(PagesClient{i, atoi(argv[i + 1]), row, atoi(argv[i]), i});
      row += atoi(argv[i + 1]);
    }
    std::vector<PagesLaunch> out;
    pages_plan(cl.data(), (int)cl.size(), atoi(argv[5]), atoi(argv[4]), atoi(argv[2]), atoi(argv[3]), 256, out);
    for (const PagesLaunch& l : out)
      for (int j = 0; j < l.c.n; ++j) {
        PagesJoin join;
        pages_join_plan(l.c, l.tiles * 16, atoi(argv[4]), &join);
        printf("%d %d %d\n", l.tiles, l.c.nsplit[j], l.c.apart ? 1 << join.log_shares : 0);
      }
    return 0;
  }
  std::mt19937 r(7);
  auto pick = [&](int lo, int hi) { return lo + (int)(r() % (unsigned)(hi - lo + 1)); };
  const int heads[][2] = {{4, 4}, {32, 8}, {40, 40}, {24, 8}, {128, 16}, {8, 1}, {256, 1}, {3, 3}, {512, 64}};
  for (int i = 0; i < 20000; ++i) {
    const int* h = heads[r() % 9];
    std::vector<PagesClient> cl;
    int row = 0;
    const int n = r() % 3 ? pick(1, 16) : pick(17, 256), longest = 1 << pick(1, 17), most = r() % 4 ? pick(1, 64) : pick(65, kPagesMaxRows);
    for (int c = 0; c < n; ++c) {
      const int rows = pick(c == 0 ? 1 : 0, most);
      cl.push_back(PagesClient{c, rows, row, rows + pick(0, longest), c * 9000});
      row += rows;
    }
    check(h[0], h[1], r() % 2 ? 128 : 64, r() % 2 ? PIPESD_BF16 : PIPESD_F32, r() % 5 ? 256 : pick(1, 304), cl);
  }
  {  // one long context among many rows that are not cut
    std::vector<PagesClient> cl;
    for (int c = 0; c < 32; ++c) cl.push_back(PagesClient{c, c ? kPagesMaxRows : 1, c * kPagesMaxRows, c ? kPagesMaxRows : 100000, c});
    for (int dtype : {PIPESD_F32, PIPESD_BF16})
      for (int hd : {64, 128}) check(256, 1, hd, dtype, 256, cl);
  }
  for (int rows : {1, kPagesMaxRows}) {
    std::vector<PagesClient> cl;
    for (int c = 0; c < 256; ++c) cl.push_back(PagesClient{c, rows, c * rows, rows + 1000 * c, c});
    for (int dtype : {PIPESD_F32, PIPESD_BF16}) check(256, 1, 64, dtype, 256, cl), check(40, 40, 128, dtype, 256, cl);
    cl.resize(1);
    cl[0].len = INT32_MAX / 2;
    for (int dtype : {PIPESD_F32, PIPESD_BF16}) check(32, 8, 128, dtype, 256, cl);
  }
  printf("%ld %ld %ld %ld\n", kinds[1], kinds[2], kinds[4], kinds[8]);
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.hip").write_text(PROGRAM)
    subprocess.run([HIPCC, "-O1", *FLAGS, "-I", CSRC, str(d / "plan.hip"), "-o", str(d / "plan")], check=True, capture_output=True)

    def run(*args):
        done = subprocess.run([str(d / "plan"), *map(str, args)], capture_output=True, text=True)
        assert done.returncode == 0, done.stdout
        return done.stdout

    return run


def kinds(plan, heads, dtype, before, rows):
    """(tiles, splits, threads that share a task of the join apart; 0: none is) of every client."""
    text = plan("kind", *heads, 0 if dtype == "f32" else 1, *[x for b, r in zip(before, rows) for x in (b + r, r)])
    return [tuple(map(int, line.split())) for line in text.splitlines()]


def test_passes_are_covered_once(plan):
    assert min(map(int, plan("sweep").split())) > 500


def test_what_passes_are_given_to(plan):
    """(tiles of a workgroup, splits) where the kinds have been measured: the fastest, or within 5 % of it (us)."""
    tiles = lambda *a: {t for t, _, _ in kinds(plan, *a)}
    h8, h64 = (32, 8, 128), (32, 8, 64)
    assert tiles(h8, "bf16", [2048], [9]) == {1}      # 11.0; 14.6 with two, 14.9 with four, 15.5 with eight
    assert tiles(h8, "bf16", [4096], [1]) == {1}      # 11.6; 13.1, 16.3, 17.0
    assert tiles(h8, "bf16", [2048], [64]) == {2}     # 16.8; 17.8 with one, 18.1 with four, 20.8 with eight
    assert tiles(h64, "bf16", [1531] * 8, [25] * 8) <= {2, 4}
    assert tiles(h8, "bf16", [131071], [9]) == {4}    # 106.6; 151, 112, 109 with eight
    assert tiles(h8, "bf16", [32768], [64]) <= {4, 8}  # 77 and 72; 155 with one, 94 with two
    assert tiles(h8, "bf16", [2048], [1024]) == {4}   # 77; 203, 112, 95
    assert tiles(h8, "f32", [8000], [1]) == {1}       # 19; 25 with two
    assert kinds(plan, h64, "bf16", [200], [1]) == [(1, 1, 0)]


def test_passes_that_are_joined_apart(plan):
    """The cases of test_gpu_pages_join.py reach one to eight threads that share a task, and clients without splits beside them."""
    one = [kinds(plan, (16, 2, dim), "bf16", [before], [rows])[0] for before in (6000, 20011, 70000) for rows in (5, 16, 33, 64, 128) for dim in (64, 128)]
    one += [kinds(plan, (8, 1, dim), "bf16", [100], [2048])[0] for dim in (64, 128)]
    assert {shares for _, _, shares in one} == {0, 1, 2, 4, 8}
    assert {tiles for tiles, _, shares in one if shares > 0} == {1, 2, 4, 8}
    before, rows = [0, 30000, 17, 4000, 200, 9000, 1], [3, 9, 40, 17, 1, 33, 64]
    for dtype in ("bf16", "f32"):
        ragged = kinds(plan, (16, 2, 128), dtype, before, rows)
        assert {s > 0 for _, _, s in ragged} == {True} and min(n for _, n, _ in ragged) == 1 and max(n for _, n, _ in ragged) > 8


def test_no_early_read_of_matrix_core_results(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    out = tmp_path / "attn.s"
    subprocess.run([HIPCC, "-O3", *FLAGS, "-S", "--cuda-device-only", "-o", str(out), os.path.join(CSRC, "kernels_pages_attn.hip")], check=True,
                   capture_output=True)
    text = out.read_text()
    assert len(re.findall(r"^_ZN6pipesd24pages_attend_wide_kernel\w+:", text, re.M)) == 4 and "v_mfma_f32_32x32x16_bf16" in text
    assert len(re.findall(r"^_ZN6pipesd19pages_attend_kernel\w+:", text, re.M)) == 8 and "v_mfma_f32_16x16x4_f32" in text
    assert isa_lint.check_mfma(str(out)) == 0
