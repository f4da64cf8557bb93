// Host side of the decision on trees of drafts: checks, and clients by the launch.
#include <algorithm>

#include "status.h"
#include "tree.h"

using namespace pipesd;

extern "C" size_t pipesd_tree_accept_workspace(void) { return tree_workspace_bytes(); }

extern "C" int pipesd_tree_accept(const float* p, int64_t p_stride, const float* q, int64_t q_stride, int32_t vocab, int32_t n_seqs, const int32_t* rows,
                                  const int32_t* tokens, const int32_t* parents, const float* uniforms, int32_t distinct, int32_t* result,
                                  int64_t result_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (!p || vocab < 1 || vocab > PIPESD_TREE_MAX_VOCAB || p_stride < vocab || (q && (q_stride < vocab || !uniforms)) || n_seqs < 1 || !rows || !tokens ||
      !parents || !result || !workspace || ((uintptr_t)workspace & 15) || workspace_bytes < tree_workspace_bytes() || ((uintptr_t)p & 3) ||
      ((uintptr_t)q & 3) || ((uintptr_t)result & 3))
    return PIPESD_EINVAL;
  int64_t total = 0;
  for (int32_t i = 0; i < n_seqs; ++i) {
    if (rows[i] < 1 || rows[i] > kTreeRows || (int64_t)rows[i] + 1 > result_stride) return PIPESD_EINVAL;
    for (int32_t r = 0; r < rows[i]; ++r) {
      const int32_t up = parents[total + r];
      if (r == 0 ? up != -1 : up < 0 || up >= r) return PIPESD_EINVAL;
      if (r > 0 && (tokens[total + r] < 0 || tokens[total + r] >= vocab)) return PIPESD_EINVAL;
      if (q && !(uniforms[total + r] >= 0.f && uniforms[total + r] < 1.f)) return PIPESD_EINVAL;
    }
    total += rows[i];
    if (total > INT32_MAX) return PIPESD_EINVAL;
  }
  TreeCall c;
  c.p_stride = p_stride;
  c.q_stride = q ? q_stride : 0;
  c.V = vocab;
  c.distinct = distinct != 0;
  c.chunks = std::min(kTreeChunks, (vocab + kTreeChunk - 1) / kTreeChunk);
  c.result_stride = result_stride;
  c.ws = tree_workspace(workspace);
  int64_t row0 = 0;  // of the launch's first client
  for (int32_t i0 = 0; i0 < n_seqs;) {
    c.n = 0;
    c.stages = 1;
    int32_t many = 0;
    while (i0 + c.n < n_seqs && c.n < kTreeClients && many + rows[i0 + c.n] <= kTreeRows) {
      const int32_t n = rows[i0 + c.n];
      c.row_off[c.n] = many;
      c.rows[c.n] = n;
      for (int32_t r = 0; r < n; ++r) c.row[many + r].children = 0;
      for (int32_t r = 0; r < n; ++r) {
        const int64_t at = row0 + many + r;
        const int32_t up = parents[at];
        TreeRow& row = c.row[many + r];
        row.token = r > 0 ? tokens[at] : 0;
        row.u = q ? uniforms[at] : 0.f;
        row.parent = (int16_t)up;
        row.nth = up < 0 ? 0 : c.row[many + up].children++;
        if (up >= 0) c.stages = std::max(c.stages, (int32_t)c.row[many + up].children);
      }
      many += n;
      ++c.n;
    }
    c.p = p + row0 * p_stride;
    c.q = q ? q + row0 * q_stride : nullptr;
    c.result = result + i0 * result_stride;
    HIP_TRY(launch_tree_accept(c, (hipStream_t)stream));
    i0 += c.n;
    row0 += many;
  }
  return PIPESD_OK;
}
