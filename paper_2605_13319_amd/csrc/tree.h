// The decision on a tree of drafts: what its launches carry.
#pragma once

#include "common.h"

namespace pipesd {

constexpr int kTreeRows = 256;      // of a client, and of the clients of a launch together
constexpr int kTreeClients = 16;    // of a launch
constexpr int kTreeChunks = 64;     // workgroups that share a row of the vocabulary, at most
constexpr int kTreeChunk = 2048;    // tokens of one, unless there are more
constexpr int kTreeSmall = 8192;    // vocabulary that one workgroup decides on alone

// what the launches of a call hand on, in the caller's memory; the counters are zero between launches
struct TreeWorkspace {
  unsigned* counters;            // [kTreeClients]
  float2* ab;                    // [kTreeRows] (a, b) that a row's child was tested with
  double* mass;                  // [kTreeRows] S of a row
  unsigned long long* partial;   // [sums][kTreeChunks]
};
inline size_t tree_workspace_bytes() {
  return kTreeClients * 16 + kTreeRows * (sizeof(float2) + sizeof(double)) + (size_t)kTreeRows * kTreeChunks * sizeof(unsigned long long);
}
inline TreeWorkspace tree_workspace(void* p) {
  char* c = (char*)p;
  TreeWorkspace w;
  w.counters = (unsigned*)c;
  c += kTreeClients * 16;
  w.ab = (float2*)c;
  c += kTreeRows * sizeof(float2);
  w.mass = (double*)c;
  c += kTreeRows * sizeof(double);
  w.partial = (unsigned long long*)c;
  return w;
}

struct TreeRow {
  int32_t token;
  float u;
  int16_t parent;          // within the client's rows
  uint8_t nth, children;   // which child of its parent it is; how many it has
};
struct TreeCall {
  const float *p, *q;      // rows of the launch's first client on; q: nullptr for token matching
  int64_t p_stride, q_stride;
  int32_t V, n, distinct;
  int32_t stages;          // children of the row that has the most
  int32_t chunks;          // workgroups that share a row of the vocabulary
  int32_t row_off[kTreeClients], rows[kTreeClients];
  TreeRow row[kTreeRows];
  int32_t* result;         // [clients][result_stride]
  int64_t result_stride;
  TreeWorkspace ws;
};
hipError_t launch_tree_accept(const TreeCall& c, hipStream_t st);

}  // namespace pipesd
