// The decision on a tree of drafts: what its launches carry.
#pragma once

#include "common.h"

namespace pipesd {

constexpr int kTreeRows = 256;      // of a client, and of the clients of a launch together
constexpr int kTreeClients = 16;    // of a launch
constexpr int kTreeChunks = 64;     // workgroups that share a row of the vocabulary

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

struct TreeCall {
  const float *p, *q;  // rows of the launch's first client on; q: nullptr for token matching
  int64_t p_stride, q_stride;
  int32_t V, n, distinct, stages;  // stages: children of the row that has the most
  int32_t row_off[kTreeClients], rows[kTreeClients];
  int32_t token[kTreeRows];
  float u[kTreeRows];
  int16_t parent[kTreeRows];       // within the client's rows
  uint8_t nth[kTreeRows], children[kTreeRows];  // which child of its parent a row is; how many it has
  int32_t* result;                 // [clients][result_stride]
  int64_t result_stride;
  TreeWorkspace ws;
};
hipError_t launch_tree_accept(const TreeCall& c, hipStream_t st);

}  // namespace pipesd
