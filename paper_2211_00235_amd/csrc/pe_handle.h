// The handle behind the C ABI and what its entry points share: the check for overlapping buffers.
#pragma once
#include <hip/hip_runtime.h>
#include <string>
#include <vector>

#include "../../include/pe.h"

struct ProfRec { const char* label; std::string kern; double flops, bytes; hipEvent_t e0, e1; };
struct pe_handle {
  int device;                       // device that was current in pe_create
  void* static_scratch;             // that device's copy of `scratch`
  hipEvent_t ev[6];
  int branches;
  int sync_debug;
  int timing;                       // PE_OPT_KERNEL_TIMING
  int side_streams;                 // PE_OPT_SIDE_STREAMS
  int stack_keep;                   // PE_OPT_STACK_KEEP_CTX
  int stack_overlap;                // PE_OPT_STACK_OVERLAP
  int stack_ckpt;                   // PE_OPT_STACK_CKPT
  hipStream_t side[2];              // side stream of the MSA branch / of the pair branch
  hipEvent_t side_ev[32];           // ring of fork/join events
  int side_ev_next;
  hipStream_t pair;                 // the pair branch's stream of calls with one stream (pair_stream); null: there is none
  bool pair_forked;                 // the call that is running has forked it from the caller's stream
  std::vector<ProfRec> recs;        // one per timed launch since the last collect
  std::vector<hipEvent_t> ev_pool;  // reusable timing events
  std::string last_error;
};

static inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const char* x = (const char*)a; const char* y = (const char*)b;
  return x < y + nb && y < x + na;
}
// a buffer of a call: written = the call writes it (outputs, ctx of the forward, workspace)
struct Region { const void* p; size_t n; bool written; };
// true when two buffers overlap of which at least one is written (null and empty buffers are skipped)
static inline bool any_alias(const Region* r, int n) {
  for (int i = 0; i < n; i++)
    for (int j = i + 1; j < n; j++)
      if ((r[i].written || r[j].written) && r[i].p && r[j].p && r[i].n && r[j].n && overlap(r[i].p, r[i].n, r[j].p, r[j].n))
        return true;
  return false;
}
