// Host launchers of the prompt's attention and of the paged cache
// (kvec_prefill.hip, kvec_append.hip, kvec_paged_decode.hip,
// kvec_paged_evict.hip), called by the C ABI in kvec_serve_api.hip.
#pragma once

#include "kvec_internal.h"
#include "kvec_prefill_plan.h"

namespace kvec {

// Division of group indices by the groups per page: floor(g / d) =
// (g * magic) >> 32 with magic = floor(2^32 / d) + 1, exact while g * d < 2^32
// (both are at most 2^16 here: 2^20 slots in groups of 16).
struct GroupDiv {
  uint64_t magic;
  int d;
};
inline GroupDiv group_div(int d) { return GroupDiv{((uint64_t)1 << 32) / (uint64_t)d + 1, d}; }

// A paged cache as the kernels see it (strides in elements).
struct PagedView {
  char* k;
  char* v;
  int64_t sp, sh, sr;
  const int32_t* table;  // [batch][max_pages]
  const int32_t* lens;   // [batch]
  int batch, H, HQ, G, D, esize;
  int ps, n_pages, max_pages, max_len;
  GroupDiv gdiv;         // groups of 16 slots per page
};

struct AppendArgs {
  int64_t n;
  const char *q, *k, *v;
  int64_t q_t, q_h, k_t, k_h, v_t, v_h, o_t, o_h;  // element strides {token, head}
  const char *wq, *wk;
  float eps;
  const int32_t* positions;
  const double* inv_freq;
  int rot;
  const int64_t* slots;
  char* q_out;
  float* acc;
  int32_t* pos;
};
hipError_t run_append(const PagedView& c, const AppendArgs& a, hipStream_t s);

struct PagedDecodePlan {
  int S;           // splits of a sequence's visible slots
  size_t part;     // bytes of the partial states [b][HQ][S][d + 2]
  size_t logits;   // bytes of the logits [b][H][G][padded max_len] (0 without acc)
  size_t total() const { return part + logits; }
};
PagedDecodePlan paged_decode_plan(const PagedView& c, int window, int sinks, bool acc);
hipError_t run_paged_decode(const PagedView& c, const void* q, const int64_t qs[2], int window, int sinks,
                            float* out, float* lse, float* acc, char* ws, hipStream_t s);

size_t paged_evict_ws(const PagedView& c, int budget);
hipError_t run_paged_evict(const PagedView& c, int budget, int window, int sinks, const int32_t* n_seen,
                           float* acc, int32_t* pos, int32_t* kept, int32_t* lens_out, char* ws,
                           hipStream_t s);

struct PrefillArgs : PrefillShape {
  const char *q, *k, *v;
  int64_t qs[3], ks[3], vs[3], os[3], ls[2];
  const int32_t *q_lens, *kv_lens;
  char* out;
  float* lse;
};
hipError_t run_prefill(const PrefillArgs& a, const PfPlan& plan, char* ws, hipStream_t s);

}  // namespace kvec
