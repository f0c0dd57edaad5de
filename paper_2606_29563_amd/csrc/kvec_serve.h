// Host launchers of the prompt's attention and of the paged cache
// (kvec_prefill.hip, kvec_append.hip, kvec_paged_decode.hip, kvec_paged_decode_q8.hip,
// kvec_paged_shared.hip, kvec_paged_read.hip, kvec_paged_evict.hip), called by the C ABI in
// kvec_serve_api.hip.
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
  int batch, H, HQ, G, D, esize, psize;  // bytes of an element of q, and of the pools
  int ps, n_pages, max_pages, max_len;
  GroupDiv gdiv;         // groups of 16 slots per page
  float *ks, *vs;        // a cache in eight bits: its scales [page][H][row]
  int format;            // ... and kvec_q8_format
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

PagedDecodePlan paged_decode_q8_plan(const PagedView& c, int window, int sinks, bool acc);
hipError_t run_paged_decode_q8(const PagedView& c, const void* q, const int64_t qs[2], int window, int sinks,
                               float* out, float* lse, float* acc, char* ws, hipStream_t s);

constexpr int kJoinSlots = 1024;  // slots whose weights a work-group of the join adds
constexpr int kJoinThreads = 256;

// What a batch's sequences begin with.
struct SharedPrefix {
  const int32_t* pages;
  const int32_t* len;  // [1]
  int n_pages, max_len;
};
struct SharedPlan {
  int kernel;            // which prefix kernel
  int tiles, Sp;         // its column tiles, and splits of the prefix
  PagedDecodePlan own;   // of the sequences' own slots
  size_t part, logits, norm;
  size_t total() const { return part + logits + norm; }
};
SharedPlan shared_plan(const PagedView& c, int max_prefix, bool acc);
hipError_t run_paged_shared(const PagedView& c, const SharedPrefix& p, const void* q, const int64_t qs[2], int window,
                            int sinks, float* out, float* lse, float* acc, char* ws, hipStream_t s);

struct ReadArgs {
  char *k, *v;
  int64_t ks[3], vs[3];  // element strides {batch, head, row}
};
hipError_t run_paged_read(const PagedView& c, const ReadArgs& a, hipStream_t s);

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
