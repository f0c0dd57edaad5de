// One new token's attention over a paged cache.
//
// Bound by reading the visible K and V rows once.  Two launches, or one:
//   partial  one work-group of four waves per (split, KV head, sequence).  The
//            visible slots of a sequence, in groups of 16 (a group lies in one
//            page), are divided evenly over the splits, from the device's own
//            lengths.  A wave takes every fourth step of its split and streams
//            it through a private LDS ring of two steps: page lookups are one step
//            ahead of the copies, copies one step ahead of the products.  The G
//            query heads are the columns of the matrix products
//            (Columns16), so every row is read once for all of them.
//            Slots that are not visible are pointed past the end of the copy's
//            buffer and read as zero: what they hold never enters.
//   combine  merges the splits of each query head, and, where the weights are
//            accumulated, goes over the logits that the first launch wrote:
//            acc[s] += mean_g 2^(x_gs - lse_g).  The logits are G floats a slot
//            and head beside 2 d elements of K and V; a second pass over K
//            would cost half of the first launch again.
// With bf16 inputs the probabilities go into the V product as two bf16 terms:
// the products are not what bounds this, and out is float32.
#include "kvec_paged_dev.h"

namespace kvec {
namespace {

template <class TT, int D>
hipError_t launch(const PdArgs& a, hipStream_t s) {
  const dim3 grid(a.S, a.c.H, a.c.batch);
  if (a.S == 1) {
    hipLaunchKernelGGL((pd_partial<TT, D, true>), grid, dim3(kPdThreads), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((pd_partial<TT, D, false>), grid, dim3(kPdThreads), 0, s, a);
  const hipError_t e1 = hipGetLastError();
  if (e1 != hipSuccess) return e1;
  return pd_join<D>(a, s);
}

}  // namespace

// Splits: 1024 work-groups over batch and heads as long as each has 1024 slots
// (16 groups a wave), more of fewer slots only to give every compute unit one,
// down to one group a wave.  us of both launches with 512 / 1024 / 4096
// work-groups, 16 sequences of 8k to 16k slots (8 heads, d 128): 169 / 163 / 170;
// with 256 / 1024 slots at least, one sequence of 32k: 35.2 / 27.5, 32 of 1k to 2k:
// 48.6 / 50.3.  Up to 256 slots are not split: the one launch (us of it / of two; one
// sequence of 128 slots 9.0 / 10.6, of 256 10.6 / 11.0, of 384 12.2 / 11.6).
PagedDecodePlan paged_decode_plan(const PagedView& c, int window, int sinks, bool acc) {
  const int64_t bh = (int64_t)c.batch * c.H;
  const int groups = most_groups(c, window, sinks);
  auto per_bh = [&](int64_t work_groups) { return (work_groups + bh - 1) / bh; };
  int64_t S = per_bh(1024);
  if (S > groups / 64) S = groups / 64;
  if (S < per_bh(256)) S = per_bh(256);
  const int most_s = (groups + kPdWaves - 1) / kPdWaves;
  if (S > most_s) S = most_s;
  if (groups <= 16) S = 1;
  return pd_plan(c, S < 1 ? 1 : S, acc);
}

hipError_t run_paged_decode(const PagedView& c, const void* q, const int64_t qs[2], int window, int sinks,
                            float* out, float* lse, float* acc, char* ws, hipStream_t s) {
  const PagedDecodePlan p = paged_decode_plan(c, window, sinks, acc != nullptr);
  const PdArgs a = pd_args(c, p, q, qs, window, sinks, out, lse, acc, ws);
  if (c.esize == 2) return c.D == 64 ? launch<BF16, 64>(a, s) : launch<BF16, 128>(a, s);
  return c.D == 64 ? launch<F32, 64>(a, s) : launch<F32, 128>(a, s);
}

}  // namespace kvec
