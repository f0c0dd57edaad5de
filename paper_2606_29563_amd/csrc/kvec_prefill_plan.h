// Which kernel runs a prompt's attention, and how many splits over the keys: an
// estimate of its time, on the host.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace kvec {

struct PrefillShape {
  int batch, H, HQ, G, D, q_len, kv_len, window, sinks, esize;
};

constexpr int kStateHead = 4;  // floats before the output in a partial state (16-byte pieces)

// Threads and packed rows of a work-group, and the keys of its step (kvec_prefill.hip).
constexpr int kPfThreads = 256, kPfRows = 64, kPfKeys = 32;
constexpr int kPf32Keys = 64;
constexpr int kPfFewThreads = 128, kPfFewRows = 32, kPfFewKeys = 32;

enum PfKernel { kRows16, kRows16Keys, kRows32, kRows32Half, kRows32Keys, kRows32Keys4, kFew };

struct PfPlan {
  PfKernel kernel;
  int S, tiles;  // splits over the keys; row tiles
  size_t bytes;  // partial states
};

inline int pf_threads(PfKernel kernel) {
  return kernel == kFew ? kPfFewThreads : kernel == kRows16 || kernel == kRows32Half ? kPfThreads : 2 * kPfThreads;
}

// Work-groups of the launch: every (row tile, split) of every (sequence, KV head), or, of
// fewer than eight of these, as many more as send each one's to XCDs of its own (pf_item).
inline int64_t pf_work_groups(const PrefillShape& a, const PfPlan& p) {
  const int64_t BH = (int64_t)a.batch * a.H, items = (int64_t)p.tiles * p.S;
  return 8 % BH == 0 ? (items + 8 / BH - 1) / (8 / BH) * 8 : items * BH;
}

inline double pf_ceil(double x) {  // 0 <= x < 2^31
  const int whole = (int)x;
  return whole + (whole < x);
}

// Kernel and splits over the keys: the pair with the least estimated time
//   max(the longest work-group, all of them over what runs at a time, K and V at 4.5 TB/s)
//     + what the join costs,
// a work-group taking so long per key tile and so long besides (first loads, masked
// tiles, stores):
//   pf_rows32, 8 waves  256 rows, 64 keys, 256 at a time: 1.9 us a tile (alone 1.85) + 6
//   pf_rows32, 4 waves  128 rows, 64 keys, 512 at a time: 2.05 us (alone 1.5) + 5
//   pf_rows32, 4 + 4    128 rows, 2 x 64 keys, 256 at a time: 2.05 us (alone 1.9) + 7
//   pf_rows32, 4 x 2    64 rows, 4 x 32 keys, 256 at a time: 1.8 us (alone 1.45) + 7.5
//   pf_few              32 rows, 2 x 32 keys, 512 at a time: 1.3 us + 5
//   pf_rows16           64 rows, 32 keys, 512 at a time: 4.8 us (alone 3.2) + 3
//   pf_rows16, 4 + 4    64 rows, 2 x 32 keys, 256 at a time: 5.2 us + 4
// (d = 64: half of pf_rows16's; four waves, 4 + 4 and, 512 at a time, 4 x 2, which is as good as pf_few on few
// rows).  A join is a launch (4 us), a round trip per 16 splits and the partial states
// there and back at 4 TB/s.
// Measured us in one piece, 8 waves / 4 / 4 + 4 / 4 x 2 / pf_few: 250 rows of 32 heads - /
// - / 12 / 11 / 10.5, 500 rows of 28 heads 23 / 18 / 16 / 14 / 16, 1000 rows of 32 34 / 28
// / 24 / 27 / 32, 1500 rows 48 / 41 / 35 / 48 / 60, 8192 rows 510 / 535 / 555 / 702 / -;
// 3000 rows 95 / 87 / 100 / 128, 1900 rows over 5900 keys 173 / 164 / 168 / -, 500 over 2000
// - / - / 34 / 27, 2048 rows of 28 heads behind a window of 4096 131 / 139 / 143 / -, 3000
// behind one of 500 56 / 44 / 53 / -; d 64, 16 heads, 4 / 4 + 4 / 4 x 2: 1000 rows 19 / 15 / 12,
// 1500 rows - / 20 / 16, 4000 rows 61 / 52 / 53, 8000 rows 150 / 172 / 176.
// float32, pf_rows16 / 4 + 4: 1000 rows of 32 heads, d 128, 115 / 98, 2000 rows 338 / 336;
// d 64, 1500 rows of 8 heads behind a window of 200 22 / 16, 1000 rows in splits 26 / 28.
inline PfPlan pf_plan(const PrefillShape& a) {
  const int64_t packed = (int64_t)a.q_len * a.G, heads = (int64_t)a.batch * a.H;
  PfPlan best = {};
  double least = 0;
  struct Cost {
    double busy, alone, besides;  // us of a tile among others and alone, us besides
  };
  auto consider = [&](PfKernel kernel, int rows, int keys, int at_a_time, Cost c) {
    const bool shared = kernel == kFew || kernel == kRows32Keys || kernel == kRows32Keys4;
    const int64_t tiles = (packed + rows - 1) / rows, groups = tiles * heads;
    // keys that a row tile sees at most, and on average
    double most = a.kv_len, mean = a.kv_len - 0.5 * (a.q_len < a.kv_len ? a.q_len : a.kv_len);
    const double span = (double)a.window + a.sinks + (double)rows / a.G;
    if (a.window > 0 && span < most) most = span;
    if (mean > most) mean = most;
    const double most_tiles = most / keys, mean_tiles = mean / keys, uneven = 1 - mean / most;
    const double state = 2.0 * a.batch * a.HQ * a.q_len * (a.D + kStateHead) * 4 / 4e6;  // us per split
    const double read = heads * most * 2 * a.D * a.esize / 4.5e6;
    // no time is below this
    const double floor = c.alone + c.besides > read ? c.alone + c.besides : read;
    const double shorter = c.busy > c.alone ? c.busy - c.alone : 0;
    for (int S = 1; S <= 64 && (S == 1 || most / S >= 64); ++S) {
      const double join = S > 1 ? 4.0 + 0.7 * ((S + 15) / 16) + S * state : 0;
      // (pf_few's probabilities are more exact: taken unless another is clearly faster)
      const double limit = least * (best.kernel == kFew && kernel != kFew ? 0.95 : 1.0);
      if (best.S != 0 && floor + join >= limit) break;  // neither this many splits nor more
      // more than one a compute unit: the longest shares it with the 257th, as long as
      // that lasts (lengths fall evenly from the longest to twice the mean less that)
      const double all_groups = (double)groups * S;
      double company = all_groups > 256 ? 1 - 256 / all_groups * 2 * uneven : 0;
      if (company < 0) company = 0;
      const double longest = pf_ceil(most_tiles / S) * (c.alone + shorter * company) + c.besides;
      // behind a window, and where the rows are few for their keys, all work-groups are
      // alike and run in whole rounds; so do short ones, whose keys are divided over waves
      double rounds = all_groups / at_a_time;
      if (rounds > 1 && (a.window > 0 || mean > 0.75 * most || shared)) rounds = pf_ceil(rounds);
      const double all = rounds * (mean_tiles / S * c.busy + c.besides);
      double t = longest > all ? longest : all;
      if (t < read) t = read;
      t += join;
      if (best.S == 0 || t < limit) {
        least = t;
        best.kernel = kernel;
        best.S = S;
        best.tiles = (int)tiles;
      }
      if (longest <= all || longest <= read) break;  // more splits only add states
    }
  };
  const bool d64 = a.D == 64;
  if (a.esize == 4) {
    consider(kRows16, kPfRows, kPfKeys, 512, d64 ? Cost{2.3, 1.6, 3} : Cost{4.8, 3.2, 3});
    consider(kRows16Keys, kPfRows, 2 * kPfKeys, d64 ? 512 : 256, d64 ? Cost{4.6, 2.7, 4.5} : Cost{5.2, 5.2, 4});
  } else if (d64) {
    consider(kRows32Half, 128, kPf32Keys, 512, Cost{1.15, 0.9, 4});
    consider(kRows32Keys, 128, 2 * kPf32Keys, 256, Cost{1.15, 0.85, 5.5});
    consider(kRows32Keys4, 64, 4 * 32, 512, Cost{1.15, 0.7, 4.3});
  } else {
    consider(kFew, kPfFewRows, 2 * kPfFewKeys, 512, Cost{1.3, 1.3, 5});
    consider(kRows32Half, 128, kPf32Keys, 512, Cost{2.05, 1.5, 5});
    consider(kRows32Keys, 128, 2 * kPf32Keys, 256, Cost{2.05, 1.9, 7});
    consider(kRows32Keys4, 64, 4 * 32, 256, Cost{1.8, 1.45, 7.5});
    consider(kRows32, 256, kPf32Keys, 256, Cost{1.9, 1.85, 6});
  }
  best.bytes = best.S > 1 ? (size_t)a.batch * a.HQ * a.q_len * best.S * (a.D + kStateHead) * 4 : 0;
  return best;
}

}  // namespace kvec
