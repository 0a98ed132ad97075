// How a call of the 8-bit cache's attention is cut up (host).
#pragma once
#include <algorithm>

#include "kv8_few.h"
#include "kv8_many.h"

namespace m2r2 {

struct Kv8Cut {
  bool many;       // k8_many
  int cols;        // of a tile
  int target;      // workgroups, about
  int max_splits;  // of a tile
  int pcols;       // columns of a partial result
  long long entries;
  size_t bytes;    // of the workspace
};

// Up to this many columns a sequence on average, k8_few, which reads the cache
// once for every sixteen; above, k8_many, whose tiles would not be filled below, with
// its second launch.  Measured at 8 heads of 128 for 4 with 64, 128 and 256 columns (us,
// k8_few / k8_many): one sequence of 400 positions 10.2/17.3, 10.2/19.4, 10.3/19.4; of
// 1500 14.5/16.0, 15.4/20.4, 19.6/22.9; four of 1000 14.9/24.2, 16.9/30.4, 24.5/31.5; four
// of 8000 36.1/45.3, 53.0/51.8, 81.2/54.1, in float32 31.8/54.1, 65.3/61.2, 91.7/83.7.  One
// sequence of 8000 would gain from fewer: 24.7/21.2, 37.0/24.8, 48.8/28.7.
constexpr int kFewMost = 128;

inline Kv8Cut kv8_cut(const Kv8Pages& kv, int hd, int n_seqs, int n_rows, int n_heads, bool bf16) {
  Kv8Cut c;
  const int H = kv.H, group = n_heads / H;
  const long long cols = (long long)n_rows * group;
  c.many = cols > (long long)kFewMost * std::max(1, n_seqs);
  c.cols = c.many ? kManyCols : kFewCols;
  // what a compute unit holds: two workgroups, three of k8_few's bfloat16 form, one of k8_many's float32 form
  c.target = (c.many == bf16 ? 2 : bf16 ? 3 : c.many ? 1 : 2) * kKv8Units;
  // joins cost a little per split: 32, or what gives every compute unit one
  c.max_splits = (int)std::max(32LL, std::min<long long>(kKv8MaxSplits, kKv8Units / std::max(1LL, (long long)n_seqs * H)));
  c.pcols = c.many ? kManyCols : (int)std::min<long long>(kFewCols, std::max<long long>(1, cols));
  const long long tiles = std::min<long long>(n_seqs, n_rows) + cols / c.cols;   // at most: ceil(a) <= a + 1 where a > 0
  const long long cap = (long long)kv.mbps * kv.bs;
  const long long most =
      tiles * (cap <= kKv8Whole ? 1 : std::min<long long>(c.max_splits, (cap + kKv8MinTokens - 1) / kKv8MinTokens));
  c.entries = std::min(most, kv8_share(c.target, H) + tiles);
  const long long slots = std::min(most, 2LL * kv8_share(c.target, H));
  c.bytes = sizeof(uint32_t) * kKv8Counters + sizeof(float) * slots * H * kv8_part_floats(c.pcols, hd);
  return c;
}

// The workspace: counters, then partial results.
inline void kv8_cut_args(Kv8AttnArgs& A, const Kv8Cut& c, void* workspace) {
  A.cnt = (uint32_t*)workspace;
  A.part = (float*)((char*)workspace + sizeof(uint32_t) * kKv8Counters);
  A.pcols = c.pcols;
  A.target = c.target;
  A.max_splits = c.max_splits;
  A.entries = (int)c.entries;
  const uint32_t d = A.kv.bs / kKv8Slab;
  A.bs_magic = ((1u << 31) + d - 1) / d;
}

}  // namespace m2r2
