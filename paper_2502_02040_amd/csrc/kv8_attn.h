// Attention over the 8-bit paged cache: what its two kernels share.
//
// k8_few takes up to 16 columns (a row of a query head each) per workgroup
// and is bound by the cache's bytes; k8_many takes 128 and is bound by the
// matrix rate.  Both number their work alike: a sequence's columns of one
// cache head are cut into tiles, its positions into splits.  Partial results of a
// tile's splits are joined by the last of them to finish (k8_few, up to 8 KB each)
// or by a second launch (k8_many, 64 KB each).
#pragma once
#include "kv8.h"

namespace m2r2 {

struct Kv8AttnArgs {
  Kv8Pages kv;
  int n_seqs, n_rows, n_heads, group;   // group: query heads of a cache head
  const int *row_start, *lens, *visible, *own;
  const void *q, *own_k, *own_v;
  void* out;
  int64_t q_row, q_head, ok_row, ok_head, ov_row, ov_head, out_row, out_head;
  int n_own;
  float scale;
  int* err;
  uint32_t* cnt;     // arrivals of split tiles, zero between calls
  float* part;       // partial results
  int pcols;         // columns of a partial result
  int target;        // workgroups that a launch is cut into, about
  int max_splits;    // of a tile
  int entries;       // (tile, split) pairs that the grid covers
  uint32_t bs_magic; // ceil(2^31 / (bs / 16))
};

constexpr int kKv8Units = 256;         // compute units
constexpr int kKv8FullTokens = 512;
constexpr int kKv8MaxSplits = 64;      // of a tile: a lane each in the join
constexpr int kKv8MinTokens = 128;     // of a split, at least: a tile of 32 for each of four waves
// Sequences up to this long are not split: the join's chain of waits costs more.
// One row of 32 heads of 96, whole and in splits of 128 (us): 130 positions 6.8 and
// 9.1, 400 8.4 and 9.2, 520 9.0 and 9.4, 700 9.7 and 9.6, 1025 11.9 and 10.7.
constexpr int kKv8Whole = 512;
// Nor are they where k8_many would cut a tile into two or three and save less than
// this: workgroups that share a compute unit gain little, and its join is a launch.
// Rows of 32 heads for 8, whole and split: 400 behind 300 positions 26.7 and 33.7, 400
// behind 600 33.9 and 36.8, 1000 behind 500 45.5 and 48.5; 400 behind 1100 41.4 and 39.5.
constexpr int kKv8FewSplits = 3, kKv8Saved = 768;
constexpr int kKv8Counters = 16384;    // split tiles of a call, at most

// Splits and counters that a call can need.  A tile is split only if its
// sequence is longer than W H / target positions, W the sum over tiles of
// their sequences' lengths, so at most target / H tiles of a head are split,
// into at most twice that many splits together.
__host__ __device__ constexpr int kv8_share(int target, int heads) { return (target + heads - 1) / heads + 1; }

typedef uint32_t u32x4_8_t __attribute__((ext_vector_type(4), aligned(8)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

template <class T>
__device__ __forceinline__ T kv8_ld(const void* p) {
  return *(const __attribute__((address_space(1))) T*)p;
}
// A load at an address that is the same in all lanes, through the scalar cache
// (nothing in the launch writes there).
template <class T>
__device__ __forceinline__ T kv8_lds(const T* p) {
  return *(const __attribute__((address_space(4))) T*)p;
}

__device__ __forceinline__ uint32_t kv8_pk(float a, float b) {   // two bfloat16, nearest even
  bf16x2_t r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}

// Codes 0, 1 (HI: 2, 3) of a word times a power of two, as two bfloat16 (exact).
template <bool HI>
__device__ __forceinline__ uint32_t kv8_up(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

// x as the sum of N bfloat16 parts (8, 16 or 24 significant bits).
template <int N, bool FINITE = true>
__device__ __forceinline__ void kv8_parts(const float (&x)[8], u32x4_t (&out)[N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const uint32_t w = kv8_pk(a, b);
      out[p][i] = w;
      a -= bf16lo(w);
      b -= bf16hi(w);
      if (!FINITE && p == 0) {   // an infinite value is its first part
        if (!(fabsf(a) < INFINITY)) a = 0.f;
        if (!(fabsf(b) < INFINITY)) b = 0.f;
      }
    }
  }
}

// Bytes of a word that are NaN codes, as a mask of whole bytes.
__device__ __forceinline__ uint32_t kv8_nan_bytes(uint32_t w) {
  const uint32_t t = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (t >> 7) * 0xffu;
}

// Integer steps across lanes without LDS: DPP within rows of 16 lanes and from
// row to row.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int kv8_dpp0(int v) {   // 0 where there is no source
  return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int kv8_wave_scan(int v) {   // inclusive sum
  v += kv8_dpp0<0x111>(v);
  v += kv8_dpp0<0x112>(v);
  v += kv8_dpp0<0x114>(v);
  v += kv8_dpp0<0x118>(v);
  v += kv8_dpp0<0x142, 0xa>(v);   // the last lane of the row before
  return v + kv8_dpp0<0x143, 0xc>(v);
}
template <int CTRL>
__device__ __forceinline__ int kv8_dpp(int v) {
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
__device__ __forceinline__ int kv8_row_max(int v) {   // over 16 lanes, in all of them
  v = max(v, kv8_dpp<kDppQuadXor1>(v));
  v = max(v, kv8_dpp<kDppQuadXor2>(v));
  v = max(v, kv8_dpp<kDppRowHalfMirror>(v));
  return max(v, kv8_dpp<kDppRowMirror>(v));
}

// One workgroup's piece of a call.
struct Kv8Work {
  int s, r0, cols, len;     // sequence, its first row, its columns (rows * group) and positions
  int tile, split, splits;  // tile of columns; split of the positions
  int t0, t1;               // the split's positions
  int slot, unit;           // split tiles only: of its first partial result, of its counter
};

// Sequence s: columns and positions; no columns if row_start is not in order.
template <int TC>
__device__ __forceinline__ void kv8_seq(const Kv8AttnArgs& A, int s, bool report, int& r0, int& cols, int& len) {
  r0 = A.row_start[s];
  const int r1 = A.row_start[s + 1], l = A.lens[s];
  const bool good = r0 >= 0 && r1 >= r0 && r1 <= A.n_rows;
  const int64_t cap = (int64_t)A.kv.mbps * A.kv.bs;
  if (report && !good) kv8_error(A.err, KV8_ERR_ROWS);
  if (report && l > cap) kv8_error(A.err, KV8_ERR_BLOCK);
  cols = good ? (r1 - r0) * A.group : 0;
  len = (int)min((int64_t)max(l, 0), cap);
}

// Piece `entry` of the launch, the same in every wave.  Splits are as long as
// an even share of all tiles' positions among the workgroups that fit the chip
// (target), so that sequences of very different lengths keep every compute unit
// busy to the end; shorter than kKv8FullTokens only as far as every compute unit
// gets one.  Measured (32 query heads over 8 of 128): one sequence of 16384
// positions 17.1 us in splits of 512, 20.9 in splits of 256; four of 8192 15.9 and
// 18.7; where the share is longer than that, a share of 768 workgroups against
// one of 256: eight sequences of 4096 (32 heads of 96) 27.8 and 32.5.
//
// k8_many's workgroups hold a compute unit to themselves or in pairs, and a few
// more than fit double the time: there a tile is cut into as many splits as
// leave the total within the target (FEWER), not one more.
struct Kv8Split {
  int per;       // positions of a split
  float share;   // of all positions, of a workgroup
};
__device__ __forceinline__ Kv8Split kv8_split(const Kv8AttnArgs& A, float sum) {
  // (a little more than the share: the float sum may be that much too small)
  const float all = min(sum * (float)A.kv.H * 1.002f, 1e18f);
  const float least = max((float)kKv8MinTokens, min(all / (float)kKv8Units, (float)kKv8FullTokens));
  const float share = all / (float)A.target;
  return {((int)min(max(share, least), 1e9f) + 63) / 64 * 64, share >= least ? share : 0.f};
}
template <int TC>
__device__ __forceinline__ bool kv8_pick(const Kv8AttnArgs& A, int entry, bool report, Kv8Work& w) {
  constexpr bool FEWER = TC > 16;   // k8_many
  const int lane = threadIdx.x & 63;
  float sum = 0.f;
  int r0 = 0, cols = 0, len = 0, tiles = 0;
  for (int c = 0; c < A.n_seqs; c += 64) {
    const bool mine = c + lane < A.n_seqs;
    kv8_seq<TC>(A, mine ? c + lane : A.n_seqs - 1, report && mine, r0, cols, len);
    tiles = mine ? (cols + TC - 1) / TC : 0;
    sum += (float)tiles * (float)len;
  }
  const Kv8Split cut = kv8_split(A, wave_sum(sum));
  int before = 0, slots = 0, units = 0;
  w.s = -1;
  for (int c = 0; c < A.n_seqs; c += 64) {
    if (A.n_seqs > 64) {
      const bool mine = c + lane < A.n_seqs;
      kv8_seq<TC>(A, mine ? c + lane : A.n_seqs - 1, false, r0, cols, len);
      tiles = mine ? (cols + TC - 1) / TC : 0;
    }
    int p = max(cut.per, ((len + A.max_splits - 1) / A.max_splits + 63) / 64 * 64);
    if (FEWER && cut.share > 0.f) {
      const int n = max(1, min(A.max_splits, (int)((float)len * 1.004f / cut.share)));
      p = ((len + n - 1) / n + 63) / 64 * 64;
    }
    int splits = len <= kKv8Whole ? 1 : (len + p - 1) / p;
    if (FEWER && splits <= kKv8FewSplits && len - p < kKv8Saved) splits = 1;
    // (row starts out of order can name rows many times over: capped, so that the
    // counts below stay in range until they are found to exceed the grid)
    const int mine = min(tiles * splits, A.entries + 1), ms = splits > 1 ? mine : 0, mu = splits > 1 ? tiles : 0;
    const int upto = kv8_wave_scan(mine), us = kv8_wave_scan(ms), uu = kv8_wave_scan(mu);
    const uint64_t hit = __ballot(entry >= before + upto - mine && entry < before + upto);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      w.s = c + l;
      w.r0 = of(r0);
      w.cols = of(cols);
      w.len = of(len);
      w.splits = of(splits);
      const int j = entry - before - of(upto - mine), pl = w.splits > 1 ? of(p) : w.len;
      // (the last tile first: of a causal sequence it sees the most)
      w.tile = of(tiles) - 1 - j / w.splits;
      w.split = j % w.splits;
      w.t0 = min(w.len, w.split * pl);
      w.t1 = min(w.len, w.t0 + pl);
      w.slot = slots + of(us - ms) + w.tile * w.splits;
      w.unit = units + of(uu - mu) + w.tile;
    }
    before = min(before + __builtin_amdgcn_readlane(upto, 63), 1 << 30);
    slots = min(slots + __builtin_amdgcn_readlane(us, 63), 1 << 30);
    units = min(units + __builtin_amdgcn_readlane(uu, 63), 1 << 30);
  }
  // row starts that overlap can ask for more than the grid holds: nothing is done then
  if (before > A.entries) {
    if (report && lane == 0) kv8_error(A.err, KV8_ERR_ROWS);
    return false;
  }
  return w.s >= 0;
}

// Positions that column c of the tile's sequence sees.
__device__ __forceinline__ int kv8_sees(const Kv8AttnArgs& A, const Kv8Work& w, int c) {
  if (c >= w.cols) return 0;
  const int i = c / A.group;
  const int v = A.visible ? A.visible[w.r0 + i] : w.len - (w.cols / A.group - 1 - i);
  return min(max(v, 0), w.len);
}

// Where the 16 positions of group t / 16 of a sequence lie: their first cache
// row (of all heads' rows of the pool) and scales.  Everything is the same in all
// lanes, so the loads are scalar ones and wait on a counter of their own.
struct Kv8Place {
  int row;       // -1: not in the pool
  float ks, vs;
};
__device__ __forceinline__ int kv8_block(const Kv8AttnArgs& A, int s, int t, int& in) {
  const uint32_t G = (uint32_t)t >> 4;
  const uint32_t lb = (uint32_t)(((uint64_t)G * A.bs_magic) >> 31);
  in = (int)(t & ~15) - (int)lb * A.kv.bs;
  return kv8_lds(A.kv.bt + (int64_t)s * A.kv.mbps + min((int)lb, A.kv.mbps - 1));
}
__device__ __forceinline__ Kv8Place kv8_place(const Kv8AttnArgs& A, int h, int blk, int in) {
  const bool ok = blk >= 0 && blk < A.kv.nb;
  const int page = (ok ? blk : 0) * A.kv.H + h;
  Kv8Place p;
  p.row = ok ? page * A.kv.bs + in : -1;
  p.ks = kv8_lds(A.kv.ks + page);
  p.vs = kv8_lds(A.kv.vs + page);
  return p;
}

template <int BF>
__device__ __forceinline__ float kv8_elem(const void* p, int64_t at) {
  if constexpr (BF) return bf16_to_f32(((const uint16_t*)p)[at]);
  else return ((const float*)p)[at];
}

// N consecutive elements (a multiple of 8, 16-byte aligned) as float.
template <int BF, int N>
__device__ __forceinline__ void kv8_row(const void* p, int64_t at, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    if constexpr (BF) {
      const u32x4_t w = kv8_ld<u32x4_t>((const uint16_t*)p + at + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i + 2 * j] = bf16lo(w[j]);
        x[i + 2 * j + 1] = bf16hi(w[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f32x4_t w = kv8_ld<f32x4_t>((const float*)p + at + i + 4 * j);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i + 4 * j + k] = w[k];
      }
    }
  }
}

// Two floats at once, as st_agent and ld_agent (8-byte aligned).
__device__ __forceinline__ void st_agent2(float* p, float a, float b) {
  const uint64_t v = __float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 ld_agent2(const float* p) {
  const uint64_t v = __hip_atomic_load((uint64_t*)const_cast<float*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Sum of an unnormalised result over its weight; nothing seen: zero.
__device__ __forceinline__ float kv8_over(float a, float l) { return l != 0.f ? a / l : 0.f; }

// Weight of a partial result with maximum m in one with maximum M (base 2);
// `l` zero: it has seen nothing (NaN weights are kept).
__device__ __forceinline__ float kv8_weight(float m, float l, float M) {
  return l != 0.f ? __builtin_amdgcn_exp2f(m - M) : 0.f;
}

constexpr float kLog2e = 1.4426950408889634f;

}  // namespace m2r2
