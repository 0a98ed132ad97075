// Appending rows to the 8-bit paged cache, with the rotation of keys and
// queries on the way.
//
// A block of one head has one scale, so its new rows are quantised together:
// a unit is one block of one sequence and one head, keys and values, and it
// needs the maximum over the block's new entries before it can write.  The
// entries stay in registers between the two.  Blocks of 16 tokens are one
// wave's (no barrier); larger ones are shared by four waves.  Queries ride in
// units of their own, a few heads each, so that a wave reads a token's cosines
// once for all of them.
//
// What bounds it: long prompts, the bytes of the rows; single tokens, the
// chain row start -> position -> block table -> scale.  Measured: a prompt of 16000
// bfloat16 rows of 32 query and 8 cache heads of 128, 82 us, 4.5 TB/s; one row, 6.2 us.
#pragma once
#include "kv8.h"

namespace m2r2 {

constexpr int kKv8AppThreads = 256;
constexpr int kKv8QHeads = 4;   // query heads of a unit

struct Kv8AppArgs {
  Kv8Pages kv;
  int n_seqs, n_rows;
  const int *row_start, *positions;
  const void *k, *v, *q;
  void* qo;
  int64_t k_row, k_head, v_row, v_head, q_row, q_head, qo_row, qo_head;
  const float* rope;
  int rope_len, n_heads, units;   // units: of one block, heads of the cache and groups of query heads
  int* err;
};

// Blocks of sequence s start at this number in the launch's count: every
// sequence has room for two more than its rows fill.
__host__ __device__ constexpr int kv8_block_base(int row_start, int s, int bs) { return row_start / bs + 2 * s; }

// Eight consecutive elements of a row as float.
template <int BF>
struct Kv8Raw {
  u32x4_t w[BF ? 1 : 2];
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    if constexpr (BF) {
      w[0] = *(const u32x4_t*)((const uint16_t*)p + at);
    } else {
      w[0] = *(const u32x4_t*)((const float*)p + at);
      w[1] = *(const u32x4_t*)((const float*)p + at + 4);
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (BF) return (i & 1) ? bf16hi(w[0][i >> 1]) : bf16lo(w[0][i >> 1]);
    else return __uint_as_float(w[i >> 2][i & 3]);
  }
};

// (lo, hi) of a pair of halves, turned by (c, s).  A product of two floats is
// exact in 64 bits, so each result is rounded once there and once to float32:
// the rounding border of a code does not depend on how the sum is formed.
__device__ __forceinline__ void kv8_turn(float& lo, float& hi, float c, float s) {
  const double a = lo, b = hi, cd = c, sd = s;
  lo = (float)(a * cd - b * sd);
  hi = (float)(b * cd + a * sd);
}

__device__ __forceinline__ bool kv8_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Four codes of values already divided by the scale.
__device__ __forceinline__ uint32_t kv8_pack4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// What is stored for y: saturated, divided by the scale; NaN where y is not finite.
__device__ __forceinline__ float kv8_scaled(float y, float inv) {
  constexpr float kTop = 448.f * 5192296858534827628530496329220096.f;   // 448 * 2^112
  return kv8_finite(y) ? fminf(fmaxf(y, -kTop), kTop) * inv : __uint_as_float(0x7fc00000u);
}

// Eight codes at `p` whose scale grew, times f (a power of two).
__device__ __forceinline__ void kv8_regrow(uint8_t* p, float f) {
  const uint2 c = *(const uint2*)p;
  uint2 o;
  const auto c0 = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, false), c1 = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, true);
  const auto c2 = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, false), c3 = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, true);
  o.x = kv8_pack4(c0[0] * f, c0[1] * f, c1[0] * f, c1[1] * f);
  o.y = kv8_pack4(c2[0] * f, c2[1] * f, c3[0] * f, c3[1] * f);
  *(uint2*)p = o;
}
// Eight values of each half, as codes.
__device__ __forceinline__ void kv8_store16(uint8_t* p, int half, const float (&y)[16], float inv) {
  float z[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) z[x] = kv8_scaled(y[x], inv);
  *(uint2*)p = make_uint2(kv8_pack4(z[0], z[1], z[2], z[3]), kv8_pack4(z[4], z[5], z[6], z[7]));
  *(uint2*)(p + half) = make_uint2(kv8_pack4(z[8], z[9], z[10], z[11]), kv8_pack4(z[12], z[13], z[14], z[15]));
}
// Maximum of their magnitudes, not counting NaN and infinities.
__device__ __forceinline__ float kv8_most16(const float (&y)[16]) {
  float m = 0.f;
#pragma unroll
  for (int x = 0; x < 16; ++x) m = fmaxf(m, kv8_finite(y[x]) ? fabsf(y[x]) : 0.f);
  return m;
}

// WPU: waves per unit; NIT: slabs of 16 tokens per wave, at most.
template <int BF, int HD, int WPU, int NIT>
__global__ __launch_bounds__(kKv8AppThreads) void k8_append(Kv8AppArgs A) {
  constexpr int NC = HD / 16;                  // lanes of a token: 8 dims of each half
  constexpr int NS = (kKv8Slab * NC + 63) / 64;   // steps of a slab
  constexpr int HALF = HD / 2;
  __shared__ float red[2][4];
  const int lane = threadIdx.x & 63, wv = WPU > 1 ? threadIdx.x >> 6 : 0;
  const int64_t gid = WPU > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int bs = A.kv.bs;
  const int entry = (int)(gid / A.units), unit = (int)(gid % A.units);
  if (entry >= kv8_block_base(A.n_rows, A.n_seqs, bs)) return;
  const int s = kv8_find(A.n_seqs, entry, [&](int i) { return kv8_block_base(A.row_start[i], i, bs); });
  const int r0 = A.row_start[s], r1 = A.row_start[s + 1], p0 = A.positions[s];
  if (r0 < 0 || r1 < r0 || r1 > A.n_rows) {
    if (lane == 0) kv8_error(A.err, KV8_ERR_ROWS);
    return;
  }
  const int j = entry - kv8_block_base(r0, s, bs);
  if (r1 == r0 || j < 0) return;
  if (p0 < 0) {
    if (lane == 0) kv8_error(A.err, KV8_ERR_BLOCK);
    return;
  }
  const int64_t cap = (int64_t)A.kv.mbps * bs, stop = (int64_t)p0 + (r1 - r0);
  const int64_t limit = A.rope ? min(cap, (int64_t)A.rope_len) : cap;
  if (j == 0 && stop > limit && lane == 0) kv8_error(A.err, limit < cap ? KV8_ERR_ROPE : KV8_ERR_BLOCK);
  const int64_t lb = p0 / bs + j;
  const int64_t begin = max((int64_t)p0, lb * bs), end = min(min(stop, limit), (lb + 1) * bs);
  if (begin >= end) return;
  const int first = (int)(begin - lb * bs), last = (int)(end - lb * bs);   // slots [first, last)
  const int blk = A.kv.bt[(int64_t)s * A.kv.mbps + lb];
  if (blk < 0 || blk >= A.kv.nb) {
    if (lane == 0) kv8_error(A.err, KV8_ERR_BLOCK);
    return;
  }
  // this lane's place in step t of slab i: a token of the block, eight dims of each half
  const int nc = NC;
  auto slot_of = [&](int i, int t) {
    const int ix = t * 64 + lane;
    return ix < kKv8Slab * nc ? (i * WPU + wv) * kKv8Slab + ix / nc : 1 << 20;
  };
  auto dim_of = [&](int t) { return (t * 64 + lane) % nc * 8; };
  const int64_t row_b = r0 + (lb * bs - p0);   // row of slot 0 (negative where that lies before the rows)

  if (unit >= A.kv.H) {   // ---- query heads ---------------------------------
    const int h0 = (unit - A.kv.H) * kKv8QHeads, h1 = min(h0 + kKv8QHeads, A.n_heads);
    for (int i = 0; i < NIT; ++i) {
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        const int slot = slot_of(i, t), d = dim_of(t);
        if (slot < first || slot >= last) continue;
        float4 cs[4];
        if (A.rope) {
          const float4* rp = (const float4*)(A.rope + ((lb * bs + slot) * HALF + d) * 2);
#pragma unroll
          for (int x = 0; x < 4; ++x) cs[x] = rp[x];
        }
        // (two heads' loads ahead of their arithmetic: 82 us for the prompt above, 86 for one head's, 84 for four)
        for (int ha = h0; ha < h1; ha += 2) {
          Kv8Raw<BF> lo[2], hi[2];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (ha + g >= h1) break;
            const int64_t at = (row_b + slot) * A.q_row + (int64_t)(ha + g) * A.q_head + d;
            lo[g].load(A.q, at);
            hi[g].load(A.q, at + HALF);
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const int h = ha + g;
            if (h >= h1) break;
            float y0[8], y1[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              y0[x] = lo[g].at(x);
              y1[x] = hi[g].at(x);
              if (A.rope) {
                const float4 f = cs[x >> 1];
                kv8_turn(y0[x], y1[x], (x & 1) ? f.z : f.x, (x & 1) ? f.w : f.y);
              }
            }
            const int64_t to = (row_b + slot) * A.qo_row + (int64_t)h * A.qo_head + d;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float(&y)[8] = z ? y1 : y0;
              if constexpr (BF) {
                bf16x8_t o;
#pragma unroll
                for (int x = 0; x < 8; ++x) o[x] = (__bf16)y[x];
                *(bf16x8_t*)((uint16_t*)A.qo + to + z * HALF) = o;
              } else {
                float* o = (float*)A.qo + to + z * HALF;
                *(float4*)o = make_float4(y[0], y[1], y[2], y[3]);
                *(float4*)(o + 4) = make_float4(y[4], y[5], y[6], y[7]);
              }
            }
          }
        }
      }
    }
    return;
  }

  // ---- one head of the cache: keys, then values ------------------------------
  const int h = unit;
  const int64_t page = (int64_t)blk * A.kv.H + h;
  for (int which = 0; which < 2; ++which) {
    const void* src = which ? A.v : A.k;
    const int64_t s_row = which ? A.v_row : A.k_row, s_head = which ? A.v_head : A.k_head;
    uint8_t* base = (which ? A.kv.v : A.kv.k) + page * bs * HD;
    float* scale = (which ? A.kv.vs : A.kv.ks) + page;
    const float old_s = *scale;
    float y[NIT][NS][16];
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        const int slot = slot_of(i, t), d = dim_of(t);
        if (slot < first || slot >= last) continue;
        Kv8Raw<BF> lo, hi;
        const int64_t at = (row_b + slot) * s_row + (int64_t)h * s_head + d;
        lo.load(src, at);
        hi.load(src, at + HALF);
        const bool turn = !which && A.rope;
        float4 cs[4];
        if (turn) {
          const float4* rp = (const float4*)(A.rope + ((lb * bs + slot) * HALF + d) * 2);
#pragma unroll
          for (int x = 0; x < 4; ++x) cs[x] = rp[x];
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          float a = lo.at(x), b = hi.at(x);
          if (turn) {
            const float4 f = cs[x >> 1];
            kv8_turn(a, b, (x & 1) ? f.z : f.x, (x & 1) ? f.w : f.y);
          }
          y[i][t][x] = a;
          y[i][t][8 + x] = b;
        }
        most = fmaxf(most, kv8_most16(y[i][t]));
      }
    most = wave_max(most);
    if constexpr (WPU > 1) {
      if (lane == 0) red[which][wv] = most;
      __syncthreads();   // (also: every wave has read the stored scale)
      most = fmaxf(fmaxf(red[which][0], red[which][1]), fmaxf(red[which][2], red[which][3]));
    }
    const int old_e = kv8_exponent(old_s);
    int e = kv8_scale_exponent(most);
    if (first > 0) e = max(e, old_e);
    const bool grown = first > 0 && e > old_e;
    const float inv = kv8_two_to(-e);
    if (grown) {   // the earlier rows' codes at the new scale
      const float f = kv8_two_to(old_e - e);
      for (int i = 0; i < NIT; ++i)
#pragma unroll
        for (int t = 0; t < NS; ++t) {
          const int slot = slot_of(i, t), d = dim_of(t);
          if (slot >= first) continue;
          kv8_regrow(base + slot * HD + d, f);
          kv8_regrow(base + slot * HD + HALF + d, f);
        }
    }
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        const int slot = slot_of(i, t), d = dim_of(t);
        if (slot < first || slot >= last) continue;
        kv8_store16(base + slot * HD + d, HALF, y[i][t], inv);
      }
    if (lane == 0 && wv == 0 && (first == 0 || grown)) *scale = kv8_two_to(e);
  }
}

}  // namespace m2r2
