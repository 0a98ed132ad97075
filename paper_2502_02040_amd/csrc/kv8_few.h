// Attention over the 8-bit cache for few columns: decoding, dual-stream rows,
// short chunks.
//
// What bounds it: the cache's bytes, read once for the 16 columns of a tile.
// A wave takes tiles of 32 positions and keeps everything between a load and
// its use in registers, with the next tile in flight; the workgroup meets once,
// at the end.
//   * S^T = K Q^T: keys are the A operand.  Row r = 4 a + b of the first product
//     is position 8 a + b, of the second 8 a + 4 + b, so that lane (q, g) gets
//     the scores of positions 8 g .. 8 g + 7 of column q, which is the B operand
//     of O^T = V^T P^T as it stands.  Lane (m, g) reads HD / 4 consecutive
//     bytes of two positions: the dims of a step are numbered to suit.
//   * A lane reads 8 bytes (dims 8 n ..) of the eight positions of its group;
//     byte permutes pair two positions' codes of a dim, which the conversion to
//     bfloat16 takes, with the block's scale, in one instruction: codes times a
//     power of two are exact there.
//   * Block ids and scales are the same for all lanes: scalar loads, one tile
//     further ahead, so that they hold up no vector load.
// Queries are bfloat16 as given, or float32 cut into three parts (24 bits).
// Probabilities are rounded to 16 bits (two parts) for bfloat16 rows and kept to 24
// for float32 rows: the matrix pipe is idle enough that both are free.
//
// Measured (a large copy reaches 5.17 TB/s here): one row of 32 heads of 128 for 8,
// behind 131001 positions, 57 us, 4.7 TB/s; 32 such sequences of up to 8192 positions
// 70 us, 4.3 TB/s; eight dual-stream pairs of float32 rows, 32 heads of 96, behind up to
// 4096 positions, 32 us, 3.5 TB/s (three products for each: 180 registers and two
// waves per SIMD); one row behind 1025 positions 10.7 us and behind 17 5.9 us, which
// are chains: launch, lengths, block ids, codes, join.
#pragma once
#include <type_traits>

#include "kv8_attn.h"

namespace m2r2 {

constexpr int kFewCols = 16;
constexpr int kFewWaves = 4;
constexpr int kFewThreads = 64 * kFewWaves;
constexpr int kFewTile = 32;

__device__ __forceinline__ f32x4_t kv8_mma16(u32x4_t a, u32x4_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                 0, 0, 0);
}
// Maximum and sum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float kv8_col_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float kv8_col_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int BF, int HD>
struct Kv8Few {
  static constexpr int NS = HD / 32;        // matrix steps of a score
  static constexpr int ND = HD / 8;         // lanes that hold dims of the output
  static constexpr int QN = BF ? 1 : 3, PN = BF ? 2 : 3;
  struct Tile {
    uint32_t k[2][2 * NS];   // the lane's bytes of two positions
    u32x2_t v[8];
  };
  struct Blocks {            // of a tile's two groups of 16 positions
    int b[2], in[2];
  };
  struct Places {
    Kv8Place p[2];
  };
  u32x4_t q[NS][QN];
  float m_run, l_run;
  f32x4_t acc[8];            // dim 8 (4 g + i) + j of column q: acc[j][i]

  __device__ __forceinline__ void init(const Kv8AttnArgs& A, const Kv8Work& w, int h, int c) {
    const int g = (threadIdx.x & 63) >> 4;
    float x[8 * NS];
    const int cc = min(c, w.cols - 1);
    kv8_row<BF>(A.q, (int64_t)(w.r0 + cc / A.group) * A.q_row + (int64_t)(h * A.group + cc % A.group) * A.q_head + g * (HD / 4), x);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = c < w.cols ? x[8 * s + i] : 0.f;
      kv8_parts<QN, false>(y, q[s]);
    }
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  static __device__ __forceinline__ Blocks blocks(const Kv8AttnArgs& A, int s, int t) {
    Blocks b;
#pragma unroll
    for (int i = 0; i < 2; ++i) b.b[i] = kv8_block(A, s, t + 16 * i, b.in[i]);
    return b;
  }
  static __device__ __forceinline__ Places places(const Kv8AttnArgs& A, int h, const Blocks& b) {
    Places p;
#pragma unroll
    for (int i = 0; i < 2; ++i) p.p[i] = kv8_place(A, h, b.b[i], b.in[i]);
    return p;
  }
  // Scalar loads return in any order: a wait for one waits for all.  This is the
  // one wait of a tile, for what the tile before requested, ahead of its own requests.
  static __device__ __forceinline__ void arrived(const Blocks& b, const Places& p) {
    asm volatile("" ::"s"(b.b[0]), "s"(b.b[1]), "s"(p.p[0].ks), "s"(p.p[0].vs), "s"(p.p[1].ks), "s"(p.p[1].vs));
    __builtin_amdgcn_sched_barrier(0);
  }
  static __device__ __forceinline__ void load(const Kv8AttnArgs& A, const Places& p, Tile& t) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const int rk = max((m >> 3) ? p.p[1].row : p.p[0].row, 0), rv = max((g >> 1) ? p.p[1].row : p.p[0].row, 0);
    const uint8_t* kp = A.kv.k + (int64_t)(rk + 8 * ((m >> 2) & 1) + (m & 3)) * HD + g * (HD / 4);
#pragma unroll
    for (int a = 0; a < 2; ++a) {
#pragma unroll
      for (int x = 0; x < 2 * NS; x += 4) {
        if (2 * NS - x >= 4) {
          const u32x4_8_t d = kv8_ld<u32x4_8_t>(kp + a * 4 * HD + 4 * x);
#pragma unroll
          for (int i = 0; i < 4; ++i) t.k[a][x + i] = d[i];
        } else {
          const u32x2_t d = kv8_ld<u32x2_t>(kp + a * 4 * HD + 4 * x);
          t.k[a][x] = d[0];
          t.k[a][x + 1] = d[1];
        }
      }
    }
    const uint8_t* vp = A.kv.v + (int64_t)(rv + 8 * (g & 1)) * HD + 8 * min(m, ND - 1);
#pragma unroll
    for (int x = 0; x < 8; ++x) t.v[x] = kv8_ld<u32x2_t>(vp + x * HD);
  }

  // Positions t .. t+31.  FULL: every live column sees all of them; else
  // column q sees those below `sees`, and none at or above `most` is seen by any.
  template <bool FULL>
  __device__ __forceinline__ void tile(Tile& t, const Places& pl, float c, int sees, int most) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
    const float ks = (m >> 3) ? pl.p[1].ks : pl.p[0].ks, vs = (g >> 1) ? pl.p[1].vs : pl.p[0].vs;
    f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
    u32x4_t k0[NS], k1[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      k0[s] = u32x4_t{kv8_up<false>(t.k[0][2 * s], ks), kv8_up<true>(t.k[0][2 * s], ks),
                      kv8_up<false>(t.k[0][2 * s + 1], ks), kv8_up<true>(t.k[0][2 * s + 1], ks)};
      k1[s] = u32x4_t{kv8_up<false>(t.k[1][2 * s], ks), kv8_up<true>(t.k[1][2 * s], ks),
                      kv8_up<false>(t.k[1][2 * s + 1], ks), kv8_up<true>(t.k[1][2 * s + 1], ks)};
    }
#pragma unroll
    for (int p = QN - 1; p >= 0; --p)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        s0 = kv8_mma16(k0[s], q[s][p], s0);
        s1 = kv8_mma16(k1[s], q[s][p], s1);
      }
    float z[8], mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      z[i] = (i < 4 ? s0[i & 3] : s1[i & 3]) * c;
      if (!FULL && 8 * g + i >= sees) z[i] = -INFINITY;
      mx = fmaxf(mx, z[i]);
    }
    const float mn = fmaxf(m_run, kv8_col_max(mx));
    const float mb = mn == -INFINITY ? 0.f : mn;   // (nothing seen yet)
    const float al = __builtin_amdgcn_exp2f(m_run - mb);
    m_run = mn;
    float p[8], ls = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(z[i] - mb);
      ls += p[i];
    }
    l_run = l_run * al + ls;
    if (__any(al != 1.f)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] *= al;
    }
    u32x4_t pp[PN];
    kv8_parts<PN>(p, pp);
    if constexpr (!FULL) {
      // codes that some column does not see must not reach it: NaN becomes
      // zero in the operand, and is added to the columns that see it
      bool odd = false;
      uint32_t ix[8], iy[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const bool live = 8 * g + x < most;
        ix[x] = live ? kv8_nan_bytes(t.v[x][0]) : 0u;
        iy[x] = live ? kv8_nan_bytes(t.v[x][1]) : 0u;
        odd |= (ix[x] | iy[x]) != 0u;
        t.v[x][0] = live ? t.v[x][0] & ~ix[x] : 0u;
        t.v[x][1] = live ? t.v[x][1] & ~iy[x] : 0u;
      }
      if (__any(odd)) {
        u32x4_t seen;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          seen[i] = (8 * g + 2 * i < sees ? 0x3f80u : 0u) | (8 * g + 2 * i + 1 < sees ? 0x3f800000u : 0u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          u32x4_t one;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a = (j < 4 ? ix[2 * i] : iy[2 * i]) >> (8 * (j & 3)), b = (j < 4 ? ix[2 * i + 1] : iy[2 * i + 1]) >> (8 * (j & 3));
            one[i] = ((a & 0xffu) ? 0x3f80u : 0u) | ((b & 0xffu) ? 0x3f800000u : 0u);
          }
          const f32x4_t n = kv8_mma16(one, seen, f32x4_t{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (n[i] > 0.f) acc[j][i] = __uint_as_float(0x7fc00000u);
        }
      }
    }
    u32x4_t vt[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const uint32_t a = __builtin_amdgcn_perm(t.v[2 * i + 1][x], t.v[2 * i][x], 0x05010400u);
        const uint32_t b = __builtin_amdgcn_perm(t.v[2 * i + 1][x], t.v[2 * i][x], 0x07030602u);
        vt[4 * x][i] = kv8_up<false>(a, vs);
        vt[4 * x + 1][i] = kv8_up<true>(a, vs);
        vt[4 * x + 2][i] = kv8_up<false>(b, vs);
        vt[4 * x + 3][i] = kv8_up<true>(b, vs);
      }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int x = PN - 1; x >= 0; --x) acc[j] = kv8_mma16(vt[j], pp[x], acc[j]);
  }

  __device__ __forceinline__ void store(float* m, float* l, float* out) {
    const int g = (threadIdx.x & 63) >> 4;
    const float ls = kv8_col_sum(l_run);
    if (g == 0) {
      *m = m_run;
      *l = ls;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = 4 * g + i;
      if (n < ND) {
        *(float4*)(out + 8 * n) = make_float4(acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
        *(float4*)(out + 8 * n + 4) = make_float4(acc[4][i], acc[5][i], acc[6][i], acc[7][i]);
      }
    }
  }
};

// Floats of a partial result: the columns' accumulators, then their maxima and sums.
__host__ __device__ constexpr int kv8_part_floats(int cols, int hd) { return cols * (hd + 2); }

// Where results go: the caller's array.
template <int BF, int HD>
struct Kv8Out {
  static constexpr bool kKeep = false;   // results of a tile are wanted together, in LDS
  struct Ahead {};                       // what finish() reads, requested early
  __device__ __forceinline__ void request(Ahead&, const Kv8AttnArgs&, int) const {}
  __device__ __forceinline__ void put(const Kv8AttnArgs& A, int row, int head, int d, float a, float b) const {
    const int64_t to = (int64_t)row * A.out_row + (int64_t)head * A.out_head + d;
    if constexpr (BF) *(uint32_t*)((uint16_t*)A.out + to) = kv8_pk(a, b);
    else *(float2*)((float*)A.out + to) = make_float2(a, b);
  }
  __device__ __forceinline__ void finish(const Ahead&, const Kv8AttnArgs&, const Kv8Work&, int, int, const float (*)[HD],
                                         float*) const {}
};

template <int BF, int HD, class Out>
__global__ __launch_bounds__(kFewThreads, 2) void k8_few(Kv8AttnArgs A, Out out) {
  constexpr int OD = HD / 16;   // dims of a thread of the own keys
  __shared__ __attribute__((aligned(16))) float acc_s[kFewWaves][kFewCols][HD];
  __shared__ float m_s[kFewWaves][kFewCols], l_s[kFewWaves][kFewCols];
  __shared__ __attribute__((aligned(16))) float ov_s[kFewCols][HD];
  __shared__ float oz_s[kFewCols];   // own values and scores (first split)
  __shared__ float mw[kFewCols][kKv8MaxSplits], li_s[kFewCols];
  __shared__ int last_s;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % A.kv.H, entry = blockIdx.x / A.kv.H;
  Kv8Work w;
  if (!kv8_pick<kFewCols>(A, entry, blockIdx.x == 0 && wv == 0, w)) return;
  const int c0 = w.tile * kFewCols, live = min(kFewCols, w.cols - c0);
  const int q = lane & 15, c = c0 + q;
  using F = Kv8Few<BF, HD>;
  int tt = wv;
  const typename F::Blocks b0 = F::blocks(A, w.s, w.t0 + tt * kFewTile);   // (needed or not)
  const int sees = kv8_sees(A, w, c);
  // positions that any, and that every live column sees
  int most = sees, least = q < live ? sees : 1 << 30;
  most = __builtin_amdgcn_readfirstlane(kv8_row_max(most));
  least = -__builtin_amdgcn_readfirstlane(kv8_row_max(-least));
  const int t1 = min(w.t1, most);
  const int ntile = t1 > w.t0 ? (t1 - w.t0 + kFewTile - 1) / kFewTile : 0;
  const float sc = A.scale * kLog2e;
  F f;
  typename Out::Ahead ahead;
  typename F::Tile ta, tb;
  typename F::Places pa, pb;
  typename F::Blocks bn;
  auto at = [&](int tt) { return w.t0 + min(tt, max(ntile - 1, 0)) * kFewTile; };
  if (tt < ntile) {
    pa = F::places(A, h, b0);
    F::load(A, pa, ta);
    bn = F::blocks(A, w.s, at(tt + kFewWaves));
  }
  // own keys and values: 16 threads per column
  const bool own = A.own && w.split == 0;
  if (own) {
    const int oc = tid >> 4, part = tid & 15, cc = min(c0 + oc, w.cols - 1);
    const int row = w.r0 + cc / A.group;
    const int o = oc < live ? A.own[row] : -1;
    if (o >= A.n_own && part == 0) kv8_error(A.err, KV8_ERR_ROWS);
    const bool has = o >= 0 && o < A.n_own;
    float z = 0.f;
    if (has) {
      const int64_t qa = (int64_t)row * A.q_row + (int64_t)(h * A.group + cc % A.group) * A.q_head + part * OD;
      const int64_t ka = (int64_t)o * A.ok_row + (int64_t)h * A.ok_head + part * OD;
      const int64_t va = (int64_t)o * A.ov_row + (int64_t)h * A.ov_head + part * OD;
#pragma unroll
      for (int d = 0; d < OD; ++d) {
        z += kv8_elem<BF>(A.q, qa + d) * kv8_elem<BF>(A.own_k, ka + d);
        ov_s[oc][part * OD + d] = kv8_elem<BF>(A.own_v, va + d);
      }
    }
    z = row_sum16(z) * sc;
    if (part == 0) oz_s[oc] = has ? z : -INFINITY;
  }
  f.init(A, w, h, c);
  out.request(ahead, A, h);
  // Tiles that every live column sees whole; the next tile's codes are in flight
  // meanwhile, whatever kind it is.
  const int nfull = min(ntile, max(0, (least - w.t0) / kFewTile));
  auto there = [](const typename F::Places& p) { return p.p[0].row >= 0 && p.p[1].row >= 0; };
  auto next = [&](const typename F::Places& have, typename F::Tile& t, typename F::Places& p) {
    F::arrived(bn, have);
    p = F::places(A, h, bn);
    bn = F::blocks(A, w.s, at(tt + 2 * kFewWaves));
    if (tt + kFewWaves < ntile) F::load(A, p, t);
    __builtin_amdgcn_sched_barrier(0);
  };
  while (tt < nfull && there(pa)) {
    next(pa, tb, pb);
    f.template tile<true>(ta, pa, sc, 0, 0);
    tt += kFewWaves;
    if (tt >= nfull || !there(pb)) {
      ta = tb;
      pa = pb;
      break;
    }
    next(pb, ta, pa);
    f.template tile<true>(tb, pb, sc, 0, 0);
    tt += kFewWaves;
  }
  // the others: at the end of what a column sees, or with positions outside the
  // pool, which are not seen
  while (tt < ntile) {
    const int t0 = w.t0 + tt * kFewTile, g = lane >> 4;
    const bool gone = (g >> 1 ? pa.p[1].row : pa.p[0].row) < 0;
    if (gone && t0 + 16 * (g >> 1) < most && (lane & 15) == 0) kv8_error(A.err, KV8_ERR_BLOCK);
    f.template tile<false>(ta, pa, sc, gone ? 0 : min(sees, t1) - t0, gone ? 0 : t1 - t0);
    tt += kFewWaves;
    if (tt < ntile) {
      pa = F::places(A, h, bn);
      F::load(A, pa, ta);
      bn = F::blocks(A, w.s, at(tt + kFewWaves));
    }
  }
  f.store(&m_s[wv][q], &l_s[wv][q], acc_s[wv][q]);
  __syncthreads();
  // ---- the waves' results, and the own key's, combined -------------------------
  float* part = A.part + ((int64_t)w.slot * A.kv.H + h) * kv8_part_floats(A.pcols, HD);
  const int64_t pstep = (int64_t)A.kv.H * kv8_part_floats(A.pcols, HD);
  constexpr int kMostPairs = kFewCols * HD / 2 / kFewThreads;   // of dims, of a thread
  auto combine = [&](auto pairs_each) {
    constexpr int EN = decltype(pairs_each)::value;
    float M[EN], l[EN], a[EN], b[EN];
#pragma unroll
    for (int k = 0; k < EN; ++k) {
      const int e = min(2 * (tid + k * kFewThreads), live * HD - 2), i = e / HD, d = e % HD;
      const float oz = own ? oz_s[i] : -INFINITY;
      M[k] = oz;
#pragma unroll
      for (int x = 0; x < kFewWaves; ++x) M[k] = fmaxf(M[k], m_s[x][i]);
      l[k] = oz != -INFINITY ? __builtin_amdgcn_exp2f(oz - M[k]) : 0.f;
      a[k] = b[k] = 0.f;
      if (l[k] != 0.f) {
        a[k] = l[k] * ov_s[i][d];
        b[k] = l[k] * ov_s[i][d + 1];
      }
#pragma unroll
      for (int x = 0; x < kFewWaves; ++x) {
        const float lx = l_s[x][i], y = kv8_weight(m_s[x][i], lx, M[k]);
        const float2 o = *(const float2*)&acc_s[x][i][d];
        // (a wave that has seen nothing leaves zeros)
        a[k] += y * o.x;
        b[k] += y * o.y;
        l[k] += lx != 0.f ? y * lx : 0.f;
      }
    }
#pragma unroll
    for (int k = 0; k < EN; ++k) {
      const int e = 2 * (tid + k * kFewThreads), i = e / HD, d = e % HD;
      if (e >= live * HD) break;
      if (w.splits == 1) {
        a[k] = kv8_over(a[k], l[k]);
        b[k] = kv8_over(b[k], l[k]);
        out.put(A, w.r0 + (c0 + i) / A.group, h * A.group + (c0 + i) % A.group, d, a[k], b[k]);
        if (Out::kKeep) *(float2*)&ov_s[i][d] = make_float2(a[k], b[k]);   // (read above, by this thread)
      } else {
        float* p = part + (int64_t)w.split * pstep;
        st_agent2(p + e, a[k], b[k]);
        if (d == 0) st_agent2(p + A.pcols * HD + 2 * i, M[k], l[k]);
      }
    }
  };
  // (several pairs at once where a thread has them: with 16 columns one at a time takes 1 us longer)
  if (live * HD > 2 * kFewThreads) combine(std::integral_constant<int, kMostPairs>{});
  else combine(std::integral_constant<int, 1>{});
  if (w.splits == 1) {
    out.finish(ahead, A, w, h, live, ov_s, &mw[0][0]);
    return;
  }
  // ---- the last split to arrive joins them ---------------------------------------
  if (!arrive_last(A.cnt + w.unit * A.kv.H + h, w.splits, &last_s)) return;
  // A thread takes pairs of dims: several where there are many columns, their
  // loads together; where a column or two leave threads over, groups of threads
  // take every so-manieth split each.  A column's weights and sum are one wave's, a
  // lane per split.  Every load of either kind is a trip to memory, so the first
  // ones do not wait for the weights, and those of the weights go out together:
  // 16 columns in 8 splits 14.6 us, 16.2 with one pair and one column at a time.
  const int pairs = live * (HD / 2);
  auto at_split = [&](int x) { return part + (int64_t)x * pstep; };
  auto weights = [&]() {
    float2 ml[kFewCols / kFewWaves];
#pragma unroll
    for (int k = 0; k < kFewCols / kFewWaves; ++k) {
      const int i = wv + k * kFewWaves;
      if (i < live) ml[k] = ld_agent2(at_split(min(lane, w.splits - 1)) + A.pcols * HD + 2 * i);
    }
#pragma unroll
    for (int k = 0; k < kFewCols / kFewWaves; ++k) {
      const int i = wv + k * kFewWaves;
      if (i >= live) break;
      const float m = lane < w.splits ? ml[k].x : -INFINITY, l = lane < w.splits ? ml[k].y : 0.f;
      const float y = kv8_weight(m, l, wave_max(m));
      mw[i][lane] = y;
      const float s = wave_sum(l != 0.f ? y * l : 0.f);
      if (lane == 0) li_s[i] = s;
    }
    __syncthreads();
  };
  auto put = [&](int e, float a, float b) {
    const int i = 2 * e / HD;
    a = kv8_over(a, li_s[i]);
    b = kv8_over(b, li_s[i]);
    out.put(A, w.r0 + (c0 + i) / A.group, h * A.group + (c0 + i) % A.group, 2 * e - i * HD, a, b);
    if (Out::kKeep) *(float2*)&ov_s[i][2 * e - i * HD] = make_float2(a, b);
  };
  auto wide = [&](auto pairs_each) {
    constexpr int EN = decltype(pairs_each)::value, UN = EN > 2 ? 8 : 16;
    float2 v[EN][UN], sum[EN];
    auto request = [&](int x) {
#pragma unroll
      for (int u = 0; u < UN; ++u)
#pragma unroll
        for (int k = 0; k < EN; ++k)
          if (x + u < w.splits) v[k][u] = ld_agent2(at_split(x + u) + 2 * min(tid + k * kFewThreads, pairs - 1));
    };
    request(0);
    weights();
#pragma unroll
    for (int k = 0; k < EN; ++k) sum[k] = make_float2(0.f, 0.f);
    for (int x = 0; x < w.splits; x += UN) {
      if (x) request(x);
#pragma unroll
      for (int u = 0; u < UN; ++u) {
#pragma unroll
        for (int k = 0; k < EN; ++k) {
          // (past the last split: weight zero)
          const float y = mw[2 * min(tid + k * kFewThreads, pairs - 1) / HD][x + u];
          sum[k].x += y != 0.f ? y * v[k][u].x : 0.f;
          sum[k].y += y != 0.f ? y * v[k][u].y : 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < EN; ++k)
      if (tid + k * kFewThreads < pairs) put(tid + k * kFewThreads, sum[k].x, sum[k].y);
  };
  if (pairs > 2 * kFewThreads) {
    wide(std::integral_constant<int, kMostPairs>{});
  } else if (pairs > kFewThreads) {
    wide(std::integral_constant<int, 2>{});
  } else {
    constexpr int UN = 16;
    const int groups = pairs <= kFewThreads / 4 ? 4 : pairs <= kFewThreads / 2 ? 2 : 1;
    const int width = kFewThreads / groups;
    const int grp = __builtin_amdgcn_readfirstlane(tid / width), e = tid % width, ee = min(e, pairs - 1), i = 2 * ee / HD;
    float2 v[UN];
    auto request = [&](int x) {   // splits x, x + groups, ...
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        v[u] = make_float2(0.f, 0.f);
        if (x + u * groups < w.splits) v[u] = ld_agent2(at_split(x + u * groups) + 2 * ee);
      }
    };
    request(grp);
    weights();
    float a = 0.f, b = 0.f;
    for (int x = grp; x < w.splits; x += UN * groups) {
      if (x != grp) request(x);
#pragma unroll
      for (int u = 0; u < UN; ++u) {
        // (past the last split: weight zero)
        const float y = x + u * groups < w.splits ? mw[i][x + u * groups] : 0.f;
        a += y != 0.f ? y * v[u].x : 0.f;
        b += y != 0.f ? y * v[u].y : 0.f;
      }
    }
    if (groups > 1) {
      float2* red = (float2*)&acc_s[0][0][0];
      if (e < pairs) red[grp * width + e] = make_float2(a, b);
      __syncthreads();
      if (grp == 0 && e < pairs) {
        a = b = 0.f;
        for (int g2 = 0; g2 < groups; ++g2) {
          a += red[g2 * width + e].x;
          b += red[g2 * width + e].y;
        }
      }
    }
    if (grp == 0 && e < pairs) put(e, a, b);
  }
  out.finish(ahead, A, w, h, live, ov_s, &mw[0][0]);
}

}  // namespace m2r2
