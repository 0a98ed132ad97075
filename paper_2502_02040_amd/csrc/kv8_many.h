// Attention over the 8-bit cache for many columns: prompts and pieces of them.
//
// What bounds it: the matrix rate, and beside it the exponentials and the LDS.
// A workgroup holds 128 columns (32 a wave) and stages tiles of 64 positions:
// codes are converted to bfloat16 (exactly: code times a power of two) and
// values transposed once for all four waves.  The codes of the next tile are in
// registers, those of the one after in flight; two buffers in LDS, one barrier
// per tile.
//   * S^T = K Q^T in 32 x 32 products.  Row m of a product is position
//     16 (m / 16) + 8 (m / 4 % 2) + 4 (m / 8 % 2) + m % 4 of its half, so that lane
//     (column, hi) gets the scores of positions 16 u + 8 hi .. + 7, which is the B
//     operand of O^T = V^T P^T as it stands.
//   * Two workgroups per compute unit, so that one's softmax runs beside the
//     other's products.
// Measured (bfloat16, 32 heads of 128 for 8): prompts of 4001 and of 500 rows 165 us,
// 0.81 PFLOP/s of the 1.31 that a large library product reaches here; 500 rows behind
// 8500 positions 95 us, 0.76 PFLOP/s, the join's launch included (4.5 us where
// nothing is split; a join inside this kernel took 106 and 162 us, but 69
// instead of 20 for 8 rows behind 8000 positions).  Counters of the prompts: the matrix
// unit busy 34 % of the time, the vector unit 45 %, the LDS 37 %; what one of two
// waves on a SIMD issues seldom overlaps the other's products.
// Probabilities of bfloat16 rows are rounded to bfloat16 (half a step of 2^-8, of
// the same size as the result's own rounding, and averaged over the positions):
// a second part would cost half of all products again.  Those of float32 rows
// are kept to 24 bits.
#pragma once
#include <type_traits>

#include "kv8_few.h"

namespace m2r2 {

constexpr int kManyCols = 128;
constexpr int kManyTile = 64;
constexpr int kManyThreads = 256;

// (the accumulators are in registers only where everything that takes them is inlined)
#define KV8_INLINE __attribute__((always_inline))

template <int HD>
struct Kv8ManyLds {
  static constexpr int KP = HD + 8;           // padded rows (elements): 16 lanes' 16 bytes hit all banks
  uint16_t k[2][kManyTile * KP];              // [position][dim]
  uint16_t v[2][HD * kManyTile];              // [dim][position], kv8_at_v
  // of a tile (four in turn): positions outside the pool; positions with NaN
  // values, of a tile that not all columns see whole, and which dims' they are
  unsigned long long gap[4], odd[4];
  int gaps;                                   // any of the first
  uint8_t nan[2][kManyTile][HD / 8];
};

// Place of positions 8 c .. 8 c + 7 of dim d: the eight 16-byte pieces of a
// row are permuted by its number, so that neither eight rows at one piece (the
// products' reads) nor sixteen rows eight apart (the transposed writes) meet in a bank.
__device__ __forceinline__ int kv8_at_v(int d, int c) { return d * kManyTile + 8 * (c ^ (d & 7) ^ (d >> 3 & 7)); }

__device__ __forceinline__ f32x16_t kv8_mma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                 0, 0, 0);
}
// Maximum and sum of lanes l and l ^ 32.
__device__ __forceinline__ float kv8_max32(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float kv8_sum32(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
// v plus both bfloat16 of w.
__device__ __forceinline__ float kv8_add2(uint32_t w, float v) {
  const bf16x2_t one = __builtin_bit_cast(bf16x2_t, 0x3f803f80u);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, w), one, v, false);
}

template <int BF, int HD>
__global__ __launch_bounds__(kManyThreads, BF ? 2 : 1) void k8_many(Kv8AttnArgs A) {
  constexpr int NQ = HD / 16;                // matrix steps of a score
  constexpr int NO = HD / 32;                // tiles of 32 output dims
  constexpr int QN = BF ? 1 : 3, PN = BF ? 1 : 3;
  using L = Kv8ManyLds<HD>;
  constexpr int KP = L::KP;
  constexpr int NK = HD / 32;                // 8-byte pieces of keys per thread
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  L& S = *(L*)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hi = lane >> 5;
  const int h = blockIdx.x % A.kv.H, entry = blockIdx.x / A.kv.H;
  Kv8Work w;
  if (!kv8_pick<kManyCols>(A, entry, blockIdx.x == 0 && wv == 0, w)) return;
  const int c0 = w.tile * kManyCols, c = c0 + 32 * wv + n;
  const bool any = c0 + 32 * wv < w.cols;   // (a wave without columns only stages)
  const bool live = c < w.cols;
  const int cc = min(c, w.cols - 1);
  const int row = w.r0 + cc / A.group, head = h * A.group + cc % A.group;
  // ---- staging ------------------------------------------------------------------
  // A wave stages 16 positions, which lie in one block: where they are is the
  // same for all lanes.  Keys: lane (position lane / 4, part lane % 4) takes
  // HD / 4 bytes; values: lane (positions 4 (lane % 4) .., dims 8 (lane / 4) ..) takes 4 x 8 bytes.
  const int kt = 16 * wv + (lane >> 2), kd = (lane & 3) * (HD / 4);
  const int vt = 16 * wv + 4 * (lane & 3), vd = 8 * (lane >> 2);
  const int vdd = min(vd, HD - 8);
  const uint32_t koff = (lane >> 2) * HD + kd, voff = 4 * (lane & 3) * HD + vdd;
  struct Raw {
    u32x2_t k[NK], v[4];
    float ks, vs;
    bool ok;   // the place exists
  };
  const int* bt = A.kv.bt + (int64_t)w.s * A.kv.mbps;
  // Vector loads all the same: they return in order, and the LDS's counter is the scalar loads' too.
  auto slot = [&](int tt, int& in) KV8_INLINE {   // logical block of the wave's positions (the last one where the table ends)
    const int tp = w.t0 + tt * kManyTile + 16 * wv;
    const uint32_t lb = (uint32_t)(((uint64_t)((uint32_t)tp >> 4) * A.bs_magic) >> 31);
    in = tp - (int)lb * A.kv.bs;
    return min((int)lb, A.kv.mbps - 1);
  };
  int zero = 0;   // (an offset that the compiler takes for a vector)
  asm("" : "+v"(zero));
  auto ask = [&](int tt) KV8_INLINE {   // block id, requested a tile before the codes
    int in;
    return kv8_ld<int>(bt + slot(tt, in) + zero);
  };
  const int i0 = ask(0), i1 = ask(1);   // (needed or not)
  const int sees = kv8_sees(A, w, c);
  // of the wave's columns, and of the workgroup's: every thread looks at all
  int most = sees, most_all = 0, least_all = 1 << 30;
#pragma unroll
  for (int x = 0; x < kManyCols / 64; ++x) {
    const int o = c0 + 64 * x + lane, v = kv8_sees(A, w, o);
    most_all = max(most_all, v);
    least_all = min(least_all, o < w.cols ? v : 1 << 30);
  }
  auto wave_most = [](int v) {
    v = kv8_row_max(v);
    v = max(v, __shfl_xor(v, 16));
    return __builtin_amdgcn_readfirstlane(max(v, __shfl_xor(v, 32)));
  };
  most = wave_most(most);
  most_all = wave_most(most_all);
  least_all = -wave_most(-least_all);
  const int t1 = min(w.t1, most_all);
  const int ntile = t1 > w.t0 ? (t1 - w.t0 + kManyTile - 1) / kManyTile : 0;
  const float sc = A.scale * kLog2e;

  auto fetch = [&](int tt, int id, Raw& r) KV8_INLINE {
    int in;
    slot(tt, in);
    const int blk = __builtin_amdgcn_readfirstlane(id);
    r.ok = (uint32_t)blk < (uint32_t)A.kv.nb;
    const int page = (r.ok ? blk : 0) * A.kv.H + h;
    r.ks = kv8_ld<float>(A.kv.ks + page + zero);
    r.vs = kv8_ld<float>(A.kv.vs + page + zero);
    const int64_t at = ((int64_t)page * A.kv.bs + in) * HD;
    const uint8_t *kp = A.kv.k + at, *vp = A.kv.v + at;
#pragma unroll
    for (int x = 0; x < NK; ++x) r.k[x] = kv8_ld<u32x2_t>(kp + koff + 8 * x);
#pragma unroll
    for (int x = 0; x < 4; ++x) r.v[x] = kv8_ld<u32x2_t>(vp + voff + x * HD);
  };
  Raw ra;
  fetch(0, i0, ra);
  bool gaps = false;   // some position of the split is outside the pool
  auto clean = [&](int tt, Raw& r, int buf) KV8_INLINE {   // a tile that not every column sees whole
    const int t = w.t0 + tt * kManyTile;
    {
      // What no column sees is zero in the products, and so is NaN, which must
      // not reach the columns that do not see it.
      if (tid == 0) {   // marks that were last read two tiles ago
        S.gap[(tt + 2) & 3] = 0;
        S.odd[(tt + 2) & 3] = 0;
      }
      if (!r.ok && lane == 0) atomicOr(&S.gap[tt & 3], 0xffffull << (16 * wv));
      {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const bool there = t + vt + x < t1 && r.ok;
          uint32_t bits = 0;
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const uint32_t nan = there ? kv8_nan_bytes(r.v[x][z]) : 0u;
            r.v[x][z] = there ? r.v[x][z] & ~nan : 0u;
            bits |= ((nan & 1) | (nan >> 7 & 2) | (nan >> 14 & 4) | (nan >> 21 & 8)) << (4 * z);
          }
          S.nan[buf][vt + x][vdd / 8] = bits;
          if (bits) atomicOr(&S.odd[tt & 3], 1ull << (vt + x));
        }
      }
    }
  };
  // Piece j of a tile into LDS: 8-byte pieces of the keys, then two dims at a time of the values.
  constexpr int NPIECE = NK + 4;
  auto piece = [&](int j, const Raw& r, int buf) KV8_INLINE {
    if (j < NK) {
      const u32x4_t o = {kv8_up<false>(r.k[j][0], r.ks), kv8_up<true>(r.k[j][0], r.ks), kv8_up<false>(r.k[j][1], r.ks),
                         kv8_up<true>(r.k[j][1], r.ks)};
      *(u32x4_t*)&S.k[buf][kt * KP + kd + 8 * j] = o;
      return;
    }
    const int x = (j - NK) >> 1, z = (j - NK) & 1;
    u32x2_t o[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w2 = __builtin_amdgcn_perm(r.v[2 * i + 1][x], r.v[2 * i][x], z ? 0x07030602u : 0x05010400u);
      o[0][i] = kv8_up<false>(w2, r.vs);
      o[1][i] = kv8_up<true>(w2, r.vs);
    }
    // (lanes without dims write the last ones' values once more)
#pragma unroll
    for (int d = 0; d < 2; ++d)
      *(u32x2_t*)&S.v[buf][kv8_at_v(vdd + 4 * x + 2 * z + d, vt >> 3) + (vt & 4)] = o[d];
  };
  auto stage = [&](int tt, Raw& r) KV8_INLINE {
    if (w.t0 + (tt + 1) * kManyTile > least_all || gaps) clean(tt, r, tt & 1);
#pragma unroll
    for (int j = 0; j < NPIECE; ++j) piece(j, r, tt & 1);
  };

  // ---- queries ----------------------------------------------------------------------
  u32x4_t q[NQ][QN];
#pragma unroll
  for (int s = 0; s < NQ; ++s) {
    float x[8];
    kv8_row<BF>(A.q, (int64_t)row * A.q_row + (int64_t)head * A.q_head + 16 * s + 8 * hi, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = live ? x[i] : 0.f;
    kv8_parts<QN, false>(x, q[s]);
  }
  float m_run = -INFINITY, l_run = 0.f;
  f32x16_t acc[NO];
#pragma unroll
  for (int d = 0; d < NO; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  if (tid < 4) {
    S.gap[tid] = 0;
    S.odd[tid] = 0;
    S.gaps = 0;
  }
  __syncthreads();
  for (int lb = w.t0 / A.kv.bs + tid; (int64_t)lb * A.kv.bs < t1; lb += kManyThreads)
    if ((uint32_t)bt[lb] >= (uint32_t)A.kv.nb) {
      S.gaps = 1;
      kv8_error(A.err, KV8_ERR_BLOCK);
    }
  __syncthreads();
  gaps = __builtin_amdgcn_readfirstlane(S.gaps) != 0;
  int id = 0;
  if (ntile > 0) {
    stage(0, ra);
    fetch(1, i1, ra);   // (beyond the last tile: some position's block, staged nowhere)
    id = ask(2);
  }
  __syncthreads();
  // row m of a product is this position of its 32
  const int krow = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  // kv8_at_v(32 d + n, 2 u + hi) is vo[u] for even d, vo[u ^ 2] for odd, plus whole rows
  int vo[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) vo[u] = kv8_at_v(n, 2 * u + hi);
  // FULL: every live column of the workgroup sees all of the tile, and it is all there
  // (so is the next one where STAGE: it is staged beside the score products,
  // which leave the vector unit idle, and the one after requested)
  auto compute = [&](int tt, auto full, auto beside) KV8_INLINE {
    constexpr bool FULL = decltype(full)::value, STAGE = decltype(beside)::value;
    const int buf = tt & 1, t0 = w.t0 + tt * kManyTile;
    // The order of this loop is meant: keys are read ahead of the products, or
    // every product waits for the LDS, and a piece of the next tile is staged
    // beside every other product.
    constexpr int NM = 2 * NQ, AHEAD = NM < 6 ? NM : 6;
    u32x4_t kf[NM];
    auto keys = [&](int i) KV8_INLINE { return *(const u32x4_t*)&S.k[buf][(32 * (i & 1) + krow) * KP + 16 * (i >> 1) + 8 * hi]; };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = keys(i);
    f32x16_t sa[2];
#pragma unroll
    for (int i = 0; i < NM; ++i) {
#pragma unroll
      for (int p = QN - 1; p >= 0; --p)
        sa[i & 1] = i < 2 && p == QN - 1 ? kv8_mma32(kf[i], q[0][p], f32x16_t{}) : kv8_mma32(kf[i], q[i >> 1][p], sa[i & 1]);
      if (i + AHEAD < NM) kf[i + AHEAD] = keys(i + AHEAD);
      if constexpr (STAGE) {
#pragma unroll
        for (int j = i * NPIECE / NM; j < (i + 1) * NPIECE / NM; ++j) piece(j, ra, buf ^ 1);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (STAGE) {
      fetch(tt + 2, id, ra);   // (beyond the last tile: some position's block, staged nowhere)
      id = ask(tt + 3);
    }
    // lane (column n, hi): scores of positions 32 x + 16 (r / 8) + 8 hi + r % 8
    const int lim = min(sees, t1) - t0;
    float mx = -INFINITY;
    if constexpr (!FULL) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * x + 16 * (r >> 3) + (r & 7) >= lim - 8 * hi) sa[x][r] = -INFINITY;
      if (const unsigned long long gap = S.gap[tt & 3]) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const uint32_t half = (uint32_t)(gap >> (32 * x)) >> (8 * hi);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((half >> (16 * (r >> 3) + (r & 7))) & 1) sa[x][r] = -INFINITY;
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sa[x][r]);
    mx = kv8_max32(mx) * sc;
    // The maximum moves only when a score is more than 2^8 times above it:
    // weights of up to 2^8 are as exact as those of up to 1, and the
    // accumulators are seldom scaled.
    if (__any(mx > m_run + 8.f)) {
      const float mn = mx > m_run + 8.f ? mx : m_run;   // (m_run -infinity: nothing seen yet)
      const float al = mn == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - mn);
      m_run = mn;
      l_run *= al;
#pragma unroll
      for (int d = 0; d < NO; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= al;
    }
    const float mb = !FULL && m_run == -INFINITY ? 0.f : m_run;
    // Weights of 16 positions at a time, each of the products beside a pair of
    // the next ones' weights.
    u32x4_t pb[2][PN], vf[2][NO];
    float ls[4] = {0.f, 0.f, 0.f, 0.f};
    auto pair = [&](int u, int i) KV8_INLINE {   // positions 16 u + 8 hi + 2 i, + 1
      float a = __builtin_amdgcn_exp2f(__builtin_fmaf(sa[u >> 1][8 * (u & 1) + 2 * i], sc, -mb));
      float b = __builtin_amdgcn_exp2f(__builtin_fmaf(sa[u >> 1][8 * (u & 1) + 2 * i + 1], sc, -mb));
      if constexpr (PN > 1) ls[i] += a + b;
#pragma unroll
      for (int p = 0; p < PN; ++p) {
        const uint32_t w2 = kv8_pk(a, b);
        pb[u & 1][p][i] = w2;
        if constexpr (PN > 1) {
          a -= bf16lo(w2);
          b -= bf16hi(w2);
        }
      }
      // (the sum is that of the weights as they are used)
      if constexpr (PN == 1) ls[i] = kv8_add2(pb[u & 1][0][i], ls[i]);
    };
    auto values = [&](int u, int d) KV8_INLINE { return *(const u32x4_t*)&S.v[buf][vo[u ^ 2 * (d & 1)] + 32 * d * kManyTile]; };
#pragma unroll
    for (int d = 0; d < NO; ++d) vf[0][d] = values(0, d);
#pragma unroll
    for (int i = 0; i < 4; ++i) pair(0, i);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if (d < NO) {
#pragma unroll
          for (int p = PN - 1; p >= 0; --p) acc[d] = kv8_mma32(vf[u & 1][d], pb[u & 1][p], acc[d]);
          if (u < 3) vf[(u + 1) & 1][d] = values(u + 1, d);
        }
        if (u < 3) pair(u + 1, d);
        __builtin_amdgcn_sched_barrier(0);
      }
    l_run += (ls[0] + ls[1]) + (ls[2] + ls[3]);
    if constexpr (!FULL) {
      // NaN values, which the products took as zero, for the columns that see them
      for (unsigned long long odd = S.odd[tt & 3]; odd; odd &= odd - 1) {
        const int p = __ffsll(odd) - 1;
        if (p < lim) {
#pragma unroll
          for (int d = 0; d < NO; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
              const uint32_t bits = S.nan[buf][p][4 * d + (r >> 2)] >> (4 * hi);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if ((bits >> i) & 1) acc[d][r + i] = __uint_as_float(0x7fc00000u);
            }
        }
      }
    }
  };
  int tt = 0;
  const int nfull = gaps ? 0 : min(ntile, max(0, (least_all - w.t0) / kManyTile));
  auto advance = [&]() KV8_INLINE {
    if (tt + 1 < ntile) {
      stage(tt + 1, ra);
      fetch(tt + 2, id, ra);
      id = ask(tt + 3);
      __syncthreads();   // the other buffer is staged; its readers passed the last barrier
    }
  };
  if (any) {
    for (; tt + 1 < nfull; ++tt) {
      compute(tt, std::true_type{}, std::true_type{});
      __syncthreads();   // (as above)
    }
    for (; tt < ntile; ++tt) {
      if (w.t0 + tt * kManyTile < most) compute(tt, std::false_type{}, std::false_type{});
      advance();
    }
  } else {
    for (; tt < ntile; ++tt) advance();
  }
  // ---- results -----------------------------------------------------------------------
  // the own key, once
  if (A.own && w.split == 0) {
    const int o = live ? A.own[row] : -1;
    if (o >= A.n_own && hi == 0) kv8_error(A.err, KV8_ERR_ROWS);
    const bool has = o >= 0 && o < A.n_own;
    float z = 0.f;
    const int oo = has ? o : 0;
#pragma unroll 4
    for (int d = 0; d < HD / 2; ++d) {
      const int dd = hi * (HD / 2) + d;
      z += kv8_elem<BF>(A.q, (int64_t)row * A.q_row + (int64_t)head * A.q_head + dd) *
           kv8_elem<BF>(A.own_k, (int64_t)oo * A.ok_row + (int64_t)h * A.ok_head + dd);
    }
    z = kv8_sum32(z) * sc;
    if (!has) z = -INFINITY;
    const float mn = fmaxf(m_run, z), mb = mn == -INFINITY ? 0.f : mn;
    const float al = __builtin_amdgcn_exp2f(m_run - mb), p = has ? __builtin_amdgcn_exp2f(z - mb) : 0.f;
    m_run = mn;
    l_run = l_run * al + (hi == 0 ? p : 0.f);
#pragma unroll
    for (int d = 0; d < NO; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int dim = 32 * d + 8 * (r >> 2) + 4 * hi + (r & 3);
        acc[d][r] *= al;
        if (has) acc[d][r] += p * kv8_elem<BF>(A.own_v, (int64_t)oo * A.ov_row + (int64_t)h * A.ov_head + dim);
      }
  }
  const float l_all = kv8_sum32(l_run);
  auto put = [&](int d, int r, float a, float b, float e, float f) KV8_INLINE {   // four dims of the lane's column
    const int64_t to = (int64_t)row * A.out_row + (int64_t)head * A.out_head + 32 * d + 8 * (r >> 2) + 4 * hi;
    if constexpr (BF) *(u32x2_t*)((uint16_t*)A.out + to) = u32x2_t{kv8_pk(a, b), kv8_pk(e, f)};
    else *(float4*)((float*)A.out + to) = make_float4(a, b, e, f);
  };
  if (w.splits == 1) {
    if (!live) return;
    const float li = l_all != 0.f ? 1.f / l_all : 0.f;
#pragma unroll
    for (int d = 0; d < NO; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        put(d, r, l_all != 0.f ? acc[d][r] * li : 0.f, l_all != 0.f ? acc[d][r + 1] * li : 0.f,
            l_all != 0.f ? acc[d][r + 2] * li : 0.f, l_all != 0.f ? acc[d][r + 3] * li : 0.f);
    return;
  }
  // Partial results as the lanes hold them (k8_join): of each wave the
  // accumulators, 16 bytes a lane, then the maximum and sum of its columns.
  if (!any) return;
  float* p = A.part + ((int64_t)(w.slot + w.split) * A.kv.H + h) * kv8_part_floats(kManyCols, HD);
#pragma unroll
  for (int d = 0; d < NO; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *(float4*)(p + ((wv * NO + d) * 4 + (r >> 2)) * 256 + 4 * lane) =
          make_float4(acc[d][r], acc[d][r + 1], acc[d][r + 2], acc[d][r + 3]);
  if (hi == 0) *(float2*)(p + kManyCols * HD + 2 * (32 * wv + n)) = make_float2(m_run, l_all);
}

// Joins the splits of tiles, in a launch of its own: the workgroups of a tile's
// splits share its results among them (a last workgroup that took them all, as
// k8_few's does, needed 1.5 us for each split's 64 KB).
template <int BF, int HD>
__global__ __launch_bounds__(kManyThreads) void k8_join(Kv8AttnArgs A) {
  constexpr int NO = HD / 32, NCH = 4 * NO;   // 1 KB pieces of a partial result per wave: 4 dims of each half of 32 columns
  __shared__ float y_s[kKv8MaxSplits][kManyCols], l_s[kManyCols];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hi = lane >> 5;
  const int h = blockIdx.x % A.kv.H, entry = blockIdx.x / A.kv.H;
  Kv8Work w;
  if (!kv8_pick<kManyCols>(A, entry, false, w) || w.splits == 1) return;
  const int pf = kv8_part_floats(kManyCols, HD);
  const float* part = A.part + ((int64_t)w.slot * A.kv.H + h) * pf;
  const int64_t pstep = (int64_t)A.kv.H * pf;
  const int c0 = w.tile * kManyCols, live = min(kManyCols, w.cols - c0);
  const int groups = (live + 31) / 32;   // of 32 columns
  if (tid < 32 * groups) {
    float M = -INFINITY, l = 0.f;
    constexpr int KEEP = 8;   // splits whose maxima and sums are read once
    float2 keep[KEEP];
    auto at = [&](int x) { return *(const float2*)(part + x * pstep + kManyCols * HD + 2 * tid); };
#pragma unroll
    for (int x = 0; x < KEEP; ++x) keep[x] = at(min(x, w.splits - 1));
#pragma unroll
    for (int x = 0; x < KEEP; ++x) M = fmaxf(M, keep[x].x);
#pragma unroll 8
    for (int x = KEEP; x < w.splits; ++x) M = fmaxf(M, at(x).x);
    auto weigh = [&](int x, float2 t) {
      const float y = kv8_weight(t.x, t.y, M);
      y_s[x][tid] = y;
      if (t.y != 0.f) l += y * t.y;
    };
#pragma unroll
    for (int x = 0; x < KEEP; ++x)
      if (x < w.splits) weigh(x, keep[x]);
#pragma unroll 4
    for (int x = KEEP; x < w.splits; ++x) weigh(x, at(x));
    l_s[tid] = l;
  }
  __syncthreads();
  const int all = groups * NCH, from = all * w.split / w.splits, to = all * (w.split + 1) / w.splits;
  // Four pieces of a wave at a time, so that a few splits keep enough loads in
  // flight (130 rows behind 870 positions 26.1 -> 22.4 us); one where there is no more.
  auto join = [&](auto pieces) KV8_INLINE {
    constexpr int NP = decltype(pieces)::value, UN = NP > 1 ? 4 : 8;
    for (int first = from + wv; first < to; first += 4 * NP) {
      float4 a[NP];
      int ch[NP], col[NP];
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        a[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        ch[k] = min(first + 4 * k, to - 1);
        col[k] = 32 * (ch[k] / NCH) + n;
      }
#pragma unroll UN
      for (int x = 0; x < w.splits; ++x) {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
          const float4 v = *(const float4*)(part + x * pstep + ch[k] * 256 + 4 * lane);
          const float y = y_s[x][col[k]];   // (zero, times zeros, for a split that the column saw nothing of)
          a[k].x += y * v.x;
          a[k].y += y * v.y;
          a[k].z += y * v.z;
          a[k].w += y * v.w;
        }
      }
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        if (first + 4 * k >= to || col[k] >= live) continue;
        const int c = col[k], d = ch[k] % NCH / 4, r4 = ch[k] % 4;
        const float l = l_s[c];
        const int row = w.r0 + (c0 + c) / A.group, head = h * A.group + (c0 + c) % A.group;
        const int64_t o = (int64_t)row * A.out_row + (int64_t)head * A.out_head + 32 * d + 8 * r4 + 4 * hi;
        const float4 z = make_float4(kv8_over(a[k].x, l), kv8_over(a[k].y, l), kv8_over(a[k].z, l), kv8_over(a[k].w, l));
        if constexpr (BF) *(u32x2_t*)((uint16_t*)A.out + o) = u32x2_t{kv8_pk(z.x, z.y), kv8_pk(z.z, z.w)};
        else *(float4*)((float*)A.out + o) = z;
      }
    }
  };
  if (to - from > 4) join(std::integral_constant<int, 4>{});
  else join(std::integral_constant<int, 1>{});
}

#undef KV8_INLINE

}  // namespace m2r2
