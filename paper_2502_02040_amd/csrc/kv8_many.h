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

template <int HD>
struct Kv8ManyLds {
  static constexpr int KP = HD + 8;           // padded rows (elements): 16 lanes' 16 bytes hit all banks
  static constexpr int VP = kManyTile + 8;
  uint16_t k[2][kManyTile * KP];              // [position][dim]
  uint16_t v[2][HD * VP];                     // [dim][position]
  // of a tile (four in turn): positions outside the pool; positions with NaN
  // values, of a tile that not all columns see whole, and which dims' they are
  unsigned long long gap[4], odd[4];
  uint8_t nan[2][kManyTile][HD / 8];
  int last;
};

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
  constexpr int KP = L::KP, VP = L::VP;
  constexpr int NK = HD / 32;                // 8-byte pieces of keys per thread: positions 4 threads each
  constexpr int ND = HD / 8;                 // groups of 8 dims: values are staged by 16 ND threads
  extern __shared__ __attribute__((aligned(16))) char lds_raw[];
  L& S = *(L*)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hi = lane >> 5;
  const int h = blockIdx.x % A.kv.H, entry = blockIdx.x / A.kv.H;
  Kv8Work w;
  if (!kv8_pick<kManyCols>(A, entry, blockIdx.x == 0 && wv == 0, w)) return;
  const int c0 = w.tile * kManyCols, c = c0 + 32 * wv + n;
  const bool live = c < w.cols;
  const int cc = min(c, w.cols - 1);
  const int row = w.r0 + cc / A.group, head = h * A.group + cc % A.group;
  const int sees = kv8_sees(A, w, c);
  // of the wave's columns, and of the workgroup's (a tile's 128 columns: every thread looks at all)
  int most = sees, most_all = 0, least_all = 1 << 30;
#pragma unroll
  for (int x = 0; x < kManyCols / 64; ++x) {
    const int o = c0 + 64 * x + lane, v = kv8_sees(A, w, o);
    most_all = max(most_all, v);
    least_all = min(least_all, o < w.cols ? v : 1 << 30);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    most = max(most, __shfl_xor(most, d));
    most_all = max(most_all, __shfl_xor(most_all, d));
    least_all = min(least_all, __shfl_xor(least_all, d));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  most_all = __builtin_amdgcn_readfirstlane(most_all);
  least_all = __builtin_amdgcn_readfirstlane(least_all);
  const int t1 = min(w.t1, most_all);
  const int ntile = t1 > w.t0 ? (t1 - w.t0 + kManyTile - 1) / kManyTile : 0;
  const float sc = A.scale * kLog2e;

  // ---- staging ------------------------------------------------------------------
  // keys: thread (position tid / 4, part tid % 4) takes HD / 4 bytes; values:
  // thread (positions 4 (tid % 16) .., dims 8 (tid / 16) ..) takes 4 x 8 bytes
  const int kt = tid >> 2, kd = (tid & 3) * (HD / 4), vt = (tid & 15) * 4, vd = (tid >> 4) * 8;
  struct Raw {
    u32x2_t k[NK], v[4];
    float ks, vs;
    bool kok, vok;   // the place exists
  };
  // block ids of a tile, requested a tile before its codes
  struct Ids {
    int k, v, kin, vin;   // block, position in it
  };
  const int* bt = A.kv.bt + (int64_t)w.s * A.kv.mbps;
  auto ask = [&](int tt) {
    const int t = w.t0 + tt * kManyTile;
    Ids id;
    auto slot = [&](int tp, int& in) {   // logical block (the last one where the table ends)
      const uint32_t lb = (uint32_t)(((uint64_t)((uint32_t)tp >> 4) * A.bs_magic) >> 31);
      in = tp - (int)lb * A.kv.bs;
      return min((int)lb, A.kv.mbps - 1);
    };
    id.k = bt[slot(t + kt, id.kin)];
    id.v = bt[slot(t + vt, id.vin)];
    return id;
  };
  const uint32_t page = A.kv.H * A.kv.bs * HD;   // bytes of a block
  const uint8_t* kb = A.kv.k + (int64_t)h * A.kv.bs * HD + kd;
  const uint8_t* vb = A.kv.v + (int64_t)h * A.kv.bs * HD + min(vd, HD - 8);
  auto fetch = [&](const Ids& id, Raw& r) {
    r.kok = (uint32_t)id.k < (uint32_t)A.kv.nb;
    r.vok = (uint32_t)id.v < (uint32_t)A.kv.nb;
    const uint32_t bk = r.kok ? id.k : 0, bv = r.vok ? id.v : 0;
    r.ks = A.kv.ks[bk * A.kv.H + h];
    r.vs = A.kv.vs[bv * A.kv.H + h];
    const uint8_t* kp = kb + (uint64_t)bk * page + id.kin * HD;
#pragma unroll
    for (int x = 0; x < NK; ++x) r.k[x] = kv8_ld<u32x2_t>(kp + 8 * x);
    const uint8_t* vp = vb + (uint64_t)bv * page + id.vin * HD;
#pragma unroll
    for (int x = 0; x < 4; ++x) r.v[x] = kv8_ld<u32x2_t>(vp + x * HD);
  };
  auto stage = [&](int tt, Raw& r, int buf) {
    const int t = w.t0 + tt * kManyTile;
    if (tid == 0) {   // marks that were last read two tiles ago
      S.gap[(tt + 2) & 3] = 0;
      S.odd[(tt + 2) & 3] = 0;
    }
    if (!r.kok) {
      atomicOr(&S.gap[tt & 3], 1ull << kt);
      if (t + kt < t1) kv8_error(A.err, KV8_ERR_BLOCK);
    }
#pragma unroll
    for (int x = 0; x < NK; ++x) {
      const u32x4_t o = {kv8_up<false>(r.k[x][0], r.ks), kv8_up<true>(r.k[x][0], r.ks), kv8_up<false>(r.k[x][1], r.ks),
                         kv8_up<true>(r.k[x][1], r.ks)};
      *(u32x4_t*)&S.k[buf][kt * KP + kd + 8 * x] = o;
    }
    if (vd < HD) {
      if (t + kManyTile > least_all || !r.vok) {
        // what no column sees is zero in the products, and so is NaN, which must
        // not reach the columns that do not see it
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const bool there = t + vt + x < t1 && r.vok;
          uint32_t bits = 0;
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const uint32_t nan = there ? kv8_nan_bytes(r.v[x][z]) : 0u;
            r.v[x][z] = there ? r.v[x][z] & ~nan : 0u;
            bits |= ((nan & 1) | (nan >> 7 & 2) | (nan >> 14 & 4) | (nan >> 21 & 8)) << (4 * z);
          }
          S.nan[buf][vt + x][vd / 8] = bits;
          if (bits) atomicOr(&S.odd[tt & 3], 1ull << (vt + x));
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t o[4][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t a = __builtin_amdgcn_perm(r.v[2 * i + 1][x], r.v[2 * i][x], 0x05010400u);
          const uint32_t b = __builtin_amdgcn_perm(r.v[2 * i + 1][x], r.v[2 * i][x], 0x07030602u);
          o[0][i] = kv8_up<false>(a, r.vs);
          o[1][i] = kv8_up<true>(a, r.vs);
          o[2][i] = kv8_up<false>(b, r.vs);
          o[3][i] = kv8_up<true>(b, r.vs);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) *(u32x2_t*)&S.v[buf][(vd + 4 * x + d) * VP + vt] = u32x2_t{o[d][0], o[d][1]};
      }
    }
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
  }
  __syncthreads();
  Raw ra;
  Ids id{};
  if (ntile > 0) {
    const Ids i0 = ask(0), i1 = ask(1);
    fetch(i0, ra);
    stage(0, ra, 0);
    fetch(i1, ra);   // (beyond the last tile: some position's block, staged nowhere)
    id = ask(2);
  }
  __syncthreads();
  // row m of a product is this position of its 32
  const int krow = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  // FULL: every live column of the workgroup sees all of the tile, and it is all there
  auto compute = [&](int tt, auto full) {
    constexpr bool FULL = decltype(full)::value;
    const int buf = tt & 1, t0 = w.t0 + tt * kManyTile;
    f32x16_t sa[2];
#pragma unroll
    for (int s = 0; s < NQ; ++s) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const u32x4_t k = *(const u32x4_t*)&S.k[buf][(32 * x + krow) * KP + 16 * s + 8 * hi];
#pragma unroll
        for (int p = QN - 1; p >= 0; --p)
          sa[x] = s == 0 && p == QN - 1 ? kv8_mma32(k, q[s][p], f32x16_t{}) : kv8_mma32(k, q[s][p], sa[x]);
      }
    }
    // keys are read ahead of the products, or every product waits for the LDS
    if constexpr (BF) {
      constexpr int AHEAD = 6;
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
      for (int i = 0; i < 2 * NQ - AHEAD; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, AHEAD, 0);
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
    u32x4_t pb[4][PN];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sa[u >> 1][8 * (u & 1) + i], sc, -mb));
      kv8_parts<PN>(p, pb[u]);
      // the sum is that of the weights as they are used
      if constexpr (PN == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) l_run = kv8_add2(pb[u][0][i], l_run);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) l_run += p[i];
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int d = 0; d < NO; ++d) {
        const u32x4_t v = *(const u32x4_t*)&S.v[buf][(32 * d + n) * VP + 16 * u + 8 * hi];
#pragma unroll
        for (int p = PN - 1; p >= 0; --p) acc[d] = kv8_mma32(v, pb[u][p], acc[d]);
      }
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
  auto advance = [&](int tt) {   // tile tt + 1 into the other buffer, whose readers passed the last barrier
    if (tt + 1 < ntile) {
      stage(tt + 1, ra, (tt + 1) & 1);
      fetch(id, ra);   // (as above)
      id = ask(tt + 3);
      __syncthreads();
    }
  };
  int tt = 0;
  const int nfull = min(ntile, max(0, (least_all - w.t0) / kManyTile));
  for (; tt < nfull && !S.gap[tt & 3]; ++tt) {
    compute(tt, std::true_type{});
    advance(tt);
  }
  for (; tt < ntile; ++tt) {
    if (w.t0 + tt * kManyTile < most) compute(tt, std::false_type{});
    advance(tt);
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
  auto put = [&](int d, int r, float a, float b, float e, float f) {   // four dims of the lane's column
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
  // Partial results as the lanes hold them: of each wave the accumulators, 16
  // bytes a lane, then the maximum and sum of its columns.
  const int pf = kv8_part_floats(kManyCols, HD);
  float* part = A.part + ((int64_t)w.slot * A.kv.H + h) * pf;
  const int64_t pstep = (int64_t)A.kv.H * pf;
  const int mine = wv * 32 * HD, ml = kManyCols * HD + 2 * (32 * wv + n);
  {
    float* p = part + (int64_t)w.split * pstep;
#pragma unroll
    for (int d = 0; d < NO; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float* o = p + mine + ((4 * d + (r >> 2)) * 64 + lane) * 4;
        st_agent2(o, acc[d][r], acc[d][r + 1]);
        st_agent2(o + 2, acc[d][r + 2], acc[d][r + 3]);
      }
    if (hi == 0) st_agent2(p + ml, m_run, l_all);
  }
  if (!arrive_last(A.cnt + w.unit * A.kv.H + h, w.splits, &S.last)) return;
  float M = -INFINITY, l = 0.f;
  for (int x = 0; x < w.splits; ++x) M = fmaxf(M, ld_agent(part + (int64_t)x * pstep + ml));
#pragma unroll
  for (int d = 0; d < NO; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  for (int x = 0; x < w.splits; ++x) {
    const float* p = part + (int64_t)x * pstep;
    const float lx = ld_agent(p + ml + 1), y = kv8_weight(ld_agent(p + ml), lx, M);
    float2 v[NO][8];
#pragma unroll
    for (int d = 0; d < NO; ++d)
#pragma unroll
      for (int r = 0; r < 8; ++r) v[d][r] = ld_agent2(p + mine + ((4 * d + (r >> 1)) * 64 + lane) * 4 + 2 * (r & 1));
    if (lx != 0.f) {
      l += y * lx;
#pragma unroll
      for (int d = 0; d < NO; ++d)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          acc[d][2 * r] += y * v[d][r].x;
          acc[d][2 * r + 1] += y * v[d][r].y;
        }
    }
  }
  if (!live) return;
#pragma unroll
  for (int d = 0; d < NO; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      put(d, r, kv8_over(acc[d][r], l), kv8_over(acc[d][r + 1], l), kv8_over(acc[d][r + 2], l), kv8_over(acc[d][r + 3], l));
}

}  // namespace m2r2
