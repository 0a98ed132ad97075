// The decode path over the 8-bit cache: per layer two launches between the
// q/k/v projections and the o projection.
//
// k8_rows, a workgroup per (head, sequence), forms the head's rows: adapter-up
// of the fast row, rotation; queries and the fast rows' own keys and values go
// to scratch in float32, the rows that write the cache are quantised and
// appended to it (a slow row sees itself as cached, a fast row its exact own
// key).  k8_few (kv8_few.h) then attends and leaves what the o projection reads.
// Separate launches, because a block's scale can grow under the codes that
// other workgroups would be reading.
#pragma once
#include "kv8_append.h"
#include "kv8_few.h"
#include "step_kernels.h"

namespace m2r2 {

// Scratch of a pass, and what k8_few is told about its rows.
struct Kv8Path {
  float *q, *ok, *ov;                          // [16][H hd] rotated queries; [nseq][H hd] own keys and values
  int *row_start, *lens, *visible, *own;       // as m2r2_kv8_query's
};
constexpr int kKv8Meta = kMaxSeq + 1 + kMaxSeq + 2 * kMaxRows;   // ints of the last four

// RMAX: rows of a sequence, at most: 2 (decoding, drafts) or 16 (a chunk of slow
// rows).  A thread forms a pair of dims (j, j + HD / 2) of a row's q, k or v; the
// rows that write meet in LDS, where a wave quantises the keys and one the
// values.  What bounds it is its chain of loads, so everything that does not
// depend on the position is requested with it, and the block's scale with the
// rotation's entries.
template <int WB, int HD, int RMAX>
__global__ __launch_bounds__(256) void k8_rows(Dims D, LayerPtrs L, RowMap rm, WS ws, StepIO io, KVPtrs kv, int layer,
                                               Kv8Path P) {
  constexpr int NC = HD / 16, HALF = HD / 2;       // lanes of a row that is quantised: 8 dims of each half
  constexpr int NS = (RMAX * NC + 63) / 64;
  constexpr int NR = (3 * RMAX * HALF + 255) / 256;   // pairs of a thread
  constexpr bool DUAL = RMAX == 2;                    // the last row may be a fast row
  __shared__ float u_s[3 * kMaxRank];
  __shared__ __attribute__((aligned(16))) float y_s[2][RMAX][HD];   // keys and values of the rows
  const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = D.r, qd = D.qdim, nqkv = 3 * qd + 3 * r;
  int first = rm.first[0], R = rm.cnt[0];
#pragma unroll
  for (int i = 1; i < kMaxSeq; ++i) {
    first = s == i ? (int)rm.first[i] : first;
    R = s == i ? (int)rm.cnt[i] : R;
  }
  const int fast_i = DUAL && rsel(rm.fast, first + R - 1) ? R - 1 : -1;   // (a fast row is its sequence's last)
  // rows that write the cache: the slow ones, a draft's fast one
  const int nw = fast_i >= 0 && !rsel(rm.wr, first + fast_i) ? R - 1 : R;
  // ---- round one: what does not depend on the position -----------------------
  const int posv = io.positions[s];
  const int exv = ws.exited[s];
  const int np = 3 * R * HALF;
  auto place = [&](int e, int& w, int& i, int& j) {   // pair e: projection, row, dim
    w = e / (R * HALF);
    i = e / HALF % R;
    j = e % HALF;
  };
  float pa[NR], pb[NR];
  u32x4_t bq[DUAL ? NR : 1][2][2];
  const bool b16 = WB && DUAL && (r == 8 || r == 16);   // B rows of one or two 16-byte pieces
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    int w, i, j;
    place(min(tid + t * 256, np - 1), w, i, j);
    const float* src = ws.QKV + (size_t)(first + i) * nqkv + w * qd + h * HD + j;
    pa[t] = src[0];
    pb[t] = src[HALF];
    if constexpr (DUAL) {
      const void* B = w == 0 ? L.B[0] : (w == 1 ? L.B[1] : L.B[2]);
      if (b16 && i == fast_i && B) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int k = 0; k < 2; ++k)
            bq[t][x][k] = ((const u32x4_t*)B)[((size_t)h * HD + j + x * HALF) * (r / 8) + min(k, r / 8 - 1)];
      }
    }
  }
  if (DUAL && fast_i >= 0 && tid < 3 * r) u_s[tid] = ws.QKV[(size_t)(first + fast_i) * nqkv + 3 * qd + tid];
  // ---- round two: rotation, the first block's scale ---------------------------
  const int pos0 = posv + rm.pos_offset;
  const bool frozen = exv != 0;   // an exited sequence only writes its cache entries
  const int cap = kv.mbps * kv.bs;
  const int p0 = max(pos0, 0), p1 = min(pos0 + nw, cap);   // positions that are written
  const bool quant = wv < 2 && p0 < p1;                    // wave 0: keys, wave 1: values
  if (tid == 0 && (pos0 < 0 || pos0 + nw > cap)) atomicOr(ws.err, 2);
  int blk = -1, old_e = 0;
  auto block = [&](int lb) { return kv.bt[(int64_t)s * kv.mbps + lb]; };
  auto page = [&]() { return ((int64_t)layer * kv.num_blocks + blk) * D.H + h; };
  auto inside = [&]() { return (uint32_t)blk < (uint32_t)kv.num_blocks; };
  if (quant) blk = block(p0 / kv.bs);
  float2 cs[NR];
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    int w, i, j;
    place(min(tid + t * 256, np - 1), w, i, j);
    int pos = pos0 + (i == fast_i ? 0 : i);   // (a fast row is at the slow one's position)
    if (pos < 0 || pos >= ws.rope_len) {
      if (w < 2) atomicOr(ws.err, 8);
      pos = 0;
    }
    cs[t] = ws.rope[(size_t)pos * HALF + j];
  }
  if (quant && inside()) old_e = kv8_exponent((wv ? kv.vs : kv.ks)[page()]);
  if (h == 0 && tid < R) {
    const int top = min(ws.rope_len, cap);
    const bool fast = tid == fast_i;
    P.visible[first + tid] = frozen ? 0 : min(max(fast ? pos0 : pos0 + tid + 1, 0), top);
    P.own[first + tid] = fast && !frozen ? s : -1;
    if (tid == 0) {
      P.row_start[s] = first;
      P.row_start[s + 1] = first + R;
      P.lens[s] = frozen ? 0 : min(max(fast_i == 0 ? pos0 : pos0 + nw, 0), top);
    }
  }
  if (DUAL && fast_i >= 0) __syncthreads();   // (uniform: u_s)
#pragma unroll
  for (int t = 0; t < NR; ++t) {
    const int e = tid + t * 256;
    if (e >= np) break;
    int w, i, j;
    place(e, w, i, j);
    float a = pa[t], b = pb[t];
    const void* B = w == 0 ? L.B[0] : (w == 1 ? L.B[1] : L.B[2]);
    const void* Am = w == 0 ? L.A[0] : (w == 1 ? L.A[1] : L.A[2]);
    if (DUAL && i == fast_i && Am && B) {
      const float* u = u_s + w * r;
      if (b16) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (8 * k >= r) break;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float u0 = u[8 * k + 2 * x], u1 = u[8 * k + 2 * x + 1];
            a += bf16lo(bq[t][0][k][x]) * u0 + bf16hi(bq[t][0][k][x]) * u1;
            b += bf16lo(bq[t][1][k][x]) * u0 + bf16hi(bq[t][1][k][x]) * u1;
          }
        }
      } else {
        a += dot_row_t<WB>(B, (size_t)h * HD + j, r, u);
        b += dot_row_t<WB>(B, (size_t)h * HD + j + HALF, r, u);
      }
    }
    if (w < 2) kv8_turn(a, b, cs[t].x, cs[t].y);
    if (w == 0) {
      float* q = P.q + (size_t)(first + i) * qd + h * HD + j;
      q[0] = a;
      q[HALF] = b;
      continue;
    }
    if (i < nw) {
      y_s[w - 1][i][j] = a;
      y_s[w - 1][i][j + HALF] = b;
    }
    if (i == fast_i) {   // its own key and value, exact
      float* o = (w == 1 ? P.ok : P.ov) + (size_t)s * qd + h * HD + j;
      o[0] = a;
      o[HALF] = b;
    }
  }
  __syncthreads();
  if (!quant) return;
  // ---- the cache: at most two blocks --------------------------------------------
  float y[NS][16];
#pragma unroll
  for (int t = 0; t < NS; ++t) {
    const int ix = t * 64 + lane, i = min(ix / NC, RMAX - 1);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float4 f = *(const float4*)&y_s[wv][i][ix % NC * 8 + (x >> 1) * HALF + 4 * (x & 1)];
      y[t][4 * x] = f.x;
      y[t][4 * x + 1] = f.y;
      y[t][4 * x + 2] = f.z;
      y[t][4 * x + 3] = f.w;
    }
  }
  for (int lb = p0 / kv.bs; lb <= (p1 - 1) / kv.bs; ++lb) {
    const int begin = max(p0, lb * kv.bs), end = min(p1, (lb + 1) * kv.bs), live = begin - lb * kv.bs;
    if (lb > p0 / kv.bs) blk = block(lb);   // (its rows begin at its first slot: no scale to keep)
    if (!inside()) {
      if (lane == 0) atomicOr(ws.err, 2);
      continue;
    }
    uint8_t* base = (uint8_t*)(wv ? kv.v : kv.k) + page() * kv.bs * HD;
    float most = 0.f;
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const int i = (t * 64 + lane) / NC, p = pos0 + i;
      if (i < nw && p >= begin && p < end) most = fmaxf(most, kv8_most16(y[t]));
    }
    int e = kv8_scale_exponent(wave_max(most));
    if (live > 0) e = max(e, old_e);
    const bool grown = live > 0 && e > old_e;
    if (grown) {
      const float f = kv8_two_to(old_e - e);
      for (int ix = lane; ix < live * NC; ix += 64) {
        uint8_t* c = base + ix / NC * HD + ix % NC * 8;
        kv8_regrow(c, f);
        kv8_regrow(c + HALF, f);
      }
    }
    const float inv = kv8_two_to(-e);
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const int ix = t * 64 + lane, i = ix / NC, p = pos0 + i;
      if (i < nw && p >= begin && p < end) kv8_store16(base + (p - lb * kv.bs) * HD + ix % NC * 8, HALF, y[t], inv);
    }
    if (lane == 0 && (live == 0 || grown)) (wv ? kv.vs : kv.ks)[page()] = kv8_two_to(e);
  }
}

// Results of the path: the o projection's operand, and the o adapter's share of
// the head for fast rows.
template <int WB, int HD>
struct Kv8PathOut {
  static constexpr bool kKeep = true;
  static constexpr int ND = HD / 8, NAO = (kMaxRank * ND + kFewThreads - 1) / kFewThreads;
  Dims D;
  RowMap rm;
  WS ws;
  const void* Ao;   // the o adapter's A, or NULL
  struct Ahead {
    u32x4_t ao[NAO];
  };
  __device__ __forceinline__ void request(Ahead& a, const Kv8AttnArgs&, int h) const {
    if (WB && Ao) {
#pragma unroll
      for (int k = 0; k < NAO; ++k) {
        const int e = min((int)threadIdx.x + k * kFewThreads, D.r * ND - 1);
        a.ao[k] = kv8_ld<u32x4_t>((const uint16_t*)Ao + (size_t)(e / ND) * D.qdim + h * HD + 8 * (e % ND));
      }
    }
  }
  __device__ __forceinline__ void put(const Kv8AttnArgs&, int row, int head, int d, float a, float b) const {
    put_o(D, rm, ws, row, head * HD + d, a);
    put_o(D, rm, ws, row, head * HD + d + 1, b);
  }
  // o: the tile's rows; sums: r * ND floats of LDS
  __device__ __forceinline__ void finish(const Ahead& a, const Kv8AttnArgs& A, const Kv8Work& w, int h, int live,
                                         const float (*o)[HD], float* sums) const {
    const int tid = threadIdx.x, r = D.r;
    const int fast = A.own[w.r0 + live - 1] >= 0 ? live - 1 : -1;
    __syncthreads();
    if (fast >= 0 && Ao) {
#pragma unroll
      for (int k = 0; k < NAO; ++k) {
        const int e = tid + k * kFewThreads;
        if (e >= r * ND) break;
        const float* x = &o[fast][8 * (e % ND)];
        float v = 0.f;
        if constexpr (WB) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v += bf16lo(a.ao[k][i]) * x[2 * i] + bf16hi(a.ao[k][i]) * x[2 * i + 1];
        } else {
          const size_t base = (size_t)(e / ND) * D.qdim + h * HD + 8 * (e % ND);
#pragma unroll
          for (int i = 0; i < 8; ++i) v += ld_wt<WB>(Ao, base + i) * x[i];
        }
        sums[e] = v;
      }
      __syncthreads();
    }
    for (int e = tid; e < live * r; e += kFewThreads) {
      const int i = e / r, j = e % r;
      float v = 0.f;
      if (fast >= 0 && Ao && i == fast)
        for (int c = 0; c < ND; ++c) v += sums[j * ND + c];
      ws.uo[((size_t)(w.r0 + i) * D.H + h) * r + j] = v;
    }
  }
};

}  // namespace m2r2
