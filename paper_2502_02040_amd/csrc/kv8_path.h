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

template <int WB, int HD>
__global__ __launch_bounds__(256) void k8_rows(Dims D, LayerPtrs L, RowMap rm, WS ws, StepIO io, KVPtrs kv, int layer,
                                               Kv8Path P) {
  constexpr int NC = HD / 16, HALF = HD / 2;       // lanes of a row: 8 dims of each half
  constexpr int NS = (kMaxRows * NC + 63) / 64;
  __shared__ float u_s[3 * kMaxRank];
  const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = D.r, qd = D.qdim, nqkv = 3 * qd + 3 * r;
  int first = rm.first[0], R = rm.cnt[0];
#pragma unroll
  for (int i = 1; i < kMaxSeq; ++i) {
    first = s == i ? (int)rm.first[i] : first;
    R = s == i ? (int)rm.cnt[i] : R;
  }
  const int fast_i = rsel(rm.fast, first + R - 1) ? R - 1 : -1;   // (a fast row is its sequence's last)
  // rows that write the cache: the slow ones, a draft's fast one
  const int nw = fast_i >= 0 && !rsel(rm.wr, first + fast_i) ? R - 1 : R;
  const int pos0 = io.positions[s] + rm.pos_offset;
  const bool frozen = ws.exited[s] != 0;   // an exited sequence only writes its cache entries
  const int cap = kv.mbps * kv.bs;
  if (fast_i >= 0 && tid < 3 * r) u_s[tid] = ws.QKV[(size_t)(first + fast_i) * nqkv + 3 * qd + tid];
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
  __syncthreads();
  // dims d .. d+7 and the same of the upper half of row i: projection w (q, k, v)
  auto form = [&](int w, int i, int d, float (&y)[16]) {
    const float* src = ws.QKV + (size_t)(first + i) * nqkv + w * qd + h * HD + d;
    if ((nqkv & 3) == 0) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float4 f = *(const float4*)(src + (x >> 1) * HALF + 4 * (x & 1));
        y[4 * x] = f.x;
        y[4 * x + 1] = f.y;
        y[4 * x + 2] = f.z;
        y[4 * x + 3] = f.w;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x) y[x] = src[(x >> 3) * HALF + (x & 7)];
    }
    float2 cs[8];
    if (w < 2) {
      int pos = pos0 + (i == fast_i ? 0 : i);   // (a fast row is at the slow one's position)
      if (pos < 0 || pos >= ws.rope_len) {
        atomicOr(ws.err, 8);
        pos = 0;
      }
      const float4* rp = (const float4*)(ws.rope + (size_t)pos * HALF + d);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float4 f = rp[x];
        cs[2 * x] = make_float2(f.x, f.y);
        cs[2 * x + 1] = make_float2(f.z, f.w);
      }
    }
    const void* B = w == 0 ? L.B[0] : (w == 1 ? L.B[1] : L.B[2]);
    const void* Am = w == 0 ? L.A[0] : (w == 1 ? L.A[1] : L.A[2]);
    if (i == fast_i && Am && B) {
#pragma unroll
      for (int x = 0; x < 16; ++x)
        y[x] += dot_row_t<WB>(B, (size_t)h * HD + d + (x >> 3) * HALF + (x & 7), r, u_s + w * r);
    }
    if (w < 2) {
#pragma unroll
      for (int x = 0; x < 8; ++x) kv8_turn(y[x], y[8 + x], cs[x].x, cs[x].y);
    }
  };
  auto keep = [&](float* to, const float (&y)[16]) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(float4*)(to + (x >> 1) * HALF + 4 * (x & 1)) = make_float4(y[4 * x], y[4 * x + 1], y[4 * x + 2], y[4 * x + 3]);
  };
  if (wv == 2) {   // ---- queries ----
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const int ix = t * 64 + lane, i = ix / NC, d = ix % NC * 8;
      if (i >= R) continue;
      float y[16];
      form(0, i, d, y);
      keep(P.q + (size_t)(first + i) * qd + h * HD + d, y);
    }
    return;
  }
  if (wv == 3) {   // ---- the fast row's own key and value ----
    const int w = 1 + lane / NC, d = lane % NC * 8;
    if (fast_i >= 0 && w <= 2) {
      float y[16];
      form(w, fast_i, d, y);
      keep((w == 1 ? P.ok : P.ov) + (size_t)s * qd + h * HD + d, y);
    }
    return;
  }
  // ---- wave 0: keys, wave 1: values, of the rows that write; at most two blocks
  float y[NS][16];
#pragma unroll
  for (int t = 0; t < NS; ++t) {
    const int ix = t * 64 + lane, i = ix / NC;
    if (i < nw) form(1 + wv, i, ix % NC * 8, y[t]);
  }
  if (lane == 0 && (pos0 < 0 || pos0 + nw > cap)) atomicOr(ws.err, 2);
  const int p0 = max(pos0, 0), p1 = min(pos0 + nw, cap);
  if (p0 >= p1) return;
  for (int lb = p0 / kv.bs; lb <= (p1 - 1) / kv.bs; ++lb) {
    const int blk = kv.bt[(int64_t)s * kv.mbps + lb];
    if (blk < 0 || blk >= kv.num_blocks) {
      if (lane == 0) atomicOr(ws.err, 2);
      continue;
    }
    const int64_t page = ((int64_t)layer * kv.num_blocks + blk) * D.H + h;
    uint8_t* base = (uint8_t*)(wv ? kv.v : kv.k) + page * kv.bs * HD;
    float* scale = (wv ? kv.vs : kv.ks) + page;
    const int begin = max(p0, lb * kv.bs), end = min(p1, (lb + 1) * kv.bs), live = begin - lb * kv.bs;
    const int old_e = kv8_exponent(*scale);
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
    if (lane == 0 && (live == 0 || grown)) *scale = kv8_two_to(e);
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
