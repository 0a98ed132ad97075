// Attention over the 8-bit paged cache: one wave per (row, query head).
#pragma once
#include "kv8.h"

namespace m2r2 {

struct Kv8AttnArgs {
  Kv8Pages kv;
  int n_seqs, n_rows, n_heads;
  const int *row_start, *lens, *visible, *own;
  const void *q, *own_k, *own_v;
  void* out;
  int64_t q_row, q_head, ok_row, ok_head, ov_row, ov_head, out_row, out_head;
  int n_own;
  float scale;
  int* err;
};

template <int BF>
__device__ __forceinline__ float kv8_elem(const void* p, int64_t at) {
  if constexpr (BF) return bf16_to_f32(((const uint16_t*)p)[at]);
  else return ((const float*)p)[at];
}

template <int BF, int HD>
__global__ __launch_bounds__(256) void k8_attn(Kv8AttnArgs A) {
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(w / A.n_heads), h = (int)(w % A.n_heads);
  if (row >= A.n_rows) return;
  const int s = kv8_find(A.n_seqs, row, [&](int i) { return A.row_start[i]; });
  const int r0 = A.row_start[s], r1 = A.row_start[s + 1];
  if (r0 < 0 || r1 < r0 || r1 > A.n_rows) {
    if (lane == 0) kv8_error(A.err, KV8_ERR_ROWS);
    return;
  }
  if (row < r0 || row >= r1) return;
  const int len = A.lens[s];
  const int64_t cap = (int64_t)A.kv.mbps * A.kv.bs;
  if (len > cap && lane == 0) kv8_error(A.err, KV8_ERR_BLOCK);
  const int n = (int)min((int64_t)max(len, 0), cap);
  const int see = min(n, A.visible ? A.visible[row] : len - (r1 - 1 - row));
  const int hk = h / (A.n_heads / A.kv.H);
  const bool on0 = lane < HD, on1 = lane + 64 < HD;
  const int64_t at = (int64_t)row * A.q_row + (int64_t)h * A.q_head + lane;
  const float q0 = on0 ? kv8_elem<BF>(A.q, at) * A.scale : 0.f, q1 = on1 ? kv8_elem<BF>(A.q, at + 64) * A.scale : 0.f;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  auto add = [&](float k0, float k1, float v0, float v1) {
    const float z = wave_sum(q0 * k0 + q1 * k1);
    const float mn = fmaxf(m, z);
    const float al = m == -INFINITY ? 0.f : __expf(m - mn), p = z == -INFINITY ? 0.f : __expf(z - mn);
    m = mn;
    l = l * al + p;
    o0 = o0 * al + p * v0;
    o1 = o1 * al + p * v1;
  };
  for (int t = 0; t < see; ++t) {
    const int lb = t / A.kv.bs, blk = A.kv.bt[(int64_t)s * A.kv.mbps + lb];
    if (blk < 0 || blk >= A.kv.nb) {
      if (lane == 0) kv8_error(A.err, KV8_ERR_BLOCK);
      continue;
    }
    const int64_t page = (int64_t)blk * A.kv.H + hk;
    const int64_t p = (page * A.kv.bs + (t - lb * A.kv.bs)) * HD + lane;
    const float ks = A.kv.ks[page], vs = A.kv.vs[page];
    const float k0 = on0 ? __builtin_amdgcn_cvt_f32_fp8(A.kv.k[p], 0) * ks : 0.f;
    const float k1 = on1 ? __builtin_amdgcn_cvt_f32_fp8(A.kv.k[p + 64], 0) * ks : 0.f;
    const float v0 = on0 ? __builtin_amdgcn_cvt_f32_fp8(A.kv.v[p], 0) * vs : 0.f;
    const float v1 = on1 ? __builtin_amdgcn_cvt_f32_fp8(A.kv.v[p + 64], 0) * vs : 0.f;
    add(k0, k1, v0, v1);
  }
  const int ow = A.own ? A.own[row] : -1;
  if (ow >= A.n_own && lane == 0) kv8_error(A.err, KV8_ERR_ROWS);
  if (ow >= 0 && ow < A.n_own) {
    const int64_t pk = (int64_t)ow * A.ok_row + (int64_t)hk * A.ok_head + lane;
    const int64_t pv = (int64_t)ow * A.ov_row + (int64_t)hk * A.ov_head + lane;
    add(on0 ? kv8_elem<BF>(A.own_k, pk) : 0.f, on1 ? kv8_elem<BF>(A.own_k, pk + 64) : 0.f,
        on0 ? kv8_elem<BF>(A.own_v, pv) : 0.f, on1 ? kv8_elem<BF>(A.own_v, pv + 64) : 0.f);
  }
  const int64_t to = (int64_t)row * A.out_row + (int64_t)h * A.out_head + lane;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  const float a = l != 0.f ? o0 * inv : 0.f, b = l != 0.f ? o1 * inv : 0.f;
  if constexpr (BF) {
    __bf16* out = (__bf16*)A.out;
    if (on0) out[to] = (__bf16)a;
    if (on1) out[to + 64] = (__bf16)b;
  } else {
    float* out = (float*)A.out;
    if (on0) out[to] = a;
    if (on1) out[to + 64] = b;
  }
}

}  // namespace m2r2
