// The paged cache held in 8 bits (include/m2r2_kv8.h): what its kernels share.
#pragma once
#include "device_common.h"

namespace m2r2 {

// One layer's cache.
struct Kv8Pages {
  uint8_t *k, *v;
  float *ks, *vs;
  const int* bt;   // [n_seqs][mbps]
  int nb, bs, mbps, H;
};

enum { KV8_ERR_BLOCK = 2, KV8_ERR_ROPE = 8, KV8_ERR_ROWS = 32 };

constexpr int kKv8MinExp = -120, kKv8MaxExp = 112;
constexpr int kKv8Slab = 16;   // block sizes are multiples of this many tokens

__device__ __forceinline__ void kv8_error(int* err, int bit) {
  if (err) atomicOr(err, bit);
}

// 2^e for e in [-126, 127], 0 below.
__device__ __forceinline__ float kv8_two_to(int e) { return e < -126 ? 0.f : __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponent of a stored scale (whatever it holds, one that a scale can have).
__device__ __forceinline__ int kv8_exponent(float s) {
  return min(max((int)((__float_as_uint(s) >> 23) & 0xff) - 127, kKv8MinExp), kKv8MaxExp);
}

// The least e in range with 448 * 2^e >= amax (finite, >= 0).  448 = 1.75 * 2^8.
__device__ __forceinline__ int kv8_scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);   // (subnormal: below the range)
  return min(max(e, kKv8MinExp), kKv8MaxExp);
}

// The last s in [0, n) with base(s) <= x, for ascending base (s = 0 if there is
// none): every lane looks at one place, 64 ways at a time.
template <class Base>
__device__ __forceinline__ int kv8_find(int n, int x, Base base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, cnt = n;
  while (cnt > 1) {
    const int step = (cnt + 63) / 64;
    const int i = lane * step;
    const bool le = i < cnt && base(lo + min(i, cnt - 1)) <= x;
    const int k = max(1, (int)__popcll(__ballot(le)));
    lo += (k - 1) * step;
    cnt = min(step, cnt - (k - 1) * step);
  }
  return lo;
}

}  // namespace m2r2
