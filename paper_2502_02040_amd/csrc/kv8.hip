// Host side of the 8-bit cache's operators (include/m2r2_kv8.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "kv8_append.h"
#include "kv8_cut.h"
#include "kv8_few.h"
#include "kv8_many.h"
#include "m2r2_kv8.h"
#include "status.h"

using namespace m2r2;

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

m2r2_status check_pages(const m2r2_kv8* kv, int32_t n_seqs) {
  if (!kv || !kv->k_pages || !kv->v_pages || !kv->k_scales || !kv->v_scales || (!kv->block_table_d && n_seqs))
    return set_error(M2R2_E_INVALID, "kv descriptor or one of its pointers is NULL");
  if (!aligned(kv->k_pages, 16) || !aligned(kv->v_pages, 16))
    return set_error(M2R2_E_INVALID, "kv pages not 16-byte aligned");
  if (!aligned(kv->k_scales, 4) || !aligned(kv->v_scales, 4) || !aligned(kv->block_table_d, 4))
    return set_error(M2R2_E_INVALID, "kv scales or block table not 4-byte aligned");
  if (kv->block_size < kKv8Slab || kv->block_size > 256 || kv->block_size % kKv8Slab)
    return set_error(M2R2_E_SHAPE, "block_size %d not a multiple of 16 in [16,256]", kv->block_size);
  if (kv->head_dim != 64 && kv->head_dim != 96 && kv->head_dim != 128)
    return set_error(M2R2_E_UNSUPPORTED, "head_dim %d (supported: 64, 96, 128)", kv->head_dim);
  if (kv->num_blocks < 1 || kv->max_blocks_per_seq < 1 || kv->n_kv_heads < 1)
    return set_error(M2R2_E_SHAPE, "kv sizes");
  if (kv->n_kv_heads > 4096) return set_error(M2R2_E_SHAPE, "n_kv_heads %d above 4096", kv->n_kv_heads);
  // rows of the pool are numbered in 32 bits, positions of a sequence too
  if ((long long)kv->num_blocks * kv->n_kv_heads * kv->block_size >= 1LL << 31)
    return set_error(M2R2_E_SHAPE, "num_blocks * n_kv_heads * block_size reaches 2^31");
  if ((long long)kv->max_blocks_per_seq * kv->block_size >= 1LL << 30)
    return set_error(M2R2_E_SHAPE, "max_blocks_per_seq * block_size reaches 2^30");
  return M2R2_OK;
}

m2r2_status check_counts(int32_t n_seqs, int32_t n_rows) {
  if (n_seqs < 0 || n_rows < 0 || n_seqs > 1 << 20 || n_rows > 1 << 26)
    return set_error(M2R2_E_SHAPE, "n_seqs %d, n_rows %d", n_seqs, n_rows);
  return M2R2_OK;
}

m2r2_status check_rows(int32_t n_seqs, int32_t n_rows, const int32_t* row_start, int32_t dtype) {
  if (m2r2_status s = check_counts(n_seqs, n_rows)) return s;
  if (!row_start || !aligned(row_start, 4)) return set_error(M2R2_E_INVALID, "row_start_d NULL or misaligned");
  if (dtype != M2R2_F32 && dtype != M2R2_BF16) return set_error(M2R2_E_DTYPE, "dtype %d", dtype);
  return M2R2_OK;
}

// (the stride of a dimension of one entry does not count)
m2r2_status check_array(const char* name, const void* p, int n, int heads, int64_t row, int64_t head, int32_t dtype) {
  if (!n) return M2R2_OK;
  if (!p) return set_error(M2R2_E_INVALID, "%s is NULL", name);
  const int64_t per = dtype == M2R2_BF16 ? 8 : 4;
  if (!aligned(p, 16) || (n > 1 && row % per) || (heads > 1 && head % per))
    return set_error(M2R2_E_INVALID, "%s: a row or head does not start on 16 bytes", name);
  const int64_t most = 1LL << 36;
  if ((n > 1 && (row < 0 || row > most)) || (heads > 1 && (head < 0 || head > most)))
    return set_error(M2R2_E_SHAPE, "%s: stride negative or above 2^36", name);
  return M2R2_OK;
}

// One that is written: its rows of heads, or its heads of rows, lie apart.
m2r2_status check_written(const char* name, const void* p, int n, int heads, int64_t row, int64_t head, int hd,
                          int32_t dtype) {
  if (m2r2_status s = check_array(name, p, n, heads, row, head, dtype)) return s;
  if (!n) return M2R2_OK;
  const bool by_row = (heads < 2 || head >= hd) && (n < 2 || row >= (heads < 2 ? 0 : (heads - 1) * head) + hd);
  const bool by_head = (n < 2 || row >= hd) && (heads < 2 || head >= (n < 2 ? 0 : (n - 1) * row) + hd);
  return by_row || by_head ? M2R2_OK : set_error(M2R2_E_INVALID, "%s: rows and heads overlap", name);
}

m2r2_status check_heads(const m2r2_kv8* kv, int32_t n_heads) {
  if (n_heads < 1 || n_heads % kv->n_kv_heads || n_heads > 65536)
    return set_error(M2R2_E_SHAPE, "n_heads %d not a multiple of n_kv_heads %d", n_heads, kv->n_kv_heads);
  return M2R2_OK;
}

Kv8Pages pages(const m2r2_kv8* kv) {
  return Kv8Pages{(uint8_t*)kv->k_pages, (uint8_t*)kv->v_pages, kv->k_scales, kv->v_scales, kv->block_table_d,
                  kv->num_blocks, kv->block_size, kv->max_blocks_per_seq, kv->n_kv_heads};
}

m2r2_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? M2R2_OK : set_error(M2R2_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

template <int BF, int HD>
void append_launch(const Kv8AppArgs& A, hipStream_t st) {
  const long long units = (long long)kv8_block_base(A.n_rows, A.n_seqs, A.kv.bs) * A.units;
  if (A.kv.bs == 16) k8_append<BF, HD, 1, 1><<<(unsigned)((units + 3) / 4), kKv8AppThreads, 0, st>>>(A);
  else if (A.kv.bs <= 64) k8_append<BF, HD, 4, 1><<<(unsigned)units, kKv8AppThreads, 0, st>>>(A);
  else if (A.kv.bs <= 128) k8_append<BF, HD, 4, 2><<<(unsigned)units, kKv8AppThreads, 0, st>>>(A);
  else k8_append<BF, HD, 4, 4><<<(unsigned)units, kKv8AppThreads, 0, st>>>(A);
}

template <int BF, int HD>
void few_launch(const Kv8AttnArgs& A, hipStream_t st) {
  k8_few<BF, HD><<<(unsigned)(A.entries * A.kv.H), kFewThreads, 0, st>>>(A, Kv8Out<BF, HD>{});
}

// A launch has fewer than 2^32 threads along x.
constexpr long long kMaxGrid = 1 << 24;
constexpr int kMaxDevices = 64;

template <int BF, int HD>
hipError_t many_setup() {   // LDS above 64 KB, once per device
  static std::atomic<bool> done[kMaxDevices];
  int dev = 0;
  if (hipError_t e = hipGetDevice(&dev)) return e;
  if (dev >= 0 && dev < kMaxDevices && done[dev].load(std::memory_order_acquire)) return hipSuccess;
  const hipError_t e = hipFuncSetAttribute((const void*)&k8_many<BF, HD>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)sizeof(Kv8ManyLds<HD>));
  if (e == hipSuccess && dev >= 0 && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
  return e;
}

template <int BF, int HD>
void many_launch(const Kv8AttnArgs& A, hipStream_t st, hipError_t* e) {
  *e = many_setup<BF, HD>();
  if (*e != hipSuccess) return;
  const unsigned grid = (unsigned)(A.entries * A.kv.H);
  k8_many<BF, HD><<<grid, kManyThreads, sizeof(Kv8ManyLds<HD>), st>>>(A);
  if ((long long)A.kv.mbps * A.kv.bs > kKv8Whole) k8_join<BF, HD><<<grid, kManyThreads, 0, st>>>(A);
}

#define M2R2_KV8_DISPATCH(FN, BFV, HDV, ...)                 \
  do {                                                       \
    if (BFV) {                                               \
      if ((HDV) == 64) FN<1, 64>(__VA_ARGS__);               \
      else if ((HDV) == 96) FN<1, 96>(__VA_ARGS__);          \
      else FN<1, 128>(__VA_ARGS__);                          \
    } else {                                                 \
      if ((HDV) == 64) FN<0, 64>(__VA_ARGS__);               \
      else if ((HDV) == 96) FN<0, 96>(__VA_ARGS__);          \
      else FN<0, 128>(__VA_ARGS__);                          \
    }                                                        \
  } while (0)

}  // namespace

extern "C" {

M2R2_API m2r2_status m2r2_kv8_append(const m2r2_kv8* kv, const m2r2_kv8_rows* r, hipStream_t stream) {
  if (!r) return set_error(M2R2_E_INVALID, "rows descriptor is NULL");
  if (m2r2_status s = check_pages(kv, r->n_seqs)) return s;
  if (m2r2_status s = check_rows(r->n_seqs, r->n_rows, r->row_start_d, r->dtype)) return s;
  if ((!r->positions_d && r->n_seqs) || !aligned(r->positions_d, 4)) return set_error(M2R2_E_INVALID, "positions_d NULL or misaligned");
  if (m2r2_status s = check_array("k", r->k, r->n_rows, kv->n_kv_heads, r->k_row, r->k_head, r->dtype)) return s;
  if (m2r2_status s = check_array("v", r->v, r->n_rows, kv->n_kv_heads, r->v_row, r->v_head, r->dtype)) return s;
  if (r->rope_d && (!aligned(r->rope_d, 16) || r->rope_len < 1))
    return set_error(M2R2_E_INVALID, "rope_d not 16-byte aligned, or rope_len %d", r->rope_len);
  if (r->n_heads) {
    if (m2r2_status s = check_heads(kv, r->n_heads)) return s;
    if (m2r2_status s = check_array("q", r->q, r->n_rows, r->n_heads, r->q_row, r->q_head, r->dtype)) return s;
    if (m2r2_status s = check_written("q_out", r->q_out, r->n_rows, r->n_heads, r->qo_row, r->qo_head, kv->head_dim,
                                      r->dtype))
      return s;
    if (r->q == r->q_out &&
        ((r->n_rows > 1 && r->q_row != r->qo_row) || (r->n_heads > 1 && r->q_head != r->qo_head)))
      return set_error(M2R2_E_INVALID, "q_out is q with other strides");
  } else if (r->q || r->q_out) {
    return set_error(M2R2_E_INVALID, "q or q_out given with n_heads 0");
  }
  if (r->err_d && !aligned(r->err_d, 4)) return set_error(M2R2_E_INVALID, "err_d misaligned");
  Kv8AppArgs A{};
  A.kv = pages(kv);
  A.n_seqs = r->n_seqs; A.n_rows = r->n_rows; A.row_start = r->row_start_d; A.positions = r->positions_d;
  A.k = r->k; A.v = r->v; A.q = r->q; A.qo = r->q_out;
  A.k_row = r->k_row; A.k_head = r->k_head; A.v_row = r->v_row; A.v_head = r->v_head;
  A.q_row = r->q_row; A.q_head = r->q_head; A.qo_row = r->qo_row; A.qo_head = r->qo_head;
  A.rope = r->rope_d; A.rope_len = r->rope_len; A.n_heads = r->n_heads; A.err = r->err_d;
  A.units = kv->n_kv_heads + (r->n_heads + kKv8QHeads - 1) / kKv8QHeads;
  if (!r->n_seqs || !r->n_rows) return M2R2_OK;
  if ((long long)kv8_block_base(r->n_rows, r->n_seqs, kv->block_size) * A.units >= kMaxGrid)
    return set_error(M2R2_E_SHAPE, "too many rows and heads for one call");
  M2R2_KV8_DISPATCH(append_launch, r->dtype == M2R2_BF16, kv->head_dim, A, stream);
  return launched("m2r2_kv8_append");
}

M2R2_API m2r2_status m2r2_kv8_workspace_size(const m2r2_kv8* kv, int32_t n_seqs, int32_t n_rows, int32_t n_heads,
                                             size_t* bytes_out) {
  if (m2r2_status s = check_counts(n_seqs, n_rows)) return s;
  if (m2r2_status s = check_pages(kv, n_seqs)) return s;
  if (m2r2_status s = check_heads(kv, n_heads)) return s;
  if (!bytes_out) return set_error(M2R2_E_INVALID, "bytes_out is NULL");
  if ((long long)n_rows * n_heads >= 1LL << 31) return set_error(M2R2_E_SHAPE, "n_rows * n_heads reaches 2^31");
  *bytes_out = 0;
  for (int bf16 = 0; bf16 < 2; ++bf16) {
    const Kv8Cut c = kv8_cut(pages(kv), kv->head_dim, n_seqs, n_rows, n_heads, bf16);
    if (c.entries * kv->n_kv_heads >= kMaxGrid) return set_error(M2R2_E_SHAPE, "too many rows and heads for one call");
    *bytes_out = std::max(*bytes_out, c.bytes);
  }
  return M2R2_OK;
}

M2R2_API m2r2_status m2r2_kv8_attention(const m2r2_kv8* kv, const m2r2_kv8_query* a, void* workspace, size_t ws_bytes,
                                        hipStream_t stream) {
  if (!a) return set_error(M2R2_E_INVALID, "query descriptor is NULL");
  if (m2r2_status s = check_pages(kv, a->n_seqs)) return s;
  if (m2r2_status s = check_rows(a->n_seqs, a->n_rows, a->row_start_d, a->dtype)) return s;
  if ((!a->lens_d && a->n_seqs) || !aligned(a->lens_d, 4)) return set_error(M2R2_E_INVALID, "lens_d NULL or misaligned");
  if (!aligned(a->visible_d, 4) || !aligned(a->own_d, 4) || !aligned(a->err_d, 4))
    return set_error(M2R2_E_INVALID, "visible_d, own_d or err_d misaligned");
  if (m2r2_status s = check_heads(kv, a->n_heads)) return s;
  size_t need = 0;
  if (m2r2_status s = m2r2_kv8_workspace_size(kv, a->n_seqs, a->n_rows, a->n_heads, &need)) return s;
  if (m2r2_status s = check_array("q", a->q, a->n_rows, a->n_heads, a->q_row, a->q_head, a->dtype)) return s;
  if (m2r2_status s = check_written("out", a->out, a->n_rows, a->n_heads, a->out_row, a->out_head, kv->head_dim,
                                    a->dtype))
    return s;
  if (a->own_d) {
    if (a->n_own < 1) return set_error(M2R2_E_SHAPE, "n_own %d", a->n_own);
    const int H = kv->n_kv_heads;
    if (m2r2_status s = check_array("own_k", a->own_k, a->n_own, H, a->ok_row, a->ok_head, a->dtype)) return s;
    if (m2r2_status s = check_array("own_v", a->own_v, a->n_own, H, a->ov_row, a->ov_head, a->dtype)) return s;
  }
  if (!(a->scale >= 0.f) || a->scale > 3e38f) return set_error(M2R2_E_INVALID, "scale");
  if (!workspace || !aligned(workspace, 256)) return set_error(M2R2_E_INVALID, "workspace NULL or not 256-byte aligned");
  if (ws_bytes < need) return set_error(M2R2_E_NOMEM, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (!a->n_seqs || !a->n_rows) return M2R2_OK;
  Kv8AttnArgs A{};
  A.kv = pages(kv);
  A.n_seqs = a->n_seqs; A.n_rows = a->n_rows; A.n_heads = a->n_heads;
  A.row_start = a->row_start_d; A.lens = a->lens_d; A.visible = a->visible_d; A.own = a->own_d;
  A.q = a->q; A.own_k = a->own_k; A.own_v = a->own_v; A.out = a->out;
  A.q_row = a->q_row; A.q_head = a->q_head; A.ok_row = a->ok_row; A.ok_head = a->ok_head;
  A.ov_row = a->ov_row; A.ov_head = a->ov_head; A.out_row = a->out_row; A.out_head = a->out_head;
  A.n_own = a->own_d ? a->n_own : 0;
  A.scale = a->scale > 0.f ? a->scale : 1.f / sqrtf((float)kv->head_dim);
  A.err = a->err_d;
  A.group = a->n_heads / kv->n_kv_heads;
  const Kv8Cut c = kv8_cut(A.kv, kv->head_dim, a->n_seqs, a->n_rows, a->n_heads, a->dtype == M2R2_BF16);
  kv8_cut_args(A, c, workspace);
  if (c.many) {
    hipError_t e = hipSuccess;
    M2R2_KV8_DISPATCH(many_launch, a->dtype == M2R2_BF16, kv->head_dim, A, stream, &e);
    if (e != hipSuccess) return set_error(M2R2_E_HIP, "m2r2_kv8_attention: %s", hipGetErrorString(e));
  } else {
    M2R2_KV8_DISPATCH(few_launch, a->dtype == M2R2_BF16, kv->head_dim, A, stream);
  }
  return launched("m2r2_kv8_attention");
}

}  // extern "C"
