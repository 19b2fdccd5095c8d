// Token rows that go into pages through a slot map: what ckv_pages_write and ckv_pages_quantize share.
#pragma once

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_internal.h"

namespace ckv {

struct RowsIn {
  const void* k;
  const void* v;
  const int32_t* deg;               // null: all ones
  int64_t k_token, k_head, v_token, v_head;  // strides in pieces of 16 bytes
  int64_t deg_token, deg_head;
  int32_t H;
};

inline RowsIn rows_in(const ckv_token_rows& r) {
  const int per = 16 / (r.dtype == CKV_F32 ? 4 : 2);
  return RowsIn{r.k, r.v, r.deg, r.k_token_stride / per, r.k_head_stride / per, r.v_token_stride / per, r.v_head_stride / per,
                r.deg_token_stride, r.deg_head_stride, r.H};
}

inline int check_rows(const ckv_token_rows* r, const int64_t* slots, int64_t n, int64_t n_pages, int32_t page_tokens) {
  if (!r || n < 0 || (n > 0 && (!slots || !r->k || !r->v)) || n_pages <= 0 || r->H <= 0) return CKV_ERR_INVALID_ARG;
  if (r->dtype != CKV_F32 && r->dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  if (r->k_token_stride < 0 || r->k_head_stride < 0 || r->v_token_stride < 0 || r->v_head_stride < 0 || r->deg_token_stride < 0 ||
      r->deg_head_stride < 0)
    return CKV_ERR_INVALID_ARG;
  if (page_shift(page_tokens) < 0 || r->D != 128 || r->H > 65535 || n > INT32_MAX || n_pages > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const int per = 16 / (r->dtype == CKV_F32 ? 4 : 2);
  if (!aligned16(r->k) || !aligned16(r->v)) return CKV_ERR_ALIGNMENT;
  // (a stride over a single token or head is never used)
  if (n > 1 && (r->k_token_stride % per || r->v_token_stride % per)) return CKV_ERR_ALIGNMENT;
  if (r->H > 1 && (r->k_head_stride % per || r->v_head_stride % per)) return CKV_ERR_ALIGNMENT;
  return CKV_OK;
}

// degrees and their logarithms of tokens i0 .. i0 + count - 1 of one head: one token per thread
__device__ __forceinline__ void write_degrees(const RowsIn& r, const int64_t* slots, int64_t n, int64_t i0, int count, int h, int32_t* deg_pages,
                                              float* logdeg_pages, int64_t n_rows, int32_t shift) {
  const int64_t mask = ((int64_t)1 << shift) - 1;
  for (int64_t i = i0 + threadIdx.x; i < min(n, i0 + count); i += blockDim.x) {
    const int64_t s = slots[i];
    if (s < 0 || s >= n_rows) continue;
    const int64_t row = (((s >> shift) * r.H + h) << shift) + (s & mask);
    const int dg = r.deg ? r.deg[i * r.deg_token + h * r.deg_head] : 1;
    if (deg_pages) deg_pages[row] = dg;
    if (logdeg_pages) logdeg_pages[row] = logf((float)dg);
  }
}

}  // namespace ckv
