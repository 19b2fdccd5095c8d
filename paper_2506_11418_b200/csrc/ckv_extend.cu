// Attention of a chunk of new tokens over a paged cache (bf16 or four-bit pages): ckv_extend_attn_paged, ckv_extend_attn_quantized.
#include <algorithm>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_decode.cuh"
#include "ckv_internal.h"
#include "ckv_ptx.cuh"

#include <cuda_fp16.h>

namespace ckv {
namespace {

constexpr int kED = 128;

struct ExtendArgs {
  const ckv_paged_view* views;
  const int64_t* q_begin;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const __nv_bfloat16* k_pages;
  const __nv_bfloat16* v_pages;
  ckv_quant_pool pool;
  const float* logdeg;
  int64_t n_rows, q_row, q_head;  // strides in elements
  int32_t Bz, H, G, shift;
  float scale;
  int32_t* status;
};

__device__ __forceinline__ float4 level4(uint32_t two_bytes, float s) {
  uint32_t h[4];
  ptx::unpack_e2m1x8(two_bytes, h);
  auto f = [](uint32_t x) { return __half2float(__ushort_as_half((unsigned short)x)); };
  return make_float4(f(h[0]) * s, f(h[0] >> 16) * s, f(h[1]) * s, f(h[1] >> 16) * s);
}

// One warp per (new token, query head), a lane has four columns; online softmax over the token's slots.
template <bool QUANT>
__global__ void __launch_bounds__(256) extend_simple_kernel(const ExtendArgs a) {
  griddep_wait();
  griddep_launch();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
  const int lane = threadIdx.x & 31, HG = a.H * a.G;
  const int64_t at = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)), row = at / HG;
  const int j = (int)(at - row * HG), h = j / a.G;
  if (row >= a.n_rows) return;
  int lo = 0, hi = a.Bz;
  if (row >= a.q_begin[a.Bz] || row < a.q_begin[0]) return;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.q_begin[mid] <= row) lo = mid; else hi = mid;
  }
  const ckv_paged_view view = a.views[lo];
  const int64_t end = view.len - (a.q_begin[lo + 1] - row) + 1;
  const float4 q = load4(a.q + row * a.q_row + j * a.q_head + 4 * lane);
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int64_t t = 0; t < end; ++t) {
    const int64_t r = (((int64_t)view.block_table[t >> a.shift] * a.H + h) << a.shift) + (t & (((int64_t)1 << a.shift) - 1));
    float4 k, v;
    if (QUANT) {
      const int jj = lane >> 3, u = lane & 7;
      const uint32_t kc = *reinterpret_cast<const uint32_t*>(a.pool.k_codes + r * 64 + 16 * (u >> 1) + 4 * jj) >> (16 * (u & 1));
      const uint32_t vc = *reinterpret_cast<const uint32_t*>(a.pool.v_codes + r * 64 + 8 * u + 4 * (jj >> 1)) >> (16 * (jj & 1));
      k = level4(kc, exp2f((float)a.pool.k_scales[r * 4 + jj] - 127.f));
      v = level4(vc, exp2f((float)a.pool.v_scales[r * 4 + jj] - 127.f));
    } else {
      k = load4(a.k_pages + r * kED + 4 * lane);
      v = load4(a.v_pages + r * kED + 4 * lane);
    }
    const float s = warp_sum(q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w) * a.scale + (a.logdeg ? a.logdeg[r] : 0.f);
    const float mm = fmaxf(m, s), base = mm == -INFINITY ? 0.f : mm;
    const float c = exp2f((m - base) * kLog2e), p = exp2f((s - base) * kLog2e);
    o = make_float4(o.x * c + p * v.x, o.y * c + p * v.y, o.z * c + p * v.z, o.w * c + p * v.w);
    l = l * c + p;
    m = mm;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store4(a.out + (row * HG + j) * kED + 4 * lane, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
}

int check_extend(const void* views, const void* q_begin, int64_t n_rows, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D, int32_t dtype,
                 const void* q, int64_t q_row, int64_t q_head, const void* out, const void* workspace, size_t workspace_bytes) {
  if (!views || !q_begin || !q || !out || n_rows < 0 || Bz <= 0 || H <= 0 || G <= 0 || q_row < 0 || q_head < 0) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_BF16 || page_shift(page_tokens) < 0 || D != kED || G > 8 || H > 8192 || Bz > 65535 || n_rows > INT32_MAX / (H * G))
    return CKV_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(out) || q_row % 8 || q_head % 8) return CKV_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < ckv_extend_workspace_bytes(n_rows, H, G, D) || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  return CKV_OK;
}

template <bool QUANT>
int run_extend(ExtendArgs& a, cudaStream_t st) {
  if (a.n_rows == 0) return CKV_OK;
  const int64_t ctas = (a.n_rows * a.H * a.G + 7) / 8;
  return launch_dependent(extend_simple_kernel<QUANT>, dim3((unsigned)ctas), dim3(256), 0, st, a) == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t ckv_extend_workspace_bytes(int64_t n_rows, int32_t H, int32_t G, int32_t D) {
  if (n_rows < 0 || H <= 0 || G <= 0 || D <= 0) return 0;
  return 256;
}

int ckv_extend_attn_paged(const ckv_paged_view* views_dev, const int64_t* q_begin, int64_t n_rows, const void* k_pages, const void* v_pages,
                          const float* logdeg_pages, int64_t n_pages, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D,
                          int32_t dtype, const void* q, int64_t q_row_stride, int64_t q_head_stride, void* out, float scale, void* workspace,
                          size_t workspace_bytes, void* cuda_stream) {
  if (!k_pages || !v_pages || n_pages <= 0) return CKV_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || (logdeg_pages && !aligned16(logdeg_pages))) return CKV_ERR_ALIGNMENT;
  const int st = check_extend(views_dev, q_begin, n_rows, page_tokens, Bz, H, G, D, dtype, q, q_row_stride, q_head_stride, out, workspace, workspace_bytes);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (n_pages > (INT32_MAX >> shift) / H) return CKV_ERR_UNSUPPORTED;  // (2^31 rows of a pool: 1 TB)
  ExtendArgs a{};
  a.views = views_dev; a.q_begin = q_begin; a.n_rows = n_rows; a.Bz = Bz; a.H = H; a.G = G; a.shift = shift; a.scale = scale;
  a.q = static_cast<const __nv_bfloat16*>(q); a.out = static_cast<__nv_bfloat16*>(out); a.q_row = q_row_stride; a.q_head = q_head_stride; a.status = static_cast<int32_t*>(workspace);
  a.k_pages = static_cast<const __nv_bfloat16*>(k_pages); a.v_pages = static_cast<const __nv_bfloat16*>(v_pages); a.logdeg = logdeg_pages;
  return run_extend<false>(a, static_cast<cudaStream_t>(cuda_stream));
}

int ckv_extend_attn_quantized(const ckv_paged_view* views_dev, const int64_t* q_begin, int64_t n_rows, const ckv_quant_pool* pool, int64_t n_pages,
                              int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D, int32_t dtype, const void* q, int64_t q_row_stride,
                              int64_t q_head_stride, void* out, float scale, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!pool || !pool->k_codes || !pool->v_codes || !pool->k_scales || !pool->v_scales || n_pages <= 0) return CKV_ERR_INVALID_ARG;
  if (!aligned16(pool->k_codes) || !aligned16(pool->v_codes) || !aligned16(pool->k_scales) || !aligned16(pool->v_scales) ||
      (pool->logdeg_pages && !aligned16(pool->logdeg_pages)))
    return CKV_ERR_ALIGNMENT;
  const int st = check_extend(views_dev, q_begin, n_rows, page_tokens, Bz, H, G, D, dtype, q, q_row_stride, q_head_stride, out, workspace, workspace_bytes);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (n_pages > (INT32_MAX >> shift) / H) return CKV_ERR_UNSUPPORTED;
  ExtendArgs a{};
  a.views = views_dev; a.q_begin = q_begin; a.n_rows = n_rows; a.Bz = Bz; a.H = H; a.G = G; a.shift = shift; a.scale = scale;
  a.q = static_cast<const __nv_bfloat16*>(q); a.out = static_cast<__nv_bfloat16*>(out); a.q_row = q_row_stride; a.q_head = q_head_stride; a.status = static_cast<int32_t*>(workspace);
  a.pool = *pool; a.logdeg = pool->logdeg_pages;
  return run_extend<true>(a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
