// Choosing the pages that a query attends to.  A page is treated as one cluster: its mean key c = sum n_t k_t / sum n_t
// and degree N = sum n_t.  By Jensen's inequality log sum_t n_t exp(q k_t) >= log N + q c, so q c * scale + log N is a
// lower bound of (and for keys that resemble each other close to) the page's share of Eq. 3's denominator, from 260
// bytes in place of the page's 64 KB of keys and values (256 + 4 of 64 * 516 B at 64 tokens).
#include <algorithm>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_internal.h"
#include "ckv_ptx.cuh"

namespace ckv {
namespace {

// ---- ckv_pages_summarize -----------------------------------------------------------------------------------------
// One CTA of four warps per (page, head); half a warp takes a key row (16 bytes per lane), so eight rows are in flight
// per step, and the partial sums meet in shared memory.  Bound by reading the keys once.
constexpr int kSumThreads = 128;

struct SummarizeArgs {
  const ckv_paged_view* views;
  const int64_t* from_lens;  // null: from the first block
  const uint4* k_pages;
  const int32_t* deg_pages;  // null: all ones
  __nv_bfloat16* c_pages;
  float* clog_pages;
  int64_t max_blocks;
  int32_t H, shift;
};

__global__ void __launch_bounds__(kSumThreads) pages_summarize_kernel(const SummarizeArgs a) {
  __shared__ float s_acc[4][128];
  __shared__ long long s_n[4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = lane & 15, r0 = warp * 2 + (lane >> 4);
  const int h = blockIdx.y, b = blockIdx.z;
  griddep_wait();
  griddep_launch();
  const ckv_paged_view view = a.views[b];
  const int64_t first = a.from_lens ? max(a.from_lens[b], (int64_t)0) >> a.shift : 0;
  for (int64_t x = blockIdx.x; x < a.max_blocks; x += gridDim.x) {
    const int64_t blk = first + x, left = view.len - (blk << a.shift);
    if (left <= 0) break;
    const int rows = (int)min(left, (int64_t)1 << a.shift);
    const int64_t ph = (int64_t)view.block_table[blk] * a.H + h, row = ph << a.shift;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    long long total = 0;
#pragma unroll 8
    for (int r = r0; r < rows; r += 8) {
      const uint4 u = a.k_pages[(row + r) * 16 + c];
      const int dg = a.deg_pages ? a.deg_pages[row + r] : 1;
      const float w = (float)dg;
      total += dg;
      const uint32_t p[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        acc[2 * i] = fmaf(w, __uint_as_float(p[i] << 16), acc[2 * i]);
        acc[2 * i + 1] = fmaf(w, __uint_as_float(p[i] & 0xffff0000u), acc[2 * i + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 16);
    total += __shfl_xor_sync(0xffffffffu, total, 16);
    if (lane < 16) {
      *reinterpret_cast<float4*>(&s_acc[warp][c * 8]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(&s_acc[warp][c * 8 + 4]) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (lane == 0) s_n[warp] = total;
    }
    __syncthreads();
    const float n = (float)(s_n[0] + s_n[1] + s_n[2] + s_n[3]);
    const float s = (s_acc[0][tid] + s_acc[1][tid]) + (s_acc[2][tid] + s_acc[3][tid]);
    a.c_pages[ph * 128 + tid] = __float2bfloat16_rn(s / n);
    if (tid == 0) a.clog_pages[ph] = logf(n);
    __syncthreads();  // the sums are read before the next block's overwrite them
  }
}

// ---- ckv_pages_select --------------------------------------------------------------------------------------------
// One thread-block cluster of CL CTAs per (sequence, KV head).  Scores are exact to the last bits of 64: products of
// bf16 are exact in it, and a choice between near pages then does not hang on the order of a 32-bit sum (with 32 bits
// about one selection in a thousand would).  A summary row is read once by half a warp, eight elements per lane, for
// all G query heads; the scores of all CTAs land as order-preserving 64-bit keys in the first CTA's shared memory,
// which finds the k-th largest by counting digits of eight bits, from the top of the range that the keys span, and
// writes the chosen blocks in ascending order.
constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelHalves = 2 * kSelWarps;      // summary rows in work at once per CTA
constexpr uint64_t kForced = ~0ull;            // key of a block that is always chosen; no score maps to it
constexpr int kSelMaxBlocks = 24576;           // 192 KB of keys

struct SelectPagesArgs {
  const ckv_paged_view* views;
  const uint4* c_pages;
  const float* clog_pages;  // null: zeros
  const __nv_bfloat16* q;
  int32_t* selected;
  int64_t max_blocks;
  float scale;
  int32_t H, shift, n_first, n_last, n_select;
};

// ascending in the score; NaN lowest, the two zeros equal
__device__ __forceinline__ uint64_t score_key(double s) {
  if (isnan(s)) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ void st_cluster_u64(uint32_t local_addr, uint32_t rank, uint64_t v) {
  uint32_t ra;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(local_addr), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(ra), "l"(v) : "memory");
}

template <int G, int CL>
__global__ void __launch_bounds__(kSelThreads, 1) pages_select_kernel(const SelectPagesArgs a) {
  extern __shared__ __align__(16) uint64_t keys[];
  __shared__ uint32_t s_hist[256];
  __shared__ uint64_t s_lo[kSelWarps], s_hi[kSelWarps];
  __shared__ int s_gt[kSelWarps], s_eq[kSelWarps], s_bin, s_above, s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  griddep_wait();
  griddep_launch();
  const ckv_paged_view view = a.views[b];
  const int64_t mask = ((int64_t)1 << a.shift) - 1;
  const int n = (int)max((int64_t)0, min((view.len + mask) >> a.shift, a.max_blocks));
  int32_t* out = a.selected + ((int64_t)b * a.H + h) * a.n_select;
  if (n <= a.n_select) {  // every block is chosen
    if (rank == 0)
      for (int i = tid; i < a.n_select; i += kSelThreads) out[i] = i < n ? i : -1;
    return;  // (the whole cluster leaves: the condition is the sequence's)
  }
  if (CL > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  // ---- scores
  {
    const int c = lane & 15, half = 2 * warp + (lane >> 4);
    double q[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint4 u = reinterpret_cast<const uint4*>(a.q + (((int64_t)b * a.H + h) * G + g) * 128)[c];
      const uint32_t p[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        q[g][2 * i] = (double)__uint_as_float(p[i] << 16);
        q[g][2 * i + 1] = (double)__uint_as_float(p[i] & 0xffff0000u);
      }
    }
    const uint32_t keys_s = (uint32_t)__cvta_generic_to_shared(keys);
    if (CL > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // the first CTA has started: its keys can be written
    constexpr int kStep = kSelHalves * CL;
    const int i0 = rank * kSelHalves + half;
    // sixteen blocks at a time: lane c holds the page of the c-th
    for (int base = 0; base < n; base += 16 * kStep) {
      const int mine = base + i0 + c * kStep;
      const int page = mine < n ? view.block_table[mine] : 0;
      for (int u0 = 0; u0 < 16 && base + u0 * kStep < n; u0 += 4) {
        uint4 rows[4];
        int64_t ph[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          ph[u] = (int64_t)__shfl_sync(0xffffffffu, page, u0 + u, 16) * a.H + h;
          rows[u] = a.c_pages[ph[u] * 16 + c];  // (a block past the end reads page 0's row and is dropped below)
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t p[4] = {rows[u].x, rows[u].y, rows[u].z, rows[u].w};
          double acc[G];
#pragma unroll
          for (int g = 0; g < G; ++g) acc[g] = 0.0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const double x = (double)__uint_as_float(p[i] << 16), y = (double)__uint_as_float(p[i] & 0xffff0000u);
#pragma unroll
            for (int g = 0; g < G; ++g) acc[g] = fma(x, q[g][2 * i], fma(y, q[g][2 * i + 1], acc[g]));
          }
#pragma unroll
          for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int g = 0; g < G; ++g) acc[g] += __shfl_xor_sync(0xffffffffu, acc[g], o);
          const int i = base + i0 + (u0 + u) * kStep;
          if (c == 0 && i < n) {
            double best = acc[0] * (double)a.scale;
#pragma unroll
            for (int g = 1; g < G; ++g) {
              const double s = acc[g] * (double)a.scale;
              if (s > best || isnan(s)) best = s;  // (a NaN stays)
            }
            if (a.clog_pages) best += (double)a.clog_pages[ph[u]];
            const bool always = i < a.n_first || i >= n - a.n_last;
            const uint64_t key = always ? kForced : score_key(best);
            if (CL == 1)
              keys[i] = key;
            else
              st_cluster_u64(keys_s + 8u * (uint32_t)i, 0, key);
          }
        }
      }
    }
  }
  if (CL > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // ---- the range of the scores, and how many are to be found among them
  uint64_t lo = kForced, hi = 0;
  int forced = 0;
  for (int i = tid; i < n; i += kSelThreads) {
    const uint64_t k = keys[i];
    if (k == kForced) {
      ++forced;
    } else {
      lo = min(lo, k);
      hi = max(hi, k);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    forced += __shfl_xor_sync(0xffffffffu, forced, o);
  }
  if (lane == 0) {
    s_lo[warp] = lo;
    s_hi[warp] = hi;
    s_gt[warp] = forced;
  }
  __syncthreads();
  forced = 0;
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) {
    lo = min(lo, s_lo[w]);
    hi = max(hi, s_hi[w]);
    forced += s_gt[w];
  }
  // chosen: keys above `edge`, and the first `ties` of those equal to it
  int need = a.n_select - forced, ties = 0;
  uint64_t edge = hi;  // need == 0: only the forced ones
  if (need > 0) {
    // digits of (key - lo), eight bits at a time from the top bit of the span
    uint64_t prefix = 0;
    int bits = hi > lo ? 64 - __clzll((long long)(hi - lo)) : 0;  // bits still open below the prefix
    bool all = false;
    while (bits > 0 && !all) {
      const int take = min(bits, 8), low = bits - take;
      s_hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kSelThreads) {
        const uint64_t k = keys[i];
        if (k == kForced) continue;
        const uint64_t d = k - lo;
        if (bits == 64 || (d >> bits) == prefix) atomicAdd(&s_hist[(uint32_t)(d >> low) & ((1u << take) - 1u)], 1u);
      }
      __syncthreads();
      if (warp == 0) {  // lane l sums digits 8 l .. 8 l + 7; suffix sums from the top digit down
        uint32_t cnt[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += cnt[j] = s_hist[8 * lane + j];
        uint32_t above = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_down_sync(0xffffffffu, above, o);
          if (lane + o < 32) above += y;
        }
        above -= sum;  // keys in the digits of higher lanes
        if ((int)above < need && (int)(above + sum) >= need) {
#pragma unroll
          for (int j = 7; j >= 0; --j) {
            if ((int)above < need && (int)(above + cnt[j]) >= need) {
              s_bin = 8 * lane + j;
              s_above = (int)above;
              s_count = (int)cnt[j];
            }
            above += cnt[j];
          }
        }
      }
      __syncthreads();
      prefix = (prefix << take) | (uint64_t)s_bin;
      need -= s_above;
      bits = low;
      all = s_count == need;  // the whole digit is chosen: no need to open it further
      __syncthreads();
    }
    const uint64_t least = lo + (bits > 0 ? prefix << bits : prefix);  // the smallest key of the digit
    if (all) {
      edge = least - 1;  // (fewer than all are chosen, so some key lies below: least is not 0)
    } else {
      edge = least;
      ties = need;
    }
  }
  // ---- the chosen blocks in ascending order: every thread takes a run of consecutive blocks
  const int per = (n + kSelThreads - 1) / kSelThreads, c0 = min(n, tid * per), c1 = min(n, c0 + per);
  int gt = 0, eq = 0;
  for (int i = c0; i < c1; ++i) {
    const uint64_t k = keys[i];
    gt += k > edge;
    eq += k == edge;
  }
  int gt_at = gt, eq_at = eq;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, gt_at, o), y = __shfl_up_sync(0xffffffffu, eq_at, o);
    if (lane >= o) {
      gt_at += x;
      eq_at += y;
    }
  }
  __syncthreads();  // (s_gt was read above)
  if (lane == 31) {
    s_gt[warp] = gt_at;
    s_eq[warp] = eq_at;
  }
  __syncthreads();
  gt_at -= gt;
  eq_at -= eq;
  for (int w = 0; w < warp; ++w) {
    gt_at += s_gt[w];
    eq_at += s_eq[w];
  }
  for (int i = c0; i < c1; ++i) {
    const uint64_t k = keys[i];
    if (k > edge) {
      out[gt_at + min(eq_at, ties)] = i;
      ++gt_at;
    } else if (k == edge) {
      if (eq_at < ties) out[gt_at + eq_at] = i;
      ++eq_at;
    }
  }
}

template <int G, int CL>
cudaError_t launch_pages_select(const SelectPagesArgs& a, int32_t Bz, cudaStream_t st) {
  const size_t smem = (size_t)a.max_blocks * 8;
  cudaError_t e = cudaFuncSetAttribute(pages_select_kernel<G, CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelMaxBlocks * 8);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(CL, (unsigned)a.H, (unsigned)Bz);
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, pages_select_kernel<G, CL>, a);
}

template <int G>
cudaError_t launch_pages_select_g(const SelectPagesArgs& a, int32_t Bz, cudaStream_t st) {
  // the scores are split over a cluster while that leaves every CTA 64 blocks to score and the SMs are not all taken
  const int64_t pairs = (int64_t)Bz * a.H, sms = sm_count();
  if (a.max_blocks >= 512 && pairs * 8 <= 2 * sms) return launch_pages_select<G, 8>(a, Bz, st);
  if (a.max_blocks >= 128 && pairs * 2 <= 2 * sms) return launch_pages_select<G, 2>(a, Bz, st);
  return launch_pages_select<G, 1>(a, Bz, st);
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

int ckv_pages_summarize(const ckv_paged_view* views_dev, const int64_t* from_lens, int32_t Bz, const void* k_pages, const int32_t* deg_pages,
                        int32_t page_tokens, int32_t H, int32_t D, int32_t dtype, int64_t max_blocks, void* c_pages, float* clog_pages,
                        void* cuda_stream) {
  if (!views_dev || !k_pages || !c_pages || !clog_pages || Bz <= 0 || H <= 0 || max_blocks < 0) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  const int shift = page_shift(page_tokens);
  if (dtype != CKV_BF16 || shift < 0 || D != 128 || H > 65535 || Bz > 65535) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(k_pages) || !aligned16(c_pages)) return CKV_ERR_ALIGNMENT;
  if (max_blocks == 0) return CKV_OK;
  SummarizeArgs a{};
  a.views = views_dev; a.from_lens = from_lens; a.k_pages = static_cast<const uint4*>(k_pages); a.deg_pages = deg_pages;
  a.c_pages = static_cast<__nv_bfloat16*>(c_pages); a.clog_pages = clog_pages;
  a.max_blocks = max_blocks; a.H = H; a.shift = shift;
  const dim3 grid((unsigned)std::min<int64_t>(max_blocks, 65535), (unsigned)H, (unsigned)Bz);
  return launch_dependent(pages_summarize_kernel, grid, dim3(kSumThreads), 0, static_cast<cudaStream_t>(cuda_stream), a) == cudaSuccess
             ? CKV_OK : CKV_ERR_CUDA;
}

int ckv_pages_select(const ckv_paged_view* views_dev, const void* c_pages, const float* clog_pages, int32_t page_tokens, int32_t Bz, int32_t H,
                     int32_t G, int32_t D, int32_t dtype, const void* q, float scale, int64_t max_len, int32_t n_first, int32_t n_last,
                     int32_t n_select, int32_t* selected, void* cuda_stream) {
  if (!views_dev || !c_pages || !q || !selected || Bz <= 0 || H <= 0 || G <= 0 || max_len < 0 || n_first < 0 || n_last < 0 || n_select <= 0 ||
      (int64_t)n_first + n_last > n_select)
    return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  const int shift = page_shift(page_tokens);
  if (dtype != CKV_BF16 || shift < 0 || D != 128 || G > 8 || H > 65535 || Bz > 65535) return CKV_ERR_UNSUPPORTED;
  const int64_t max_blocks = max_len / page_tokens + (max_len % page_tokens ? 1 : 0);
  if (max_blocks > kSelMaxBlocks) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(c_pages) || !aligned16(q)) return CKV_ERR_ALIGNMENT;
  SelectPagesArgs a{};
  a.views = views_dev; a.c_pages = static_cast<const uint4*>(c_pages); a.clog_pages = clog_pages;
  a.q = static_cast<const __nv_bfloat16*>(q); a.selected = selected;
  a.max_blocks = max_blocks; a.scale = scale; a.H = H; a.shift = shift;
  a.n_first = n_first; a.n_last = n_last; a.n_select = n_select;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaErrorInvalidValue;
  switch (G) {
    case 1: e = launch_pages_select_g<1>(a, Bz, st); break;
    case 2: e = launch_pages_select_g<2>(a, Bz, st); break;
    case 3: e = launch_pages_select_g<3>(a, Bz, st); break;
    case 4: e = launch_pages_select_g<4>(a, Bz, st); break;
    case 5: e = launch_pages_select_g<5>(a, Bz, st); break;
    case 6: e = launch_pages_select_g<6>(a, Bz, st); break;
    case 7: e = launch_pages_select_g<7>(a, Bz, st); break;
    case 8: e = launch_pages_select_g<8>(a, Bz, st); break;
  }
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // extern "C"
