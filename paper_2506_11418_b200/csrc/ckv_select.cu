// Choosing the pages that a query attends to.  A page is treated as one cluster: its mean key c = sum n_t k_t / sum n_t
// and degree N = sum n_t.  By Jensen's inequality log sum_t n_t exp(q k_t) >= log N + q c, so q c * scale + log N is a
// lower bound of (and for keys that resemble each other close to) the page's share of Eq. 3's denominator, from 260
// bytes in place of the 33 KB that 64 tokens' keys, values and log-degrees take.
#include <algorithm>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_internal.h"
#include "ckv_ptx.cuh"

namespace ckv {
namespace {

// ---- ckv_pages_summarize -----------------------------------------------------------------------------------------
// WPH warps per (page, head): one for a prompt's many pages (the eight warps of a CTA take neighbouring heads, and none waits
// for another), four for a step's few (the page's rows are in flight at once; the partial sums meet
// in shared memory).  Half a warp takes a key row, 16 bytes per lane, eight rows in flight per lane.  Bound by reading the
// keys once: 190 MB of a prompt batch in 32.0 us = 0.92 of the measured bandwidth (four warps per page and head: 43 us); the
// last pages of 64 sequences x 8 heads in 3.0 us.
constexpr int kSumThreads = 256;

struct SummarizeArgs {
  const ckv_paged_view* views;
  const int64_t* from_lens;  // null: from the first block; above the length: from the last
  const uint4* k_pages;
  const int32_t* deg_pages;  // null: all ones
  __nv_bfloat16* c_pages;
  float* clog_pages;
  int64_t max_blocks;
  int32_t H, shift;
};

template <int WPH>
__global__ void __launch_bounds__(kSumThreads) pages_summarize_kernel(const SummarizeArgs a) {
  constexpr int kHeads = kSumThreads / 32 / WPH, kRows = 8;
  __shared__ __align__(16) float s_acc[WPH > 1 ? kSumThreads / 32 : 1][128];
  __shared__ long long s_n[kSumThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 15, part = warp % WPH;
  const int64_t unit = (int64_t)blockIdx.x * kHeads + warp / WPH, x = unit / a.H;  // (block, head) of the sequence
  const int h = (int)(unit - x * a.H), b = blockIdx.y;
  griddep_wait();
  griddep_launch();
  const ckv_paged_view view = a.views[b];
  int64_t from = a.from_lens ? a.from_lens[b] : 0;
  if (from > view.len) from = view.len - 1;  // (a sequence that shrank: its last block lost tokens)
  const int64_t blk = (max(from, (int64_t)0) >> a.shift) + x, left = view.len - (blk << a.shift);
  const int rows = x < a.max_blocks && left > 0 ? (int)min(left, (int64_t)1 << a.shift) : 0;
  if (WPH == 1 && rows == 0) return;
  const int64_t ph = rows > 0 ? (int64_t)view.block_table[blk] * a.H + h : 0, row = ph << a.shift;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  long long total = 0;
  for (int r0 = 2 * part + (lane >> 4); r0 < rows; r0 += 2 * WPH * kRows) {
    uint4 u[kRows];
    int dg[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = r0 + 2 * WPH * i;
      const bool ok = r < rows;
      u[i] = ok ? a.k_pages[(row + r) * 16 + c] : make_uint4(0u, 0u, 0u, 0u);
      dg[i] = ok ? (a.deg_pages ? a.deg_pages[row + r] : 1) : 0;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float w = (float)dg[i];
      total += dg[i];
      const uint32_t p[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[2 * j] = fmaf(w, __uint_as_float(p[j] << 16), acc[2 * j]);
        acc[2 * j + 1] = fmaf(w, __uint_as_float(p[j] & 0xffff0000u), acc[2 * j + 1]);
      }
    }
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 16);
  total += __shfl_xor_sync(0xffffffffu, total, 16);
  if constexpr (WPH == 1) {
    if (rows > 0 && lane < 16) {
      const float n = (float)total;
      reinterpret_cast<uint4*>(a.c_pages)[ph * 16 + c] =
          make_uint4(pack_bf16x2(acc[0] / n, acc[1] / n), pack_bf16x2(acc[2] / n, acc[3] / n), pack_bf16x2(acc[4] / n, acc[5] / n),
                     pack_bf16x2(acc[6] / n, acc[7] / n));
      if (lane == 0) a.clog_pages[ph] = logf(n);
    }
  } else {
    if (lane < 16) {
      *reinterpret_cast<float4*>(&s_acc[warp][c * 8]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(&s_acc[warp][c * 8 + 4]) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (lane == 0) s_n[warp] = total;
    }
    __syncthreads();
    if (rows > 0) {
      const int w0 = warp - part, d = part * 32 + lane;
      static_assert(WPH == 1 || WPH == 4, "a warp finishes 32 of the 128 columns");
      const float n = (float)(s_n[w0] + s_n[w0 + 1] + s_n[w0 + 2] + s_n[w0 + 3]);
      const float s = (s_acc[w0][d] + s_acc[w0 + 1][d]) + (s_acc[w0 + 2][d] + s_acc[w0 + 3][d]);
      a.c_pages[ph * 128 + d] = __float2bfloat16_rn(s / n);
      if (d == 0) a.clog_pages[ph] = logf(n);
    }
  }
}

// ---- ckv_pages_select --------------------------------------------------------------------------------------------
// The result is that of scores computed in 64 bits: a choice between near pages must not hang on the order of a 32-bit sum
// (it would for about one selection in a thousand).  Few pages are near the border, so only those are scored in 64 bits:
//  1. All scores in fp32 on the tensor cores, with a bound on how far they may be off: bf16 products are exact in fp32, and
//     128 additions, cut off rather than rounded, lose at most 2^-23 of sum |q c| each: 2^-15 has a factor of two to spare.
//     A summary row is read once, straight into the lanes that multiply it, for all G heads.  The CTAs of a thread-block
//     cluster share the pages; scores land in the first CTA's shared memory.
//  2. That CTA finds a narrow interval that holds the k-th largest: a histogram over the scores' range, the bin that holds
//     it, a histogram over that bin if it is still full.
//  3. Pages above the interval by more than twice the error are chosen, those below by as much are not; the others (a few)
//     are scored in 64 bits and ranked.  If they are many (equal pages, or scores that are not finite), all pages are scored
//     in 64 bits and the k-th is found digit by digit.
//  4. The chosen blocks are written in ascending order.
// Bound by the latency of these steps: 12.4 us for 256 (sequence, head) pairs of up to 1024 pages (23 MB of summaries: 3.6 us),
// 16.8 us when the summaries are not in the L2; 9.0 us (11.1) for 8 pairs of 2048 pages (scores 2.9, interval 1.6, border 2.5, order 1.3); with all scores in 64 bits the former
// took 47 us.
constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelBins = 1024;
constexpr int kSelNear = 512;                  // pages near the border that are ranked against each other
constexpr int kSelZoom = 4;                    // histograms at most
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
  int32_t H, G, shift, n_first, n_last, n_select;
};

// ascending in the score; NaN lowest, the two zeros equal
__device__ __forceinline__ uint64_t score_key(double s) {
  if (isnan(s)) return 0;
  const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ void st_cluster_f32(uint32_t local_addr, uint32_t rank, float v) {
  uint32_t ra;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(local_addr), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(ra), "f"(v) : "memory");
}

// score of one block in 64 bits, by eight lanes (x = 0 .. 7) that have sixteen elements each: pieces x and x + 8 of the row;
// q: the heads' rows in shared memory.  All 32 lanes call; lanes with ok = false read nothing.
__device__ __forceinline__ uint64_t exact_key(const SelectPagesArgs& a, const uint4* q, int64_t ph, int x, bool ok) {
  double c[16];
  auto unpack = [](const uint4& u, double* d) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      d[2 * i] = (double)__uint_as_float(w[i] << 16);
      d[2 * i + 1] = (double)__uint_as_float(w[i] & 0xffff0000u);
    }
  };
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  unpack(ok ? a.c_pages[ph * 16 + x] : zero, c);
  unpack(ok ? a.c_pages[ph * 16 + 8 + x] : zero, c + 8);
  const double lg = ok && a.clog_pages ? (double)a.clog_pages[ph] : 0.0;
  double best = 0.0;
#pragma unroll 2
  for (int g = 0; g < a.G; ++g) {
    double w[16], s = 0.0, r = 0.0;
    unpack(q[g * 16 + x], w);
    unpack(q[g * 16 + 8 + x], w + 8);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s = fma(c[i], w[i], s);
      r = fma(c[8 + i], w[8 + i], r);
    }
    s += r;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= (double)a.scale;
    if (g == 0 || s > best || isnan(s)) best = s;  // (a NaN stays)
  }
  return score_key(best + lg);
}

struct SelectShared {
  uint4 q[8 * 16];           // the query heads' rows
  uint32_t hist[kSelBins + 2];
  uint64_t near_key[kSelNear];
  int32_t near_id[kSelNear];
  float err[8 * kSelWarps];  // of each scoring warp of the cluster: the bound on its scores' error,
  float lo[8 * kSelWarps];   // its lowest score and its highest, without the blocks that are always chosen
  float hi[8 * kSelWarps];
  uint64_t key_lo[kSelWarps], key_hi[kSelWarps];
  int gt[kSelWarps], eq[kSelWarps];
  int bin, above, count, n_near;
  uint32_t more[kSelMaxBlocks / 32], same[kSelMaxBlocks / 32];  // a bit per block: chosen; equal to the border
};

// the sum of x over the threads before this one; `part` is scratch for a sum per warp.  All threads call.
__device__ __forceinline__ int sum_before(int x, int* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  if (lane == 31) part[warp] = y;
  __syncthreads();
  y -= x;
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) y += w < warp ? part[w] : 0;
  return y;
}

// The k-th largest of keys[0, n) without the forced ones, k = need > 0 and fewer than all: chosen are keys above `edge` and the
// first `ties` of those equal to it.  Digits of eight bits from the top of the range that the keys span.
__device__ void radix_select(const uint64_t* keys, int n, int need, SelectShared& sh, uint64_t& edge, int& ties) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint64_t lo = kForced, hi = 0;
  for (int i = tid; i < n; i += kSelThreads) {
    const uint64_t k = keys[i];
    if (k != kForced) {
      lo = min(lo, k);
      hi = max(hi, k);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  if (lane == 0) {
    sh.key_lo[warp] = lo;
    sh.key_hi[warp] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) {
    lo = min(lo, sh.key_lo[w]);
    hi = max(hi, sh.key_hi[w]);
  }
  uint64_t prefix = 0;
  int bits = hi > lo ? 64 - __clzll((long long)(hi - lo)) : 0;  // bits still open below the prefix
  bool all = false;
  while (bits > 0 && !all) {
    const int take = min(bits, 8), low = bits - take;
    sh.hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {
      const uint64_t k = keys[i];
      if (k == kForced) continue;
      const uint64_t d = k - lo;
      if (bits == 64 || (d >> bits) == prefix) atomicAdd(&sh.hist[(uint32_t)(d >> low) & ((1u << take) - 1u)], 1u);
    }
    __syncthreads();
    if (warp == 0) {  // lane l sums digits 8 l .. 8 l + 7; suffix sums from the top digit down
      uint32_t cnt[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += cnt[j] = sh.hist[8 * lane + j];
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
            sh.bin = 8 * lane + j;
            sh.above = (int)above;
            sh.count = (int)cnt[j];
          }
          above += cnt[j];
        }
      }
    }
    __syncthreads();
    prefix = (prefix << take) | (uint64_t)sh.bin;
    need -= sh.above;
    bits = low;
    all = sh.count == need;  // the whole digit is chosen: no need to open it further
    __syncthreads();
  }
  const uint64_t least = lo + (bits > 0 ? prefix << bits : prefix);  // the smallest key of the digit
  edge = all ? least - 1 : least;  // (fewer than all are chosen, so some key lies below a digit that is: least is not 0)
  ties = all ? 0 : need;
}

template <int CL>
__global__ void __launch_bounds__(kSelThreads, 2) pages_select_kernel(const SelectPagesArgs a) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ SelectShared sh;
  float* const score = reinterpret_cast<float*>(dyn);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  griddep_wait();
  griddep_launch();
  const ckv_paged_view view = a.views[b];
  const int64_t mask = ((int64_t)1 << a.shift) - 1;
  const int n = (int)max((int64_t)0, min((view.len + mask) >> a.shift, a.max_blocks));
  int32_t* const out = a.selected + ((int64_t)b * a.H + h) * a.n_select;
  if (n <= a.n_select) {  // every block is chosen
    if (rank == 0)
      for (int i = tid; i < a.n_select; i += kSelThreads) out[i] = i < n ? i : -1;
    return;  // (the whole cluster leaves: the condition is the sequence's)
  }
  if (CL > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  const int f0 = a.n_first, f1 = n - a.n_last, need = a.n_select - a.n_first - a.n_last;  // the others are f0 <= i < f1
  const uint4* const q_rows = reinterpret_cast<const uint4*>(a.q + ((int64_t)b * a.H + h) * a.G * 128);
  if (rank == 0)
    for (int i = tid; i < a.G * 16; i += kSelThreads) sh.q[i] = q_rows[i];

  // ---- 1. scores in fp32.  Lane (g, t) has elements 8 (t + 4 i) .. + 7 (i < 4) of rows g and g + 8 of a block of sixteen, and
  // of query head g: the same elements in the same k steps, which is all that a product needs.
  {
    uint4 qf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) qf[i] = g < a.G ? q_rows[g * 16 + t + 4 * i] : make_uint4(0u, 0u, 0u, 0u);
    if (CL > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // the first CTA has started: its scores can be written
    const uint32_t score_s = (uint32_t)__cvta_generic_to_shared(score);
    const bool h0 = 2 * t < a.G, h1 = 2 * t + 1 < a.G;
    float err = 0.f, lo = INFINITY, hi = -INFINITY;
    constexpr int kStep = 16 * kSelWarps * CL;
    int base = 16 * (rank * kSelWarps + warp);
    int page = base + (lane & 15) < n ? view.block_table[base + (lane & 15)] : 0;
    for (; base < n; base += kStep) {
      const int64_t pa = (int64_t)__shfl_sync(0xffffffffu, page, g) * a.H + h, pb = (int64_t)__shfl_sync(0xffffffffu, page, g + 8) * a.H + h;
      uint4 ra[4], rb[4];  // (rows past the end are page 0's, and dropped below)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ra[i] = a.c_pages[pa * 16 + t + 4 * i];
        rb[i] = a.c_pages[pb * 16 + t + 4 * i];
      }
      const float la = a.clog_pages ? a.clog_pages[pa] : 0.f, lb = a.clog_pages ? a.clog_pages[pb] : 0.f;
      const int next = base + kStep + (lane & 15);
      page = next < n ? view.block_table[next] : 0;
      float c[4] = {0.f, 0.f, 0.f, 0.f}, m[4] = {0.f, 0.f, 0.f, 0.f};  // q c, and |q| |c|
      constexpr uint32_t kAbs = 0x7fff7fffu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ptx::mma_bf16(c, ra[i].x, rb[i].x, ra[i].y, rb[i].y, qf[i].x, qf[i].y);
        ptx::mma_bf16(c, ra[i].z, rb[i].z, ra[i].w, rb[i].w, qf[i].z, qf[i].w);
        ptx::mma_bf16(m, ra[i].x & kAbs, rb[i].x & kAbs, ra[i].y & kAbs, rb[i].y & kAbs, qf[i].x & kAbs, qf[i].y & kAbs);
        ptx::mma_bf16(m, ra[i].z & kAbs, rb[i].z & kAbs, ra[i].w & kAbs, rb[i].w & kAbs, qf[i].z & kAbs, qf[i].w & kAbs);
      }
      // heads 2 t and 2 t + 1 of rows g and g + 8, then all heads over the four lanes of a row
      float sa = fmaxf(h0 ? c[0] * a.scale : -INFINITY, h1 ? c[1] * a.scale : -INFINITY);
      float sb = fmaxf(h0 ? c[2] * a.scale : -INFINITY, h1 ? c[3] * a.scale : -INFINITY);
      // (a sum, not a maximum: it keeps infinities and NaN)
      float ea = (m[0] + m[1]), eb = (m[2] + m[3]);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        sa = fmaxf(sa, __shfl_xor_sync(0xffffffffu, sa, o));
        sb = fmaxf(sb, __shfl_xor_sync(0xffffffffu, sb, o));
        ea += __shfl_xor_sync(0xffffffffu, ea, o);
        eb += __shfl_xor_sync(0xffffffffu, eb, o);
      }
      if (t < 2) {  // lanes 4 g: row g; 4 g + 1: row g + 8
        const int i = base + g + 8 * t;
        const float s = (t ? sb : sa) + (t ? lb : la);
        // (|q| |c| + 2^-125) scale 2^-15, and the roundings after the sum; 2^-140 is what 128 subnormal products and additions can
        // lose, with a factor of two to spare
        const float e = (t ? eb : ea) * fabsf(a.scale) * 0x1p-15f + fabsf(a.scale) * 0x1p-140f + fabsf(t ? lb : la) * 0x1p-20f + 0x1p-120f;
        if (i < n) {
          err = fmaxf(err, e < 1e30f ? e : INFINITY);  // (NaN becomes infinite)
          if (i >= f0 && i < f1) {
            lo = fminf(lo, s);
            hi = fmaxf(hi, s);
          }
          if (CL == 1)
            score[i] = s;
          else
            st_cluster_f32(score_s + 4u * (uint32_t)i, 0, s);
        }
      }
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      err = fmaxf(err, __shfl_xor_sync(0xffffffffu, err, o));
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    if (lane < 3) {
      float* const to = (lane == 0 ? sh.err : lane == 1 ? sh.lo : sh.hi) + rank * kSelWarps + warp;
      const float v = lane == 0 ? err : lane == 1 ? lo : hi;
      if (CL == 1)
        *to = v;
      else
        st_cluster_f32((uint32_t)__cvta_generic_to_shared(to), 0, v);
    }
  }
  if (CL > 1) {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    if (rank != 0) return;
  }

  // ---- 2. an interval that holds the k-th largest of the blocks that are not always chosen
  float lo = INFINITY, hi = -INFINITY, err = 0.f;
  if (tid == 0) sh.n_near = 0;
  __syncthreads();
  for (int w = lane; w < kSelWarps * CL; w += 32) {
    lo = fminf(lo, sh.lo[w]);
    hi = fmaxf(hi, sh.hi[w]);
    err = fmaxf(err, sh.err[w]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    err = fmaxf(err, __shfl_xor_sync(0xffffffffu, err, o));
  }
  bool fine = err < 1e30f;  // every score is finite and its error known
  fine &= lo > -1e30f && hi < 1e30f;
  uint64_t edge = 0;
  int ties = 0;
  float top = INFINITY, bottom = INFINITY;  // chosen above `top`, not chosen below `bottom`, to be seen in between
  if (need > 0 && fine) {
    for (int zoom = 0; zoom < kSelZoom; ++zoom) {
      const float width = (hi - lo) * (1.f / kSelBins), inv = 1.f / width;
      if (!(width > 1e-30f) || !(inv > 0.f)) break;
      for (int i = tid; i < kSelBins + 2; i += kSelThreads) sh.hist[i] = 0;
      __syncthreads();
#pragma unroll 4
      for (int i = f0 + tid; i < f1; i += kSelThreads) {
        const float s = score[i];
        const int bin = s < lo ? 0 : s > hi ? kSelBins + 1 : 1 + min(kSelBins - 1, (int)((s - lo) * inv));
        atomicAdd(&sh.hist[bin], 1u);
      }
      __syncthreads();
      // thread x sums bins 4 x + 1 .. 4 x + 4, from the top down
      const int x = tid;
      int cnt[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += cnt[j] = (int)sh.hist[4 * x + 1 + j];
      int above = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_down_sync(0xffffffffu, above, o);
        if (lane + o < 32) above += y;
      }
      if (lane == 0) sh.gt[warp] = above;
      __syncthreads();
      above += (int)sh.hist[kSelBins + 1] - sum;
      for (int w = warp + 1; w < kSelWarps; ++w) above += sh.gt[w];
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        if (above < need && above + cnt[j] >= need) {
          sh.bin = 4 * x + j;
          sh.count = cnt[j];
        }
        above += cnt[j];
      }
      __syncthreads();
      // the bin's range, and room for the rounding of its borders
      const float at = lo + width * (float)sh.bin, room = 0.125f * width + 0x1p-21f * fmaxf(fabsf(lo), fabsf(hi));
      const int count = sh.count;
      lo = at - room;
      hi = at + width + room;
      if (count <= 32 || width <= err) break;
      __syncthreads();  // (the counters are read)
    }
    top = hi + 2.f * err;
    bottom = lo - 2.f * err;
  }

  // ---- 3. the blocks in between
  int above = 0;
  if (need > 0 && fine) {
#pragma unroll 4
    for (int i = f0 + tid; i < f1; i += kSelThreads) {
      const float s = score[i];
      above += s > top;
      if (s <= top && s >= bottom) {
        const int at = atomicAdd(&sh.n_near, 1);
        if (at < kSelNear) sh.near_id[at] = i;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
    if (lane == 0) sh.eq[warp] = above;
  }
  __syncthreads();
  const int n_near = sh.n_near;
  uint64_t* const keys = reinterpret_cast<uint64_t*>(dyn);  // (in the scores' place)
  const bool few = need == 0 || (fine && n_near <= kSelNear);
  if (need > 0 && few) {
    above = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) above += sh.eq[w];
    for (int j0 = 4 * warp; j0 < n_near; j0 += 4 * kSelWarps) {
      const int j = j0 + (lane >> 3);
      const bool ok = j < n_near;
      const uint64_t k = exact_key(a, sh.q, ok ? (int64_t)view.block_table[sh.near_id[j]] * a.H + h : 0, lane & 7, ok);
      if (ok && (lane & 7) == 0) sh.near_key[j] = k;
    }
    __syncthreads();
    // ranked by key, then by number: the best need - above of them are chosen (their scores become infinite)
    for (int j = tid; j < n_near; j += kSelThreads) {
      const uint64_t k = sh.near_key[j];
      const int id = sh.near_id[j];
      int better = 0;
      for (int x = 0; x < n_near; ++x) better += sh.near_key[x] > k || (sh.near_key[x] == k && sh.near_id[x] < id);
      score[id] = better < need - above ? INFINITY : -INFINITY;
    }
    __syncthreads();
  } else if (need > 0) {
    for (int i0 = 4 * warp; i0 < n; i0 += 4 * kSelWarps) {
      const int i = i0 + (lane >> 3);
      const bool ok = i >= f0 && i < f1;
      const uint64_t k = exact_key(a, sh.q, ok ? (int64_t)view.block_table[i] * a.H + h : 0, lane & 7, ok);
      if (i < n && (lane & 7) == 0) keys[i] = ok ? k : kForced;
    }
    __syncthreads();
    radix_select(keys, n, need, sh, edge, ties);
  }

  // ---- 4. in ascending order: a bit per block, a place per word of 32 blocks, then a lane per block
  const int words = (n + 31) / 32;
  if (few && words <= 32 * kSelWarps) {  // up to 8192 blocks: each warp has a run of words, one per lane, and nothing goes through memory
    const int run = (words + kSelWarps - 1) / kSelWarps, first = min(words, warp * run), last = min(words, first + run);
    uint32_t bits = 0;
#pragma unroll 4
    for (int w = first; w < last; ++w) {
      const int i = 32 * w + lane;
      const uint32_t m = __ballot_sync(0xffffffffu, i < n && (i < f0 || i >= f1 || (need > 0 && score[i] > top)));
      if (lane == w - first) bits = m;
    }
    int at = sum_before(__popc(bits), sh.gt);
#pragma unroll 4
    for (int w = first; w < last; ++w) {
      const uint32_t m = __shfl_sync(0xffffffffu, bits, w - first);
      const int to = __shfl_sync(0xffffffffu, at, w - first) + __popc(m & ((1u << lane) - 1u));
      if ((m >> lane & 1u) && to < a.n_select) out[to] = 32 * w + lane;
    }
    return;
  }
#pragma unroll 4
  for (int w = warp; w < words; w += kSelWarps) {
    const int i = 32 * w + lane;
    bool more = false, same = false;
    if (i < n) {
      if (few) {
        more = i < f0 || i >= f1 || (need > 0 && score[i] > top);
      } else {
        const uint64_t k = keys[i];
        more = k > edge;
        same = k == edge;
      }
    }
    const uint32_t bm = __ballot_sync(0xffffffffu, more), bs = few ? 0u : __ballot_sync(0xffffffffu, same);
    if (lane == 0) {
      sh.more[w] = bm;
      sh.same[w] = bs;
    }
  }
  __syncthreads();
  const int per = (words + kSelThreads - 1) / kSelThreads, w0 = min(words, tid * per), w1 = min(words, w0 + per);
  if (!few) {  // of the equal ones the first `ties`
    int equal = 0;
    for (int w = w0; w < w1; ++w) equal += __popc(sh.same[w]);
    int left = ties - sum_before(equal, sh.eq);
    for (int w = w0; w < w1; ++w)
      for (uint32_t bits = sh.same[w]; bits && left > 0; bits &= bits - 1, --left) sh.more[w] |= bits & -bits;
  }
  int chosen = 0;
  for (int w = w0; w < w1; ++w) chosen += __popc(sh.more[w]);
  int at = sum_before(chosen, sh.gt);
  for (int w = w0; w < w1; ++w) {  // where each word's blocks go
    sh.same[w] = (uint32_t)at;
    at += __popc(sh.more[w]);
  }
  __syncthreads();
#pragma unroll 4
  for (int w = warp; w < words; w += kSelWarps) {
    const uint32_t bits = sh.more[w];
    const int to = (int)sh.same[w] + __popc(bits & ((1u << lane) - 1u));
    if ((bits >> lane & 1u) && to < a.n_select) out[to] = 32 * w + lane;
  }
}

template <int CL>
cudaError_t launch_pages_select(const SelectPagesArgs& a, int32_t Bz, cudaStream_t st) {
  static std::atomic<bool> ready[64];  // per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !ready[dev].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(pages_select_kernel<CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelMaxBlocks * 8);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) ready[dev].store(true, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(CL, (unsigned)a.H, (unsigned)Bz);
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = (size_t)a.max_blocks * 8;
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
  return cudaLaunchKernelEx(&cfg, pages_select_kernel<CL>, a);
}

cudaError_t launch_pages_select_any(const SelectPagesArgs& a, int32_t Bz, cudaStream_t st) {
  // the scores are split over a cluster while that leaves every warp a block of sixteen or more and the SMs are not all taken
  const int64_t pairs = (int64_t)Bz * a.H, sms = sm_count();
  if (a.max_blocks >= 1024 && pairs * 8 <= sms) return launch_pages_select<8>(a, Bz, st);
  if (a.max_blocks >= 512 && pairs * 4 <= 2 * sms) return launch_pages_select<4>(a, Bz, st);
  if (a.max_blocks >= 256 && pairs * 2 <= 2 * sms) return launch_pages_select<2>(a, Bz, st);
  return launch_pages_select<1>(a, Bz, st);
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
  if (dtype != CKV_BF16 || shift < 0 || D != 128 || H > 65535 || Bz > 65535 || max_blocks > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(k_pages) || !aligned16(c_pages)) return CKV_ERR_ALIGNMENT;
  if (max_blocks == 0) return CKV_OK;
  SummarizeArgs a{};
  a.views = views_dev; a.from_lens = from_lens; a.k_pages = static_cast<const uint4*>(k_pages); a.deg_pages = deg_pages;
  a.c_pages = static_cast<__nv_bfloat16*>(c_pages); a.clog_pages = clog_pages;
  a.max_blocks = max_blocks; a.H = H; a.shift = shift;
  // one warp per (page, head) once that gives every SM's warp slots something to do
  const bool many = max_blocks * H * Bz >= (int64_t)32 * sm_count();
  const int64_t units = many ? 8 : 2, ctas = (max_blocks * H + units - 1) / units;
  if (ctas > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)ctas, (unsigned)Bz);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = many ? launch_dependent(pages_summarize_kernel<1>, grid, dim3(kSumThreads), 0, st, a)
                             : launch_dependent(pages_summarize_kernel<4>, grid, dim3(kSumThreads), 0, st, a);
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
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
  a.max_blocks = max_blocks; a.scale = scale; a.H = H; a.G = G; a.shift = shift;
  a.n_first = n_first; a.n_last = n_last; a.n_select = n_select;
  return launch_pages_select_any(a, Bz, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // extern "C"
