// Block tables and slot maps of a paged cache built on the GPU from sequence lengths, and writes through a slot map.
#include <algorithm>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_internal.h"
#include "ckv_rows.cuh"

namespace ckv {
namespace {

// ---- ckv_pages_resize ----------------------------------------------------------------------------------------------
// With have = ceil(len / P) and want = ceil(new_len / P) of every sequence:
//   given = max(0, have - want) pages go to the back of the ring, taken = max(0, want - have) come from its front, both
//   in the order of the sequences; grown = max(0, new_len - len) tokens get slots.
// Everything is a function of the three exclusive sums over the sequences, so there is one launch and no hand-over
// between CTAs: each CTA computes the sums for itself (a batch's lengths are a few KB in L2) and then does its share of
// the pages and tokens, finding the sequence of a page or token by bisection in shared memory.  No CTA reads what
// another writes: a page that is taken is read from the ring, or, when the ring runs out, from the row of the sequence
// that gives it; rows only ever change behind a growing sequence's last page; given pages land behind the ring's last;
// lengths and the ring's state have separate outputs.  Bound by latency (lengths, sums, table or ring, slot): 4.9 us for a step
// of 64 sequences, 8.1 us for 512 sequences with 600 thousand new tokens.
constexpr int kResizeThreads = 256;
constexpr int kResizeWarps = kResizeThreads / 32;
constexpr int kResizeMaxSeqs = 8192;  // three sums of four bytes for each in shared memory: 96 KB

struct ResizeArgs {
  const int64_t* lens;
  const int64_t* new_lens;
  int32_t* tables;
  int32_t* ring;
  const int64_t* ring_state;
  int64_t* slots;
  int64_t* slot_begin;
  int64_t* lens_out;
  int64_t* ring_state_out;
  int32_t* status;
  ckv_paged_view* views;
  int64_t table_stride, n_pages, n_slots;
  int32_t Bz, shift;
};

struct ResizeNeeds {
  int64_t grow;
  int64_t take, give;
  int flags;  // bit 0: a negative length or one whose row the table cannot hold now; bit 1: new length above the row
};

__device__ __forceinline__ ResizeNeeds resize_needs(const ResizeArgs& a, int b) {
  ResizeNeeds r{0, 0, 0, 0};
  const int64_t o = a.lens[b], n = a.new_lens[b], room = a.table_stride << a.shift;
  if (o < 0 || n < 0 || o > room) {
    r.flags = 1;
  } else if (n > room) {
    r.flags = 2;
  } else {
    const int64_t mask = ((int64_t)1 << a.shift) - 1;
    const int64_t have = (o + mask) >> a.shift, want = (n + mask) >> a.shift;
    r.grow = max(n - o, (int64_t)0);
    r.take = max(want - have, (int64_t)0);
    r.give = max(have - want, (int64_t)0);
  }
  return r;
}

// the last b with begin[b] <= i (begin ascending, begin[0] = 0, i < begin[n])
__device__ __forceinline__ int find_seq(const int32_t* begin, int n, int32_t i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin[mid] <= i)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kResizeThreads) pages_resize_kernel(const ResizeArgs a) {
  extern __shared__ int32_t sums[];  // [3][Bz + 1] exclusive sums: tokens grown, pages taken, pages given
  __shared__ int64_t s_warp[3][kResizeWarps];
  __shared__ int64_t s_total[3];
  __shared__ int s_flags;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.Bz;
  int32_t* grow_begin = sums;
  int32_t* take_begin = sums + (n + 1);
  int32_t* give_begin = sums + 2 * (n + 1);
  if (tid == 0) s_flags = 0;
  griddep_wait();
  griddep_launch();
  __syncthreads();

  // sums: every thread takes a run of consecutive sequences
  const int per = (n + kResizeThreads - 1) / kResizeThreads, b0 = min(n, tid * per), b1 = min(n, b0 + per);
  int64_t v[3] = {0, 0, 0};
  int flags = 0;
  for (int b = b0; b < b1; ++b) {
    const ResizeNeeds r = resize_needs(a, b);
    v[0] += r.grow;
    v[1] += r.take;
    v[2] += r.give;
    flags |= r.flags;
  }
  if (flags) atomicOr(&s_flags, flags);
  int64_t at[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    int64_t x = v[k];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    at[k] = x - v[k];
    if (lane == 31) s_warp[k][warp] = x;
  }
  __syncthreads();
  if (tid < 3) {
    int64_t x = 0;
    for (int w = 0; w < kResizeWarps; ++w) {
      const int64_t y = s_warp[tid][w];
      s_warp[tid][w] = x;
      x += y;
    }
    s_total[tid] = x;
  }
  __syncthreads();
  const int64_t head = a.ring_state[0], count = a.ring_state[1];
  const int64_t grown = s_total[0], taken = s_total[1], given = s_total[2];
  int status = 0;
  if ((s_flags & 1) || head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages || given > a.n_pages - count)
    status = CKV_RESIZE_INCONSISTENT;
  else if (s_flags & 2)
    status = CKV_RESIZE_TABLE_FULL;
  else if (grown > a.n_slots)
    status = CKV_RESIZE_SLOTS_FULL;
  else if (taken > count + given)
    status = CKV_RESIZE_NO_PAGES;

  const int64_t gid = (int64_t)blockIdx.x * kResizeThreads + tid, gsize = (int64_t)gridDim.x * kResizeThreads;
  if (status != 0) {  // nothing is assigned: lengths, tables and ring stay as they are, no token has a slot, no view passes its row
    for (int64_t i = gid; i < a.n_slots; i += gsize) a.slots[i] = -1;
    for (int64_t b = gid; b <= n; b += gsize) {
      a.slot_begin[b] = 0;
      if (b < n) {
        const int64_t o = a.lens[b];
        a.lens_out[b] = o;
        if (a.views) a.views[b] = ckv_paged_view{a.tables + b * a.table_stride, min(max(o, (int64_t)0), a.table_stride << a.shift)};
      }
    }
    if (gid == 0) {
      a.ring_state_out[0] = head;
      a.ring_state_out[1] = count;
      *a.status = status;
    }
    return;
  }
  // (the sums fit 32 bits now: grown <= n_slots, taken and given are pages of one pool; a sum of tokens that passed 63 bits
  // would have taken more pages than any pool has)
#pragma unroll
  for (int k = 0; k < 3; ++k) at[k] += s_warp[k][warp];
  for (int b = b0; b < b1; ++b) {
    const ResizeNeeds r = resize_needs(a, b);
    grow_begin[b] = (int32_t)at[0];
    take_begin[b] = (int32_t)at[1];
    give_begin[b] = (int32_t)at[2];
    at[0] += r.grow;
    at[1] += r.take;
    at[2] += r.give;
  }
  if (tid == 0) {
    grow_begin[n] = (int32_t)grown;
    take_begin[n] = (int32_t)taken;
    give_begin[n] = (int32_t)given;
  }
  __syncthreads();

  const int64_t mask = ((int64_t)1 << a.shift) - 1;
  auto given_page = [&](int64_t j) -> int32_t {
    const int b = find_seq(give_begin, n, (int32_t)j);
    const int64_t want = (a.new_lens[b] + mask) >> a.shift;
    return a.tables[b * a.table_stride + want + (j - give_begin[b])];
  };
  auto supply = [&](int64_t j) -> int32_t {  // the j-th page that is taken
    if (j >= count) return given_page(j - count);
    int64_t p = head + j;
    if (p >= a.n_pages) p -= a.n_pages;
    return a.ring[p];
  };
  // tokens: a warp takes runs of 128 slots, each lane every 32nd, so that one bisection serves four
  for (int64_t i0 = gid / 32 * 128; i0 < a.n_slots; i0 += gsize / 32 * 128) {
    int b = -1;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u + lane;
      if (i >= a.n_slots) break;
      int64_t slot = -1;
      if (i < grown) {
        if (b < 0) b = find_seq(grow_begin, n, (int32_t)i);
        while (grow_begin[b + 1] <= (int32_t)i) ++b;
        const int64_t o = a.lens[b], pos = o + (i - grow_begin[b]), blk = pos >> a.shift, have = (o + mask) >> a.shift;
        const int32_t page = blk < have ? a.tables[b * a.table_stride + blk] : supply(take_begin[b] + (blk - have));
        slot = ((int64_t)page << a.shift) + (pos & mask);
      }
      a.slots[i] = slot;
    }
  }
  for (int64_t j = gid; j < given; j += gsize) {
    int64_t p = head + count + j;
    if (p >= a.n_pages) p -= a.n_pages;
    a.ring[p] = given_page(j);
  }
  for (int64_t j = gid; j < taken; j += gsize) {
    const int b = find_seq(take_begin, n, (int32_t)j);
    const int64_t have = (a.lens[b] + mask) >> a.shift;
    a.tables[b * a.table_stride + have + (j - take_begin[b])] = supply(j);
  }
  for (int64_t b = gid; b <= n; b += gsize) {
    a.slot_begin[b] = grow_begin[b];
    if (b < n) {
      const int64_t len = a.new_lens[b];
      a.lens_out[b] = len;
      if (a.views) a.views[b] = ckv_paged_view{a.tables + b * a.table_stride, len};
    }
  }
  if (gid == 0) {
    a.ring_state_out[0] = (head + taken) % a.n_pages;
    a.ring_state_out[1] = count + given - taken;
    *a.status = 0;
  }
}

// ---- ckv_pages_write -------------------------------------------------------------------------------------------------
// grid (token groups, KV head).  A row of K or V is VEC pieces of 16 bytes; a CTA moves 256 / VEC * U tokens, all of a
// thread's loads in flight before its first store.  Bound by the bytes of the rows, read once and written once: 29999 tokens
// x 8 heads with degrees (249 MB) in 42 us = 0.91 of the measured bandwidth; a step's 64 tokens in 2.0 us.
constexpr int kWriteThreads = 256;

template <int VEC, int U>
__global__ void __launch_bounds__(kWriteThreads) pages_write_kernel(const RowsIn r, const int64_t* slots, int64_t n, uint4* k_pages, uint4* v_pages,
                                                                    int32_t* deg_pages, float* logdeg_pages, int64_t n_rows, int32_t shift) {
  constexpr int kRows = kWriteThreads / VEC;
  const int h = blockIdx.y, c = threadIdx.x % VEC, r0 = threadIdx.x / VEC;
  const int64_t i0 = (int64_t)blockIdx.x * (kRows * U);
  const uint32_t mask = (1u << shift) - 1u;
  griddep_wait();
  griddep_launch();
  const uint4* const k_from = reinterpret_cast<const uint4*>(r.k) + h * r.k_head + c;
  const uint4* const v_from = reinterpret_cast<const uint4*>(r.v) + h * r.v_head + c;
  uint32_t row[U];  // (the rows of a pool fit 31 bits: the host checks)
  uint4 k[U], v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * kRows + r0;
    const uint64_t s = i < n ? (uint64_t)slots[i] : ~0ull;
    row[u] = ~0u;
    if (s < (uint64_t)n_rows) {
      row[u] = ((((uint32_t)s >> shift) * r.H + h) << shift) + ((uint32_t)s & mask);
      k[u] = k_from[i * r.k_token];
      v[u] = v_from[i * r.v_token];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] == ~0u) continue;
    k_pages[(size_t)row[u] * VEC + c] = k[u];
    v_pages[(size_t)row[u] * VEC + c] = v[u];
  }
  if (deg_pages || logdeg_pages) write_degrees(r, slots, n, i0, kRows * U, h, deg_pages, logdeg_pages, n_rows, shift);
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

int ckv_pages_resize(const int64_t* lens, const int64_t* new_lens, int32_t Bz, int32_t page_tokens, int32_t* block_tables, int64_t table_stride,
                     int32_t* ring, int64_t n_pages, const int64_t* ring_state, int64_t* slots, int64_t n_slots, int64_t* slot_begin,
                     int64_t* lens_out, int64_t* ring_state_out, int32_t* status, ckv_paged_view* views_dev, void* cuda_stream) {
  if (!lens || !new_lens || !block_tables || !ring || !ring_state || !slot_begin || !lens_out || !ring_state_out || !status || Bz <= 0 ||
      table_stride <= 0 || n_pages <= 0 || n_slots < 0 || (n_slots > 0 && !slots))
    return CKV_ERR_INVALID_ARG;
  const size_t lb = (size_t)Bz * 8;
  if (overlaps(lens_out, lb, lens, lb) || overlaps(lens_out, lb, new_lens, lb) || overlaps(ring_state_out, 16, ring_state, 16)) return CKV_ERR_INVALID_ARG;
  const int shift = page_shift(page_tokens);
  if (shift < 0 || Bz > kResizeMaxSeqs || n_pages > INT32_MAX || n_slots > INT32_MAX || table_stride > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  ResizeArgs a{};
  a.lens = lens; a.new_lens = new_lens; a.tables = block_tables; a.ring = ring; a.ring_state = ring_state;
  a.slots = slots; a.slot_begin = slot_begin; a.lens_out = lens_out; a.ring_state_out = ring_state_out; a.status = status; a.views = views_dev;
  a.table_stride = table_stride; a.n_pages = n_pages; a.n_slots = n_slots; a.Bz = Bz; a.shift = shift;
  // one run of 128 slots per warp, but every CTA repeats the sums: at most two CTAs per SM
  const int64_t ctas = std::min<int64_t>(std::max<int64_t>((n_slots + 128 * kResizeWarps - 1) / (128 * kResizeWarps), 1), 2 * sm_count());
  const size_t smem = (size_t)3 * (Bz + 1) * 4;
  // (48 KB come without asking, but hold the kernel's static arrays too)
  if (smem > 40 * 1024 &&
      cudaFuncSetAttribute(pages_resize_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (kResizeMaxSeqs + 1) * 4) != cudaSuccess)
    return CKV_ERR_CUDA;
  return launch_dependent(pages_resize_kernel, dim3((unsigned)ctas), dim3(kResizeThreads), smem, static_cast<cudaStream_t>(cuda_stream), a) == cudaSuccess
             ? CKV_OK : CKV_ERR_CUDA;
}

int ckv_pages_write(const ckv_token_rows* rows, const int64_t* slots, int64_t n, void* k_pages, void* v_pages, int32_t* deg_pages,
                    float* logdeg_pages, int64_t n_pages, int32_t page_tokens, void* cuda_stream) {
  int st = check_rows(rows, slots, n, n_pages, page_tokens);
  if (st != CKV_OK) return st;
  if (!k_pages || !v_pages) return CKV_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages)) return CKV_ERR_ALIGNMENT;
  if (n == 0) return CKV_OK;
  const RowsIn r = rows_in(*rows);
  const int shift = page_shift(page_tokens);
  const int64_t n_rows = n_pages << shift;
  if (n_rows > INT32_MAX / rows->H) return CKV_ERR_UNSUPPORTED;  // (2^31 rows of a bf16 pool: 1 TB)
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto kernel, int rows_per_cta) {
    const dim3 grid((unsigned)((n + rows_per_cta - 1) / rows_per_cta), (unsigned)rows->H);
    return launch_dependent(kernel, grid, dim3(kWriteThreads), 0, stream, r, slots, n, static_cast<uint4*>(k_pages), static_cast<uint4*>(v_pages),
                            deg_pages, logdeg_pages, n_rows, (int32_t)shift);
  };
  // four rows per thread once that still gives every SM a CTA, else one (a decoding step's few tokens: latency counts)
  const bool many = n * rows->H >= (int64_t)64 * sm_count();
  const cudaError_t e = rows->dtype == CKV_BF16 ? (many ? go(pages_write_kernel<16, 4>, 64) : go(pages_write_kernel<16, 1>, 16))
                                                : (many ? go(pages_write_kernel<32, 4>, 32) : go(pages_write_kernel<32, 1>, 8));
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // extern "C"
