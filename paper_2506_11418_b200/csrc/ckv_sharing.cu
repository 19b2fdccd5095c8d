// Sequences that share pages: forking, freeing (ckv_pages_fork), making a pool compact (ckv_pages_compact), and the copies of pages that
// both ask for (ckv_pages_copy).
#include <algorithm>
#include <climits>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_decode.cuh"
#include "ckv_internal.h"

namespace ckv {
namespace {

// Both table kernels are one cluster of eight thread blocks: their phases hand counts of pages over to one another (a few
// hundred KB, in L2), and a barrier of the cluster (about a microsecond) is cheaper than a launch.  Bound by latency: a phase
// is a chain of two or three loads.  A small pool takes one block and has the counts in shared memory.
constexpr int kCtas = 8;
constexpr int64_t kSmallPool = 16384;  // pages
constexpr int kSmallRows = 1024;
template <int CL>
__device__ __forceinline__ void sync_all() {
  if constexpr (CL > 1)
    cluster_sync_all();
  else
    __syncthreads();
}
// a count that other threads have changed
template <int CL>
__device__ __forceinline__ int32_t count_of(const int32_t* p) {
  if constexpr (CL > 1)
    return __ldcg(p);
  else
    return *p;
}
constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxRows = 8192;

// Sums of one value per thread over the CTA: the sum of all, and of those before this thread.
__device__ __forceinline__ int block_scan(int v, int* s_warp, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();  // (s_warp may still be read from the last time)
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int y = s_warp[w];
    before += w < warp ? y : 0;
    total += y;
  }
  return before + x - v;
}

struct Shared {  // the head of a workspace
  int32_t flags;          // 1: inconsistent, 2: a list is full
  int32_t count[kCtas];   // of a CTA's pages: freed (fork), held (compact)
  int32_t front;          // held pages in front of the border (compact)
};
constexpr size_t kHead = 256;

// ---- ckv_pages_fork --------------------------------------------------------------------------------------------------
// Holders of a page after the call, apart from rows that go on writing to it: shared + 1 - (old rows that list it) + (new rows that
// hold it whole).  The first child of a row cancels out for the blocks that it keeps whole, so in a step in which most rows go on
// as they are, hardly a counter is touched.
struct ForkArgs {
  const int64_t* lens;
  const int32_t* parents;
  const int64_t* keep;
  const int32_t* tables;
  int32_t* tables_out;
  const int32_t* shared;
  int32_t* shared_out;
  int32_t* ring;
  const int64_t* ring_state;
  int32_t* copies;
  int64_t* lens_out;
  int64_t* ring_state_out;
  int32_t* status;
  ckv_paged_view* views;
  Shared* head;
  int32_t* delta;   // [n_pages] holders gained and lost
  int32_t* first;   // [n_pages] the first new row that goes on writing to it
  int64_t stride, n_pages;
  int32_t n_in, n_out, shift;
};

struct ForkRow {
  int p;         // parent, -1: none
  int64_t n;     // tokens kept
  bool ok;
};
__device__ __forceinline__ ForkRow fork_row(const ForkArgs& a, int b) {
  ForkRow r{a.parents[b], 0, true};
  if (r.p < -1 || r.p >= a.n_in) return ForkRow{-1, 0, false};
  if (r.p < 0) return r;
  const int64_t len = a.lens[r.p];
  r.n = a.keep ? a.keep[b] : len;
  if (len < 0 || len > a.stride << a.shift || r.n < 0 || r.n > len) return ForkRow{-1, 0, false};
  return r;
}

template <int CL>
__global__ void __launch_bounds__(kThreads) pages_fork_kernel(const ForkArgs a) {
  // [n_out] tokens kept, parent, the page that is filled in part (-1: none), takes before; [n_in] first child; one block: the pages' counts
  extern __shared__ int64_t rows[];
  __shared__ int s_warp[kWarps];
  int64_t* const kept = rows;
  int32_t* const parent = reinterpret_cast<int32_t*>(kept + a.n_out);
  int32_t* const tail = parent + a.n_out;
  int32_t* const before = tail + a.n_out;
  int32_t* const child = before + a.n_out;
  int32_t* const delta = CL > 1 ? a.delta : child + a.n_in;
  int32_t* const first = CL > 1 ? a.first : delta + a.n_pages;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
  const int gwarp = cta * kWarps + warp, n_warps = CL * kWarps;
  const int64_t gid = (int64_t)cta * kThreads + tid, gsize = CL * kThreads, mask = ((int64_t)1 << a.shift) - 1;
  griddep_wait();
  griddep_launch();
  for (int64_t p = gid; p < a.n_pages; p += gsize) {
    delta[p] = 0;
    first[p] = INT_MAX;
  }
  if (gid == 0) a.head->flags = 0;
  for (int b = tid; b < a.n_in; b += kThreads) child[b] = INT_MAX;
  __syncthreads();
  bool bad = false;
  for (int b = tid; b < a.n_out; b += kThreads) {
    const ForkRow r = fork_row(a, b);
    bad |= !r.ok;
    kept[b] = r.n;
    parent[b] = r.p;
    int32_t page = -1;
    if (r.p >= 0) {
      atomicMin(&child[r.p], b);
      if (r.n & mask) {
        page = a.tables[r.p * a.stride + (r.n >> a.shift)];
        if ((uint32_t)page >= (uint32_t)a.n_pages) {
          bad = true;
          page = -1;
        }
      }
    }
    tail[b] = page;
  }
  const int64_t head = a.ring_state[0], count = a.ring_state[1];
  bad |= head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages;
  sync_all<CL>();

  // a warp per row: blocks that an old row lists and its first child does not hold whole; blocks that further children hold whole
  for (int b = gwarp; b < a.n_in; b += n_warps) {
    const int64_t len = a.lens[b];
    if (len < 0 || len > a.stride << a.shift) {
      bad = true;
      continue;
    }
    const int64_t have = (len + mask) >> a.shift, from = child[b] == INT_MAX ? 0 : kept[child[b]] >> a.shift;
    for (int64_t i = lane; i < have; i += 32) {
      const int32_t page = a.tables[b * a.stride + i];
      if ((uint32_t)page >= (uint32_t)a.n_pages)
        bad = true;
      else if (i >= from)
        atomicSub(&delta[page], 1);
    }
  }
  for (int b = gwarp; b < a.n_out; b += n_warps) {
    if (parent[b] < 0 || child[parent[b]] == b) continue;
    const int32_t* const row = a.tables + parent[b] * a.stride;
    for (int64_t i = lane; i < kept[b] >> a.shift; i += 32) {
      const int32_t page = row[i];
      if ((uint32_t)page < (uint32_t)a.n_pages) atomicAdd(&delta[page], 1);
    }
  }
  for (int b = (int)gid; b < a.n_out; b += (int)gsize)
    if (tail[b] >= 0) atomicMin(&first[tail[b]], b);
  if (bad) atomicOr(&a.head->flags, 1);
  sync_all<CL>();

  // new rows that need a page of their own, in order (every CTA for itself); pages nobody holds any more, a run of pages per CTA
  int taken = 0;
  bad = false;
  for (int b0 = 0; b0 < a.n_out; b0 += kThreads) {
    const int b = b0 + tid;
    const int32_t page = b < a.n_out ? tail[b] : -1;
    const int take = page >= 0 && !(a.shared[page] + 1 + count_of<CL>(&delta[page]) == 0 && count_of<CL>(&first[page]) == b);
    int total;
    const int x = block_scan(take, s_warp, total);
    if (b < a.n_out) before[b] = take ? taken + x : -1 - (taken + x);  // (negative: it takes none)
    taken += total;
  }
  const int64_t per = (a.n_pages + CL - 1) / CL, p0 = min(a.n_pages, cta * per), p1 = min(a.n_pages, p0 + per);
  auto is_freed = [&](int64_t p, int32_t& left) {
    const int32_t d = count_of<CL>(&delta[p]);
    left = a.shared[p] + d;
    bad |= left < -1 || a.shared[p] < 0;
    return d < 0 && left == -1 && count_of<CL>(&first[p]) == INT_MAX;
  };
  int freed = 0;
  for (int64_t p = p0 + tid; p < p1; p += kThreads) {
    int32_t left;
    freed += is_freed(p, left);
  }
  int total;
  block_scan(freed, s_warp, total);
  if (bad) atomicOr(&a.head->flags, 1);
  if (tid == 0) a.head->count[cta] = total;
  sync_all<CL>();

  int64_t freed_before = 0, freed_all = 0;
  for (int c = 0; c < CL; ++c) {
    const int x = __ldcg(&a.head->count[c]);
    freed_before += c < cta ? x : 0;
    freed_all += x;
  }
  const int status = (__ldcg(&a.head->flags) & 1) || freed_all > a.n_pages - count ? CKV_RESIZE_INCONSISTENT
                     : taken > count + freed_all                                   ? CKV_RESIZE_NO_PAGES
                                                                                   : CKV_RESIZE_OK;
  // counts and, behind the queue's last page, what is free now (in the order of the pages: a thread has a run of them each time)
  for (int64_t q0 = p0; q0 < p1; q0 += 4 * kThreads) {
    const int64_t q = q0 + 4 * tid;
    int32_t left[4];
    int f[4], n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      left[k] = 0;
      f[k] = q + k < p1 ? is_freed(q + k, left[k]) : 0;
      n += f[k];
    }
    int64_t at = head + count + freed_before + block_scan(n, s_warp, total);
    freed_before += total;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (q + k >= p1) break;
      a.shared_out[q + k] = status ? a.shared[q + k] : max(left[k], 0);
      if (f[k] && !status) a.ring[at % a.n_pages] = (int32_t)(q + k);
      at += f[k];
    }
  }
  if (gid == 0) {
    a.ring_state_out[0] = status ? head : (head + taken) % a.n_pages;
    a.ring_state_out[1] = status ? count : count + freed_all - taken;
    *a.status = status;
  }
  for (int b = (int)gid; b < a.n_out; b += (int)gsize) {
    if (status || b >= taken) a.copies[3 * b] = a.copies[3 * b + 1] = a.copies[3 * b + 2] = -1;
  }
  sync_all<CL>();
  if (status) return;
  for (int b = gwarp; b < a.n_out; b += n_warps) {
    const int64_t n = kept[b], whole = n >> a.shift, blocks = (n + mask) >> a.shift;
    const int32_t* const from = a.tables + max(parent[b], 0) * a.stride;
    int32_t* const to = a.tables_out + b * a.stride;
    for (int64_t i = lane; i < blocks; i += 32) {
      int32_t page = from[i];
      if (i == whole && before[b] >= 0) {
        int64_t at = head + before[b];
        if (at >= a.n_pages) at -= a.n_pages;
        const int32_t mine = __ldcg(&a.ring[at]);
        int32_t* const c = a.copies + 3 * before[b];
        c[0] = page; c[1] = mine; c[2] = (int32_t)(n & mask);
        page = mine;
      }
      to[i] = page;
    }
    if (lane == 0) {
      a.lens_out[b] = n;
      if (a.views) a.views[b] = ckv_paged_view{to, n};
    }
  }
}

// ---- ckv_pages_compact -----------------------------------------------------------------------------------------------
// With U pages held, the k-th held page from U on moves to the k-th page in front of U that is not held.
struct CompactArgs {
  const int64_t* lens;
  const int32_t* tables;
  int32_t* tables_out;
  const int32_t* shared;
  int32_t* shared_out;
  int32_t* ring;
  int32_t* copies;
  int64_t* ring_state_out;
  int32_t* status;
  ckv_paged_view* views;
  Shared* head;
  int32_t* mark;   // [n_pages] held; then 1 + the number of its move
  int64_t stride, n_pages, n_copies;
  int32_t Bz, shift;
};

template <int CL>
__global__ void __launch_bounds__(kThreads) pages_compact_kernel(const CompactArgs a) {
  extern __shared__ int32_t s_mark[];  // one block: the pages' marks
  __shared__ int s_warp[kWarps];
  int32_t* const mark = CL > 1 ? a.mark : s_mark;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
  const int gwarp = cta * kWarps + warp, n_warps = CL * kWarps;
  const int64_t gid = (int64_t)cta * kThreads + tid, gsize = CL * kThreads, mask = ((int64_t)1 << a.shift) - 1;
  griddep_wait();
  griddep_launch();
  for (int64_t p = gid; p < a.n_pages; p += gsize) mark[p] = 0;
  if (gid == 0) {
    a.head->flags = 0;
    a.head->front = 0;
  }
  sync_all<CL>();
  bool bad = false;
  for (int b = gwarp; b < a.Bz; b += n_warps) {
    const int64_t len = a.lens[b];
    if (len < 0 || len > a.stride << a.shift) {
      bad = true;
      continue;
    }
    for (int64_t i = lane; i < (len + mask) >> a.shift; i += 32) {
      const int32_t page = a.tables[b * a.stride + i];
      if ((uint32_t)page >= (uint32_t)a.n_pages)
        bad = true;
      else
        mark[page] = 1;
    }
  }
  if (bad) atomicOr(&a.head->flags, 1);
  sync_all<CL>();
  const int64_t per = (a.n_pages + CL - 1) / CL, p0 = min(a.n_pages, cta * per), p1 = min(a.n_pages, p0 + per);
  int held = 0, total;
  for (int64_t p = p0 + tid; p < p1; p += kThreads) held += count_of<CL>(&mark[p]);
  block_scan(held, s_warp, total);
  if (tid == 0) a.head->count[cta] = total;
  sync_all<CL>();
  int64_t held_before = 0, U = 0;
  for (int c = 0; c < CL; ++c) {
    const int x = __ldcg(&a.head->count[c]);
    held_before += c < cta ? x : 0;
    U += x;
  }
  const int64_t first_before = held_before;
  held = 0;
  for (int64_t p = p0 + tid; p < min(p1, U); p += kThreads) held += count_of<CL>(&mark[p]);
  if (held) atomicAdd(&a.head->front, held);
  sync_all<CL>();
  const int64_t front = __ldcg(&a.head->front), moves = U - front;
  const int status = (__ldcg(&a.head->flags) & 1) ? CKV_RESIZE_INCONSISTENT : moves > a.n_copies ? CKV_RESIZE_SLOTS_FULL : CKV_RESIZE_OK;
  if (status == 0) {
    for (int64_t q0 = p0; q0 < p1; q0 += 4 * kThreads) {
      const int64_t q = q0 + 4 * tid;
      int h[4], n = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        h[k] = q + k < p1 ? count_of<CL>(&mark[q + k]) : 0;
        n += h[k];
      }
      int64_t at = held_before + block_scan(n, s_warp, total);  // held pages in front of q
      held_before += total;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t p = q + k;
        if (p >= p1) break;
        if (p >= U && h[k]) {
          a.copies[3 * (at - front)] = (int32_t)p;
          a.copies[3 * (at - front) + 2] = (int32_t)mask + 1;
          mark[p] = (int32_t)(at - front) + 1;
        } else if (p < U && !h[k]) {
          a.copies[3 * (p - at) + 1] = (int32_t)p;
        }
        at += h[k];
      }
    }
  }
  for (int64_t i = gid; i < a.n_copies; i += gsize)
    if (status || i >= moves) a.copies[3 * i] = a.copies[3 * i + 1] = a.copies[3 * i + 2] = -1;
  if (gid == 0) {
    *a.status = status;
    if (status == 0) {
      a.ring_state_out[0] = 0;
      a.ring_state_out[1] = a.n_pages - U;
    }
  }
  sync_all<CL>();
  if (status) return;
  held_before = first_before;
  for (int64_t q0 = p0; q0 < p1; q0 += 4 * kThreads) {  // (pages in front of U keep their mark: 0 or 1)
    const int64_t q = q0 + 4 * tid;
    int h[4], n = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[k] = q + k < p1 && count_of<CL>(&mark[q + k]) != 0;
      n += h[k];
    }
    int64_t at = held_before + block_scan(n, s_warp, total);
    held_before += total;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t p = q + k;
      if (p >= p1) break;
      a.shared_out[p] = p >= U ? 0 : h[k] ? a.shared[p] : a.shared[__ldcg(&a.copies[3 * (p - at)])];
      if (p >= U) a.ring[p - U] = (int32_t)p;
      at += h[k];
    }
  }
  for (int b = gwarp; b < a.Bz; b += n_warps) {
    const int64_t len = a.lens[b];
    int32_t* const to = a.tables_out + b * a.stride;
    for (int64_t i = lane; i < (len + mask) >> a.shift; i += 32) {
      const int32_t page = a.tables[b * a.stride + i];
      to[i] = page < U ? page : __ldcg(&a.copies[3 * (count_of<CL>(&mark[page]) - 1) + 1]);
    }
    if (lane == 0 && a.views) a.views[b] = ckv_paged_view{to, len};
  }
}

// ---- ckv_pages_copy --------------------------------------------------------------------------------------------------
// A unit of work is the rows of one head of one page in one layer, in all arrays; CTAs go round the units.  Bound by the bytes of the
// rows, read once and written once.
constexpr int kCopyThreads = 128;  // (256: a compacted pool of 2.8 GB takes 541 us, so 486)
constexpr int kMaxArrays = 64;

struct CopyPagesArgs {
  ckv_page_array arrays[kMaxArrays];
  const int32_t* copies;
  int64_t n, n_pages;
  int32_t n_arrays, H, layers;
};

// The same run of two arrays, all loads of a round before its first store (one array after the other would wait twice).  STREAM: past the
// caches, which a short list's few pages gain from (64 beams: 24.7 -> 23.0 us) and a pool's do not (486 -> 507).
template <typename T, bool STREAM>
__device__ __forceinline__ void copy_runs(unsigned char* to0, const unsigned char* from0, unsigned char* to1, const unsigned char* from1, int64_t bytes) {
  const int64_t n = bytes / (int64_t)sizeof(T);
  constexpr int U = 4;
  auto load = [](const unsigned char* p, int64_t i) { return STREAM ? __ldcs(reinterpret_cast<const T*>(p) + i) : reinterpret_cast<const T*>(p)[i]; };
  auto store = [](unsigned char* p, int64_t i, T x) {
    if (STREAM)
      __stcs(reinterpret_cast<T*>(p) + i, x);
    else
      reinterpret_cast<T*>(p)[i] = x;
  };
  for (int64_t i = threadIdx.x; i < n; i += U * kCopyThreads) {
    T x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * kCopyThreads >= n) break;
      x[u] = load(from0, i + u * kCopyThreads);
      if (to1) y[u] = load(from1, i + u * kCopyThreads);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * kCopyThreads >= n) break;
      store(to0, i + u * kCopyThreads, x[u]);
      if (to1) store(to1, i + u * kCopyThreads, y[u]);
    }
  }
}

template <bool COUNT>
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const __grid_constant__ CopyPagesArgs a) {
  griddep_wait();
  griddep_launch();
  int64_t lo = 0, n = a.n;
  if (COUNT) {  // the list ends at its first entry without a source: found in two strides
    while (n > lo) {
      const int64_t step = (n - lo + kCopyThreads - 1) / kCopyThreads, i = lo + threadIdx.x * step;
      const int some = __syncthreads_count(i < n && a.copies[3 * i] >= 0);  // entries lo, lo + step, ... that list something
      if (some == 0) {
        n = lo;
      } else if (step == 1) {
        lo = n = lo + some;
      } else {
        const int64_t last = lo + (some - 1) * step;
        n = min(n, last + step);
        lo = last + 1;
      }
    }
  }
  const int64_t per = (int64_t)a.layers * a.H, units = n * per;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t c = u / per;
    const int rest = (int)(u - c * per), layer = rest / a.H, h = rest - layer * a.H;
    const int64_t src = a.copies[3 * c], dst = a.copies[3 * c + 1];
    const int tokens = a.copies[3 * c + 2];
    if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages || src == dst || tokens <= 0) continue;
    for (int k = 0; k < a.n_arrays; ++k) {
      auto run = [&](int k, unsigned char*& to, const unsigned char*& from, int64_t& bytes) {
        const ckv_page_array& r = a.arrays[k];
        unsigned char* const base = static_cast<unsigned char*>(r.base) + layer * r.layer_bytes;
        const int64_t head_bytes = (int64_t)r.rows * r.row_bytes;
        bytes = layer < r.layers ? (int64_t)min(tokens, r.rows) * r.row_bytes : 0;
        to = base + (dst * a.H + h) * head_bytes;
        from = base + (src * a.H + h) * head_bytes;
      };
      unsigned char *to0, *to1 = nullptr;
      const unsigned char *from0, *from1 = nullptr;
      int64_t bytes, more = 0;
      run(k, to0, from0, bytes);
      if (k + 1 < a.n_arrays) run(k + 1, to1, from1, more);
      if (more != bytes) {
        to1 = nullptr;
        from1 = nullptr;
      } else {
        ++k;
      }
      if (((reinterpret_cast<uintptr_t>(to0) | reinterpret_cast<uintptr_t>(from0) | reinterpret_cast<uintptr_t>(to1) | reinterpret_cast<uintptr_t>(from1) |
            (uintptr_t)bytes) & 15) == 0)
        copy_runs<uint4, !COUNT>(to0, from0, to1, from1, bytes);
      else
        copy_runs<uint32_t, !COUNT>(to0, from0, to1, from1, bytes);
    }
  }
}

template <typename Args>
cudaError_t launch_cluster(void (*kernel)(Args), int ctas, size_t smem, cudaStream_t st, const Args& a) {
  if (smem > 40 * 1024) {  // (48 KB come without asking, but hold the kernel's static arrays too)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

size_t fork_bytes(int64_t n_pages) { return kHead + (size_t)n_pages * 8; }

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t ckv_pages_fork_workspace_bytes(int64_t n_pages) { return n_pages <= 0 || n_pages > INT32_MAX ? 0 : fork_bytes(n_pages); }

int ckv_pages_fork(const int64_t* lens, int32_t n_in, const int32_t* parents, const int64_t* keep, int32_t n_out, int32_t page_tokens,
                   const int32_t* block_tables, int32_t* block_tables_out, int64_t table_stride, const int32_t* shared, int32_t* shared_out,
                   int32_t* ring, int64_t n_pages, const int64_t* ring_state, int32_t* copies, int64_t* lens_out, int64_t* ring_state_out,
                   int32_t* status, ckv_paged_view* views_dev, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!lens || !parents || !block_tables || !block_tables_out || !shared || !shared_out || !ring || !ring_state || !copies || !lens_out || !ring_state_out ||
      !status || n_in <= 0 || n_out <= 0 || table_stride <= 0 || n_pages <= 0)
    return CKV_ERR_INVALID_ARG;
  const int shift = page_shift(page_tokens);
  if (shift < 0 || n_in > kMaxRows || n_out > kMaxRows || n_pages > INT32_MAX || table_stride > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const size_t out_bytes = (size_t)n_out * table_stride * 4;
  if (overlaps(block_tables_out, out_bytes, block_tables, (size_t)n_in * table_stride * 4) || overlaps(shared_out, (size_t)n_pages * 4, shared, (size_t)n_pages * 4) ||
      overlaps(lens_out, (size_t)n_out * 8, lens, (size_t)n_in * 8) || (keep && overlaps(lens_out, (size_t)n_out * 8, keep, (size_t)n_out * 8)) ||
      overlaps(ring_state_out, 16, ring_state, 16))
    return CKV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < fork_bytes(n_pages) || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  ForkArgs a{};
  a.lens = lens; a.parents = parents; a.keep = keep; a.tables = block_tables; a.tables_out = block_tables_out; a.shared = shared; a.shared_out = shared_out;
  a.ring = ring; a.ring_state = ring_state; a.copies = copies; a.lens_out = lens_out; a.ring_state_out = ring_state_out; a.status = status; a.views = views_dev;
  a.head = static_cast<Shared*>(workspace);
  a.delta = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + kHead);
  a.first = a.delta + n_pages;
  a.stride = table_stride; a.n_pages = n_pages; a.n_in = n_in; a.n_out = n_out; a.shift = shift;
  const bool small = n_pages <= kSmallPool && n_in <= kSmallRows && n_out <= kSmallRows;
  const size_t smem = (size_t)n_out * 20 + (size_t)n_in * 4 + (small ? (size_t)n_pages * 8 : 0);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = small ? launch_cluster(pages_fork_kernel<1>, 1, smem, st, a) : launch_cluster(pages_fork_kernel<kCtas>, kCtas, smem, st, a);
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

size_t ckv_pages_compact_workspace_bytes(int64_t n_pages) { return n_pages <= 0 || n_pages > INT32_MAX ? 0 : kHead + (size_t)n_pages * 4; }

int ckv_pages_compact(const int64_t* lens, int32_t Bz, int32_t page_tokens, const int32_t* block_tables, int32_t* block_tables_out, int64_t table_stride,
                      const int32_t* shared, int32_t* shared_out, int32_t* ring, int64_t n_pages, int32_t* copies, int64_t n_copies,
                      int64_t* ring_state_out, int32_t* status, ckv_paged_view* views_dev, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!lens || !block_tables || !block_tables_out || !shared || !shared_out || !ring || (n_copies > 0 && !copies) || n_copies < 0 || !ring_state_out || !status ||
      Bz <= 0 || table_stride <= 0 || n_pages <= 0)
    return CKV_ERR_INVALID_ARG;
  const int shift = page_shift(page_tokens);
  if (shift < 0 || Bz > kMaxRows || n_pages > INT32_MAX || n_copies > INT32_MAX || table_stride > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const size_t table_bytes = (size_t)Bz * table_stride * 4;
  if (overlaps(block_tables_out, table_bytes, block_tables, table_bytes) || overlaps(shared_out, (size_t)n_pages * 4, shared, (size_t)n_pages * 4))
    return CKV_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < ckv_pages_compact_workspace_bytes(n_pages) || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  CompactArgs a{};
  a.lens = lens; a.tables = block_tables; a.tables_out = block_tables_out; a.shared = shared; a.shared_out = shared_out; a.ring = ring; a.copies = copies;
  a.ring_state_out = ring_state_out; a.status = status; a.views = views_dev;
  a.head = static_cast<Shared*>(workspace);
  a.mark = reinterpret_cast<int32_t*>(static_cast<unsigned char*>(workspace) + kHead);
  a.stride = table_stride; a.n_pages = n_pages; a.n_copies = n_copies; a.Bz = Bz; a.shift = shift;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = n_pages <= kSmallPool && Bz <= kSmallRows ? launch_cluster(pages_compact_kernel<1>, 1, (size_t)n_pages * 4, st, a)
                                                                  : launch_cluster(pages_compact_kernel<kCtas>, kCtas, 0, st, a);
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

int ckv_pages_copy(const ckv_page_array* arrays, int32_t n_arrays, int32_t H, const int32_t* copies, int64_t n, int64_t n_pages, void* cuda_stream) {
  if (!arrays || n_arrays <= 0 || H <= 0 || n < 0 || (n > 0 && !copies) || n_pages <= 0) return CKV_ERR_INVALID_ARG;
  CopyPagesArgs a{};
  for (int i = 0; i < n_arrays; ++i) {
    const ckv_page_array& r = arrays[i];
    if (!r.base || r.layers <= 0 || r.row_bytes <= 0 || r.rows <= 0 || r.layer_bytes < 0) return CKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(r.base) | (uintptr_t)r.row_bytes | (uintptr_t)r.layer_bytes) & 3) return CKV_ERR_ALIGNMENT;
    if (r.layers > 65535) return CKV_ERR_UNSUPPORTED;
  }
  if (n > INT32_MAX || n_pages > INT32_MAX || H > 65535) return CKV_ERR_UNSUPPORTED;
  if (n == 0) return CKV_OK;
  a.copies = copies; a.n = n; a.n_pages = n_pages; a.H = H;
  for (int at = 0; at < n_arrays; at += kMaxArrays) {
    a.n_arrays = std::min(n_arrays - at, kMaxArrays);
    a.layers = 0;
    for (int i = 0; i < a.n_arrays; ++i) {
      a.arrays[i] = arrays[at + i];
      a.layers = std::max(a.layers, arrays[at + i].layers);
    }
    // a block per unit, where one that has nothing to do costs less than finding the end of the list first, else blocks that go round
    const int64_t units = n * (int64_t)a.layers * H;  // (both at most 2^31)
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = units <= 64 * sm_count() ? launch_dependent(pages_copy_kernel<false>, dim3((unsigned)units), dim3(kCopyThreads), 0, st, a)
                                                   : launch_dependent(pages_copy_kernel<true>, dim3((unsigned)(16 * sm_count())), dim3(kCopyThreads), 0, st, a);
    if (e != cudaSuccess) return CKV_ERR_CUDA;
  }
  return CKV_OK;
}

}  // extern "C"
