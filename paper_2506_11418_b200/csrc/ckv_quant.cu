// Four-bit pages: keys and values as e2m1 codes in groups of 32 elements that share a power of two (the microscaling
// format MXFP4 of the OCP specification 1.0), and the decode attention that reads them: 140 bytes per cached token and head
// in place of 516.
//
// Value of an element = level(code) * 2^(scale - 127); level: sign bit, then 0, 0.5, 1, 1.5, 2, 3, 4, 6.  Scale byte 255 is NaN.
// A row's 64 bytes are ordered for the lanes that multiply them (two elements per byte, the even one in the low half):
//   keys    byte 16 t + 4 j + i holds elements 32 j + 8 t + 2 i, + 1   (t, j, i < 4): lane (g, t) of a warp reads its 16 bytes
//           of token g in one piece: eight consecutive elements of each of the four groups
//   values  byte  8 g + 2 j + i holds elements 32 j + 4 g + 2 i, + 1   (g < 8, j < 4, i < 2): lane (g, t) reads 8 bytes: four
//           elements of each group, so that every 16-row tile of V^T lies in one group
#include <algorithm>
#include <cuda_fp16.h>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_decode.cuh"
#include "ckv_internal.h"
#include "ckv_ptx.cuh"
#include "ckv_rows.cuh"

namespace ckv {
namespace {

constexpr int kD = 128;
constexpr int kCodeBytes = 64, kScaleBytes = 4;  // per row

// ---- ckv_pages_quantize ----------------------------------------------------------------------------------------------
// Half a warp per row, eight elements per lane; a group is four lanes.  Shared exponent = floor(log2 of the group's largest
// magnitude) - 2, so that the largest element lies in [4, 8) steps and codes end at 6; elements round to the nearest even
// code.  A group with an element that is not finite becomes NaN as a whole (scale 255, codes 0).

__device__ __forceinline__ void load8(const void* p, int64_t vec, int lane16, bool f32, float (&x)[8]) {
  if (f32) {
    const float4* f = reinterpret_cast<const float4*>(p) + vec + 2 * lane16;
    const float4 a = f[0], b = f[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 u = reinterpret_cast<const uint4*>(p)[vec + lane16];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// codes of a lane's eight elements, and the row's four scale bytes (every lane of the half warp has them)
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], int lane16, uint32_t& scales) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const int field = (int)(top >> 23);  // exponent field of the largest magnitude; 255: infinity or NaN
  const bool finite = field != 255;
  const int byte = finite ? max(field - 2, 0) : 255;
  const float f = finite ? __uint_as_float((uint32_t)(254 - byte) << 23) : 0.f;  // 2^(127 - byte), byte <= 252
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = finite ? x[i] * f : 0.f;  // exact
  scales = (uint32_t)byte << (8 * (lane16 >> 2));
  scales |= __shfl_xor_sync(0xffffffffu, scales, 4);
  scales |= __shfl_xor_sync(0xffffffffu, scales, 8);
  return ptx::pack_e2m1x8(y);
}

constexpr int kQuantThreads = 256;

template <bool F32, int U>
__global__ void __launch_bounds__(kQuantThreads) pages_quantize_kernel(const RowsIn r, const int64_t* slots, int64_t n, const ckv_quant_pool pool,
                                                                       int64_t n_rows, int32_t shift) {
  constexpr int kRows = kQuantThreads / 16;
  const int h = blockIdx.y, lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4;
  const int64_t i0 = (int64_t)blockIdx.x * (kRows * U), mask = ((int64_t)1 << shift) - 1;
  griddep_wait();
  griddep_launch();
  int64_t row[U];
  float k[U][8], v[U][8];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * kRows + r0;
    const int64_t s = i < n ? slots[i] : -1;
    row[u] = (s >= 0 && s < n_rows) ? (((s >> shift) * r.H + h) << shift) + (s & mask) : -1;
    if (row[u] >= 0) {
      load8(r.k, i * r.token_vecs + h * r.head_vecs, lane16, F32, k[u]);
      load8(r.v, i * r.token_vecs + h * r.head_vecs, lane16, F32, v[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) k[u][e] = v[u][e] = 0.f;
    }
  }
  const int j = lane16 >> 2, t = lane16 & 3;  // this lane's elements: 32 j + 8 t ..
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t ks, vs;
    const uint32_t kc = encode8(k[u], lane16, ks), vc = encode8(v[u], lane16, vs);
    if (row[u] < 0) continue;
    reinterpret_cast<uint32_t*>(pool.k_codes)[row[u] * 16 + 4 * t + j] = kc;
    uint16_t* vd = reinterpret_cast<uint16_t*>(pool.v_codes) + row[u] * 32 + 8 * t + j;  // g = 2 t and 2 t + 1
    vd[0] = (uint16_t)vc;
    vd[4] = (uint16_t)(vc >> 16);
    if (lane16 == 0) reinterpret_cast<uint32_t*>(pool.k_scales)[row[u]] = ks;
    if (lane16 == 1) reinterpret_cast<uint32_t*>(pool.v_scales)[row[u]] = vs;
  }
  if (pool.deg_pages || pool.logdeg_pages) write_degrees(r, slots, n, i0, kRows * U, h, pool.deg_pages, pool.logdeg_pages, n_rows, shift);
}

// ---- ckv_pages_dequantize --------------------------------------------------------------------------------------------
// Half a warp per row, eight elements per lane, as above; every value is exact in bf16 and fp32.

__device__ __forceinline__ float scale_value(uint32_t byte) {  // 2^(byte - 127); 255: NaN
  return byte == 255 ? __uint_as_float(0x7fffffffu) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

__device__ __forceinline__ void store8(void* p, int64_t vec, int lane16, bool f32, uint32_t codes, float s) {
  uint32_t h[4];
  ptx::unpack_e2m1x8(codes, h);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    x[2 * i] = f.x * s;
    x[2 * i + 1] = f.y * s;
  }
  if (f32) {
    float4* f = reinterpret_cast<float4*>(p) + vec + 2 * lane16;
    f[0] = make_float4(x[0], x[1], x[2], x[3]);
    f[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    reinterpret_cast<uint4*>(p)[vec + lane16] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
}

struct DequantArgs {
  const int32_t* table;
  int64_t len, cap;
  ckv_quant_pool pool;
  void* k;
  void* v;
  int32_t* deg;
  float* logdeg;
  int32_t H, shift;
};

template <bool F32, int U>
__global__ void __launch_bounds__(kQuantThreads) pages_dequantize_kernel(const DequantArgs a) {
  constexpr int kRows = kQuantThreads / 16, kVecs = F32 ? 32 : 16;
  const int h = blockIdx.y, lane16 = threadIdx.x & 15, r0 = threadIdx.x >> 4, j = lane16 >> 2, t = lane16 & 3;
  const int64_t i0 = (int64_t)blockIdx.x * (kRows * U), mask = ((int64_t)1 << a.shift) - 1;
  griddep_wait();
  griddep_launch();
  uint32_t kc[U], vc[U], ks[U], vs[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * kRows + r0;
    if (i >= a.len) continue;
    const int64_t row = (((int64_t)a.table[i >> a.shift] * a.H + h) << a.shift) + (i & mask);
    kc[u] = reinterpret_cast<const uint32_t*>(a.pool.k_codes)[row * 16 + 4 * t + j];
    const uint16_t* vd = reinterpret_cast<const uint16_t*>(a.pool.v_codes) + row * 32 + 8 * t + j;
    vc[u] = (uint32_t)vd[0] | ((uint32_t)vd[4] << 16);
    ks[u] = reinterpret_cast<const uint32_t*>(a.pool.k_scales)[row];
    vs[u] = reinterpret_cast<const uint32_t*>(a.pool.v_scales)[row];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * kRows + r0;
    if (i >= a.len) continue;
    const int64_t vec = ((int64_t)h * a.cap + i) * kVecs;
    store8(a.k, vec, lane16, F32, kc[u], scale_value((ks[u] >> (8 * j)) & 255u));
    store8(a.v, vec, lane16, F32, vc[u], scale_value((vs[u] >> (8 * j)) & 255u));
  }
  if (a.deg || a.logdeg)
    for (int64_t i = i0 + threadIdx.x; i < min(a.len, i0 + kRows * U); i += blockDim.x) {
      const int dg = a.pool.deg_pages ? a.pool.deg_pages[(((int64_t)a.table[i >> a.shift] * a.H + h) << a.shift) + (i & mask)] : 1;
      if (a.deg) a.deg[(int64_t)h * a.cap + i] = dg;
      if (a.logdeg) a.logdeg[(int64_t)h * a.cap + i] = logf((float)dg);
    }
}

// ---- ckv_decode_attn_quantized ----------------------------------------------------------------------------------------
// As the bf16 kernel: every warp walks its own span of a sequence in tiles of 32 tokens through a ring of cp.async copies,
// scores and outputs on mma.sync (fp16 inputs: e2m1 levels are exact in fp16, and so are the query's elements after the
// row is scaled by a power of two), softmax online in the exp2 domain, and partials that are joined in the cluster or by
// the combine kernel.  With four bits per element the tensor cores and the copies are no longer what counts: unpacking
// and scaling are, so both are arranged to cost as little as they can:
//   S   a group's 32 elements are two k steps of the product; their sum is multiplied by the token's scale of that group
//       (one FFMA per token, head and group in place of 32 products with the scale)
//   O   V's scale belongs to a token and a group, as the weight p belongs to a token: the weight of token t in group j is
//       p_t 2^e_tj, one B operand per group.  It goes to fp16 relative to the largest one so far (a running power of two
//       per head and group, with its own rescaling of the accumulators), so that whatever the scales are the tokens that
//       matter keep 11 bits and only weights below 2^-28 of the largest lose any.
//   V   two tokens' codes are interleaved by nibble before they are unpacked, which gives the operand's pairs of
//       neighbouring tokens without permuting fp16 values.
constexpr int kQT = 32;  // tokens per tile
constexpr int kQWarps = 4;
constexpr int kQStages = 3;
constexpr int kQCodes = kQT * kCodeBytes;
constexpr int kQStageBytes = 2 * kQCodes + 2 * kQT * kScaleBytes + kQT * 4;  // codes of K, V; scales of K, V; log-degrees
constexpr size_t kQRingBytes = (size_t)kQWarps * kQStages * kQStageBytes;
static_assert(kQRingBytes >= (size_t)kQWarps * 8 * kPartial * 4 + (size_t)kQWarps * kQWarps * 16 * 4, "cluster_combine's rows and weights fit");

struct QuantArgs {
  DecodeArgs d;  // views, q, out, partial, shapes, n_splits, page_shift
  ckv_quant_pool pool;
};

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// a row's four scale bytes as fp32: 2^(byte - 127), 255 NaN (bf16 holds them all exactly)
__device__ __forceinline__ void scales_f32(uint32_t w, float (&s)[4]) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %0, a;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  s[0] = __uint_as_float(lo << 16);
  s[1] = __uint_as_float(lo & 0xffff0000u);
  s[2] = __uint_as_float(hi << 16);
  s[3] = __uint_as_float(hi & 0xffff0000u);
}

// Where row r of a tile of V codes sits, and its 16-byte piece c: even rows first, pieces exchanged every other row pair, so
// that the lanes' reads of rows 2 t (+ 1, 8, 9) at 8 g fall on different banks
__device__ __forceinline__ uint32_t v_off(int r, int c) {
  const int s = (r >> 1) + (r & 1) * (kQT / 2);
  return (uint32_t)(s * kCodeBytes + ((c ^ (s & 2)) << 4));
}

template <int CL>
__global__ void __launch_bounds__(kQWarps * 32, 4) decode_quant_kernel(const QuantArgs qa_) {
  constexpr int TT = kQT, NW = kQWarps, ST = kQStages;
  const DecodeArgs& a = qa_.d;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x * NW + warp;
  griddep_wait();
  griddep_launch();
  if (CL == 0 && split >= a.n_splits) return;
  const int h = blockIdx.y, b = blockIdx.z, G = a.G;
  const ckv_paged_view view = reinterpret_cast<const ckv_paged_view*>(a.views)[b];
  const int64_t len = view.len;
  const int64_t seq_tiles = (len + TT - 1) / TT;
  const int64_t t_begin = TT * (seq_tiles * split / a.n_splits);
  const int64_t t_end = min(len, TT * (seq_tiles * (split + 1) / a.n_splits));
  const int ntiles = (int)((t_end - t_begin + TT - 1) / TT);
  const int64_t n_blocks = (len + ((int64_t)1 << a.page_shift) - 1) >> a.page_shift;
  int64_t blk0 = t_begin >> a.page_shift;
  int my_page = (ntiles > 0 && blk0 + lane < n_blocks) ? view.block_table[blk0 + lane] : 0;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem_raw) + (uint32_t)warp * ST * kQStageBytes;
  const float* logdeg = qa_.pool.logdeg_pages;

  auto issue = [&](int tile) {
    const int64_t t0 = t_begin + (int64_t)tile * TT;
    const uint32_t st = ring + (uint32_t)(tile % ST) * kQStageBytes;
    const int64_t blk = t0 >> a.page_shift;
    if (blk >= blk0 + 32) {  // next 32 entries of the table (tiles are issued in order)
      blk0 = blk;
      my_page = blk0 + lane < n_blocks ? view.block_table[blk0 + lane] : 0;
    }
    const int page = __shfl_sync(0xffffffffu, my_page, (int)(blk - blk0));
    const int64_t row0 = (((int64_t)page * a.H + h) << a.page_shift) + (t0 & (((int64_t)1 << a.page_shift) - 1));
    const int nt = (int)min((int64_t)TT, t_end - t0);
    const unsigned char* kc = qa_.pool.k_codes + row0 * kCodeBytes;
    const unsigned char* vc = qa_.pool.v_codes + row0 * kCodeBytes;
#pragma unroll
    for (int i = 0; i < TT / 8; ++i) {
      const int r = 8 * i + (lane >> 2), c = lane & 3;
      const uint32_t ok = r < nt ? 16u : 0u;
      const int off = r < nt ? r * kCodeBytes + c * 16 : 0;  // clamped address, zero-filled when out of range
      cp_async16(st + (uint32_t)(r * kCodeBytes + c * 16), kc + off, ok);
      cp_async16(st + kQCodes + v_off(r, c), vc + off, ok);
    }
    if (lane < 16) {  // scales: eight pieces of four rows each, for K and for V
      const int c = lane & 7;
      const int bytes = max(0, min(16, (nt - 4 * c) * kScaleBytes));
      const unsigned char* s = (lane < 8 ? qa_.pool.k_scales : qa_.pool.v_scales) + row0 * kScaleBytes;
      cp_async16(st + 2 * kQCodes + (uint32_t)((lane < 8 ? 0 : TT * kScaleBytes) + c * 16), s + (bytes > 0 ? c * 16 : 0), (uint32_t)bytes);
    }
    if (logdeg) cp_async4(st + 2 * kQCodes + 2 * TT * kScaleBytes + lane * 4, logdeg + (lane < nt ? row0 + lane : row0), lane < nt ? 4u : 0u);
  };

  // query fragments: head g's elements 32 j + 8 t .. + 7, scaled by a power of two that puts the row's largest at 2^14
  uint32_t qa[4][4];
  float sc;  // what turns the products into exponents of two
  {
    float x[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint4 u = make_uint4(0u, 0u, 0u, 0u);
      if (g < G) u = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + (((int64_t)b * a.H + h) * G + g) * kD)[4 * j + t];
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[j][2 * i] = __uint_as_float(w[i] << 16);
        x[j][2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        top = max(top, max((w[i] << 16) & 0x7fffffffu, w[i] & 0x7fff0000u));
      }
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int field = min(max((int)(top >> 23), 41), 254);  // (2^100 at most, also for a row of zeros)
    const float f = __uint_as_float((uint32_t)(141 - field + 127) << 23);  // 2^(14 - (field - 127))
    sc = a.scale * kLog2e * __uint_as_float((uint32_t)(field - 14) << 23);  // 1 / f = 2^(field - 141)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) qa[j][i] = pack_f16x2(x[j][2 * i] * f, x[j][2 * i + 1] * f);
  }

  float oacc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) oacc[i][0] = oacc[i][1] = oacc[i][2] = oacc[i][3] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;            // for head g (this thread's share of the tokens)
  float wmax[4] = {0.f, 0.f, 0.f, 0.f};            // largest weight p 2^e of head g in each group
  uint32_t fref[4] = {253u << 23, 253u << 23, 253u << 23, 253u << 23};  // bits of the power of two that the weights are multiplied by

#pragma unroll
  for (int i = 0; i < ST - 1; ++i) {
    if (i < ntiles) issue(i);
    cp_async_commit();
  }
  for (int tile = 0; tile < ntiles; ++tile) {
    cp_async_wait<ST - 2>();
    __syncwarp();
    if (tile + ST - 1 < ntiles) issue(tile + ST - 1);
    cp_async_commit();
    const unsigned char* st = smem_raw + (size_t)(warp * ST + tile % ST) * kQStageBytes;
    const int nt = (int)min((int64_t)TT, t_end - (t_begin + (int64_t)tile * TT));

    // ---- scores of tokens 8 n + 2 t, + 1 with head g
    float p[4][2];
    float tmax = -INFINITY;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint4 kw = *reinterpret_cast<const uint4*>(st + (8 * n + g) * kCodeBytes + 16 * t);
      const uint2 ks = *reinterpret_cast<const uint2*>(st + 2 * kQCodes + (8 * n + 2 * t) * kScaleBytes);
      float s0 = 0.f, s1 = 0.f, k0[4], k1[4];
      scales_f32(ks.x, k0);
      scales_f32(ks.y, k1);
      const uint32_t kj[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t e[4];
        ptx::unpack_e2m1x8(kj[j], e);
        float c[4];
        ptx::mma_f16_first(c, qa[j][0], 0u, qa[j][1], 0u, e[0], e[1]);
        ptx::mma_f16(c, qa[j][2], 0u, qa[j][3], 0u, e[2], e[3]);
        s0 = fmaf(c[0], k0[j], s0);
        s1 = fmaf(c[1], k1[j], s1);
      }
      float2 bias = make_float2(0.f, 0.f);
      if (logdeg) bias = *reinterpret_cast<const float2*>(st + 2 * kQCodes + 2 * TT * kScaleBytes + (8 * n + 2 * t) * 4);
      s0 = 8 * n + 2 * t < nt ? fmaf(s0, sc, bias.x * kLog2e) : -INFINITY;
      s1 = 8 * n + 2 * t + 1 < nt ? fmaf(s1, sc, bias.y * kLog2e) : -INFINITY;
      p[n][0] = s0;
      p[n][1] = s1;
      tmax = fmaxf(tmax, fmaxf(s0, s1));
    }
    // ---- online softmax
    tmax = fmaxf(tmax, __shfl_xor_sync(0xffffffffu, tmax, 1));
    tmax = fmaxf(tmax, __shfl_xor_sync(0xffffffffu, tmax, 2));
    const float m_new = fmaxf(m_run, tmax);
    const float m_use = m_new == -INFINITY ? 0.f : m_new;  // nothing but -inf so far: weights of zero, not inf - inf
    const float corr = exp2f(m_run - m_use);
    m_run = m_new;
    float psum = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      p[n][0] = exp2f(p[n][0] - m_use);
      p[n][1] = exp2f(p[n][1] - m_use);
      psum += p[n][0] + p[n][1];
    }
    l_run = l_run * corr + psum;
    // ---- weights p 2^e of every group in fp16, relative to the largest so far
    float vs[4][2][4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint2 w = *reinterpret_cast<const uint2*>(st + 2 * kQCodes + TT * kScaleBytes + (8 * n + 2 * t) * kScaleBytes);
      scales_f32(w.x, vs[n][0]);
      scales_f32(w.y, vs[n][1]);
    }
    uint32_t pb[4][4];  // [group][n]: tokens 8 n + 2 t, + 1
    float ratio[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float w[4][2], top = 0.f;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        w[n][0] = p[n][0] * vs[n][0][j];
        w[n][1] = p[n][1] * vs[n][1][j];
        top = fmaxf(top, fmaxf(w[n][0], w[n][1]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      wmax[j] = fmaxf(wmax[j] * corr, top);
      // f = 2^(14 - floor(log2 wmax)), 2^126 at most
      const uint32_t f = (268u << 23) - max(__float_as_uint(wmax[j]) & 0x7f800000u, 15u << 23);
      ratio[j] = corr * __uint_as_float(f) * __uint_as_float((254u << 23) - fref[j]);
      fref[j] = f;
#pragma unroll
      for (int n = 0; n < 4; ++n) pb[j][n] = pack_f16x2(w[n][0] * __uint_as_float(f), w[n][1] * __uint_as_float(f));
    }
    if (__any_sync(0xffffffffu, ratio[0] != 1.f || ratio[1] != 1.f || ratio[2] != 1.f || ratio[3] != 1.f)) {
      // the accumulators hold heads 2 t and 2 t + 1: their factors are in quads 2 t and 2 t + 1
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float r0 = __shfl_sync(0xffffffffu, ratio[j], 8 * t), r1 = __shfl_sync(0xffffffffu, ratio[j], 8 * t + 4);
#pragma unroll
        for (int i = 2 * j; i < 2 * j + 2; ++i) {
          oacc[i][0] *= r0; oacc[i][1] *= r1; oacc[i][2] *= r0; oacc[i][3] *= r1;
        }
      }
    }
    // ---- O^T += V^T P: step s covers tokens 16 s .. 16 s + 15; m tile 2 j + i holds elements 32 j + 4 g + 2 i (row g), + 1 (row g + 8)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const unsigned char* vt = st + kQCodes;
      uint2 v4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
        const int r = 16 * s + 2 * t + (e & 1) + 8 * (e >> 1);
        v4[e] = *reinterpret_cast<const uint2*>(vt + v_off(r, g >> 1) + (g & 1) * 8);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {  // groups 2 u and 2 u + 1
        const uint32_t a0 = u ? v4[0].y : v4[0].x, b0 = u ? v4[1].y : v4[1].x, a1 = u ? v4[2].y : v4[2].x, b1 = u ? v4[3].y : v4[3].x;
        constexpr uint32_t lo = 0x0f0f0f0fu, hi = 0xf0f0f0f0u;
        uint32_t e0[4], o0[4], e1[4], o1[4];  // even / odd elements of tokens (2 t, + 1) and (2 t + 8, + 9)
        ptx::unpack_e2m1x8((a0 & lo) | ((b0 << 4) & hi), e0);
        ptx::unpack_e2m1x8(((a0 >> 4) & lo) | (b0 & hi), o0);
        ptx::unpack_e2m1x8((a1 & lo) | ((b1 << 4) & hi), e1);
        ptx::unpack_e2m1x8(((a1 >> 4) & lo) | (b1 & hi), o1);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int j = 2 * u + (x >> 1);
          ptx::mma_f16(oacc[4 * u + x], e0[x], o0[x], e1[x], o1[x], pb[j][2 * s], pb[j][2 * s + 1]);
        }
      }
    }
  }
  cp_async_wait<0>();

  l_run += __shfl_xor_sync(0xffffffffu, l_run, 1);
  l_run += __shfl_xor_sync(0xffffffffu, l_run, 2);
  // back from each group's own power of two
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float inv = __uint_as_float((254u << 23) - fref[j]);
    const float r0 = __shfl_sync(0xffffffffu, inv, 8 * t), r1 = __shfl_sync(0xffffffffu, inv, 8 * t + 4);
#pragma unroll
    for (int i = 2 * j; i < 2 * j + 2; ++i) {
      oacc[i][0] *= r0; oacc[i][1] *= r1; oacc[i][2] *= r0; oacc[i][3] *= r1;
    }
  }
  auto park = [&](float* dst, int64_t hstride, int heads) {
    if (t == 0 && g < heads) {
      dst[g * hstride + kD] = m_run;
      dst[g * hstride + kD + 1] = l_run;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (2 * t + e >= heads) continue;
      float* o = dst + (2 * t + e) * hstride + 4 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(o + 32 * j) = make_float4(oacc[2 * j][e], oacc[2 * j][2 + e], oacc[2 * j + 1][e], oacc[2 * j + 1][2 + e]);
    }
  };
  if constexpr (CL > 0) {
    cluster_combine<CL, NW>(smem_raw, warp, lane, G, reinterpret_cast<__nv_bfloat16*>(a.out) + ((int64_t)b * a.H + h) * G * kD,
                            [&](float* part) { park(part, kPartial, 8); });
  } else {
    park(a.partial + ((((int64_t)b * a.H + h) * G) * a.n_splits + split) * kPartial, (int64_t)a.n_splits * kPartial, G);
  }
}

template <int CL>
bool quant_ready() {  // sets the kernel's shared memory once per device
  constexpr int kMaxDev = 64;
  static std::atomic<bool> done[kMaxDev];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev >= 0 && dev < kMaxDev && done[dev].load(std::memory_order_relaxed)) return true;
  if (cudaFuncSetAttribute(decode_quant_kernel<CL>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kQRingBytes) != cudaSuccess) return false;
  if (dev >= 0 && dev < kMaxDev) done[dev].store(true, std::memory_order_relaxed);
  return true;
}

template <int CL>
cudaError_t launch_quant(QuantArgs a, cudaStream_t st) {
  if (!quant_ready<CL>()) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  const int ctas = CL > 0 ? CL : (a.d.n_splits + kQWarps - 1) / kQWarps;
  if (CL > 0) a.d.n_splits = CL * kQWarps;
  cfg.gridDim = dim3((unsigned)ctas, (unsigned)a.d.H, (unsigned)a.d.Bz);
  cfg.blockDim = dim3(kQWarps * 32);
  cfg.dynamicSmemBytes = kQRingBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL > 0 ? CL : 1;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 0 ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, decode_quant_kernel<CL>, a);
  if (e != cudaSuccess || CL > 0) return e;
  return launch_decode_combine(a.d, st);
}

// Splits of a launch that joins its partials in a second kernel: four CTAs per SM, four splits per CTA; the count that
// minimises waves x (tiles per warp + a fixed cost of two tiles), with at least two tiles per warp.
int32_t quant_splits(int32_t Bz, int32_t H, int64_t max_len) {
  const int64_t pairs = (int64_t)Bz * H, slots = 4ll * sm_count();
  const int64_t tiles = std::max<int64_t>(1, (max_len + kQT - 1) / kQT);
  const int64_t most = std::min<int64_t>(64, std::max<int64_t>(1, tiles / (2 * kQWarps)));
  int64_t best = 1, best_cost = INT64_MAX;
  for (int64_t c = 1; c <= most; ++c) {
    const int64_t cost = ((pairs * c + slots - 1) / slots) * ((tiles + c * kQWarps - 1) / (c * kQWarps) + 2);
    if (cost < best_cost) {
      best_cost = cost;
      best = c;
    }
  }
  return (int32_t)(best * kQWarps);
}

int check_pool(const ckv_quant_pool* p) {
  if (!p || !p->k_codes || !p->v_codes || !p->k_scales || !p->v_scales) return CKV_ERR_INVALID_ARG;
  if (!aligned16(p->k_codes) || !aligned16(p->v_codes) || !aligned16(p->k_scales) || !aligned16(p->v_scales)) return CKV_ERR_ALIGNMENT;
  return CKV_OK;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

int ckv_pages_quantize(const ckv_token_rows* rows, const int64_t* slots, int64_t n, const ckv_quant_pool* pool, int64_t n_pages, int32_t page_tokens,
                       void* cuda_stream) {
  int st = check_rows(rows, slots, n, n_pages, page_tokens);
  if (st != CKV_OK || (st = check_pool(pool)) != CKV_OK) return st;
  if (n == 0) return CKV_OK;
  const RowsIn r = rows_in(*rows);
  const int shift = page_shift(page_tokens);
  const int64_t n_rows = n_pages << shift;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto kernel, int rows_per_cta) {
    const dim3 grid((unsigned)((n + rows_per_cta - 1) / rows_per_cta), (unsigned)rows->H);
    return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, stream, r, slots, n, *pool, n_rows, (int32_t)shift);
  };
  const bool many = n * rows->H >= (int64_t)32 * sm_count();  // two rows per half warp once that fills the SMs
  const cudaError_t e = rows->dtype == CKV_F32 ? (many ? go(pages_quantize_kernel<true, 2>, 32) : go(pages_quantize_kernel<true, 1>, 16))
                                               : (many ? go(pages_quantize_kernel<false, 2>, 32) : go(pages_quantize_kernel<false, 1>, 16));
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

int ckv_pages_dequantize(const int32_t* block_table, int64_t len, const ckv_quant_pool* pool, int32_t page_tokens, int32_t H, int32_t D,
                         int32_t dtype, void* k, void* v, int32_t* deg, float* logdeg, int64_t cap, void* cuda_stream) {
  if (!block_table || !k || !v || len < 0 || H <= 0 || cap < len) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  int st = check_pool(pool);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (shift < 0 || D != kD || H > 65535) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(k) || !aligned16(v)) return CKV_ERR_ALIGNMENT;
  if (len == 0) return CKV_OK;
  DequantArgs a{};
  a.table = block_table; a.len = len; a.cap = cap; a.pool = *pool; a.k = k; a.v = v; a.deg = deg; a.logdeg = logdeg; a.H = H; a.shift = shift;
  const bool many = len * H >= (int64_t)64 * sm_count();
  const int rows = many ? 64 : 16;
  const int64_t ctas = (len + rows - 1) / rows;
  if (ctas > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)ctas, (unsigned)H);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, stream, a); };
  const cudaError_t e = dtype == CKV_F32 ? (many ? go(pages_dequantize_kernel<true, 4>) : go(pages_dequantize_kernel<true, 1>))
                                         : (many ? go(pages_dequantize_kernel<false, 4>) : go(pages_dequantize_kernel<false, 1>));
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

size_t ckv_decode_quantized_workspace_bytes(int32_t Bz, int32_t H, int32_t G, int32_t D, int64_t max_len) {
  if (Bz <= 0 || H <= 0 || G <= 0 || D <= 0 || max_len < 0) return 0;
  return ((size_t)Bz * H * G * quant_splits(Bz, H, max_len) * kPartial * sizeof(float) + 255) / 256 * 256;
}

int ckv_decode_attn_quantized(const ckv_paged_view* views_dev, const ckv_quant_pool* pool, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G,
                              int32_t D, int32_t dtype, const void* q, void* out, float scale, int64_t max_len, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  if (!views_dev || !q || !out || Bz <= 0 || H <= 0 || G <= 0 || max_len < 0) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  int st = check_pool(pool);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (dtype != CKV_BF16 || shift < 0 || D != kD || G > 8 || H > 65535 || Bz > 65535) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(out)) return CKV_ERR_ALIGNMENT;
  const size_t need = ckv_decode_quantized_workspace_bytes(Bz, H, G, D, max_len);
  if (!workspace || workspace_bytes < need || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  QuantArgs a{};
  a.d.views = views_dev; a.d.q = q; a.d.out = out;
  a.d.partial = static_cast<float*>(workspace);
  a.d.Bz = Bz; a.d.H = H; a.d.G = G;
  a.d.n_splits = quant_splits(Bz, H, max_len);
  a.d.max_len = max_len;
  a.d.scale = scale;
  a.d.page_shift = shift;
  a.pool = *pool;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  // few pairs: one cluster of eight CTAs each, joined on the chip, while all are resident at once (four CTAs per SM)
  const cudaError_t e = (int64_t)Bz * H * 8 <= 4ll * sm_count() ? launch_quant<8>(a, stream) : launch_quant<0>(a, stream);
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // extern "C"
