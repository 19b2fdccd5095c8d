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
// magnitude) - 2, so that the largest element lies in [4, 8) steps and codes end at 6; elements round to the nearest code,
// ties to the even one.  A group with an element that is not finite becomes NaN as a whole (scale 255, codes 0).  32749 tokens
// x 8 heads of bf16, from a graph: 34 us = 0.79 of the measured bandwidth, and 33 us (0.81) back; of fp32: 47 us (1.0) and 50.5
// us (0.93).

// a lane's eight elements as they lie in memory
template <bool F32>
struct Eight {
  uint4 u[F32 ? 2 : 1];
};

template <bool F32>
__device__ __forceinline__ Eight<F32> load8(const void* p, int64_t vec, int lane16) {
  Eight<F32> r;
  if constexpr (F32) {
    r.u[0] = reinterpret_cast<const uint4*>(p)[vec + 2 * lane16];
    r.u[1] = reinterpret_cast<const uint4*>(p)[vec + 2 * lane16 + 1];
  } else {
    r.u[0] = reinterpret_cast<const uint4*>(p)[vec + lane16];
  }
  return r;
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The bits of a lane's largest magnitude, as far as the exponent needs them: the upper 16.  Magnitudes compare as their bits do,
// NaN above infinity.
template <bool F32>
__device__ __forceinline__ uint32_t top16(const Eight<F32>& v) {
  constexpr uint32_t kAbs = 0x7fff7fffu;
  uint32_t w[4];
  if constexpr (F32) {  // (of two fp32 the upper halves in one register)
    w[0] = __byte_perm(v.u[0].x, v.u[0].y, 0x7632);
    w[1] = __byte_perm(v.u[0].z, v.u[0].w, 0x7632);
    w[2] = __byte_perm(v.u[1].x, v.u[1].y, 0x7632);
    w[3] = __byte_perm(v.u[1].z, v.u[1].w, 0x7632);
  } else {
    w[0] = v.u[0].x; w[1] = v.u[0].y; w[2] = v.u[0].z; w[3] = v.u[0].w;
  }
  const uint32_t t = max_u16x2(max_u16x2(w[0] & kAbs, w[1] & kAbs), max_u16x2(w[2] & kAbs, w[3] & kAbs));
  return max(t >> 16, t & 0xffffu);
}

// codes of a lane's eight elements, and its group's scale byte; top: the group's largest magnitude, its upper 16 bits
template <bool F32>
__device__ __forceinline__ uint32_t encode8(const Eight<F32>& v, uint32_t top, uint32_t& byte) {
  const uint32_t field = top >> 7;  // its exponent field; 255: infinity or NaN
  byte = field == 255 ? 255u : (uint32_t)max((int)field - 2, 0);
  const float f = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte), byte <= 252: products are exact
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    if constexpr (F32) {
      a = __uint_as_float((i & 1) ? v.u[i >> 1].z : v.u[i >> 1].x);
      b = __uint_as_float((i & 1) ? v.u[i >> 1].w : v.u[i >> 1].y);
    } else {
      const uint32_t w = i == 0 ? v.u[0].x : i == 1 ? v.u[0].y : i == 2 ? v.u[0].z : v.u[0].w;
      a = __uint_as_float(w << 16);
      b = __uint_as_float(w & 0xffff0000u);
    }
    ptx::mul_f32x2(x[2 * i], x[2 * i + 1], a, b, f);
  }
  return field == 255 ? 0u : ptx::pack_e2m1x8(x);
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
  uint32_t row[U];  // (the rows of a pool fit 31 bits: the host checks)
  Eight<F32> k[U] = {}, v[U] = {};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = i0 + u * kRows + r0;
    const uint64_t s = i < n ? (uint64_t)slots[i] : ~0ull;
    row[u] = ~0u;
    if (s < (uint64_t)n_rows) {
      row[u] = ((((uint32_t)s >> shift) * r.H + h) << shift) + ((uint32_t)s & (uint32_t)mask);
      k[u] = load8<F32>(r.k, i * r.k_token + h * r.k_head, lane16);
      v[u] = load8<F32>(r.v, i * r.v_token + h * r.v_head, lane16);
    }
  }
  const int j = lane16 >> 2, t = lane16 & 3;  // this lane's elements: 32 j + 8 t ..
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // K's largest in the lower half, V's in the upper: one exchange for both over the group's four lanes
    uint32_t top = top16<F32>(k[u]) | top16<F32>(v[u]) << 16, ks, vs;
    top = max_u16x2(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max_u16x2(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (row[u] == ~0u) continue;
    const uint32_t kc = encode8<F32>(k[u], top & 0xffffu, ks), vc = encode8<F32>(v[u], top >> 16, vs);
    reinterpret_cast<uint32_t*>(pool.k_codes)[(size_t)row[u] * 16 + 4 * t + j] = kc;
    uint16_t* vd = reinterpret_cast<uint16_t*>(pool.v_codes) + (size_t)row[u] * 32 + 8 * t + j;  // g = 2 t and 2 t + 1
    vd[0] = (uint16_t)vc;
    vd[4] = (uint16_t)(vc >> 16);
    if (t == 0) {
      pool.k_scales[(size_t)row[u] * 4 + j] = (uint8_t)ks;
      pool.v_scales[(size_t)row[u] * 4 + j] = (uint8_t)vs;
    }
  }
  if (pool.deg_pages || pool.logdeg_pages) write_degrees(r, slots, n, i0, kRows * U, h, pool.deg_pages, pool.logdeg_pages, n_rows, shift);
}

// ---- ckv_pages_dequantize --------------------------------------------------------------------------------------------
// Half a warp per row, eight elements per lane, as above; every value is exact in bf16 and fp32.

__device__ __forceinline__ float scale_value(uint32_t byte) {  // 2^(byte - 127); 255: NaN
  return byte == 255 ? __uint_as_float(0x7fffffffu) : byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

// (all lanes of the warp call; those with ok = false store nothing)
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t vec, int lane16, bool ok, uint32_t codes, float s) {
  uint32_t h[4];
  ptx::unpack_e2m1x8(codes, h);
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    x[2 * i] = f.x * s;
    x[2 * i + 1] = f.y * s;
  }
  if constexpr (F32) {
    // lanes 2 i and 2 i + 1 write the 32 bytes of the one, then of the other: whole sectors per instruction
    const bool odd = lane16 & 1;
    float4 mine = odd ? make_float4(x[0], x[1], x[2], x[3]) : make_float4(x[4], x[5], x[6], x[7]), theirs;
    theirs.x = __shfl_xor_sync(0xffffffffu, mine.x, 1);
    theirs.y = __shfl_xor_sync(0xffffffffu, mine.y, 1);
    theirs.z = __shfl_xor_sync(0xffffffffu, mine.z, 1);
    theirs.w = __shfl_xor_sync(0xffffffffu, mine.w, 1);
    if (!ok) return;
    float4* f = reinterpret_cast<float4*>(p) + vec + 2 * (lane16 & ~1);
    f[lane16 & 1] = odd ? theirs : make_float4(x[0], x[1], x[2], x[3]);
    f[2 + (lane16 & 1)] = odd ? make_float4(x[4], x[5], x[6], x[7]) : theirs;
  } else if (ok) {
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
  uint32_t kc[U] = {}, vc[U] = {}, ks[U] = {}, vs[U] = {};
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
    const int64_t vec = ((int64_t)h * a.cap + i) * kVecs;
    store8<F32>(a.k, vec, lane16, i < a.len, kc[u], scale_value((ks[u] >> (8 * j)) & 255u));
    store8<F32>(a.v, vec, lane16, i < a.len, vc[u], scale_value((vs[u] >> (8 * j)) & 255u));
  }
  if (!a.deg && a.logdeg && a.pool.logdeg_pages && !a.pool.deg_pages) {  // known by their logarithms only
    for (int64_t i = i0 + threadIdx.x; i < min(a.len, i0 + kRows * U); i += blockDim.x)
      a.logdeg[(int64_t)h * a.cap + i] = a.pool.logdeg_pages[(((int64_t)a.table[i >> a.shift] * a.H + h) << a.shift) + (i & mask)];
  } else if (a.deg || a.logdeg) {
    for (int64_t i = i0 + threadIdx.x; i < min(a.len, i0 + kRows * U); i += blockDim.x) {
      const int dg = a.pool.deg_pages ? a.pool.deg_pages[(((int64_t)a.table[i >> a.shift] * a.H + h) << a.shift) + (i & mask)] : 1;
      if (a.deg) a.deg[(int64_t)h * a.cap + i] = dg;
      if (a.logdeg) a.logdeg[(int64_t)h * a.cap + i] = logf((float)dg);
    }
  }
}

// ---- ckv_decode_attn_quantized ----------------------------------------------------------------------------------------
// As the bf16 kernel: every warp walks its own span of a sequence in tiles of 32 tokens through a ring of cp.async copies,
// scores and outputs on mma.sync (fp16 inputs: e2m1 levels are exact in fp16, and so are the query's elements after the
// row is scaled by a power of two, down to 2^-31 of its largest; smaller ones are off by 2^-39 of it at most), softmax online in the exp2 domain, and partials that are joined in the cluster or by
// a second kernel.  With four bits per element the issue slots are what counts (a tile's 4480 bytes take 192 cycles of an
// SM's share of the measured bandwidth), so unpacking and scaling are arranged to cost as few instructions as they can:
//   S   S^T = K Q^T: tokens fill the 16 rows of the A operand and up to eight heads the columns of B, so no row is padding.  A
//       group's 32 elements are two k steps; their sum is multiplied by the token's scale of that group (one multiply-add
//       per token, head and group in place of 32 products with the scale), two heads per instruction
//   O   V's scale belongs to a token and a group, as the weight p belongs to a token: the weight of token t in group j is
//       p_t 2^e_tj, one B operand per group, turned from S^T's layout by movmatrix.  It goes to fp16 times a power of two F
//       that is the head's and the group's own and follows the largest such weight so far, so that however far the scales lie
//       apart the tokens that matter keep 11 bits: weights from 2^-21 of the largest on, and below that 2^-32 of the largest.
//       Sums are fp32 and divided last: p goes up to 2^6, so 2^6 times the tokens times the largest value has to stay in range.
//   m   the softmax's reference and F move only when a tile needs it (an exponent above 6, a weight that would pass 2^15):
//       after a sequence's first tiles that is rare, and the accumulators are left alone.
//   e   lanes share tokens: each tile's 256 scales are converted once, one token per lane, and read back as fp32 (doubled in
//       registers; kept doubled in shared memory they cost 73 us below, in place of 71)
//   V   two tokens' codes are interleaved by nibble before they are unpacked, which gives the operand's pairs of
//       neighbouring tokens without permuting fp16 values.
// Batch 32, 4097 .. 16384 tokens, 8 KV heads of 4 query heads: 71 us = 0.77 of the measured bandwidth at an SM clock of 1965 MHz;
// in a long loop the power limit takes the clock to 1740, and a call 80 us.  With 8 query heads: 77 us.  About 580 instructions per
// tile at 2.4 per cycle and SM, 128 of them cvt on the half-rate ALU pipe: that pipe is 57 % busy, the tensor pipe 25 %, and four
// warps per scheduler leave the rest to latency.
constexpr int kQT = 32;  // tokens per tile
constexpr int kQShareWarps = 16, kQShareStages = 2;      // the launch by shares: one CTA per SM, 128 registers per thread
constexpr int kQClusterWarps = 8, kQClusterStages = 3;   // the launch by clusters
constexpr int kQCodes = kQT * kCodeBytes;
constexpr int kQStageBytes = 2 * kQCodes + 2 * kQT * kScaleBytes + kQT * 4;  // codes of K, V; scales of K, V; log-degrees
constexpr int kQScaleOut = 2 * kQT * 16;                                     // a tile's scales of K, V as fp32
constexpr int quant_warp_bytes(int stages) { return stages * kQStageBytes + kQScaleOut; }
static_assert(quant_warp_bytes(kQClusterStages) >= 8 * kPartial * 4 + kQClusterWarps * 16 * 4, "cluster_combine's rows and weights take a warp's part or less");
static_assert(quant_warp_bytes(kQShareStages) >= 8 * kPartial * 4, "a warp's partial takes its ring's place");
constexpr float kQLazy = 6.f;           // exponents up to this above the reference are let through
constexpr uint32_t kQFactor = 7u;       // F puts the largest weight at 2^7 .. 2^8 when it is set; it may grow to 2^15

struct QuantArgs {
  DecodeArgs d;        // views, q, out, partial ([warp + pair][G][kPartial], launch by shares), shapes, page_shift
  int32_t* plan;       // launch by shares, for the combine kernel: tiles of one head before each sequence [Bz + 1], tiles per warp
  ckv_quant_pool pool;
};

// tiles of a length; a batch's tiles over all heads fit 31 bits (the host checks, from max_len)
__device__ __forceinline__ int tiles_of(int64_t len) { return (int)((max(len, (int64_t)0) + kQT - 1) / kQT); }

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ float ex2(float x) {  // 2^x, results below 2^-126 are 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// pairs of fp32 in one register pair: two products or multiply-adds per instruction, each rounded as the scalar one
struct f32x2 {
  uint64_t v;
  __device__ __forceinline__ f32x2() {}
  __device__ __forceinline__ f32x2(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
  __device__ __forceinline__ void get(float& a, float& b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}

__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}

__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// four scale bytes as fp32: 2^(byte - 127), 255 NaN (bf16 holds them all exactly)
__device__ __forceinline__ void scales_f32(uint32_t w, float4* out) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %0, a;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  const float s0 = __uint_as_float(lo << 16), s1 = __uint_as_float(lo & 0xffff0000u);
  const float s2 = __uint_as_float(hi << 16), s3 = __uint_as_float(hi & 0xffff0000u);
  *out = make_float4(s0, s1, s2, s3);
}

// Where row r of a tile of V codes sits, and its 16-byte piece c: even rows first, pieces exchanged every other row pair, so
// that the lanes' reads of rows 2 t (+ 1, 8, 9) at 8 g fall on different banks
__device__ __forceinline__ uint32_t v_off(int r, int c) {
  const int s = (r >> 1) + (r & 1) * (kQT / 2);
  return (uint32_t)(s * kCodeBytes + ((c ^ (s & 2)) << 4));
}

// HALF: at most four query heads.  They stand twice in the columns of S^T, and a lane weighs its two heads for two of the
// four groups: of the outputs' columns the first four then hold groups 0 and 1, the others 2 and 3.
//
// CL > 0: one cluster per (sequence, KV head), its warps share the tiles evenly and join their partials on the chip.
// CL = 0: one CTA of sixteen warps per SM (twelve warps without the few spills of 128 registers: 77 us); each warp takes an
// equal share of all tiles of the batch, in the order of the pairs, so a ragged batch is balanced to a tile and every warp
// runs from start to end.  A share may end in one pair and go on in the next: each stretch leaves a partial at index share +
// pair, which no other stretch has.
template <int CL, bool HALF>
__global__ void __launch_bounds__((CL > 0 ? kQClusterWarps : kQShareWarps) * 32, 1) decode_quant_kernel(const QuantArgs qa_) {
  constexpr int TT = kQT, NW = CL > 0 ? kQClusterWarps : kQShareWarps, ST = CL > 0 ? kQClusterStages : kQShareStages;
  constexpr int kQWarpBytes = ST * kQStageBytes + kQScaleOut;
  constexpr int NU = HALF ? 1 : 2;  // pairs of groups that a lane weighs
  const DecodeArgs& a = qa_.d;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t = lane & 3;
  const int head0 = 2 * (HALF ? t & 1 : t);  // this lane's heads: head0, head0 + 1
  griddep_wait();
  griddep_launch();
  const ckv_paged_view* const views = reinterpret_cast<const ckv_paged_view*>(a.views);
  const int G = a.G;
  int b, h, tile0;  // where this warp is, and its first tile there
  int share = 0;    // tiles that it has to do from there (CL = 0)
  ckv_paged_view view;
  // (shares go round the SMs first, so that a small batch is spread over all of them)
  const int gw = CL > 0 ? (int)blockIdx.x * NW + warp : warp * (int)gridDim.x + (int)blockIdx.x;
  if constexpr (CL > 0) {
    b = blockIdx.z;
    h = blockIdx.y;
    view = views[b];
    tile0 = (int)((int64_t)tiles_of(view.len) * gw / (CL * NW));
  } else {
    // tiles of 32 sequences, one per lane, summed up to and with each
    auto scan = [&](int i, ckv_paged_view& v, int& n) {
      v = ckv_paged_view{nullptr, 0};
      if (i + lane < a.Bz) v = views[i + lane];
      n = tiles_of(v.len);
      int sum = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
      }
      return sum;
    };
    ckv_paged_view v;
    int n, sum = 0, total = 0, longest = 0;  // tiles of one head; of the longest sequence
    for (int i = 0; i < a.Bz; i += 32) {
      sum = scan(i, v, n);
      if (gw == 0 && i + lane < a.Bz) qa_.plan[i + lane] = total + sum - n;
      total += __shfl_sync(0xffffffffu, sum, 31);
      longest = max(longest, __reduce_max_sync(0xffffffffu, n));
    }
    const uint32_t all = (uint32_t)total * a.H, warps = gridDim.x * NW;
    // (not so small that one pair is cut into many more stretches than its combining warps have in flight: one head of 66000
    // tokens takes 15.6 us, by single tiles 29.5)
    share = max(max((int)((all + warps - 1) / warps), (longest + 511) / 512), 1);
    if (gw == 0 && lane == 0) {
      qa_.plan[a.Bz] = total;
      qa_.plan[a.Bz + 1] = share;
    }
    const int64_t start64 = (int64_t)gw * share;
    if (start64 >= all) return;
    const int start = (int)start64;
    share = min(share, (int)(all - start));
    int before = 0;  // tiles of all heads before the 32 sequences
    for (b = 0;; b += 32) {
      if (a.Bz > 32) sum = scan(b, v, n);  // (else they are at hand)
      const uint32_t past = __ballot_sync(0xffffffffu, before + sum * a.H > start);
      if (past) {
        const int l = __ffs((int)past) - 1, of_b = __shfl_sync(0xffffffffu, n, l);
        const int rest = start - before - __shfl_sync(0xffffffffu, sum - n, l) * a.H;
        b += l;
        h = rest / of_b;
        tile0 = rest - h * of_b;
        view.block_table = reinterpret_cast<const int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(v.block_table), l));
        view.len = __shfl_sync(0xffffffffu, v.len, l);
        break;
      }
      before += __shfl_sync(0xffffffffu, sum, 31) * a.H;
    }
  }
  unsigned char* const mine = smem_raw + (size_t)warp * kQWarpBytes;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(mine);
  float4* const sc_out = reinterpret_cast<float4*>(mine + ST * kQStageBytes);  // [K, V][token][group]
  const float* logdeg = qa_.pool.logdeg_pages;

  for (;;) {  // one stretch of tiles of one (sequence, KV head)
  const int seq_tiles = tiles_of(view.len);
  const int ntiles = CL > 0 ? (int)((int64_t)seq_tiles * (gw + 1) / (CL * NW)) - tile0 : min(share, seq_tiles - tile0);
  const int n_tail = (int)(view.len - (int64_t)(seq_tiles - 1) * TT);  // tokens of the sequence's last tile
  const int tile_shift = a.page_shift - 5;        // tiles per page
  const int n_blocks = (seq_tiles + (1 << tile_shift) - 1) >> tile_shift;
  int blk0 = tile0 >> tile_shift;
  int my_page = (ntiles > 0 && blk0 + lane < n_blocks) ? view.block_table[blk0 + lane] : 0;

  // piece i of a tile of codes is row 8 i + lane / 4, 16 bytes lane % 4: 512 bytes on in memory, 256 in the tile of V
  const uint32_t v_dst = kQCodes + v_off(lane >> 2, lane & 3);
  auto issue = [&](int tile) {
    const uint32_t st = ring + (uint32_t)(tile % ST) * kQStageBytes;
    const int at = tile0 + tile, blk = at >> tile_shift;
    if (blk >= blk0 + 32) {  // next 32 entries of the table (tiles are issued in order)
      blk0 = blk;
      my_page = blk0 + lane < n_blocks ? view.block_table[blk0 + lane] : 0;
    }
    const int page = __shfl_sync(0xffffffffu, my_page, blk - blk0);
    const int64_t row0 = (((int64_t)page * a.H + h) << a.page_shift) + (at & ((1 << tile_shift) - 1)) * TT;
    const int nt = at == seq_tiles - 1 ? n_tail : TT;
    const unsigned char* kc = qa_.pool.k_codes + row0 * kCodeBytes + lane * 16;
    const unsigned char* vc = qa_.pool.v_codes + row0 * kCodeBytes + lane * 16;
    const unsigned char* s = (lane < 8 ? qa_.pool.k_scales : qa_.pool.v_scales) + row0 * kScaleBytes + (lane & 7) * 16;
    const uint32_t s_dst = st + 2 * kQCodes + (uint32_t)lane * 16;  // lanes 0 .. 7: K's scales, 8 .. 15: V's
    const uint32_t l_dst = st + 2 * kQCodes + 2 * TT * kScaleBytes + (uint32_t)lane * 4;
    if (nt == TT) {
#pragma unroll
      for (int i = 0; i < TT / 8; ++i) {
        cp_async16(st + (uint32_t)(lane * 16 + i * 512), kc + i * 512, 16u);
        cp_async16(st + v_dst + (uint32_t)(i * 256), vc + i * 512, 16u);
      }
      if (lane < 16) cp_async16(s_dst, s, 16u);
      if (logdeg) cp_async4(l_dst, logdeg + row0 + lane, 4u);
    } else {  // the sequence's last tile: rows past its end are zero-filled, from addresses inside the tile's first row
#pragma unroll
      for (int i = 0; i < TT / 8; ++i) {
        const bool ok = 8 * i + (lane >> 2) < nt;
        cp_async16(st + (uint32_t)(lane * 16 + i * 512), ok ? kc + i * 512 : kc - lane * 16, ok ? 16u : 0u);
        cp_async16(st + v_dst + (uint32_t)(i * 256), ok ? vc + i * 512 : vc - lane * 16, ok ? 16u : 0u);
      }
      const int bytes = max(0, min(16, (nt - 4 * (lane & 7)) * kScaleBytes));
      if (lane < 16) cp_async16(s_dst, bytes > 0 ? s : s - (lane & 7) * 16, (uint32_t)bytes);
      if (logdeg) cp_async4(l_dst, logdeg + (lane < nt ? row0 + lane : row0), lane < nt ? 4u : 0u);
    }
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
      const int head = HALF ? g & 3 : g;
      if (head < G) u = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + (((int64_t)b * a.H + h) * G + head) * kD)[4 * j + t];
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
  const f32x2 sc2(__shfl_sync(0xffffffffu, sc, 4 * head0), __shfl_sync(0xffffffffu, sc, 4 * head0 + 4));
  float m_ref[2] = {0.f, 0.f};          // the exponents' reference
  bool seen[2] = {false, false};        // a score above -inf has been met
  f32x2 l_run(0.f, 0.f);                // this thread's share of the sum
  f32x2 fac[2 * NU];                    // F of each group
  uint32_t wtop[2 * NU];                // this thread's largest weight of each group, times F, in fp16
#pragma unroll
  for (int j = 0; j < 2 * NU; ++j) {
    fac[j] = f32x2(__uint_as_float(253u << 23), __uint_as_float(253u << 23));
    wtop[j] = 0u;
  }

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
    const unsigned char* st = mine + (size_t)(tile % ST) * kQStageBytes;
    const int nt = tile0 + tile == seq_tiles - 1 ? n_tail : TT;

    // ---- scales: one token per lane
    {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(st + 2 * kQCodes);
      scales_f32(w[lane], sc_out + lane);
      scales_f32(w[TT + lane], sc_out + TT + lane);
      __syncwarp();
    }
    // ---- exponents of tokens 8 n + g with this lane's heads, relative to the reference
    f32x2 x[4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint4 ka = *reinterpret_cast<const uint4*>(st + (16 * s + g) * kCodeBytes + 16 * t);
      const uint4 kb = *reinterpret_cast<const uint4*>(st + (16 * s + 8 + g) * kCodeBytes + 16 * t);
      const uint32_t wa[4] = {ka.x, ka.y, ka.z, ka.w}, wb[4] = {kb.x, kb.y, kb.z, kb.w};
      const float4 fa = sc_out[16 * s + g], fb = sc_out[16 * s + 8 + g];
      const f32x2 sa[4] = {f32x2(fa.x, fa.x), f32x2(fa.y, fa.y), f32x2(fa.z, fa.z), f32x2(fa.w, fa.w)};
      const f32x2 sb[4] = {f32x2(fb.x, fb.x), f32x2(fb.y, fb.y), f32x2(fb.z, fb.z), f32x2(fb.w, fb.w)};
      f32x2 xa, xb;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t ea[4], eb[4];
        ptx::unpack_e2m1x8(wa[j], ea);
        ptx::unpack_e2m1x8(wb[j], eb);
        float c[4];
        ptx::mma_f16_first(c, ea[0], eb[0], ea[1], eb[1], qa[j][0], qa[j][1]);
        ptx::mma_f16(c, ea[2], eb[2], ea[3], eb[3], qa[j][2], qa[j][3]);
        xa = j == 0 ? mul2(f32x2(c[0], c[1]), sa[j]) : fma2(f32x2(c[0], c[1]), sa[j], xa);
        xb = j == 0 ? mul2(f32x2(c[2], c[3]), sb[j]) : fma2(f32x2(c[2], c[3]), sb[j], xb);
      }
      float ba = 0.f, bb = 0.f;
      if (logdeg) {
        const float* ld = reinterpret_cast<const float*>(st + 2 * kQCodes + 2 * TT * kScaleBytes) + 16 * s + g;
        ba = ld[0];
        bb = ld[8];
      }
      x[2 * s] = fma2(xa, sc2, f32x2(fmaf(ba, kLog2e, -m_ref[0]), fmaf(ba, kLog2e, -m_ref[1])));
      x[2 * s + 1] = fma2(xb, sc2, f32x2(fmaf(bb, kLog2e, -m_ref[0]), fmaf(bb, kLog2e, -m_ref[1])));
    }
    if (nt < TT) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (8 * n + g >= nt) x[n] = f32x2(-INFINITY, -INFINITY);
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      float x0, x1;
      x[n].get(x0, x1);
      top[0] = fmaxf(top[0], x0);
      top[1] = fmaxf(top[1], x1);
    }
    float corr[2] = {1.f, 1.f};
    const bool move = __any_sync(0xffffffffu, fmaxf(top[0], top[1]) > kQLazy || !(seen[0] && seen[1]));
    if (move) {  // the reference goes to the largest score so far
      float up[2] = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], o));
        if (top[e] > -INFINITY) {
          up[e] = seen[e] ? fmaxf(top[e], 0.f) : top[e];
          corr[e] = seen[e] ? ex2(-up[e]) : 0.f;
          seen[e] = true;
          m_ref[e] += up[e];
        }
      }
      const f32x2 down(-up[0], -up[1]);
#pragma unroll
      for (int n = 0; n < 4; ++n) x[n] = add2(x[n], down);
      l_run = mul2(l_run, f32x2(corr[0], corr[1]));
    }
    f32x2 p[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      float x0, x1;
      x[n].get(x0, x1);
      p[n] = f32x2(ex2(x0), ex2(x1));
      l_run = add2(l_run, p[n]);
    }
    // ---- weights p 2^e of two groups times F in fp16, then their O^T += V^T P
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const float2* const v_scales = reinterpret_cast<const float2*>(sc_out + TT + g) + (HALF ? t >> 1 : u);
      uint32_t pk[2][4];  // [group][n]: token 8 n + g, this lane's heads
      bool over = move;
#pragma unroll 1
      for (;;) {
        if (over) {  // F moves (rarely)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float f[2], q[2];
            fac[2 * u + j].get(f[0], f[1]);
            const float2 past = __half22float2(*reinterpret_cast<const __half2*>(&wtop[2 * u + j]));
            float old[2] = {past.x * corr[0], past.y * corr[1]};  // largest weight before this tile, times the old F
            float now[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              const float v = reinterpret_cast<const float*>(v_scales + 16 * n)[j];
              float p0, p1;
              p[n].get(p0, p1);
              now[0] = fmaxf(now[0], p0 * v);
              now[1] = fmaxf(now[1], p1 * v);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float inv = __uint_as_float((254u << 23) - __float_as_uint(f[e]));
              q[e] = fmaxf(old[e] * inv, now[e]);
#pragma unroll
              for (int o = 4; o < 32; o <<= 1) q[e] = fmaxf(q[e], __shfl_xor_sync(0xffffffffu, q[e], o));
              // F = 2^(7 - floor(log2 q)), 2^126 at most
              f[e] = __uint_as_float(((254u + kQFactor) << 23) - max(__float_as_uint(q[e]) & 0x7f800000u, (kQFactor + 1u) << 23));
              const float ratio = corr[e] * f[e] * inv;
              old[e] = old[e] * inv * f[e];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                oacc[2 * (2 * u + j) + i][e] *= ratio;
                oacc[2 * (2 * u + j) + i][2 + e] *= ratio;
                if (HALF) {
                  oacc[2 * (2 + j) + i][e] *= ratio;
                  oacc[2 * (2 + j) + i][2 + e] *= ratio;
                }
              }
            }
            fac[2 * u + j] = f32x2(f[0], f[1]);
            wtop[2 * u + j] = pack_f16x2(old[0], old[1]);
          }
        }
        uint32_t high[2] = {wtop[2 * u], wtop[2 * u + 1]};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const float2 s01 = v_scales[16 * n];
          const f32x2 vs[2] = {f32x2(s01.x, s01.x), f32x2(s01.y, s01.y)};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float w0, w1;
            mul2(mul2(p[n], vs[j]), fac[2 * u + j]).get(w0, w1);
            pk[j][n] = pack_f16x2(w0, w1);
            high[j] = max_f16x2(high[j], pk[j][n]);
          }
        }
        const uint32_t all = max_f16x2(high[0], high[1]);
        const bool too_large = (all & 0x7fffu) > 0x7800u || all > 0x7800ffffu;  // above 2^15 (the weights are not negative)
        if (over || !__any_sync(0xffffffffu, too_large)) {  // (still too large after F has moved: NaN)
          wtop[2 * u] = high[0];
          wtop[2 * u + 1] = high[1];
          break;
        }
        over = true;
      }
      // step s covers tokens 16 s .. 16 s + 15; m tile 2 j + i holds elements 32 j + 4 g + 2 i (row g), + 1 (row g + 8)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        uint32_t v[4][3 - NU], pb[2][2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {  // tokens 2 t, 2 t + 1, 2 t + 8, 2 t + 9
          const int r = 16 * s + 2 * t + (e & 1) + 8 * (e >> 1);
          const unsigned char* at = st + kQCodes + v_off(r, g >> 1) + (g & 1) * 8;
          if constexpr (HALF) {
            const uint2 x = *reinterpret_cast<const uint2*>(at);
            v[e][0] = x.x;
            v[e][1] = x.y;
          } else {
            v[e][0] = *reinterpret_cast<const uint32_t*>(at + 4 * u);
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) pb[j][i] = transpose8x8(pk[j][2 * s + i]);  // tokens 8 n + 2 t, + 1, column g
#pragma unroll
        for (int y = 0; y < 3 - NU; ++y) {
          constexpr uint32_t lo = 0x0f0f0f0fu, hi = 0xf0f0f0f0u;
          uint32_t e0[4], o0[4], e1[4], o1[4];  // even / odd elements of tokens (2 t, + 1) and (2 t + 8, + 9)
          ptx::unpack_e2m1x8((v[0][y] & lo) | ((v[1][y] << 4) & hi), e0);
          ptx::unpack_e2m1x8(((v[0][y] >> 4) & lo) | (v[1][y] & hi), o0);
          ptx::unpack_e2m1x8((v[2][y] & lo) | ((v[3][y] << 4) & hi), e1);
          ptx::unpack_e2m1x8(((v[2][y] >> 4) & lo) | (v[3][y] & hi), o1);
#pragma unroll
          for (int i = 0; i < 4; ++i) ptx::mma_f16(oacc[4 * (u + y) + i], e0[i], o0[i], e1[i], o1[i], pb[i >> 1][0], pb[i >> 1][1]);
        }
      }
    }
  }
  cp_async_wait<0>();

  float l[2], m_out[2];
  l_run.get(l[0], l[1]);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], o);
    m_out[e] = l[e] == 0.f ? -INFINITY : m_ref[e];
  }
  // back from each group's own power of two
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float f0, f1;
    fac[HALF ? j & 1 : j].get(f0, f1);
    const float r0 = __uint_as_float((254u << 23) - __float_as_uint(f0)), r1 = __uint_as_float((254u << 23) - __float_as_uint(f1));
#pragma unroll
    for (int i = 2 * j; i < 2 * j + 2; ++i) {
      oacc[i][0] *= r0; oacc[i][1] *= r1; oacc[i][2] *= r0; oacc[i][3] *= r1;
    }
  }
  auto park = [&](float* part) {
    if (g == 0 && (!HALF || t < 2)) {
#pragma unroll
      for (int e = 0; e < 2; ++e) *reinterpret_cast<float2*>(part + (head0 + e) * kPartial + kD) = make_float2(m_out[e], l[e]);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float* o = part + (head0 + e) * kPartial + 4 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!HALF || (j >> 1) == (t >> 1))
          *reinterpret_cast<float4*>(o + 32 * j) = make_float4(oacc[2 * j][e], oacc[2 * j][2 + e], oacc[2 * j + 1][e], oacc[2 * j + 1][2 + e]);
    }
  };
  if constexpr (CL > 0) {
    cluster_combine<CL, NW>(smem_raw, warp, lane, G, reinterpret_cast<__nv_bfloat16*>(a.out) + ((int64_t)b * a.H + h) * G * kD, park);
    return;
  }
  __syncwarp();  // the ring is read: the partial takes its place, and leaves in whole rows
  float* const part = reinterpret_cast<float*>(mine);
  park(part);
  __syncwarp();
  float4* const dst = reinterpret_cast<float4*>(a.partial + (gw + (int64_t)b * a.H + h) * G * kPartial);
  for (int i = lane; i < G * (kPartial / 4); i += 32) dst[i] = reinterpret_cast<const float4*>(part)[i];
  share -= ntiles;
  if (share <= 0) return;
  __syncwarp();
  tile0 = 0;
  if (++h == a.H) {
    h = 0;
    do view = views[++b];
    while (view.len <= 0);  // (tiles are left, so a later sequence has some)
  }
  }
}

// One CTA per (sequence, query head) joins the partials of the stretches that cover its pair: its W warps take every W-th, a
// lane owns four columns, and the loads of four partials are in flight at once.  The host gives each warp four or so: few pairs
// are spread over many stretches (8 pairs of 131072 tokens over 296 each: 38 us with 32 warps, 50 with eight).
constexpr int kQCombThreads = 1024;

__global__ void __launch_bounds__(kQCombThreads) quant_combine_kernel(const QuantArgs qa_) {
  const int W = blockDim.x / 32;
  __shared__ float2 s_ml[kQCombThreads / 32];
  __shared__ float4 s_out[kQCombThreads / 32][32];
  const DecodeArgs& a = qa_.d;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x, pair = row / a.G, b = pair / a.H, h = pair - b * a.H;
  griddep_wait();
  griddep_launch();
  const int t0 = qa_.plan[b], tiles = qa_.plan[b + 1] - t0, share = qa_.plan[a.Bz + 1];
  const int first = t0 * a.H + h * tiles;                // of all tiles, in the order of the pairs
  const int w0 = first / share, n = tiles > 0 ? (first + tiles - 1) / share - w0 + 1 : 0;
  const int64_t step = (int64_t)a.G * kPartial;
  const float* p = a.partial + ((int64_t)(w0 + pair) * a.G + (row - pair * a.G)) * kPartial;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, float4 y) {  // out, max and sum of one more partial
    const float mm = fmaxf(m, ml.x);
    if (mm == -INFINITY && !(ml.y != 0.f)) return;  // (no tokens, or only tokens of weight zero)
    const float c = m == -INFINITY ? 0.f : exp2f(m - mm), f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mm);
    o.x = fmaf(f, y.x, o.x * c); o.y = fmaf(f, y.y, o.y * c); o.z = fmaf(f, y.z, o.z * c); o.w = fmaf(f, y.w, o.w * c);
    l = fmaf(f, ml.y, l * c);
    m = mm;
  };
  for (int s = warp; s < n; s += 4 * W) {
    float2 ml[4];
    float4 y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool ok = s + u * W < n;
      const float* r = p + (s + u * W) * step;
      ml[u] = ok ? *reinterpret_cast<const float2*>(r + kD) : make_float2(-INFINITY, 0.f);
      y[u] = ok ? *reinterpret_cast<const float4*>(r + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) add(ml[u], y[u]);
  }
  s_out[warp][lane] = o;
  if (lane == 0) s_ml[warp] = make_float2(m, l);
  __syncthreads();
  if (warp == 0) {
    const float2 ml = lane < W ? s_ml[lane] : make_float2(-INFINITY, 0.f);
    m = warp_max(ml.x);
    const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - m);
    l = warp_sum(f * ml.y);
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int w = 0; w < W; ++w) {
      const float fw = __shfl_sync(0xffffffffu, f, w);
      const float4 y = s_out[w][lane];
      o.x = fmaf(fw, y.x, o.x); o.y = fmaf(fw, y.y, o.y); o.z = fmaf(fw, y.z, o.z); o.w = fmaf(fw, y.w, o.w);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    store4(reinterpret_cast<__nv_bfloat16*>(a.out) + (int64_t)row * kD + lane * 4, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  }
}

// Sets the kernel's shared memory (and a cluster size above 8) once per device; how many clusters fit at once, 0: none
template <int CL, bool HALF>
int quant_clusters() {
  constexpr int NW = CL > 0 ? kQClusterWarps : kQShareWarps, kSmem = NW * quant_warp_bytes(CL > 0 ? kQClusterStages : kQShareStages);
  constexpr int kMaxDev = 64;
  static std::atomic<int> cached[kMaxDev];  // 0 = not asked yet, else the answer + 1
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDev) return 0;
  if ((n = cached[dev].load(std::memory_order_relaxed)) > 0) return n - 1;
  auto kern = decode_quant_kernel<CL, HALF>;
  bool ok = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) == cudaSuccess;
  if (ok && CL > 8) ok = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
  if (ok && CL == 0) n = 1;
  if (ok && CL > 0) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(CL, 1, 1);
    cfg.blockDim = dim3(NW * 32);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CL;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
      n = 0;
      cudaGetLastError();  // a refusal here only means "not this cluster size"
    }
  }
  cached[dev].store(n + 1, std::memory_order_relaxed);
  return n;
}

// CTAs of the launch by shares: one per SM, or one per tile where max_len says that there are fewer
int64_t quant_ctas(int32_t Bz, int32_t H, int64_t max_len) {
  const int64_t sms = sm_count(), tiles = std::min<int64_t>(max_len / kQT + (max_len % kQT ? 1 : 0), sms);
  return std::max<int64_t>(1, std::min<int64_t>(sms, std::min<int64_t>((int64_t)Bz * H, sms) * tiles));
}

inline size_t quant_plan_bytes(int32_t Bz) { return ((size_t)(Bz + 2) * 4 + 255) / 256 * 256; }

template <int CL, bool HALF>
cudaError_t launch_quant(const QuantArgs& a, cudaStream_t st) {
  constexpr int NW = CL > 0 ? kQClusterWarps : kQShareWarps;
  if (quant_clusters<CL, HALF>() < 1) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = CL > 0 ? dim3(CL, (unsigned)a.d.H, (unsigned)a.d.Bz) : dim3((unsigned)quant_ctas(a.d.Bz, a.d.H, a.d.max_len));
  cfg.blockDim = dim3(NW * 32);
  cfg.dynamicSmemBytes = NW * quant_warp_bytes(CL > 0 ? kQClusterStages : kQShareStages);
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, decode_quant_kernel<CL, HALF>, a);
  if (e != cudaSuccess || CL > 0) return e;
  const int64_t pairs = (int64_t)a.d.Bz * a.d.H, each = quant_ctas(a.d.Bz, a.d.H, a.d.max_len) * kQShareWarps / pairs;  // stretches per pair
  const int warps = each > 64 ? 32 : each > 32 ? 16 : each > 16 ? 8 : 4;
  return launch_dependent(quant_combine_kernel, dim3((unsigned)(pairs * a.d.G)), dim3(warps * 32), 0, st, a);
}

template <bool HALF>
cudaError_t launch_quant_heads(const QuantArgs& a, cudaStream_t st) {
  // Few pairs: one cluster each, the largest of which all are resident at once, unless the sequences are so long that the
  // SMs a cluster cannot use (all but 80 of 148 for 8 pairs) count for more than the second kernel (about 3 us).  8 pairs
  // of 8000 tokens: 10.7 us by clusters, 11.6 by shares; of 16416: 14.5 both; of 33000: 22.0 and 18.0.
  const int64_t pairs = (int64_t)a.d.Bz * a.d.H, tiles = (a.d.max_len + kQT - 1) / kQT;
  auto fits = [&](int clusters, int cl) { return clusters >= pairs && tiles <= (int64_t)64 * cl; };
  if (fits(quant_clusters<16, HALF>(), 16)) return launch_quant<16, HALF>(a, st);
  if (fits(quant_clusters<10, HALF>(), 10)) return launch_quant<10, HALF>(a, st);
  if (fits(quant_clusters<8, HALF>(), 8)) return launch_quant<8, HALF>(a, st);
  return launch_quant<0, HALF>(a, st);
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
  if (n_rows > INT32_MAX / rows->H) return CKV_ERR_UNSUPPORTED;  // (2^31 rows of a pool: 290 GB)
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto kernel, int rows_per_cta) {
    const dim3 grid((unsigned)((n + rows_per_cta - 1) / rows_per_cta), (unsigned)rows->H);
    return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, stream, r, slots, n, *pool, n_rows, (int32_t)shift);
  };
  // a half warp takes several rows once that fills the SMs, four of bf16 (32749 tokens x 8 heads: 32 us, with one row 39) or two
  // of fp32, which are as many bytes in flight (47 and 49; four rows 49); of 1200 tokens one row each is faster, 3.0 and 3.4
  const bool many = n * rows->H >= (int64_t)128 * sm_count();
  const cudaError_t e = rows->dtype == CKV_F32 ? (many ? go(pages_quantize_kernel<true, 2>, 32) : go(pages_quantize_kernel<true, 1>, 16))
                                               : (many ? go(pages_quantize_kernel<false, 4>, 64) : go(pages_quantize_kernel<false, 1>, 16));
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

int ckv_pages_dequantize(const int32_t* block_table, int64_t len, const ckv_quant_pool* pool, int32_t page_tokens, int32_t H, int32_t D,
                         int32_t dtype, void* k, void* v, int32_t* deg, float* logdeg, int64_t cap, void* cuda_stream) {
  if (!block_table || !k || !v || len < 0 || H <= 0 || cap < len) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  int st = check_pool(pool);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (deg && pool->logdeg_pages && !pool->deg_pages) return CKV_ERR_INVALID_ARG;  // (the degrees are known by their logarithms only)
  if (shift < 0 || D != kD || H > 65535) return CKV_ERR_UNSUPPORTED;
  if (!aligned16(k) || !aligned16(v)) return CKV_ERR_ALIGNMENT;
  if (len == 0) return CKV_OK;
  DequantArgs a{};
  a.table = block_table; a.len = len; a.cap = cap; a.pool = *pool; a.k = k; a.v = v; a.deg = deg; a.logdeg = logdeg; a.H = H; a.shift = shift;
  // writes are what counts, and one row per half warp gives the shortest chains before them; two of bf16 for many rows (32749
  // tokens x 8 heads: 30.1 us, one row 31.6, four 33; of 3000 tokens: 4.2, 3.6, 4.1); fp32 by one row always (48.6, by two 49.4)
  const bool many = dtype == CKV_BF16 && len * H >= (int64_t)512 * sm_count();
  const int rows = many ? 32 : 16;
  const int64_t ctas = (len + rows - 1) / rows;
  if (ctas > INT32_MAX) return CKV_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)ctas, (unsigned)H);
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, stream, a); };
  const cudaError_t e = dtype == CKV_F32 ? go(pages_dequantize_kernel<true, 1>)
                                         : (many ? go(pages_dequantize_kernel<false, 2>) : go(pages_dequantize_kernel<false, 1>));
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

size_t ckv_decode_quantized_workspace_bytes(int32_t Bz, int32_t H, int32_t G, int32_t D, int64_t max_len) {
  if (Bz <= 0 || H <= 0 || G <= 0 || D <= 0 || max_len < 0) return 0;
  const size_t stretches = (size_t)quant_ctas(Bz, H, max_len) * kQShareWarps + (size_t)Bz * H;
  return quant_plan_bytes(Bz) + (stretches * G * kPartial * sizeof(float) + 255) / 256 * 256;
}

int ckv_decode_attn_quantized(const ckv_paged_view* views_dev, const ckv_quant_pool* pool, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G,
                              int32_t D, int32_t dtype, const void* q, void* out, float scale, int64_t max_len, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
  if (!views_dev || !q || !out || Bz <= 0 || H <= 0 || G <= 0 || max_len < 0) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  int st = check_pool(pool);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (dtype != CKV_BF16 || shift < 0 || D != kD || G > 8 || H > 65535 || Bz > 65535 || (int64_t)Bz * H * G > INT32_MAX ||
      max_len > (((int64_t)1 << 36) - 1) / ((int64_t)Bz * H) - kQT)  // (tiles of all pairs are counted in 31 bits)
    return CKV_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(out)) return CKV_ERR_ALIGNMENT;
  const size_t need = ckv_decode_quantized_workspace_bytes(Bz, H, G, D, max_len);
  if (!workspace || workspace_bytes < need || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  QuantArgs a{};
  a.d.views = views_dev; a.d.q = q; a.d.out = out;
  a.plan = static_cast<int32_t*>(workspace);
  a.d.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + quant_plan_bytes(Bz));
  a.d.Bz = Bz; a.d.H = H; a.d.G = G;
  a.d.max_len = max_len;
  a.d.scale = scale;
  a.d.page_shift = shift;
  a.pool = *pool;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = G <= 4 ? launch_quant_heads<true>(a, stream) : launch_quant_heads<false>(a, stream);
  return e == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // extern "C"
