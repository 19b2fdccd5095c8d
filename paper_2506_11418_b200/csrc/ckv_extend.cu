// Attention of a chunk of new tokens over a paged cache (bf16 or four-bit pages): ckv_extend_attn_paged, ckv_extend_attn_quantized.
//
// Rows.  The new tokens of a sequence and the G query heads of one KV head are the rows of one problem: row r of a tile is token
// r / G, head r % G, T = 128 / G tokens in a tile of 128 rows, so every key and value that is fetched serves all of them.  An
// item is two tiles of consecutive tokens of one (sequence, KV head) and the slots that the last of them sees.
//
// One CTA per SM, persistent.  S = Q K^T and O += P V run on tcgen05.mma (128 x 128 x 16, operands in shared memory with the
// 128-byte swizzle, P read from tensor memory), slots in steps of 128:
//   warps 0-3, 4-7  softmax of tile 0 and of tile 1, a row per thread: S from tensor memory, weights e^(scale (s - m)) to bf16
//                   over S's place, their sum in fp32 registers.  m is the largest s when the tile's rows began,
//                   and moves (the row of O is then scaled in tensor memory) only when a later one would weigh
//                   more than 2^kSlack, so that O is rarely touched.  The log-degree is in s already (warp 11).
//   warp 8          walks the CTA's work and passes it on; TMA: the item's queries and log-degrees, and keys and values through a ring
//                   of four 32 KB stages
//   warp 9          issues the MMAs: PV of one tile and the next QK^T of it while the other tile's softmax runs
//   warp 10         bf16 pages: values behind an item's last slot to zero; four-bit pages: copies codes and scales as they are
//   warp 11         log-degrees as three more columns of K
//   warps 12-19     over four-bit pages only: codes and scales to bf16 tiles, slots behind the last to zero
// Tensor memory: S0 | S1 | O0 | O1, 128 columns each, all 512.
// An item with one tile only (single tokens, short chunks) uses the second set for every other step of slots: two softmax
// states of the same rows, joined at the end.  Otherwise such an item would wait for its softmax at every step.
//
// Sharing the work.  All items' lengths (slots, three quarters of them where there is one tile, + kItemCost each) are laid end to end, in the order (sequence, KV head, tile
// pair), and every CTA takes an equal stretch, wherever it begins and ends, so a ragged batch, few rows over a long cache and
// many rows are all balanced to a step.  (Of one large chunk, whole items are dealt first: see there.)  Each CTA finds its stretch
// by itself from lengths on the device: the sum over a sequence's items is an arithmetic series.  A piece that is not a whole item leaves (O, m, sum) in the workspace, and extend_join_kernel
// joins them, in order, so results do not depend on timing.
//
// What bounds it.  A step of a pair of tiles is 2176 cycles of the tensor core and, for each tile, about 2000 of softmax with its two
// products behind it, so the tensor core is busy for 62 % (3440 cycles per step).  2048 tokens over 32768 slots, 8 x 4 heads: 878 us =
// 1214 TFLOP/s, 0.75 of a plain matrix product's burst rate at an SM clock of 1.7 GHz (power); an item's start and end take some 6000
// cycles (eight prompts of 100 to 2048 tokens: 122 us, 590 TFLOP/s).  Over four-bit pages the unpacking bounds it: 1024 tokens over 32768
// slots 557 us = 971 TFLOP/s, 32 sequences of 4097 to 16384 slots with five tokens each 241 us.
//
// Waits are bounded; one that gives up sets the status word at the start of the workspace, and the other roles follow.
#include <cuda.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/ckv.h"
#include "ckv_common.cuh"
#include "ckv_decode.cuh"
#include "ckv_internal.h"
#include "ckv_ptx.cuh"

namespace ckv {
namespace {

using namespace ptx;

constexpr int kED = 128;            // head_dim
constexpr int kEN = 128;            // slots per step; rows per tile
constexpr int kEStages = 4;         // bf16 tiles in flight: keys in the even ones, values in the odd
constexpr int kERawSlots = 2;       // four-bit pages: tiles as they are, keys and values in turn
constexpr int kETile = kEN * kED * 2;
constexpr int kEHalf = kETile / 2;  // 64 columns of a tile: 128 rows of 128 bytes
constexpr int kEBiasSlots = 4;
// Threads and registers: two softmax warps, one of warps 8-11 and, over four-bit pages, two that unpack on each quarter of an SM;
// their shares add up to what the block is launched with (3 x 168, 5 x 96).
template <bool QUANT> constexpr int kEWarps = QUANT ? 20 : 12;
template <bool QUANT> constexpr int kESoftmaxRegs = QUANT ? 160 : 216;
template <bool QUANT> constexpr int kEOtherRegs = QUANT ? 64 : 72;
constexpr int kEUnpackRegs = 48, kEUnpackWarps = 8;
constexpr int kItemCost = 320;      // what an item costs beside its slots (queries in, rows out), in slots (eight prompts: 124 us, with 128 142)
constexpr int kMinShare = 256;      // slots that a CTA takes at least (17 tokens over 4113 slots: 20.4 us, with 192 21.7, with 512 22.1)
constexpr float kSlack = 8.f;       // weights below 2^8
constexpr int kMaxStarts = 220;     // CTAs whose stretches' begins fit beside the sums
constexpr int kPartRow = 132;       // floats of a partial row: O, m, sum, pad; a piece's rows lie side by side, four floats of each
// shared memory, from a 1024-byte boundary
constexpr int oQ = 0;
constexpr int oRing = oQ + 2 * kETile;
constexpr int oBias = oRing + kEStages * kETile;
constexpr int oAug = oBias + kEBiasSlots * kEN * 4;       // 16 bytes per slot: its log-degree in three bf16, kEBiasSlots steps
constexpr int oOnes = oAug + kEBiasSlots * kEN * 16;       // 16 bytes per row of Q: three ones
constexpr int oZero = oOnes + kEN * 16;                    // the other eight columns of both
constexpr int oState = oZero + kEN * 16;  // float2 [256]: m and sum of every row, exchanged by one-tile items
constexpr int kERaw = kEN * (64 + 4);                      // codes and scales of one tile
constexpr int oRaw = oState + 256 * 8;
constexpr int oBar = oRaw + kERawSlots * kERaw;
constexpr int oPieces = oBar + 512;
constexpr int oMisc = oPieces + 256;
constexpr int kEBytes = oMisc + 128;

struct ExtendArgs {
  const ckv_paged_view* views;
  const int64_t* q_begin;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const __nv_bfloat16* k_pages;
  const __nv_bfloat16* v_pages;
  ckv_quant_pool pool;
  const float* logdeg;
  int64_t n_rows, max_slots, q_row, q_head;  // (strides in elements)
  int32_t Bz, H, G, T, shift;
  float scale;          // above zero
  uint32_t desc_qk;     // (a negative scale negates Q)
  int32_t* status;      // workspace: status word | pieces [CTAs] | partial rows
  struct ExtendPiece* pieces;
  float* partial;       // [2 CTAs][slot_rows][kPartRow]
  int32_t slot_rows;
};

// What the joining kernel needs to know of a CTA's stretch.  Slot 1 of a CTA holds a piece of the item that begins in its
// stretch and does not end there, slot 0 one of the item that began in an earlier CTA's.
struct ExtendPiece {
  int64_t row0;      // the item that this CTA ends and did not begin: its first row of q,
  int32_t h, ntok;   // KV head, tokens (0: there is none),
  int32_t first;     // and the CTA that began it
  int32_t held[2];   // whether the slots hold something
};

// One sequence's part of the work
template <bool DEAL>
struct ExtendSeq {
  int64_t row0;   // first of its rows of q
  int32_t n;      // new tokens
  int32_t len;    // slots
  __device__ __forceinline__ int items(int T2) const { return (n + T2 - 1) / T2; }
  // slots that item j's last token sees
  __device__ __forceinline__ int end(int j, int T2) const { return max(0, len - n + min((j + 1) * T2, n)); }
  // Whether item j has one tile of rows (only a sequence's last may), and what its slots then count: a step of it takes 1.4 us next to 2.0,
  // over four-bit pages 1.7 next to 2.3 (four chunks among twelve single tokens: 380 us, counted alike 395).
  // A sequence whose items are dealt has too few of them to matter.
  __device__ __forceinline__ bool one(int j, int T2) const { return n - j * T2 <= T2 / 2; }
  __host__ __device__ __forceinline__ static constexpr int weigh(int slots, bool one) { return one && !DEAL ? slots - slots / 4 : slots; }
  // cost of items 0 .. m - 1 of one head
  __device__ __forceinline__ int64_t before(int m, int T2) const {
    const int base = len - n, last = items(T2) - 1;
    const int j0 = base >= 0 ? 0 : -base / T2, e = max(min(m, last), j0);
    int64_t c = (int64_t)m * kItemCost + (int64_t)(e - j0) * base + (int64_t)T2 * (((int64_t)e * (e + 1) - (int64_t)j0 * (j0 + 1)) / 2);
    if (m > last) c += weigh(len, one(last, T2));
    return c;
  }
};

template <bool DEAL>
__device__ __forceinline__ ExtendSeq<DEAL> extend_seq(const ExtendArgs& a, int b) {
  ExtendSeq<DEAL> s;
  const int64_t r0 = min(max(a.q_begin[b], (int64_t)0), a.n_rows), r1 = min(max(a.q_begin[b + 1], r0), a.n_rows);
  s.row0 = r0;
  s.n = (int32_t)(r1 - r0);
  s.len = (int32_t)min(max(a.views[b].len, (int64_t)0), a.max_slots);
  return s;
}

// A piece of an item: steps lo .. hi - 1 of its slots.  The TMA warp walks the CTA's stretch and passes its pieces to the other warps
// through a ring in shared memory.
constexpr int kEPieces = 4;
enum : int { kOneTile = 1, kWhole = 2, kFirst = 4, kStop = 8 };
struct __align__(16) Piece {
  int64_t row0;   // first row of q
  int h, ntok;    // KV head, tokens
  int base, end;  // slot at which the item's first token stands, slots that its last token sees
  int lo, hi;
  int flags;      // one tile of rows; the whole item; the item begins in this stretch; there is no piece any more
  int seq;
};

template <bool DEAL>
struct Walk {
  int64_t left, x;  // what is left of the stretch; offset in the item
  ExtendSeq<DEAL> s;
  int b, h, j;
  int dealt, item;  // whole items that come before the stretch (one sequence only), and the next of them
  // the next piece that has something to do
  __device__ __forceinline__ bool next(const ExtendArgs& a, Piece& p) {
    const int T2 = 2 * a.T;
    while ((DEAL && dealt > 0) || left > 0) {
      const bool deal = DEAL && dealt > 0;
      const int items = s.items(T2), at_h = deal ? item / items : h, at_j = deal ? item - at_h * items : j;
      const int end = s.end(at_j, T2), steps = (end + kEN - 1) / kEN;
      const bool one = s.one(at_j, T2);
      const int64_t cost = (int64_t)s.weigh(end, one) + kItemCost, from = deal ? 0 : x, to = deal ? cost : min(x + left, cost);
      auto step_of = [&](int64_t y) {
        const uint32_t z = (uint32_t)max(y - kItemCost, (int64_t)0);
        constexpr uint32_t S2 = kEN, S1 = ExtendSeq<DEAL>::weigh(kEN, true);
        return (int)min(one ? (z + S1 / 2) / S1 : (z + S2 / 2) / S2, (uint32_t)steps);
      };
      const bool ends = to == cost;
      p.lo = step_of(from);
      p.hi = ends ? steps : step_of(to);
      p.row0 = s.row0 + (int64_t)at_j * T2;
      p.h = at_h;
      p.ntok = min(T2, s.n - at_j * T2);
      p.base = s.len - s.n + at_j * T2;
      p.end = end;
      p.flags = (one ? kOneTile : 0) | (p.lo == 0 && p.hi == steps ? kWhole : 0) | (from == 0 ? kFirst : 0);
      p.seq = b;
      if (deal) {
        --dealt;
        item += gridDim.x;
      } else {
        left -= to - x;
        x = to;
        if (ends) {
          x = 0;
          if (++j >= items) {
            j = 0;
            if (++h == a.H) {
              h = 0;
              s.n = 0;
              while (left > 0 && s.n == 0) {  // (what is left belongs to a later sequence)
                if (++b < a.Bz)
                  s = extend_seq<DEAL>(a, b);
                else
                  left = 0;
              }
            }
          }
        }
      }
      if (p.lo < p.hi || (steps == 0 && ends)) return true;
    }
    return false;
  }
};

__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// D[tmem] (+)= A[tmem] * B[smem desc]
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// eight columns
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 128 columns of 32 lanes into registers, and the wait in the same statement (no use can move above it)
__device__ __forceinline__ void tmem_ld128(uint32_t taddr, float (&v)[128]) {
  asm volatile(
      "{\n\t.reg .b32 t1, t2, t3;\n\t"
      "add.u32 t1, %128, 32;\n\tadd.u32 t2, %128, 64;\n\tadd.u32 t3, %128, 96;\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%128];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
      "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [t1];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%64,%65,%66,%67,%68,%69,%70,%71,%72,%73,%74,%75,%76,%77,%78,%79,"
      "%80,%81,%82,%83,%84,%85,%86,%87,%88,%89,%90,%91,%92,%93,%94,%95}, [t2];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%96,%97,%98,%99,%100,%101,%102,%103,%104,%105,%106,%107,%108,%109,%110,%111,"
      "%112,%113,%114,%115,%116,%117,%118,%119,%120,%121,%122,%123,%124,%125,%126,%127}, [t3];\n\t"
      "tcgen05.wait::ld.sync.aligned;\n\t}"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31]),
        "=f"(v[32]), "=f"(v[33]), "=f"(v[34]), "=f"(v[35]), "=f"(v[36]), "=f"(v[37]), "=f"(v[38]), "=f"(v[39]),
        "=f"(v[40]), "=f"(v[41]), "=f"(v[42]), "=f"(v[43]), "=f"(v[44]), "=f"(v[45]), "=f"(v[46]), "=f"(v[47]),
        "=f"(v[48]), "=f"(v[49]), "=f"(v[50]), "=f"(v[51]), "=f"(v[52]), "=f"(v[53]), "=f"(v[54]), "=f"(v[55]),
        "=f"(v[56]), "=f"(v[57]), "=f"(v[58]), "=f"(v[59]), "=f"(v[60]), "=f"(v[61]), "=f"(v[62]), "=f"(v[63]),
        "=f"(v[64]), "=f"(v[65]), "=f"(v[66]), "=f"(v[67]), "=f"(v[68]), "=f"(v[69]), "=f"(v[70]), "=f"(v[71]),
        "=f"(v[72]), "=f"(v[73]), "=f"(v[74]), "=f"(v[75]), "=f"(v[76]), "=f"(v[77]), "=f"(v[78]), "=f"(v[79]),
        "=f"(v[80]), "=f"(v[81]), "=f"(v[82]), "=f"(v[83]), "=f"(v[84]), "=f"(v[85]), "=f"(v[86]), "=f"(v[87]),
        "=f"(v[88]), "=f"(v[89]), "=f"(v[90]), "=f"(v[91]), "=f"(v[92]), "=f"(v[93]), "=f"(v[94]), "=f"(v[95]),
        "=f"(v[96]), "=f"(v[97]), "=f"(v[98]), "=f"(v[99]), "=f"(v[100]), "=f"(v[101]), "=f"(v[102]), "=f"(v[103]),
        "=f"(v[104]), "=f"(v[105]), "=f"(v[106]), "=f"(v[107]), "=f"(v[108]), "=f"(v[109]), "=f"(v[110]), "=f"(v[111]),
        "=f"(v[112]), "=f"(v[113]), "=f"(v[114]), "=f"(v[115]), "=f"(v[116]), "=f"(v[117]), "=f"(v[118]), "=f"(v[119]),
        "=f"(v[120]), "=f"(v[121]), "=f"(v[122]), "=f"(v[123]), "=f"(v[124]), "=f"(v[125]), "=f"(v[126]), "=f"(v[127])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
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

// tcgen05 instruction descriptors: bf16 x bf16 -> fp32, M = N = 128; B K-major (keys) or N-major (values)
constexpr uint32_t kDescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t kNegateA = 1u << 13;
constexpr uint32_t kDescPV = kDescQK | (1u << 16);

template <int N>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Shared-memory matrix descriptor of an operand without swizzle
__device__ __forceinline__ uint64_t umma_desc_plain(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return (uint64_t)((smem_addr >> 4) & 0x3fffu) | ((uint64_t)((lbo_bytes >> 4) & 0x3fffu) << 16) | ((uint64_t)((sbo_bytes >> 4) & 0x3fffu) << 32) | (1ull << 46);
}
// 32 bytes, a whole sector
__device__ __forceinline__ void st_global_v8(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p) : "memory"); }
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// one arrival of every lane once its copies so far are there
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
  return ok != 0;
}

// Bounded wait.  A poll sleeps until the barrier's phase ends or some time has passed (4 us were measured), so that the warps that wait
// (most of the time there are eight) do not take issue slots from those that compute.  The limit is about four seconds: a warp that
// forms rows anew (values that are not finite) may take long.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kSpinLimit / 4; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(1000u)
        : "memory");
    if (ok) return true;
  }
  return false;
}

__device__ __forceinline__ uint32_t ld_shared_u32(uint32_t addr) {
  uint32_t x;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
  return x;
}
// Four scale bytes as pairs of equal bf16: 2^(byte - 127), 255 NaN
__device__ __forceinline__ void scales_bf16x2(uint32_t w, uint32_t (&out)[4]) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %0, a;\n\t"
      "cvt.rn.bf16x2.ue8m0x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
  out[0] = __byte_perm(lo, lo, 0x1010); out[1] = __byte_perm(lo, lo, 0x3232);
  out[2] = __byte_perm(hi, hi, 0x1010); out[3] = __byte_perm(hi, hi, 0x3232);
}
// Eight e2m1 codes, lowest four bits first, times a power of two: bf16, exactly.  The eight levels' bytes are looked up four codes at a time
// (__byte_perm takes three bits of a code as an index); signs are moved beside them.
__device__ __forceinline__ void unpack8_bf16(uint32_t w, uint32_t scale, uint32_t (&out)[4]) {
  constexpr uint32_t lo0 = 0xc0800000u, lo1 = 0xc0804000u;  // 0, 0.5, 1, 1.5 and 2, 3, 4, 6: low bytes of 0000 3f00 3f80 3fc0, 4000 4040 4080 40c0
  constexpr uint32_t hi0 = 0x3f3f3f00u, hi1 = 0x40404040u;  // and high ones
  const uint32_t even = (w << 4) & 0x80808080u, odd = w & 0x80808080u;  // signs of codes 0 2 4 6, 1 3 5 7, one per byte
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t sel = (w >> (16 * k)) & 0x7777u;
    const uint32_t lo = __byte_perm(lo0, lo1, sel), hi = __byte_perm(hi0, hi1, sel) | __byte_perm(even, odd, k ? 0x7362 : 0x5140);
    const uint32_t a = __byte_perm(lo, hi, 0x5140), b = __byte_perm(lo, hi, 0x7362);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(out[2 * k]) : "r"(a), "r"(scale));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(out[2 * k + 1]) : "r"(b), "r"(scale));
  }
}

// A warp's wait: false if any lane gave up
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, bar_wait(bar, parity)); }

// Elements 4 lane .. 4 lane + 3 of a row of keys or values
template <bool QUANT>
__device__ __forceinline__ float4 row4(const ExtendArgs& a, int64_t row, bool value, int lane) {
  if constexpr (!QUANT) {
    return load4((value ? a.v_pages : a.k_pages) + row * kED + 4 * lane);
  } else {
    const int j = lane >> 3, u = lane & 7;
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>((value ? a.pool.v_codes : a.pool.k_codes) + row * 64);
    const uint32_t w = value ? codes[2 * u + (j >> 1)] >> (16 * (j & 1)) : codes[4 * (u >> 1) + j] >> (16 * (u & 1));
    const uint32_t s = (value ? a.pool.v_scales : a.pool.k_scales)[row * 4 + j];
    uint32_t scale[4], x[4];
    scales_bf16x2(s, scale);
    unpack8_bf16(w & 0xffffu, scale[0], x);
    return make_float4(__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16), __uint_as_float(x[1] & 0xffff0000u));
  }
}

// DEAL: one sequence, and rows enough for an item per CTA
template <bool QUANT, bool DEAL>
__global__ void __launch_bounds__(kEWarps<QUANT> * 32, 1) extend_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                                                              const __grid_constant__ CUtensorMap tm_v, const ExtendArgs a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t s0 = smem_u32(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // barriers: full [stage] | empty [stage] | log-degrees full, free, in bf16, free [slot] | S full [tile] | P full [tile, half] | O full [tile] | Q full, empty | exchange | values ready [stage / 2] | piece, free [slot] | codes, free [slot]
  auto bar = [&](int i) { return s0 + oBar + 8u * i; };
  auto b_full = [&](int i) { return bar(i); };
  auto b_empty = [&](int i) { return bar(kEStages + i); };
  auto b_bias = [&](int i) { return bar(2 * kEStages + i); };
  auto b_bias_free = [&](int i) { return bar(2 * kEStages + kEBiasSlots + i); };
  auto b_bias_ready = [&](int i) { return bar(2 * kEStages + 2 * kEBiasSlots + i); };
  auto b_aug_free = [&](int i) { return bar(2 * kEStages + 3 * kEBiasSlots + i); };
  constexpr int kRest = 2 * kEStages + 4 * kEBiasSlots;
  auto b_s = [&](int g) { return bar(kRest + g); };
  auto b_p = [&](int g, int half) { return bar(kRest + 2 + 2 * g + half); };  // (columns 0-63, 64-127)
  auto b_o = [&](int g) { return bar(kRest + 6 + g); };
  const uint32_t b_q = bar(kRest + 8), b_q_free = bar(kRest + 9), b_x = bar(kRest + 10);
  auto b_v = [&](int i) { return bar(kRest + 11 + i); };
  auto b_piece = [&](int i) { return bar(kRest + 11 + kEStages / 2 + i); };
  auto b_piece_free = [&](int i) { return bar(kRest + 11 + kEStages / 2 + kEPieces + i); };
  auto b_raw = [&](int i) { return bar(kRest + 11 + kEStages / 2 + 2 * kEPieces + i); };
  auto b_raw_free = [&](int i) { return bar(kRest + 11 + kEStages / 2 + 2 * kEPieces + kERawSlots + i); };
  Piece* const pieces = reinterpret_cast<Piece*>(smem + oPieces);
  int64_t* const s_start = reinterpret_cast<int64_t*>(smem + oMisc);            // the stretch's offset in its sequence, sequence
  int64_t* const s_sum = reinterpret_cast<int64_t*>(smem + oState);             // (before the roles begin)
  int64_t* const s_starts = s_sum + 32;
  volatile uint32_t* const s_tmem = reinterpret_cast<volatile uint32_t*>(smem + oMisc + 64);

  if (tid == 0) {
    for (int i = 0; i < kEStages; ++i) {
      mbar_init(b_full(i), QUANT ? kEUnpackWarps : 1);
      mbar_init(b_empty(i), 1);
    }
    for (int i = 0; i < kEBiasSlots; ++i) {
      mbar_init(b_bias(i), 1);
      mbar_init(b_bias_free(i), 1);
      mbar_init(b_bias_ready(i), 1);
      mbar_init(b_aug_free(i), 1);
    }
    for (int g = 0; g < 2; ++g) {
      mbar_init(b_s(g), 1);
      mbar_init(b_p(g, 0), 4);
      mbar_init(b_p(g, 1), 4);
      mbar_init(b_o(g), 1);
    }
    mbar_init(b_q, 1);
    mbar_init(b_q_free, 1);
    mbar_init(b_x, 8);
    for (int i = 0; i < kEStages / 2; ++i) mbar_init(b_v(i), 1);
    for (int i = 0; i < kERawSlots; ++i) {
      mbar_init(b_raw(i), 32);
      mbar_init(b_raw_free(i), kEUnpackWarps);
    }
    for (int i = 0; i < kEPieces; ++i) {
      mbar_init(b_piece(i), 1);
      mbar_init(b_piece_free(i), 10 + (QUANT ? kEUnpackWarps : 0) + (a.logdeg ? 1 : 0));  // softmax warps, MMA, unpacking warps, warps 10 and 11
    }
    mbar_init_fence();
    s_start[0] = -1;
    prefetch_map(&tm_q);
    if (!QUANT) {
      prefetch_map(&tm_k);
      prefetch_map(&tm_v);
    }
  }
  if (tid < kEN) {
    st_shared_v4(s0 + oOnes + tid * 16, make_uint4(0x3f803f80u, 0x00003f80u, 0, 0));
    st_shared_v4(s0 + oZero + tid * 16, make_uint4(0, 0, 0, 0));
    fence_async_smem();
  }
  if (warp == 9) tmem_alloc(s0 + oMisc + 64, 512);
  griddep_wait();
  griddep_launch();
  if (blockIdx.x == 0 && tid == 0) *a.status = 0;
  const int T2 = 2 * a.T;

  // this CTA's stretch: every thread sums a run of sequences
  constexpr int kThreads = kEWarps<QUANT> * 32;
  const int per = (a.Bz + kThreads - 1) / kThreads, q0 = min(a.Bz, tid * per), q1 = min(a.Bz, q0 + per);
  int64_t mine = 0;
  for (int b = q0; b < q1; ++b) {
    const ExtendSeq<DEAL> s = extend_seq<DEAL>(a, b);
    if (s.n > 0) mine += s.before(s.items(T2), T2) * a.H;
  }
  int64_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s_sum[warp] = upto;
  tc_fence_before();
  __syncthreads();
  int64_t total = 0, at = upto - mine;
  for (int w = 0; w < kEWarps<QUANT>; ++w) {
    if (w < warp) at += s_sum[w];
    total += s_sum[w];
  }
  const int64_t share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)kMinShare);
  int64_t begin = min(share * blockIdx.x, total), left = min(share, total - begin);
  // One sequence with more items than CTAs (a large chunk): as many items as an even share holds are dealt to the CTAs whole, in
  // turn, and only the rest is laid out in stretches.  CTAs then go through the same keys at the same time, and L2 has them (2048 tokens over
  // 32768 slots: 0.4 GB from memory in place of 1.9).
  int dealt = 0;
  if (DEAL && total > 0) {
    const ExtendSeq<DEAL> s = extend_seq<DEAL>(a, 0);
    const int items = s.items(T2), n = (int)gridDim.x;
    const int64_t of_head = s.before(items, T2);
    dealt = (int)min(total / n / (of_head - s.before(items - 1, T2)), (int64_t)items * a.H / n);  // (the last item of a head is the longest)
    if (dealt > 0) {
      int64_t whole = 0;
      if (tid < n)
        for (int w = 0; w < dealt; ++w) {
          const int j = (tid + w * n) % items;
          whole += s.before(j + 1, T2) - s.before(j, T2);
        }
      int64_t upto = whole;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      __syncthreads();
      if (lane == 31) s_sum[warp] = upto;
      __syncthreads();
      upto -= whole;
      for (int w = 0; w < warp; ++w) upto += s_sum[w];
      // where every CTA's stretch begins: behind the dealt items, after what is left of the even shares of the CTAs before
      const int64_t behind = (int64_t)(dealt * n / items) * of_head + s.before(dealt * n % items, T2);
      if (tid <= n) s_starts[tid] = behind + tid * total / n - upto;
      __syncthreads();
      begin = s_starts[blockIdx.x];
      left = s_starts[blockIdx.x + 1] - begin;
      if (tid == 0) {
        s_start[0] = begin;
        s_start[1] = 0;
      }
    }
  }
  if ((!DEAL || dealt == 0) && left > 0 && begin >= at && begin < at + mine) {
    for (int b = q0; b < q1; ++b) {
      const ExtendSeq<DEAL> s = extend_seq<DEAL>(a, b);
      if (s.n == 0) continue;
      const int64_t c = s.before(s.items(T2), T2) * a.H;
      if (begin < at + c) {
        s_start[0] = begin - at;
        s_start[1] = b;
        break;
      }
      at += c;
    }
  }
  __syncthreads();
  const int64_t offset = s_start[0];
  ExtendPiece* const mark = a.pieces + blockIdx.x;
  if (offset < 0) {  // no work
    if (tid == 0) *mark = ExtendPiece{0, 0, 0, 0, {0, 0}};
    if (warp == 9) tmem_dealloc(*s_tmem, 512);
    return;
  }
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  bool ok = true;
  // the other warps' side of the ring of pieces: the next one, or none; one arrival per warp gives a slot back
  int np = 0;
  auto next_piece = [&](auto wait) {
    if (!(ok = wait(b_piece(np % kEPieces), (uint32_t)((np / kEPieces) & 1)))) return false;
    return !(pieces[np % kEPieces].flags & kStop);
  };
  auto piece_done = [&] {
    mbar_arrive(b_piece_free(np % kEPieces));
    ++np;
  };

  if (QUANT && warp >= 12) {
    // ---------------------------------------------------------------- four-bit pages: codes and scales to bf16 tiles, exactly
    give_registers<kEUnpackRegs>();
    // Lane l has its row's 16-byte piece l % 4.  Of keys and values alike such a piece holds, for each of the row's four groups j,
    // elements 32 j + 8 (l % 4) .. + 7: 16 bytes of the tile.  The two rows that a store's eight lanes write differ in bit 2, which the
    // swizzle turns into the other half of the banks.
    const int w = warp - 12, piece = lane & 3, in8 = (lane >> 3) + 4 * ((lane >> 2) & 1);
    int idx = 0;
    while (next_piece(warp_wait)) {
      const int end = pieces[np % kEPieces].end, lo = pieces[np % kEPieces].lo, hi = pieces[np % kEPieces].hi;
      __syncwarp();
      if (lane == 0) piece_done(); else ++np;
      for (int i = 2 * lo; i < 2 * hi; ++i, ++idx) {  // keys, values, keys, ...
        const int seen = end - (i >> 1) * kEN, st = idx % kEStages, slot = idx % kERawSlots;
        const uint32_t from = s0 + oRaw + slot * kERaw, tile = s0 + oRing + (uint32_t)st * kETile;
        if (!(ok = warp_wait(b_raw(slot), (uint32_t)((idx / kERawSlots) & 1)) && warp_wait(b_empty(st), (uint32_t)(((idx / kEStages) & 1) ^ 1)))) break;
#pragma unroll 1
        for (int k = 0; k < kEN / (8 * kEUnpackWarps); ++k) {  // (not unrolled: the roles' code together would not stay in the instruction cache)
          const int r = (kEN / kEUnpackWarps) * w + 8 * k + in8;
          uint4 c;
          ld_shared_v4(from + r * 64 + piece * 16, c);
          uint32_t sc[4];
          scales_bf16x2(ld_shared_u32(from + kEN * 64 + r * 4), sc);
          if (r >= seen) {  // slots behind the last: zeros, whatever is there
            c = make_uint4(0, 0, 0, 0);
            sc[0] = sc[1] = sc[2] = sc[3] = 0;
          }
          uint32_t word[4] = {c.x, c.y, c.z, c.w};  // keys: word j has group j's eight codes; values: half words j and j + 4
          if (i & 1) {
            word[0] = __byte_perm(c.x, c.z, 0x5410); word[1] = __byte_perm(c.x, c.z, 0x7632);
            word[2] = __byte_perm(c.y, c.w, 0x5410); word[3] = __byte_perm(c.y, c.w, 0x7632);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t v[4];
            unpack8_bf16(word[j], sc[j], v);
            st_shared_v4(tile + (j >> 1) * kEHalf + r * 128 + ((((j & 1) * 4 + piece) ^ in8) << 4), make_uint4(v[0], v[1], v[2], v[3]));
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(b_raw_free(slot));
          mbar_arrive(b_full(st));
        }
      }
      if (!ok) break;
    }
  } else if (warp >= 8) {
  give_registers<kEOtherRegs<QUANT>>();
  if (warp == 8) {
    // ---------------------------------------------------------------- TMA, and the walk along the stretch
    Walk<DEAL> walk;
    walk.b = (int)s_start[1];
    walk.s = extend_seq<DEAL>(a, walk.b);
    walk.left = left;
    walk.dealt = dealt;
    walk.item = (int)blockIdx.x;
    walk.h = walk.j = 0;
    walk.x = 0;
    ExtendPiece note{0, 0, 0, 0, {0, 0}};
    if (left > 0) {
      const int items = walk.s.items(T2);
      const int64_t of_head = walk.s.before(items, T2);
      walk.h = (int)(offset / of_head);
      const int64_t in_head = offset - walk.h * of_head;
      int lo = 0, hi = items;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (walk.s.before(mid, T2) <= in_head) lo = mid; else hi = mid;
      }
      walk.j = lo;
      walk.x = in_head - walk.s.before(lo, T2);
      // the CTA in whose stretch this item begins: the last that does not begin behind it
      const int64_t item_begin = begin - walk.x;
      if (DEAL && dealt > 0) {
        note.first = -1;
        for (int c = 0; c < (int)gridDim.x; c += 32)
          note.first += __popc(__ballot_sync(0xffffffffu, c + lane < (int)gridDim.x && s_starts[c + lane] <= item_begin));
      } else {
        note.first = (int32_t)(item_begin / share);
      }
    }
    const int run = min(kEN, 1 << a.shift), runs = kEN / run;  // slots of a step that lie in one page
    const int rr = (lane >> 1) % runs, half = lane & 1;
    int n = 0, nq = 0;                                         // steps so far, pieces with steps
    Piece p;
    while (true) {
      const bool more = walk.next(a, p);
      if (!more) p.flags = kStop;
      if (!(ok = warp_wait(b_piece_free(np % kEPieces), (uint32_t)(((np / kEPieces) & 1) ^ 1)))) break;
      if (lane == 0) {
        pieces[np % kEPieces] = p;
        mbar_arrive(b_piece(np % kEPieces));
      }
      ++np;
      if (!more) break;
      if (!(p.flags & kWhole)) {
        note.held[p.flags & kFirst ? 1 : 0] = 1;
        if (p.lo > 0 && p.hi * kEN >= p.end) {  // it ends an item that it did not begin
          note.row0 = p.row0;
          note.h = p.h;
          note.ntok = p.ntok;
        }
      }
      const int32_t* const table = a.views[p.seq].block_table;
      const int n_blocks = (p.end + (1 << a.shift) - 1) >> a.shift;
      int win = -32;
      int32_t cur = 0, nxt = 0;
      for (int i = p.lo; i < p.hi; ++i, ++n) {
        const int t0 = i * kEN, blk0 = t0 >> a.shift;
        if ((blk0 & ~31) != win) {
          const bool first = win < 0 || (blk0 & ~31) != win + 32;
          win = blk0 & ~31;
          cur = first ? (win + lane < n_blocks ? table[win + lane] : 0) : nxt;
          nxt = win + 32 + lane < n_blocks ? table[win + 32 + lane] : 0;
        }
        const int slot = t0 + rr * run;                        // this lane's run of slots
        const int page = __shfl_sync(0xffffffffu, cur, (slot >> a.shift) & 31);
        const int row = ((page * a.H + p.h) << a.shift) + (slot & ((1 << a.shift) - 1));
        const int live = min(runs, (p.end - t0 + run - 1) / run);  // runs that hold something
        const bool mine_ = lane < 2 * runs && rr < live;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if constexpr (!QUANT) {
            const int idx = 2 * n + kv, st = idx % kEStages;
            if (!(ok = warp_wait(b_empty(st), (uint32_t)(((idx / kEStages) & 1) ^ 1)))) break;
            if (lane == 0) mbar_arrive_expect_tx(b_full(st), (uint32_t)(live * run * 256));
            __syncwarp();
            if (mine_) tma_load_2d(s0 + oRing + st * kETile + half * kEHalf + rr * run * 128, kv ? &tm_v : &tm_k, 64 * half, row, b_full(st));
          }
          if (kv == 0 && a.logdeg) {
            const int bs = n % kEBiasSlots;
            if (!(ok = warp_wait(b_bias_free(bs), (uint32_t)(((n / kEBiasSlots) & 1) ^ 1)))) break;
            if (lane == 0) mbar_arrive_expect_tx(b_bias(bs), (uint32_t)(live * run * 4));
            __syncwarp();
            if (mine_ && half == 0) bulk_load(s0 + oBias + (bs * kEN + rr * run) * 4, a.logdeg + row, run * 4, b_bias(bs));
          }
        }
        if (ok && i == p.lo) {  // the queries' place is free only when the last item's products are done: its first keys come before
          if (!(ok = warp_wait(b_q_free, (uint32_t)((nq++ & 1) ^ 1)))) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(b_q, (uint32_t)(4 * a.T * a.G * 128));
            for (int g = 0; g < 2; ++g)
              for (int f = 0; f < 2; ++f)
                tma_load_3d(s0 + oQ + g * kETile + f * kEHalf, &tm_q, 64 * f, p.h * a.G, (int)p.row0 + (p.flags & kOneTile ? 0 : g * a.T), b_q);
          }
        }
        if (!ok) break;
      }
      if (!ok) break;
    }
    if (lane == 0) *mark = note;
  } else if (warp == 9) {
    // ---------------------------------------------------------------- MMA: one thread
    if (elect_one()) {
      int n = 0, nq = 0;                     // steps, pieces with steps so far
      uint32_t par[2] = {0, 0};              // of P
      const uint64_t d_q = umma_desc_sw128(s0 + oQ, 16, 1024), d_k = umma_desc_sw128(s0 + oRing, 16, 1024), d_v = umma_desc_sw128(s0 + oRing, kEHalf, 1024);
      // (no swizzle: rows of 16 bytes, eight of them in 128; the second eight columns are the zeros, at the leading offset)
      const uint64_t d_ones = umma_desc_plain(s0 + oOnes, oZero - oOnes, 128), d_aug = umma_desc_plain(s0 + oAug, oZero - oAug, 128);
      constexpr uint64_t kAugStep = (uint64_t)(kEN * 16 >> 4) - ((uint64_t)(kEN * 16 >> 4) << 16);  // the next slot begins later: its zeros are nearer
      auto qk = [&](int g, int i) {          // S of tile g at the piece's step i, and its arrival
        const uint64_t dk = d_k + (uint64_t)((2 * (n + i)) % kEStages) * (kETile >> 4), dq = d_q + (uint64_t)g * (kETile >> 4);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const uint64_t off = (uint64_t)((ks >> 2) * (kEHalf >> 4) + (ks & 3) * 2);
          umma_bf16(tmem + (uint32_t)g * 128, dq + off, dk + off, a.desc_qk, ks ? 1u : 0u);
        }
        if (a.logdeg) umma_bf16(tmem + (uint32_t)g * 128, d_ones, d_aug + (uint64_t)((n + i) % kEBiasSlots) * kAugStep, kDescQK, 1u);
        umma_commit(b_s(g));
      };
      auto pv = [&](int g, int i, bool more) {
        const uint64_t dv = d_v + (uint64_t)((2 * (n + i) + 1) % kEStages) * (kETile >> 4);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {  // as the weights arrive
          if (!(ok = bar_wait(b_p(g, half), par[g]))) return;
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            umma_bf16_ts(tmem + 256 + (uint32_t)g * 128, tmem + (uint32_t)g * 128 + 32 * half + 8 * ks, dv + (uint64_t)(4 * half + ks) * 128, kDescPV,
                         (more || half || ks) ? 1u : 0u);
        }
        par[g] ^= 1;
      };
      auto stage_full = [&](int idx) { return bar_wait(b_full(idx % kEStages), (uint32_t)((idx / kEStages) & 1)); };
      auto keys = [&](int i) {               // of the piece's step i, and its log-degrees
        return stage_full(2 * (n + i)) &&
               (!a.logdeg || bar_wait(b_bias_ready((n + i) % kEBiasSlots), (uint32_t)(((n + i) / kEBiasSlots) & 1)));
      };
      auto values = [&](int i) {
        return QUANT ? stage_full(2 * (n + i) + 1) : bar_wait(b_v((n + i) % (kEStages / 2)), (uint32_t)(((n + i) / (kEStages / 2)) & 1));
      };
      while (next_piece(bar_wait)) {
        const int steps = pieces[np % kEPieces].hi - pieces[np % kEPieces].lo;
        const bool one = pieces[np % kEPieces].flags & kOneTile;
        piece_done();
        if (steps <= 0) continue;
        // Tiles of scores in the order of their products: of a pair's two tiles in turn, of a single one's steps in turn.  PV of tile j is
        // followed by QK^T of tile j + 2, which takes its place.
        const int tiles = one ? steps : 2 * steps;
        if (!(ok = bar_wait(b_q, (uint32_t)(nq++ & 1)))) break;
#pragma unroll 1
        for (int j = -2; j < tiles; ++j) {
          const int g = j & 1;
          if (j >= 0) {
            const int i = one ? j : j >> 1;
            if ((one || g == 0) && !(ok = values(i))) break;
            pv(g, i, j >= 2);
            if (!ok) break;
            if (one || g == 1) umma_commit(b_empty((2 * (n + i) + 1) % kEStages));
            if (!one && j >= tiles - 2) umma_commit(b_o(g));
          }
          if (j + 2 < tiles) {
            const int i = one ? j + 2 : (j + 2) >> 1;
            if ((one || g == 0) && !(ok = keys(i))) break;
            tc_fence_after();
            qk(g, i);
            if (one || g == 1) {
              umma_commit(b_empty(2 * (n + i) % kEStages));
              if (a.logdeg) umma_commit(b_aug_free((n + i) % kEBiasSlots));
            }
            if (j + 3 == tiles) umma_commit(b_q_free);
          }
        }
        if (!ok) break;
        if (one) {
          umma_commit(b_o(0));
          umma_commit(b_o(1));
        }
        n += steps;
      }
    }
  } else if (QUANT && warp == 10) {
    // ---------------------------------------------------------------- four-bit pages: codes and scales of a tile, as they are.  (Bulk copies of
    // a page's few KB each take about 50 ns to issue; these are 17 instructions per tile.)  What comes two steps later is
    // brought into L2.
    int n = 0;
    while (next_piece(warp_wait)) {
      const Piece& p = pieces[np % kEPieces];
      const int end = p.end, lo = p.lo, hi = p.hi, h = p.h;
      const int32_t* const table = a.views[p.seq].block_table;
      __syncwarp();
      if (lane == 0) piece_done(); else ++np;
      // rows of the pool at which the 32 slots of quarter lane / 8 of step i begin; none behind the last slot
      auto row_of = [&](int i) -> int {
        const int slot = i * kEN + 32 * (lane >> 3);
        return i < hi && slot < end ? ((table[slot >> a.shift] * a.H + h) << a.shift) + (slot & ((1 << a.shift) - 1)) : -1;
      };
      auto fetch_l2 = [&](int row) {
        if (row < 0) return;
        const int c = lane & 7;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const uint8_t* const codes = (kv ? a.pool.v_codes : a.pool.k_codes) + (int64_t)row * 64;
          prefetch_l2(codes + c * 128);
          prefetch_l2(codes + (c + 8) * 128);
          if (c == 0) prefetch_l2((kv ? a.pool.v_scales : a.pool.k_scales) + (int64_t)row * 4);
        }
      };
      int r0 = row_of(lo), r1 = row_of(lo + 1), r2 = row_of(lo + 2);
      fetch_l2(r1);
      for (int i = lo; i < hi; ++i, ++n) {
        fetch_l2(r2);
        const int r3 = row_of(i + 3);
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          const int slot = (2 * n + kv) % kERawSlots;
          if (!(ok = warp_wait(b_raw_free(slot), (uint32_t)((((2 * n + kv) / kERawSlots) & 1) ^ 1)))) break;
          const uint32_t to = s0 + oRaw + slot * kERaw + (lane >> 3) * 2048 + (lane & 7) * 16;
          const uint8_t* const codes = (kv ? a.pool.v_codes : a.pool.k_codes);
          const uint8_t* const from = codes + (r0 < 0 ? 0 : (int64_t)r0 * 64 + (lane & 7) * 16);
          const uint32_t bytes = r0 < 0 ? 0 : 16;
#pragma unroll
          for (int k = 0; k < 16; ++k) cp_async16(to + k * 128, from + (r0 < 0 ? 0 : k * 128), bytes);
          const uint8_t* const scales = kv ? a.pool.v_scales : a.pool.k_scales;
          cp_async16(s0 + oRaw + slot * kERaw + kEN * 64 + lane * 16, scales + (r0 < 0 ? 0 : (int64_t)r0 * 4 + (lane & 7) * 16), bytes);
          cp_async_arrive(b_raw(slot));
        }
        if (!ok) break;
        r0 = r1;
        r1 = r2;
        r2 = r3;
      }
      if (!ok) break;
    }
    cp_async_wait_all();
  } else if (warp == 10) {
    // ---------------------------------------------------------------- slots behind the last that an item sees: whatever their values
    // are, they must not meet a weight of zero
    int n = 0;
    while (next_piece(warp_wait)) {
      const int end = pieces[np % kEPieces].end, lo = pieces[np % kEPieces].lo, hi = pieces[np % kEPieces].hi;
      __syncwarp();
      if (lane == 0) piece_done(); else ++np;
      for (int i = lo; i < hi; ++i, ++n) {
        const int st = (2 * n + 1) % kEStages, seen = end - i * kEN;
        if (!(ok = warp_wait(b_full(st), (uint32_t)(((2 * n + 1) / kEStages) & 1)))) break;
        if (seen < kEN) {
          const uint32_t vt = s0 + oRing + (uint32_t)st * kETile;
          for (int c = seen * 8 + lane; c < kEN * 8; c += 32) {
            st_shared_v4(vt + c * 16, make_uint4(0, 0, 0, 0));
            st_shared_v4(vt + kEHalf + c * 16, make_uint4(0, 0, 0, 0));
          }
          fence_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b_v(st / 2));
      }
      if (!ok) break;
    }
  } else if (warp == 11 && a.logdeg) {
    // ---------------------------------------------------------------- log-degrees: three more columns of K, next to three ones in Q.  log n / |scale|
    // as the sum of three bf16 holds 24 bits of it.  What the type's largest values become stays finite, here and times
    // scale * log2 e: where a caller masks slots with them, scores minus their maximum have to be numbers.
    const float inv = 1.f / a.scale, most = fminf(3.3e38f, 3e38f / (a.scale * kLog2e));
    int n = 0;
    while (next_piece(warp_wait)) {
      const int steps = pieces[np % kEPieces].hi - pieces[np % kEPieces].lo;
      __syncwarp();
      if (lane == 0) piece_done(); else ++np;
      for (int i = 0; i < steps; ++i, ++n) {
        const int bs = n % kEBiasSlots;
        if (!(ok = warp_wait(b_bias(bs), (uint32_t)((n / kEBiasSlots) & 1)) && warp_wait(b_aug_free(bs), (uint32_t)(((n / kEBiasSlots) & 1) ^ 1)))) break;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int t = lane + 32 * k;
          const float x = reinterpret_cast<const float*>(smem + oBias)[bs * kEN + t];
          float b = x * inv;
          if (fabsf(b) > most && fabsf(x) != INFINITY) b = copysignf(most, b);
          const __nv_bfloat16 hi = __float2bfloat16_rn(b);
          const float r1 = fabsf(b) < INFINITY ? b - __bfloat162float(hi) : 0.f;
          const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
          st_shared_v4(s0 + oAug + (bs * kEN + t) * 16, make_uint4((uint32_t)__bfloat16_as_ushort(hi) | (uint32_t)__bfloat16_as_ushort(mid) << 16,
                                                                  pack_bf16x2(r1 - __bfloat162float(mid), 0.f), 0, 0));
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(b_bias_free(bs));
          mbar_arrive(b_bias_ready(bs));
        }
      }
      if (!ok) break;
    }
  }
  } else {
    // ---------------------------------------------------------------- softmax of tile g, one row per thread
    take_registers<kESoftmaxRegs<QUANT>>();
    const int g = warp >> 2, r = tid & 127, tok = r / a.G, head = r - tok * a.G;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // (32 lanes of tensor memory per warp, lane number in the upper half word)
    const uint32_t t_s = tmem + lanes + (uint32_t)g * 128, t_o = t_s + 256;
    float2* const state = reinterpret_cast<float2*>(smem + oState);
    const float scale = a.scale * kLog2e, slack = kSlack / scale;  // (a.scale is positive)
    int ns = 0, no = 0, nx = 0;  // own steps, pieces with steps, exchanges so far
    while (next_piece(warp_wait)) {
      const Piece& p = pieces[np % kEPieces];
      const int lo = p.lo, steps = p.hi - lo;
      const bool one = p.flags & kOneTile;
      const int my_tok = tok + (one ? 0 : g * a.T);
      const bool valid = tok < a.T && my_tok < p.ntok;
      const bool busy = __any_sync(0xffffffffu, valid);
      const int lim = valid ? p.base + my_tok + 1 - lo * kEN : 0;  // slots of the piece that this row sees
      const int lim_min = __reduce_min_sync(0xffffffffu, valid ? lim : INT32_MAX);
      float m = -INFINITY;
      f32x2 l2(0.f, 0.f);
      for (int i = 0; i < steps; ++i) {
        const bool own = !one || (i & 1) == g;
        if (own) {
          if (!(ok = warp_wait(b_s(g), (uint32_t)(ns++ & 1)))) break;
          tc_fence_after();
          // one step of this row; MASK: some row of the warp does not see all of the step's slots.  (Two copies of the code: with
          // the selection as a branch inside, the compiler moves all 128 registers around it.)
          auto step = [&](auto mask) {
            constexpr bool MASK = decltype(mask)::value;
            float y[128];
            tmem_ld128(t_s, y);
            if constexpr (MASK) {
              const int seen = lim - i * kEN;
#pragma unroll
              for (int c = 0; c < 128; ++c) y[c] = c < seen ? y[c] : -INFINITY;
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 128; c += 8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], y[c + 2 * k], y[c + 2 * k + 1]);
            }
            const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
            if (__any_sync(0xffffffffu, top > m + slack)) {
              const bool up = top > m;
              const float f = up ? ex2((m - top) * scale) : 1.f;
              if (__any_sync(0xffffffffu, m > -INFINITY)) {  // O holds something (its last product is complete: S came behind it)
#pragma unroll 1
                for (int c = 0; c < 128; c += 8) {
                  float o[8];
                  tmem_ld8(t_o + c, o);
#pragma unroll
                  for (int k = 0; k < 8; ++k) o[k] *= f;
                  tmem_st8(t_o + c, o);
                }
              }
              l2 = mul2(l2, f32x2(f, f));
              m = up ? top : m;
            }
            float off = m == -INFINITY ? 0.f : -m * scale;
            // (what the rounding of m * scale leaves is the same factor for all of a row's weights, unless m is a mask of the type's
            // largest values)
            if (__any_sync(0xffffffffu, fabsf(fmaf(m, scale, off)) > 0x1p-12f && m > -INFINITY)) {
#pragma unroll
              for (int c = 0; c < 128; ++c) y[c] -= m > -INFINITY ? m : 0.f;
              off = 0.f;
            }
            const f32x2 sc(scale, scale), mm(off, off);
            f32x2 la(0.f, 0.f), lb(0.f, 0.f);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
              for (int c0 = 64 * half; c0 < 64 * half + 64; c0 += 16) {
                float pk[8];
#pragma unroll
                for (int c = c0; c < c0 + 16; c += 4) {
                  float e[4];
                  fma2(f32x2(y[c], y[c + 1]), sc, mm).get(e[0], e[1]);
                  fma2(f32x2(y[c + 2], y[c + 3]), sc, mm).get(e[2], e[3]);
#pragma unroll
                  for (int k = 0; k < 4; ++k) e[k] = ex2(e[k]);
                  la = add2(la, f32x2(e[0], e[1]));
                  lb = add2(lb, f32x2(e[2], e[3]));
                  pk[(c - c0) / 2] = __uint_as_float(pack_bf16x2(e[0], e[1]));
                  pk[(c - c0) / 2 + 1] = __uint_as_float(pack_bf16x2(e[2], e[3]));
                }
                tmem_st8(t_s + c0 / 2, pk);
              }
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(b_p(g, half));
            }
            l2 = add2(l2, add2(la, lb));
          };
          if (busy) {
            if ((i + 1) * kEN > lim_min)
              step(std::true_type{});
            else
              step(std::false_type{});
          } else {
            tc_fence_before();
            if (lane == 0) {
              mbar_arrive(b_p(g, 0));
              mbar_arrive(b_p(g, 1));
            }
          }
        }
      }
      if (!ok) break;
      m *= scale;  // (in base two from here on)
      float l;
      {
        float x, y;
        l2.get(x, y);
        l = x + y;
      }
      // ------------------------------------------------------------ rows out
      if (steps > 0) {
        if (!(ok = warp_wait(b_o(g), (uint32_t)(no++ & 1)))) break;
        tc_fence_after();
      }
      const bool whole = p.flags & kWhole;
      const int slot = p.flags & kFirst ? 1 : 0;
      float4* const part = reinterpret_cast<float4*>(a.partial + (int64_t)(2 * blockIdx.x + slot) * a.slot_rows * kPartRow) + my_tok * a.G + head;
      float f0 = l == 0.f ? 0.f : 1.f, f1 = 0.f;  // (a row that sees nothing: zeros, whatever the values are)
      if (one && steps > 0) {  // two states of the same rows
        state[tid] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(b_x);
        if (!(ok = warp_wait(b_x, (uint32_t)(nx++ & 1)))) break;
        const float2 x0 = state[r], x1 = state[128 + r];
        m = fmaxf(x0.x, x1.x);
        f0 = x0.x == -INFINITY ? 0.f : ex2(x0.x - m);
        f1 = x1.x == -INFINITY ? 0.f : ex2(x1.x - m);
        l = x0.y * f0 + x1.y * f1;
      }
      if (busy) {
        __nv_bfloat16* const out = a.out + ((p.row0 + my_tok) * a.H * a.G + p.h * a.G + head) * kED;
        const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
        // a one-tile item's columns are shared between the two tiles' warps
        const int c0 = one && steps > 0 ? 2 * g : 0, c1 = one && steps > 0 ? c0 + 2 : (one && g == 1) ? 0 : 4;
        const float a0 = f0 * inv, a1 = f1 * inv;
        const bool plain = !one && !__any_sync(0xffffffffu, f0 == 0.f);
        f32x2 finite2(0.f, 0.f);  // or NaN
#pragma unroll 1
        for (int c = c0; c < c1; ++c) {
          float o[32];
          if (steps > 0) {
            tmem_ld32((one ? tmem + lanes + 256 : t_o) + 32 * c, o);
            if (plain) {
#pragma unroll
              for (int k = 0; k < 32; k += 2) mul2(f32x2(o[k], o[k + 1]), f32x2(a0, a0)).get(o[k], o[k + 1]);
            } else {
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = f0 == 0.f ? 0.f : o[k] * a0;
            }
            if (one && steps > 1) {
              float u[32];
              tmem_ld32(tmem + lanes + 384 + 32 * c, u);
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] += f1 == 0.f ? 0.f : u[k] * a1;
            }
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = 0.f;
          }
#pragma unroll
          for (int k = 0; k < 32; k += 2) finite2 = fma2(f32x2(o[k], o[k + 1]), f32x2(0.f, 0.f), finite2);
          if (valid && whole) {
#pragma unroll
            for (int k = 0; k < 32; k += 16)
              st_global_v8(out + 32 * c + k, pack_bf16x2(o[k], o[k + 1]), pack_bf16x2(o[k + 2], o[k + 3]), pack_bf16x2(o[k + 4], o[k + 5]),
                           pack_bf16x2(o[k + 6], o[k + 7]), pack_bf16x2(o[k + 8], o[k + 9]), pack_bf16x2(o[k + 10], o[k + 11]),
                           pack_bf16x2(o[k + 12], o[k + 13]), pack_bf16x2(o[k + 14], o[k + 15]));
          } else if (valid) {
#pragma unroll
            for (int k = 0; k < 8; ++k) part[(8 * c + k) * a.slot_rows] = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
          }
        }
        float finite, other;
        finite2.get(finite, other);
        finite += other;
        // An infinity or NaN among the values of later new tokens has met weights of zero in the rows that do not see them.  Such rows'
        // products are formed anew over what they see, a row at a time; m and l are right.
        __syncwarp();
        for (uint32_t again = __ballot_sync(0xffffffffu, valid && finite != 0.f && fabsf(l) < INFINITY && fabsf(m) < INFINITY); again; again &= again - 1) {
          const int from = __ffs((int)again) - 1;
          const int r_tok = __shfl_sync(0xffffffffu, my_tok, from), r_head = __shfl_sync(0xffffffffu, head, from);
          const float r_m = __shfl_sync(0xffffffffu, m, from), r_inv = __shfl_sync(0xffffffffu, inv, from);
          const int begin = lo * kEN, upto = min(p.end, (lo + steps) * kEN), see = min(upto, p.base + r_tok + 1);
          const int32_t* const table = a.views[p.seq].block_table;
          auto value_row = [&](int t) { return (((int64_t)table[t >> a.shift] * a.H + p.h) << a.shift) + (t & ((1 << a.shift) - 1)); };
          bool hit = false;
          for (int t = max(see, begin); t < upto; ++t) {
            const float4 v = row4<QUANT>(a, value_row(t), true, lane);
            hit |= !(fmaf(v.x, 0.f, fmaf(v.y, 0.f, fmaf(v.z, 0.f, v.w * 0.f))) == 0.f);
          }
          if (!__any_sync(0xffffffffu, hit)) continue;  // (what is not finite is what the row sees)
          const float4 q = load4(a.q + (p.row0 + r_tok) * a.q_row + (p.h * a.G + r_head) * a.q_head + 4 * lane);
          const float sign = a.desc_qk & kNegateA ? -a.scale : a.scale;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int t = begin; t < see; t += 4) {  // (four slots' loads on their way at once)
            float4 k[4], v[4];
            float y[4], bias[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int64_t row = value_row(min(t + x, see - 1));
              k[x] = row4<QUANT>(a, row, false, lane);
              v[x] = row4<QUANT>(a, row, true, lane);
              bias[x] = a.logdeg ? a.logdeg[row] : 0.f;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = warp_sum(q.x * k[x].x + q.y * k[x].y + q.z * k[x].z + q.w * k[x].w) * sign + bias[x];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if (t + x >= see) break;
              const float w = ex2(fmaf(y[x], kLog2e, -r_m));
              o = make_float4(fmaf(w, v[x].x, o.x), fmaf(w, v[x].y, o.y), fmaf(w, v[x].z, o.z), fmaf(w, v[x].w, o.w));
            }
          }
          if (lane >= 8 * c0 && lane < 8 * c1) {
            const int64_t at = (p.row0 + r_tok) * a.H * a.G + p.h * a.G + r_head;
            if (whole)
              store4(a.out + at * kED + 4 * lane, make_float4(o.x * r_inv, o.y * r_inv, o.z * r_inv, o.w * r_inv));
            else
              reinterpret_cast<float4*>(a.partial + (int64_t)(2 * blockIdx.x + slot) * a.slot_rows * kPartRow)[lane * a.slot_rows + r_tok * a.G + r_head] = o;
          }
        }
        if (valid && !whole && (!one || g == 0)) part[32 * a.slot_rows] = make_float4(m, l, 0.f, 0.f);
      }
      if (one && steps > 0) {  // nobody goes on to the next piece's products before both have read
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_x);
        if (!(ok = warp_wait(b_x, (uint32_t)(nx++ & 1)))) break;
      }
      __syncwarp();
      if (lane == 0) piece_done(); else ++np;
    }
  }
  if (!ok) {
    *a.status = 1;
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);  // copies and products that are still under way
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// Joins the pieces of the item that CTA blockIdx.x of the kernel above ended and did not begin, 32 rows per CTA, 16 columns per warp.  A
// lane has a row, so that loads are whole lines and a store is a sector; where there are few rows (single tokens over a long cache, and
// then many pieces), the lanes that are left share a row's pieces.
constexpr int kJoinWarps = 8;
constexpr int kJoinRows = 32;

__global__ void __launch_bounds__(kJoinWarps * 32) extend_join_kernel(const ExtendArgs a) {
  griddep_wait();
  griddep_launch();
  const ExtendPiece last = a.pieces[blockIdx.x];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = (int)blockIdx.x - last.first + 1, row0 = (int)blockIdx.y * kJoinRows, rows = min(last.ntok * a.G - row0, kJoinRows);
  if (rows <= 0) return;
  const int RB = rows > 16 ? 32 : rows > 8 ? 16 : rows > 4 ? 8 : 4, S = 32 / RB;  // lanes with a row each, times lanes that share its pieces
  const int r = row0 + min(lane % RB, rows - 1);
  float m = -INFINITY, l = 0.f;
  float o[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) o[k] = 0.f;
  auto add = [&](float pm, float pl, const float (&y)[16]) {
    const float mm = fmaxf(m, pm);
    if (mm == -INFINITY && !(pl != 0.f)) return;  // (no slots, or only such of weight zero)
    const float c = m == -INFINITY ? 0.f : exp2f(m - mm), f = pm == -INFINITY ? 0.f : exp2f(pm - mm);
#pragma unroll
    for (int k = 0; k < 16; ++k) o[k] = fmaf(f, y[k], o[k] * c);
    l = fmaf(f, pl, l * c);
    m = mm;
  };
  constexpr int U = 4;
  for (int p = lane / RB; p < n; p += U * S) {
    float4 ml[U], y[U][4];
    int held[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (every address is in the workspace, whether something was left there or not)
      const int q = min(p + u * S, n - 1), c = last.first + q, slot = q == 0 ? 1 : 0;
      const float4* const at = reinterpret_cast<const float4*>(a.partial + (int64_t)(2 * c + slot) * a.slot_rows * kPartRow) + r;
      held[u] = a.pieces[c].held[slot];
      ml[u] = at[32 * a.slot_rows];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[u][k] = at[(4 * warp + k) * a.slot_rows];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p + u * S >= n || !held[u]) continue;
      const float x[16] = {y[u][0].x, y[u][0].y, y[u][0].z, y[u][0].w, y[u][1].x, y[u][1].y, y[u][1].z, y[u][1].w,
                           y[u][2].x, y[u][2].y, y[u][2].z, y[u][2].w, y[u][3].x, y[u][3].y, y[u][3].z, y[u][3].w};
      add(ml[u].x, ml[u].y, x);
    }
  }
  for (int d = RB; d < 32; d <<= 1) {
    const float pm = __shfl_xor_sync(0xffffffffu, m, d), pl = __shfl_xor_sync(0xffffffffu, l, d);
    float x[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) x[k] = __shfl_xor_sync(0xffffffffu, o[k], d);
    add(pm, pl, x);
  }
  if (lane >= rows) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int tok = r / a.G, head = r - tok * a.G;
  uint4* const out = reinterpret_cast<uint4*>(a.out + ((last.row0 + tok) * a.H * a.G + last.h * a.G + head) * kED + 16 * warp);
#pragma unroll
  for (int k = 0; k < 16; k += 8)
    out[k / 8] = make_uint4(pack_bf16x2(o[k] * inv, o[k + 1] * inv), pack_bf16x2(o[k + 2] * inv, o[k + 3] * inv), pack_bf16x2(o[k + 4] * inv, o[k + 5] * inv),
                            pack_bf16x2(o[k + 6] * inv, o[k + 7] * inv));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn extend_encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess
               ? reinterpret_cast<EncodeTiledFn>(p)
               : nullptr;
  }();
  return fn;
}

bool encode(CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const cuuint32_t es[3] = {1, 1, 1};
  return extend_encode_fn() && extend_encode_fn()(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, es,
                                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Sets the kernel's shared memory once per device
template <bool QUANT, bool DEAL>
bool extend_ready() {
  constexpr int kMaxDev = 64;
  static std::atomic<bool> done[kMaxDev];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDev) return false;
  if (done[dev].load(std::memory_order_relaxed)) return true;
  if (cudaFuncSetAttribute(extend_kernel<QUANT, DEAL>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEBytes + 1024) != cudaSuccess) return false;
  done[dev].store(true, std::memory_order_relaxed);
  return true;
}

int32_t slot_rows(int64_t n_rows, int32_t G) { return (int32_t)std::min<int64_t>(2 * (kEN / G) * G, n_rows * G); }
size_t pieces_bytes() { return ((size_t)sm_count() * sizeof(ExtendPiece) + 255) / 256 * 256; }

int check_extend(const void* views, const void* q_begin, int64_t n_rows, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D, int32_t dtype,
                 const void* q, int64_t q_row, int64_t q_head, const void* out, float scale, const void* workspace, size_t workspace_bytes) {
  if (!views || !q_begin || !q || !out || n_rows < 0 || Bz <= 0 || H <= 0 || G <= 0 || q_row < 0 || q_head < 0 ||
      !std::isfinite(scale))
    return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_F32 && dtype != CKV_BF16) return CKV_ERR_INVALID_ARG;
  if (dtype != CKV_BF16 || page_shift(page_tokens) < 0 || D != kED || G > 8 || H > 8192 || Bz > 65535 || n_rows > INT32_MAX / (H * G))
    return CKV_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(out) || q_row % 8 || q_head % 8) return CKV_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < ckv_extend_workspace_bytes(n_rows, H, G, D) || !aligned16(workspace)) return CKV_ERR_WORKSPACE;
  return CKV_OK;
}

// Fills in what both calls have in common and launches
template <bool QUANT>
int run_extend(ExtendArgs& a, const void* q, int64_t q_row, int64_t q_head, const void* k, const void* v, int64_t n_pages, void* workspace, cudaStream_t st) {
  if (a.n_rows == 0) return CKV_OK;
  a.q = static_cast<const __nv_bfloat16*>(q); a.q_row = q_row; a.q_head = q_head;
  a.k_pages = static_cast<const __nv_bfloat16*>(k); a.v_pages = static_cast<const __nv_bfloat16*>(v);
  a.T = kEN / a.G;
  // log-degrees are divided by the scale: next to 1e-30 products vanish as they do next to zero
  a.desc_qk = kDescQK | (a.scale < 0 ? kNegateA : 0u);
  a.scale = std::max(std::fabs(a.scale), 1e-30f);
  a.max_slots = n_pages << a.shift;
  a.status = static_cast<int32_t*>(workspace);
  a.pieces = reinterpret_cast<ExtendPiece*>(static_cast<unsigned char*>(workspace) + 256);
  a.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + 256 + pieces_bytes());
  a.slot_rows = slot_rows(a.n_rows, a.G);
  CUtensorMap tm[3] = {};
  const cuuint64_t HG = (cuuint64_t)a.H * a.G, rows = ((cuuint64_t)n_pages * a.H) << a.shift;
  {  // (the stride of a single head or row is never used)
    const cuuint64_t dims[3] = {kED, HG, (cuuint64_t)a.n_rows}, strides[2] = {HG > 1 ? (cuuint64_t)q_head * 2 : 256, a.n_rows > 1 ? (cuuint64_t)q_row * 2 : 256};
    const cuuint32_t box[3] = {64, (cuuint32_t)a.G, (cuuint32_t)a.T};
    if (!encode(&tm[0], q, 3, dims, strides, box)) return CKV_ERR_UNSUPPORTED;
  }
  for (int i = 0; i < (QUANT ? 0 : 2); ++i) {
    const cuuint64_t dims[2] = {kED, rows}, strides[1] = {kED * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)std::min(kEN, 1 << a.shift)};
    if (!encode(&tm[1 + i], i ? v : k, 2, dims, strides, box)) return CKV_ERR_UNSUPPORTED;
  }
  const unsigned ctas = (unsigned)sm_count();
  cudaStream_t stream = st;
  auto go = [&](auto deal) {
    constexpr bool DEAL = decltype(deal)::value;
    return extend_ready<QUANT, DEAL>() && launch_dependent(extend_kernel<QUANT, DEAL>, dim3(ctas), dim3(kEWarps<QUANT> * 32), kEBytes + 1024, stream, tm[0], tm[1],
                                                           tm[2], a) == cudaSuccess;
  };
  // (a kernel of its own: what it does at its start would cost small calls 2 to 6 us)
  const bool deal = a.Bz == 1 && (a.n_rows + 2 * a.T - 1) / (2 * a.T) * a.H >= ctas && ctas < kMaxStarts;
  if (!(deal ? go(std::true_type{}) : go(std::false_type{}))) return CKV_ERR_CUDA;
  return launch_dependent(extend_join_kernel, dim3(ctas, (unsigned)(a.slot_rows + kJoinRows - 1) / kJoinRows), dim3(kJoinWarps * 32), 0, st, a) == cudaSuccess ? CKV_OK : CKV_ERR_CUDA;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t ckv_extend_workspace_bytes(int64_t n_rows, int32_t H, int32_t G, int32_t D) {
  if (n_rows < 0 || H <= 0 || G <= 0 || D <= 0) return 0;
  return 256 + pieces_bytes() + (size_t)2 * sm_count() * slot_rows(n_rows, G) * kPartRow * sizeof(float);
}

int ckv_extend_attn_paged(const ckv_paged_view* views_dev, const int64_t* q_begin, int64_t n_rows, const void* k_pages, const void* v_pages,
                          const float* logdeg_pages, int64_t n_pages, int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D,
                          int32_t dtype, const void* q, int64_t q_row_stride, int64_t q_head_stride, void* out, float scale, void* workspace,
                          size_t workspace_bytes, void* cuda_stream) {
  if (!k_pages || !v_pages || n_pages <= 0) return CKV_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || (logdeg_pages && !aligned16(logdeg_pages))) return CKV_ERR_ALIGNMENT;
  const int st = check_extend(views_dev, q_begin, n_rows, page_tokens, Bz, H, G, D, dtype, q, q_row_stride, q_head_stride, out, scale, workspace,
                              workspace_bytes);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (n_pages > (INT32_MAX >> shift) / H) return CKV_ERR_UNSUPPORTED;  // (2^31 rows of a pool: 1 TB)
  ExtendArgs a{};
  a.views = views_dev; a.q_begin = q_begin; a.n_rows = n_rows; a.Bz = Bz; a.H = H; a.G = G; a.shift = shift; a.scale = scale;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.logdeg = logdeg_pages;
  return run_extend<false>(a, q, q_row_stride, q_head_stride, k_pages, v_pages, n_pages, workspace, static_cast<cudaStream_t>(cuda_stream));
}

int ckv_extend_attn_quantized(const ckv_paged_view* views_dev, const int64_t* q_begin, int64_t n_rows, const ckv_quant_pool* pool, int64_t n_pages,
                              int32_t page_tokens, int32_t Bz, int32_t H, int32_t G, int32_t D, int32_t dtype, const void* q, int64_t q_row_stride,
                              int64_t q_head_stride, void* out, float scale, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (!pool || !pool->k_codes || !pool->v_codes || !pool->k_scales || !pool->v_scales || n_pages <= 0) return CKV_ERR_INVALID_ARG;
  if (!aligned16(pool->k_codes) || !aligned16(pool->v_codes) || !aligned16(pool->k_scales) || !aligned16(pool->v_scales) ||
      (pool->logdeg_pages && !aligned16(pool->logdeg_pages)))
    return CKV_ERR_ALIGNMENT;
  const int st = check_extend(views_dev, q_begin, n_rows, page_tokens, Bz, H, G, D, dtype, q, q_row_stride, q_head_stride, out, scale, workspace,
                              workspace_bytes);
  if (st != CKV_OK) return st;
  const int shift = page_shift(page_tokens);
  if (n_pages > (INT32_MAX >> shift) / H) return CKV_ERR_UNSUPPORTED;
  ExtendArgs a{};
  a.views = views_dev; a.q_begin = q_begin; a.n_rows = n_rows; a.Bz = Bz; a.H = H; a.G = G; a.shift = shift; a.scale = scale;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.pool = *pool; a.logdeg = pool->logdeg_pages;
  return run_extend<true>(a, q, q_row_stride, q_head_stride, nullptr, nullptr, n_pages, workspace, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
