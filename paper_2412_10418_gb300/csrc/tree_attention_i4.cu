// tree_attention_i4.cu -- cdsl_tree_attention over a 4-bit cache: float32 queries, and bf16 ones of at most 16 query
// vectors per K/V head (more: tree_attention_rows.cu).
//
// A row of 128 values is 72 bytes, so that what bounds a large pass is less the bytes than the work on each of them: in the
// time in which HBM brings an SM two chunks of 64 slots its four schedulers issue 3,000 instructions, for 32,768 codes.
// Slots are the MMA's M as in tree_attention_tc.cu, but codes go from shared memory to registers, become 16-bit operands
// there and are multiplied there (mma.sync m16n8k16); through shared memory to tcgen05 they would be written and read once
// more, in 16 bits four times their size, which alone takes longer than HBM does. A row's groups take turns by four
// values, so that one 8- or 16-byte load gives a lane the fragments of all groups.
//
//   S^T = K Q^T    K's operand is a code plus 8 as the bits of an fp16 number below 2^-14, one instruction for two of
//                  them: (word & 0x000f000f) ^ 0x00080008 = (code + 8) 2^-24, the next four bits 2^-20. What the 8
//                  adds, -8 times the sum of the group's q, is what the accumulators start from (float32 queries: the
//                  codes themselves, an fma more, as those sums are larger and so are their roundings). Groups are summed
//                  apart and multiplied by their scales in fp32. q is held in fp16 planes under a power of two that takes the
//                  row's largest to 2^14 or more: exact down to 2^-27 of it from bf16 (one plane), to 2^-35 of it from float32 (three).
//   O^T = V^T P^T  V's operand is the value in bf16, exact (a code's 3 bits by a scale's 4): bits 3 .. 6 of
//                  128 + 8 (code + 8), then one fma of two by (scale / 8, -24 scale). P is the sum of two bf16
//                  planes (2^-16 of itself; three for float32 queries, 2^-24): fp32's range, whatever lies next to what.
//                  Up to four vectors have two of the MMA's eight columns each, of P's two planes: one product for both.
//
// Scores go through shared memory once, to where a lane has 16 slots of one vector: maxima take two exchanges there, and
// probabilities are P's fragments as they are. O^T is one chain over kChain stretches of 64 slots and is then added to fp32
// sums (in the workspace: few passes are as long), as a tensor core's additions truncate; its reference is the running
// maximum, and few stretches raise it. (float32 queries: every product is added up in fp32.) A warp has a run of its own and
// no barrier but its own; its K and V come by bulk copies, the next stretch's K while this one's softmax and P V run, and V
// beside the next scores.
//
// Measured, 32 heads over 8 of 128: 64 sequences of up to 8192 tokens, one token (453 MB): 113 us, 59 % of the copy
// bandwidth; 8 sequences of 16,384, 4 / 8 / 16 vectors: 47 / 50 / 70 us; one of 512 tokens 8.9 us in a graph with the joining. Bound by
// instructions: 2,900 a chunk of 128 slots, 2.2 a cycle and SM, half of the integer pipe's rate (masks, shifts, byte moves) and
// a third of the tensor cores'. Steps on the way (us, the large case): by the CUDA cores 505; codes turned as above, K's
// and V's rows by a warp of 64 slots 181; no selects on V's scales 148; scores through shared memory and loops rolled, masks as one
// instruction, pages 32 at a time 126; V's scales by pairs once, units of 64 slots 121; 12 warps an SM with two to four
// tiles side by side, in place of 16 with one, 115; blocks of four warps, one to a scheduler, 111 with four vectors twice.
// Right shifts as high halves of products, on the FMA pipe: 132 for 122. V's rows four slots apart in a lane, so that
// four lanes' meet half as many banks twice: no difference.
//
// Waits are bounded by a number of tries (wait_for): on expiry CDSL_ETIMEOUT is latched and the warp exits once its copies
// have landed or been given up on as well.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "once.h"
#include "tree_attention.cuh"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {

constexpr int kStretch = 64;                   // slots at a time: a unit
constexpr int kTiles = kStretch / 16;
constexpr int kWarps = 4;                      // of a block: one to each of an SM's four schedulers
constexpr int kPitch = kStretch + 4;           // floats of a vector's scores
constexpr int kChain = 64;                     // stretches of O^T's chain (512 products: 2^-15 of it at worst)

template <int HD, int NQ, bool F32>
struct Cfg {
  static constexpr int G = HD / kGroup, RB = HD / 2, SB = 2 * G;   // groups; bytes of a row's codes and scales
  static constexpr int NT = NQ == 16 ? 2 : 1;                      // the MMA's columns by eights
  // four vectors: each has two columns, of P's two planes, which one MMA then takes for two
  static constexpr bool TWICE = NQ == 4;
  static constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : TWICE ? 1 : 2;   // planes of q, and of p in a column
  // of K's scales: 128 products of 2^15 (a query) and 2^120 (a key's value) stay within float32 (codes times 2^-24 do as they are)
  static constexpr float DOWN = F32 ? 0x1p-15f : 1.f;
  static constexpr uint32_t CODES = kStretch * RB, SCALES = kStretch * SB;
  static constexpr uint32_t V_OFF = CODES + SCALES;
  static constexpr uint32_t F_OFF = 2 * V_OFF;                     // V's scales / 8 by pairs of slots
  static constexpr uint32_t P_OFF = F_OFF + SCALES;
  // scores, then P's fragments: PP planes of two words for each tile and lane
  static constexpr uint32_t S_BYTES = 8 * NT * kPitch * 4, F_BYTES = NT * kTiles * 32 * PP * 8;
  static constexpr uint32_t MASK_OFF = P_OFF + (S_BYTES > F_BYTES ? S_BYTES : F_BYTES);
  static constexpr uint32_t WARP_BYTES = (MASK_OFF + NQ * (kWords + 1) * 4 + 127) / 128 * 128;
  static constexpr uint32_t PLAN_OFF = kWarps * WARP_BYTES;
  // of an SM, by registers (16 of 128 registers: 117 us for 111; NQ 16 with 12: 93 for 72, float32 34 for 30)
  static constexpr int WARPS = F32 || NQ == 16 ? 8 : 12;
  static constexpr int K_TILES = NT == 2 ? 2 : 4, V_TILES = NT == 2 ? 1 : 2;   // side by side
  static constexpr size_t smem(int batch) { return PLAN_OFF + plan_bytes(batch); }
};

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }
// The pieces (16 bits, four codes) of group g (even: the low one) of two words.
__device__ __forceinline__ uint32_t both(uint32_t a, uint32_t b, int g) { return prmt(a, b, g & 1 ? 0x7632 : 0x5410); }

// d = a b + (c0, c1, c2, c3) (d itself would have to be set first)
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1,
                                        float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, float c0, float c1,
                                         float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
// (a, b) as two bf16, a low.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The codes in bits BIT .. BIT + 3 of both halves of x (mask: those) as fp16: themselves, or (code + 8) 2^(BIT - 24).
template <bool EXACT, int BIT>
__device__ __forceinline__ uint32_t code_f16(uint32_t x, uint32_t mask) {
  constexpr uint32_t eights = 0x00080008u << BIT;
  if constexpr (!EXACT) return and_xor(x, mask, eights);
  uint32_t d;                                  // of 1024 + (code + 8) 2^BIT
  asm("fma.rn.f16x2 %0, %1, %2, %3;"
      : "=r"(d)
      : "r"(and_xor(x, mask, 0x64006400u | eights)), "r"(BIT ? 0x2c002c00u : 0x3c003c00u),
        "r"(BIT ? 0xd480d480u : 0xe408e408u));   // times 1 / 16, less 72; less 1032
  return d;
}

template <int HD, int NQ, bool F32>
__global__ void __launch_bounds__(32 * kWarps, Cfg<HD, NQ, F32>::WARPS / kWarps) k_tree_i4(TreeArgs a) {
  using C = Cfg<HD, NQ, F32>;
  using T = std::conditional_t<F32, float, __nv_bfloat16>;
  constexpr int G = C::G, NT = C::NT, QP = C::QP, PP = C::PP;
  constexpr bool TWICE = C::TWICE;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t s_full[kWarps][2];   // K, V
  __shared__ uint32_t s_masks[4];
  __shared__ Segment s_segs[kWarps][2];        // this segment and the next (registers are dear)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, run = blockIdx.x * kWarps + warp;
  uint8_t* const sm = smem + warp * C::WARP_BYTES;
  uint64_t* const full = s_full[warp];
  Segment* const s_seg = s_segs[warp];
  float* const s_p = reinterpret_cast<float*>(sm + C::P_OFF);
  uint32_t* const s_mask = reinterpret_cast<uint32_t*>(sm + C::MASK_OFF);
  int* const s_first = reinterpret_cast<int*>(smem + C::PLAN_OFF);
  const Cache& c = a.c;
  const int r = lane >> 2, q4 = lane & 3;   // fragments' row (or column) and quarter
  if (lane == 0) {
    tc::mbar_init(&full[0], 1);
    tc::mbar_init(&full[1], 1);
    tc::fence_mbar_init();
  }
  if (threadIdx.x < 3) s_masks[lane] = lane == 0 ? 0x000f000fu : lane == 1 ? 0x00f000f0u : 0x00780078u;
  pdl_wait();
  pdl_launch_dependents();
  build_plan(a, s_first);                      // (ends in a block barrier)
  if (blockIdx.x == 0) check_lens(a);
  const int total = s_first[c.batch], runs = runs_of(a, total);
  if (run >= runs) return;
  const int end = run_begin(run + 1, total, runs);
  // of all scores: 2^-14 of the queries, 2^24 of the codes or 2^15 of their scales (DOWN)
  const float fa = a.scale * (F32 ? 2.f : 0x1p10f);
  // (through shared memory, or the compiler knows them as constants and takes two instructions)
  const volatile uint32_t* const masks = s_masks;
  const uint32_t k0 = masks[0], k4 = masks[1], kv = masks[2];
  const int P = 1 << c.page_shift, rows = min(P, kStretch), shift = min(c.page_shift, 6);

  // The copies of a stretch: its pieces (of a page, or of 64 slots) by a lane each. Pages come 32 pieces at a time, or each
  // copy would wait for its page first.
  const int per = kStretch >> shift;           // pieces of a stretch
  int pages = -1, window = 0;                  // this lane's piece of the window, and the window's first slot
  struct Stretch {
    int page;
    uint32_t live;                             // pieces that have a page
  };
  auto look = [&](const Segment& s, int slot) {
    window = slot;
    const int mine = slot + (lane << shift);
    pages = -1;
    if (mine < min(s.keys, s.c1 * kStretch)) {
      pages = page_of(c, s.b, mine);
      if (pages < 0) set_status(a.status, CDSL_ERANGE);
    }
  };
  auto locate = [&](const Segment& s, int slot) {
    if ((slot - window) >> shift >= 32) look(s, slot);
    Stretch x;
    x.page = __shfl_sync(0xffffffffu, pages, ((slot - window) >> shift) + lane & 31);
    if (lane >= per) x.page = -1;
    x.live = __ballot_sync(0xffffffffu, x.page >= 0);
    return x;
  };
  const size_t page_rows = (size_t)2 * c.kvh << c.page_shift, layer_row = row_of(c, a.layer, 0, 0, 0, 0);
  auto load = [&](const Segment& s, int slot, const Stretch& x, int kv) {
    if (lane == 0) tc::mbar_expect_tx(&full[kv], __popc(x.live) * rows * (C::RB + C::SB));
    __syncwarp();
    if (x.page >= 0) {
      const size_t row = layer_row + x.page * page_rows + ((kv * c.kvh + s.h) << c.page_shift) + ((slot + (lane << shift)) & (P - 1));
      uint8_t* const to = sm + kv * C::V_OFF;
      tc::bulk_load(to + lane * rows * C::RB, c.pool + row * C::RB, rows * C::RB, &full[kv]);
      tc::bulk_load(to + C::CODES + lane * rows * C::SB, c.scale + row * C::SB, rows * C::SB, &full[kv]);
    }
  };

  int it = 0;                                  // stretches
  int unit = run_begin(run, total, runs), turn = 0;
  if (lane == 0) s_seg[0] = segment_at(a, s_first, unit, end);
  __syncwarp();
  Stretch x = {};
  bool loaded = false;                         // x is the segment's first stretch and on its way
#pragma unroll 1
  for (; unit < end; turn ^= 1) {
    const Segment& s = s_seg[turn];
    const Segment& next = s_seg[turn ^ 1];
    if (!loaded && s.keys > 0) {
      look(s, s.c0 * kStretch);
      x = locate(s, s.c0 * kStretch);
      load(s, s.c0 * kStretch, x, 0);
      load(s, s.c0 * kStretch, x, 1);
    }
    loaded = false;
    unit += s.c1 - s.c0;
    __syncwarp();                              // (the segment before is done with shared memory)
    if (lane == 0 && unit < end) s_seg[turn ^ 1] = segment_at(a, s_first, unit, end);
    for (int i = lane; i < NQ * (kWords + 1); i += 32) {
      const int v = i / (kWords + 1), w = i % (kWords + 1);
      s_mask[i] = v < s.nq && w < a.W ? a.mask[((size_t)s.b * a.T + vector_of(a, s.h, s.qb, v).t) * a.W + w] : 0u;
    }
    // ---- queries: this lane has dimensions 32 g + 8 q4 .. of vectors r (+ 8) as the MMA's columns
    uint32_t qf[NT][QP][G][4];                 // of both steps of a group
    float from[NT][G][2];                      // what the accumulators of vectors 2 q4, 2 q4 + 1 (+ 8) start from
    float fb[NT];                              // factors of the scores of vectors r (+ 8)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int v = TWICE ? r & 3 : 8 * n + r;
      const bool any = v < s.nq;
      const Vec w = vector_of(a, s.h, s.qb, any ? v : 0);
      const T* const q = static_cast<const T*>(a.q) + s.b * a.sq[0] + w.t * a.sq[1] + w.h * a.sq[2] + 8 * q4;
      float y[G][8];
      uint32_t top = 0;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[g][e] = any ? to_f32<T>(q[g * kGroup + e]) : 0.f;
          top = max(top, __float_as_uint(y[g][e]) & 0x7fffffffu);
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e2 = max((int)(top >> 23) - 127, -100);          // (a row that is not finite: 128)
      // (to 2^14 .. 2^15: up to twice that could round to infinity)
      const float up = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : exp2f((float)(14 - e2));
      float sum[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        sum[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[g][e] *= !F32 && e & 1 ? up * 0.0625f : up;   // (the second and fourth of four: codes 2^4 higher)
#pragma unroll
        for (int p = 0; p < QP; ++p)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t two = pack_f16(y[g][i], y[g][4 + i]);
            const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&two));
            qf[n][p][g][i] = two;
            sum[g] += (z.x + z.y) * (i & 1 ? 16.f : 1.f);
            y[g][i] -= z.x;
            y[g][4 + i] -= z.y;
          }
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
#pragma unroll
        for (int e = 0; e < 2; ++e) from[n][g][e] = F32 ? 0.f : __shfl_sync(0xffffffffu, sum[g], 4 * (2 * q4 + e)) * -0x1p-21f;
      }
      fb[n] = any ? exp2f((float)e2) : 0.f;
    }
    __syncwarp();                              // (the masks)

    float o[G][2][NT][4];                      // dimensions 32 g + 4 r + 2 half (+ 1) of vectors 2 q4, 2 q4 + 1 (+ 8)
    float m[NT], l[NT];                        // of vectors r (+ 8): the maxima so far, and this lane's slots' share of the sums
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n] = -INFINITY;
      l[n] = 0.f;
    }
    const auto clear = [&] {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][h][n][e] = 0.f;
    };
    clear();
    const size_t part = (size_t)run * 2 + (s.c0 == 0);
    // The sums behind O^T's chain: in the part's place in the workspace, relative to the maxima m_then. (A whole item's is
    // free while the run is at it: it ends before the run's last part begins.)
    bool chained = false;
    float m_then[NT];
    const auto add_chain = [&] {               // o += the sums
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float f = m_then[n] == -INFINITY ? 0.f : ex2(m_then[n] - m[n]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float by = __shfl_sync(0xffffffffu, f, 4 * (2 * q4 + e));
          if (TWICE && q4 >= 2) continue;      // (put wrote the planes' sum)
          const float* const from = a.part_o + (part * NQ + 8 * n + 2 * q4 + e) * HD + 4 * r;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float4 y = *reinterpret_cast<const float4*>(from + g * kGroup);
            o[g][0][n][e] = fmaf(y.x, by, o[g][0][n][e]);
            o[g][0][n][2 + e] = fmaf(y.y, by, o[g][0][n][2 + e]);
            o[g][1][n][e] = fmaf(y.z, by, o[g][1][n][e]);
            o[g][1][n][2 + e] = fmaf(y.w, by, o[g][1][n][2 + e]);
          }
        }
      }
    };
    const auto one_plane = [&] {               // o of a vector's two columns together in the first
      if constexpr (TWICE)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[g][h][0][e] += __shfl_xor_sync(0xffffffffu, o[g][h][0][e], 2);
    };
    const auto put = [&](int n, int e, float by) {   // o to the part's place
      if (TWICE && q4 >= 2) return;
      float* const to = a.part_o + (part * NQ + 8 * n + 2 * q4 + e) * HD + 4 * r;
#pragma unroll
      for (int g = 0; g < G; ++g)
        *reinterpret_cast<float4*>(to + g * kGroup) =
            make_float4(o[g][0][n][e] * by, o[g][0][n][2 + e] * by, o[g][1][n][e] * by, o[g][1][n][2 + e] * by);
    };

    const int last = min(s.keys, s.c1 * kStretch);
#pragma unroll 1
    for (int slot = s.c0 * kStretch, links = 0; slot < last; slot += kStretch, ++it) {
      // ---- scores of slots 16 tile + r, + 8 and vectors 2 q4, + 1
      if (!__all_sync(0xffffffffu, wait_for(&full[0], it & 1, a.status))) {
        wait_for(&full[1], it & 1, a.status);
        return;
      }
      const uint32_t* const k_scales = reinterpret_cast<const uint32_t*>(sm + C::CODES);
#pragma unroll C::K_TILES
      for (int i = 0; i < kTiles; ++i) {
        float t[NT][4];
        uint32_t w[2][G], sc[2][G / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = 16 * i + r + 8 * h;
          if constexpr (G == 4) {
            const uint4 u = *reinterpret_cast<const uint4*>(sm + row * C::RB + 16 * q4);
            w[h][0] = u.x; w[h][1] = u.y; w[h][2] = u.z; w[h][3] = u.w;
            const uint2 z = *reinterpret_cast<const uint2*>(k_scales + row * 2);
            sc[h][0] = z.x; sc[h][1] = z.y;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(sm + row * C::RB + 8 * q4);
            w[h][0] = u.x; w[h][1] = u.y;
            sc[h][0] = k_scales[row];
          }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t x0 = both(w[0][g / 2], w[0][G / 2 + g / 2], g), x1 = both(w[1][g / 2], w[1][G / 2 + g / 2], g);
          const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
          const uint32_t lo[4] = {code_f16<F32, 0>(x0, k0), code_f16<F32, 0>(x1, k0), code_f16<F32, 4>(x0, k4), code_f16<F32, 4>(x1, k4)};
          const uint32_t hi[4] = {code_f16<F32, 0>(y0, k0), code_f16<F32, 0>(y1, k0), code_f16<F32, 4>(y0, k4), code_f16<F32, 4>(y1, k4)};
          const float s0 = bf16_at(sc[0][g / 2], g & 1) * C::DOWN, s1 = bf16_at(sc[1][g / 2], g & 1) * C::DOWN;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float d[4];
            mma_f16(d, lo, qf[n][QP - 1][g][0], qf[n][QP - 1][g][1], from[n][g][0], from[n][g][1], from[n][g][0], from[n][g][1]);
            mma_f16(d, hi, qf[n][QP - 1][g][2], qf[n][QP - 1][g][3], d[0], d[1], d[2], d[3]);
#pragma unroll
            for (int p = QP - 2; p >= 0; --p) {
              mma_f16(d, lo, qf[n][p][g][0], qf[n][p][g][1], d[0], d[1], d[2], d[3]);
              mma_f16(d, hi, qf[n][p][g][2], qf[n][p][g][3], d[0], d[1], d[2], d[3]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              t[n][e] = g == 0 ? d[e] * (e < 2 ? s0 : s1) : fmaf(d[e], e < 2 ? s0 : s1, t[n][e]);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s_p[(8 * n + 2 * q4 + (e & 1)) * kPitch + 16 * i + r + 8 * (e >> 1)] = t[n][e];
      }
      // Scales times 0, of two slots a lane: is one of them not finite?
      uint32_t k_bad[2] = {0u, 0u};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < G / 2; ++i) k_bad[h] = fma_bf16x2(k_scales[(lane + 32 * h) * (G / 2) + i], 0u, k_bad[h]);
      __syncwarp();                            // (K has been read; the scores)
      // ---- the next K
      const uint32_t live_now = x.live;
      const int there = last - slot;           // slots that there are, if fewer than 64
      const bool more = slot + kStretch < last, beyond = !more && unit < end && next.keys > 0;
      const Segment& after = more ? s : next;
      const int to = more ? slot + kStretch : next.c0 * kStretch;
      if (more || beyond) {
        if (beyond) look(after, to);
        x = locate(after, to);
        load(after, to, x, 0);
      }
      if (!__all_sync(0xffffffffu, wait_for(&full[1], it & 1, a.status))) {
        if (more || beyond) wait_for(&full[0], (it + 1) & 1, a.status);
        return;
      }
      uint8_t* const v_scales = sm + C::V_OFF + C::CODES;
      // V's scales of the slots of a pair of the MMA's k, s0 and s0 + 4; and are they finite?
      const int s0 = 16 * (lane >> 3) + 8 * (lane >> 2 & 1) + (lane & 3);
      uint32_t even[G / 2], odd[G / 2];
      if constexpr (G == 4) {
        const uint2 u = reinterpret_cast<const uint2*>(v_scales)[s0], z = reinterpret_cast<const uint2*>(v_scales)[s0 + 4];
        even[0] = u.x; even[1] = u.y; odd[0] = z.x; odd[1] = z.y;
      } else {
        even[0] = reinterpret_cast<const uint32_t*>(v_scales)[s0];
        odd[0] = reinterpret_cast<const uint32_t*>(v_scales)[s0 + 4];
      }
      uint32_t even_bad = 0, odd_bad = 0;
#pragma unroll
      for (int i = 0; i < G / 2; ++i) {
        even_bad = fma_bf16x2(even[i], 0u, even_bad);
        odd_bad = fma_bf16x2(odd[i], 0u, odd_bad);
      }
      const auto nan = [](uint32_t x) { return (x & 0x7fff7fffu) != 0; };   // (else 0 or -0)
      // rows of V that are not finite, as bits of the lanes' first and second slots; of K: their scores become NaN, which an
      // infinite scale alone would not make them (-inf is nothing to a maximum)
      uint32_t v_bad[2] = {0u, 0u};
      if (__any_sync(0xffffffffu, nan(even_bad | odd_bad | k_bad[0] | k_bad[1]))) {
        v_bad[0] = __ballot_sync(0xffffffffu, nan(even_bad));
        v_bad[1] = __ballot_sync(0xffffffffu, nan(odd_bad));
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (nan(k_bad[h]))
#pragma unroll 1
            for (int v = 0; v < 8 * NT; ++v) s_p[v * kPitch + lane + 32 * h] = __uint_as_float(0x7fc00000u);
        __syncwarp();
      }
      // slots that there are, as bits
      uint64_t valid = there >= 64 ? ~0ull : (1ull << there) - 1;
      const uint32_t pieces = shift == 6 ? 1u : shift == 5 ? 3u : 15u;
      if (live_now != pieces)
#pragma unroll 1
        for (int i = 0; i < kStretch >> shift; ++i)
          if (!(live_now >> i & 1)) valid &= ~((shift == 6 ? ~0ull : (1ull << rows) - 1) << (i << shift));
      // Code of its own for stretches with slots of the tree, past the item's, without a page or with a row that is not
      // finite: as one, every score has selects.
      const bool masked = valid != ~0ull || slot + kStretch > s.len || (v_bad[0] | v_bad[1]) != 0;
      // ---- maxima, probabilities, sums: slots 16 tile + q4, + 4, + 8, + 12 of vector r (+ 8)
      uint32_t pf[NT][kTiles][PP][2];
      bool raised = false;
      float alpha[NT];
      auto softmax = [&](auto general) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int v = TWICE ? r & 3 : 8 * n + r;
          // (the query's power of two before the maximum where it is small and after it where it is large: no step leaves
          // float32's range where the score is inside it)
          const float f1 = fa * fminf(fb[n], 1.f), f2 = fmaxf(fb[n], 1.f);
          uint64_t seen = ~0ull;
          if constexpr (general) {
            const uint32_t* const w = s_mask + v * (kWords + 1);
            seen = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int f = slot - s.len + 32 * h;   // the tree's node in the first slot
              uint32_t y;
              if (f <= -32) y = ~0u;
              else if (f < 0) y = ((1u << -f) - 1) | w[0] << -f;
              else if (f >= 32 * kWords) y = 0u;
              else y = __funnelshift_r(w[f >> 5], w[(f >> 5) + 1], f & 31);
              seen |= (uint64_t)y << (32 * h);
            }
            seen = v < s.nq ? (seen & valid) >> q4 : 0ull;
          }
          float t[kTiles][4], top = -INFINITY;
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              t[i][e] = s_p[v * kPitch + 16 * i + 4 * e + q4] * f1;
              if constexpr (general) {
                if (!(seen >> (16 * i + 4 * e) & 1)) continue;
              }
              top = fmaxf(top, t[i][e]);
            }
          }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float mq = top == -INFINITY ? top : top * f2;
          const float was = m[n], mn = fmaxf(was, mq);
          alpha[n] = was == mn ? 1.f : was == -INFINITY ? 0.f : ex2(was - mn);
          raised = raised || was != mn;
          m[n] = mn;
          const float off = mn == -INFINITY ? 0.f : mn;
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kTiles; ++i) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[e] = ex2(fmaf(t[i][e], f2, -off));
              if constexpr (general) {
                if (!(seen >> (16 * i + 4 * e) & 1)) y[e] = 0.f;
                sum += y[e];
                if (y[e] != 0.f && v_bad[e & 1] >> (8 * i + 4 * (e >> 1) + q4) & 1) y[e] = __uint_as_float(0x7fc00000u);
              } else {
                sum += y[e];
              }
            }
#pragma unroll
            for (int p = 0; p < PP; ++p)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t two = pack_bf16(y[2 * h], y[2 * h + 1]);
                if constexpr (TWICE) {
                  const uint32_t rest = pack_bf16(y[2 * h] - __uint_as_float(two << 16), y[2 * h + 1] - __uint_as_float(two & 0xffff0000u));
                  if (r >= 4) two = rest;
                }
                pf[n][i][p][h] = two;
                if (p + 1 < PP) {
                  y[2 * h] -= __uint_as_float(two << 16);
                  y[2 * h + 1] -= __uint_as_float(two & 0xffff0000u);
                }
              }
          }
          l[n] = fmaf(l[n], alpha[n], sum);
        }
      };
      if (masked) {
        softmax(std::true_type());
        // nothing of a slot that is not there, or whose V is not finite, may reach the sums
        const bool e0 = valid >> s0 & 1 && !(v_bad[0] >> lane & 1), e1 = valid >> (s0 + 4) & 1 && !(v_bad[1] >> lane & 1);
#pragma unroll
        for (int i = 0; i < G / 2; ++i) {
          if (!e0) even[i] = 0u;
          if (!e1) odd[i] = 0u;
        }
      } else {
        softmax(std::false_type());
      }
      {
        uint32_t f[G];
#pragma unroll
        for (int g = 0; g < G; ++g) f[g] = mul_bf16x2(both(even[g / 2], odd[g / 2], g), 0x3e003e00u);   // 1 / 8
        uint8_t* const to = sm + C::F_OFF + ((lane & 0x18) + 2 * (lane & 3) + (lane >> 2 & 1)) * (4 * G);   // [tile][q4][half]
        if constexpr (G == 4) *reinterpret_cast<uint4*>(to) = make_uint4(f[0], f[1], f[2], f[3]);
        else *reinterpret_cast<uint2*>(to) = make_uint2(f[0], f[1]);
      }
      if (__any_sync(0xffffffffu, raised)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float by = __shfl_sync(0xffffffffu, alpha[n], 4 * (2 * q4 + e));
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                o[g][h][n][e] *= by;
                o[g][h][n][2 + e] *= by;
              }
          }
      }
      __syncwarp();                            // (scores are read, V's scales are written)
      uint32_t* const s_f = reinterpret_cast<uint32_t*>(s_p) + lane * (2 * PP);   // (of this lane alone)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          uint32_t* const to = s_f + (n * kTiles + i) * (64 * PP);
          if constexpr (PP == 1) {
            *reinterpret_cast<uint2*>(to) = make_uint2(pf[n][i][0][0], pf[n][i][0][1]);
          } else if constexpr (PP == 2) {
            *reinterpret_cast<uint4*>(to) = make_uint4(pf[n][i][0][0], pf[n][i][0][1], pf[n][i][1][0], pf[n][i][1][1]);
          } else {
#pragma unroll
            for (int p = 0; p < PP; ++p) *reinterpret_cast<uint2*>(to + 2 * p) = make_uint2(pf[n][i][p][0], pf[n][i][p][1]);
          }
        }
      // ---- O^T += V^T P^T: slots 16 tile + q4, + 4, + 8, + 12 are the lane's k (so that four lanes' rows lie next to one another)
#pragma unroll C::V_TILES
      for (int i = 0; i < kTiles; ++i) {
        uint32_t b[NT][PP][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint32_t* const from = s_f + (n * kTiles + i) * (64 * PP);
          if constexpr (PP == 2) {
            const uint4 u = *reinterpret_cast<const uint4*>(from);
            b[n][0][0] = u.x; b[n][0][1] = u.y; b[n][1][0] = u.z; b[n][1][1] = u.w;
          } else {
#pragma unroll
            for (int p = 0; p < PP; ++p) {
              const uint2 u = *reinterpret_cast<const uint2*>(from + 2 * p);
              b[n][p][0] = u.x; b[n][p][1] = u.y;
            }
          }
        }
        uint32_t w[4][G / 2], f[2][G];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint8_t* const from = sm + C::V_OFF + (16 * i + 4 * e + q4) * C::RB + r * (C::RB / 8);
          if constexpr (G == 4) {
            const uint2 u = *reinterpret_cast<const uint2*>(from);
            w[e][0] = u.x; w[e][1] = u.y;
          } else {
            w[e][0] = *reinterpret_cast<const uint32_t*>(from);
          }
        }
        {
          const uint4* const from = reinterpret_cast<const uint4*>(sm + C::F_OFF + (8 * i + 2 * q4) * (4 * G));
          const uint4 u = from[0];
          if constexpr (G == 4) {
            const uint4 z = from[1];
            f[0][0] = u.x; f[0][1] = u.y; f[0][2] = u.z; f[0][3] = u.w;
            f[1][0] = z.x; f[1][1] = z.y; f[1][2] = z.z; f[1][3] = z.w;
          } else {
            f[0][0] = u.x; f[0][1] = u.y; f[1][0] = u.z; f[1][1] = u.w;
          }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t x01 = both(w[0][g / 2], w[1][g / 2], g), x23 = both(w[2][g / 2], w[3][g / 2], g);
          const uint32_t a8 = f[0][g], am = mul_bf16x2(a8, 0xc340c340u), b8 = f[1][g], bm = mul_bf16x2(b8, 0xc340c340u);   // -192
          const uint32_t va[2][4] = {{value_bf16<0>(x01, kv, a8, am), value_bf16<1>(x01, kv, a8, am), value_bf16<0>(x23, kv, b8, bm),
                                      value_bf16<1>(x23, kv, b8, bm)},
                                     {value_bf16<2>(x01, kv, a8, am), value_bf16<3>(x01, kv, a8, am), value_bf16<2>(x23, kv, b8, bm),
                                      value_bf16<3>(x23, kv, b8, bm)}};
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int p = PP - 1; p >= 0; --p)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                float (&z)[4] = o[g][h][n];
                if constexpr (F32) {           // (rounded sums: a plane of 16 slots at a time)
                  float d[4];
                  mma_bf16(d, va[h], b[n][p][0], b[n][p][1], 0.f, 0.f, 0.f, 0.f);
#pragma unroll
                  for (int e = 0; e < 4; ++e) z[e] += d[e];
                } else {
                  mma_bf16(z, va[h], b[n][p][0], b[n][p][1], z[0], z[1], z[2], z[3]);
                }
              }
        }
      }
      __syncwarp();                            // (V and P are read)
      if (more || beyond) load(after, to, x, 1);
      loaded = beyond;
      if (!F32 && ++links == kChain && more) {
        if (chained) add_chain();
        one_plane();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          put(n, 0, 1.f);
          put(n, 1, 1.f);
          m_then[n] = m[n];
        }
        chained = true;
        links = 0;
        clear();
      }
    }
    // ---- the item's (or its part's) sums
    if (chained) add_chain();
    one_plane();
    const bool whole = s.c0 == 0 && s.c1 == s.units;
    const int live = min(NQ, a.T * a.G - s.qb * NQ);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int v = 8 * n + r;
      float sum = l[n];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (v >= s.nq) sum = 0.f;                // (a vector past the nodes: zeros)
      const float top = sum == 0.f ? -INFINITY : m[n] == -INFINITY ? 0.f : m[n];   // (NaN scores: no maximum)
      const float inv = sum == 0.f ? 0.f : whole ? 1.f / sum : 1.f;
      if (q4 == 0 && v < live) {
        if (whole) {
          store_lse(a, s.b, vector_of(a, s.h, s.qb, v), top, sum);
        } else {
          a.part_ml[(part * 2) * NQ + v] = top;
          a.part_ml[(part * 2 + 1) * NQ + v] = sum;
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int to = 8 * n + 2 * q4 + e;
        const float by = __shfl_sync(0xffffffffu, inv, 4 * (2 * q4 + e));
        if (to >= live) continue;
        if (by == 0.f)
#pragma unroll
          for (int g = 0; g < G; ++g) o[g][0][n][e] = o[g][0][n][2 + e] = o[g][1][n][e] = o[g][1][n][2 + e] = 0.f;
        if (!whole) {
          put(n, e, by);
          continue;
        }
        const Vec w = vector_of(a, s.h, s.qb, to);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int d = 0; d < 4; ++d) store_out<T>(a, s.b, w, g * kGroup + 4 * r + d, o[g][d / 2][n][d % 2 * 2 + e] * by);
      }
    }
  }
}

template <int HD, int NQ, bool F32>
cudaError_t launch(const TreeArgs& a, cudaStream_t s) {
  using C = Cfg<HD, NQ, F32>;
  const auto k = k_tree_i4<HD, NQ, F32>;
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, k, C::smem(CDSL_TREE_MAX_BATCH))) return e;
  return launch_pdl(k, dim3((a.blocks + kWarps - 1) / kWarps), dim3(32 * kWarps), C::smem(a.c.batch), s, a);
}

template <typename F>
auto by_shape(const Cache& c, int NQ, bool f32, F&& f) {   // f(Cfg's parameters as constants)
  using std::bool_constant;
  using std::integral_constant;
  auto g = [&](auto hd, auto nq) { return f32 ? f(hd, nq, bool_constant<true>()) : f(hd, nq, bool_constant<false>()); };
  auto h = [&](auto hd) {
    if (NQ == 8) return g(hd, integral_constant<int, 8>());
    return NQ == 4 ? f(hd, integral_constant<int, 4>(), bool_constant<false>()) : f(hd, integral_constant<int, 16>(), bool_constant<false>());
  };
  return c.hd == 128 ? h(integral_constant<int, 128>()) : h(integral_constant<int, 64>());
}

}  // namespace

int i4_blocks_per_sm(const Cache& c, int NQ, bool f32) {
  return by_shape(c, NQ, f32, [](auto hd, auto nq, auto f) { return Cfg<hd(), nq(), f()>::WARPS; });
}

cudaError_t launch_tree_i4(const TreeArgs& a, cudaStream_t s) {
  return by_shape(a.c, a.NQ, a.dtype == CDSL_DTYPE_F32, [&](auto hd, auto nq, auto f) { return launch<hd(), nq(), f()>(a, s); });
}

}  // namespace tree
}  // namespace cdsl
