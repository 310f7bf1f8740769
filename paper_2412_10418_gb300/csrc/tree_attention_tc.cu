// tree_attention_tc.cu -- cdsl_tree_attention of bf16 queries on the 5th-generation tensor cores.
//
// Codes go from HBM to the MMA as they are. A chunk of 128 slots is the MMA's M = 128, the query vectors its
// N (16, 32 or 64: a tree has few of them, and as M they would be padded to 128), so that the work
// follows the number of queries:
//   S^T = K Q^T   M = 128 slots, N = NQ vectors, K = head_dim      K tile K-major, as TMA lands it
//   O^T = V^T P^T  M = head_dim, N = NQ (x planes), K = 128 slots   V tile MN-major, as TMA lands it
// An e4m3 cache takes kind::f8f6f4, twice the rate and half the shared memory of bf16 and no
// conversion of K and V at all. What is not e4m3 is split into e4m3 planes instead: a query row, scaled
// by a power of two to at most 448, is hi + lo, each to 4 bits, together bf16's 8 (to 2^-18 of the row's
// largest); a probability is hi + lo / 32 (to 2^-10 of itself), the planes side by side along N with
// sums of their own in TMEM. A bf16 cache takes kind::f16 with Q as it is and P in two bf16 planes.
// The rows' power-of-two scales never touch the codes: K's multiplies the thread's scores, V's the
// thread's probabilities (relative to the largest V scale so far, so that they use e4m3's range).
//
// Every chunk's P is relative to that chunk's own column maxima and largest V scale, and its O^T starts
// anew in TMEM and is added to fp32 sums in registers with the factor that this takes, so that small
// probabilities keep their bits beside one large one chunks away, and no sum is a chain of the tensor
// core's truncating additions. The sums' own reference is raised only when a maximum passes it by
// more than 2^kMargin.
//
// Warps: one loads the chunks by TMA into a ring (a box per page piece, the scale bytes with V), one issues
// the MMAs, the next chunk's S while this one's softmax runs (S has two buffers in TMEM), and four, or
// eight at NQ = 64 (half of the columns each), do the softmax: a thread owns a slot (a TMEM lane) of the chunk and
// walks the query vectors (columns), and later one dimension of O^T. Column maxima come from redux.sync over
// a warp and shared memory over the warps. Each thread keeps its own slots' share of the sums l.
//
// Waits are bounded (tc::kWaitLimitNs): on expiry CDSL_ETIMEOUT is latched, the role winds down and
// the block frees its TMEM and exits.
#include <cuda.h>

#include <algorithm>

#include "gemm.cuh"
#include "kernels.h"
#include "tree_attention.cuh"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {


template <int HD, int NQ, bool F8>
struct Cfg {
  static constexpr int EB = F8 ? 1 : 2;
  static constexpr int CQ = NQ < 32 ? NQ : 32;             // columns of a softmax thread
  static constexpr int SOFT = kKeys * (NQ / CQ);           // softmax threads
  static constexpr int THREADS = SOFT + 64;                // and warps SOFT / 32 (loads), SOFT / 32 + 1 (MMAs)
  static constexpr int KROW = HD * EB;                     // bytes of a K or V row
  static constexpr int BW = KROW < 128 ? KROW : 128;       // of it per tile block
  static constexpr int NB = KROW / BW;                     // blocks
  static constexpr uint32_t BLOCK = kKeys * BW;            // bytes of a block of a chunk
  static constexpr uint32_t TILE = NB * BLOCK;             // K or V of a chunk
  static constexpr int QP = F8 ? 2 : 1;                    // planes of Q
  static constexpr uint32_t Q_PLANE = NQ * KROW;
  static constexpr int RB = 2 * NQ;                        // bytes of a P row (slot): e4m3 both planes, bf16 one
  static constexpr int PP = F8 ? 1 : 2;                    // P tiles
  static constexpr uint32_t P_TILE = kKeys * RB;
  static constexpr uint32_t FIXED = QP * Q_PLANE + PP * P_TILE;
  // two blocks per SM where two stages and the registers of one group of softmax warps fit, else one
  static constexpr uint32_t LIMIT2 = 109 * 1024, LIMIT1 = 216 * 1024;
  static constexpr int CTAS = SOFT == kKeys && FIXED + 4 * TILE <= LIMIT2 ? 2 : 1;
  static constexpr int FIT = ((CTAS == 2 ? LIMIT2 : LIMIT1) - FIXED) / (2 * TILE);
  static constexpr int NST = FIT > 4 ? 4 : FIT;            // ring stages of K and V
  static_assert(NST >= 2, "stages");
  static constexpr uint32_t Q_OFF = 0;
  static constexpr uint32_t P_OFF = Q_OFF + QP * Q_PLANE;
  static constexpr uint32_t KV_OFF = (P_OFF + PP * P_TILE + 1023) / 1024 * 1024;
  static constexpr uint32_t SCALE_OFF = KV_OFF + NST * 2 * TILE;   // a byte per slot, K and V
  static constexpr uint32_t PLAN_OFF = SCALE_OFF + NST * 2 * kKeys;
  static constexpr int OC = F8 ? 2 * NQ : NQ;              // TMEM columns of O^T
  static constexpr uint32_t TMEM = 4 * NQ;                 // S twice, O
  static constexpr size_t smem(int batch) { return 1024 + PLAN_OFF + (batch + 1) * 4; }
};

template <int HD, int NQ, bool F8>
__global__ void __launch_bounds__(Cfg<HD, NQ, F8>::THREADS, Cfg<HD, NQ, F8>::CTAS)
    k_tree_tc(TreeArgs a, const __grid_constant__ CUtensorMap map) {
  using C = Cfg<HD, NQ, F8>;
  constexpr int NST = C::NST, kSoft = C::SOFT, kProducer = kSoft / 32, kIssuer = kProducer + 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const sm = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
  int* const s_first = reinterpret_cast<int*>(sm + C::PLAN_OFF);
  __shared__ __align__(8) uint64_t k_full[NST], v_full[NST], k_empty[NST], v_empty[NST];
  __shared__ __align__(8) uint64_t s_full[2], s_empty[2], p_full, p_empty, q_full, done;
  __shared__ uint32_t s_tmem;
  // per query vector: score factor (softmax scale and the row's own), the chunk's maximum in base 2, its
  // factors to the sums (of l, and of O^T with V's scale: two chunks' in turn), the sums' reference, factor of a raise
  __shared__ __align__(16) float s_qs[NQ], s_mq[NQ], s_b[NQ], s_bo[2][NQ], s_f[NQ], s_inv[NQ];
  __shared__ float s_ref[NQ], s_wmax[4][NQ], s_l[4][NQ];
  __shared__ int s_bad[NQ];                    // the query is not finite
  __shared__ long long s_out[NQ];              // where its output begins
  __shared__ uint32_t s_mask[NQ + 1][kWords];  // of the block's nodes
  __shared__ uint32_t s_pieces[NST];           // pieces of a stage's chunk that hold slots, as bits
  __shared__ int s_wv[4];
  const Cache& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      tc::mbar_init(&k_full[i], 1);
      tc::mbar_init(&v_full[i], 1);
      tc::mbar_init(&k_empty[i], 1);
      tc::mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&s_full[i], 1);
      tc::mbar_init(&s_empty[i], kSoft);
    }
    tc::mbar_init(&p_full, kSoft);
    tc::mbar_init(&p_empty, 1);
    tc::mbar_init(&q_full, kSoft);
    tc::mbar_init(&done, 1);
    tc::fence_mbar_init();
  }
  if (warp == kIssuer) tc::tmem_alloc(&s_tmem, C::TMEM);
  if (warp == kProducer && lane == 0) tc::tma_prefetch_map(&map);
  pdl_wait();
  pdl_launch_dependents();
  tc::tc_fence_before();
  build_plan(a, s_first);                      // (ends in a block barrier)
  tc::tc_fence_after();
  const uint32_t tmem = s_tmem, t_o = tmem + 2 * NQ;
  const uint32_t sbase = tc::smem_u32(sm);
  if (blockIdx.x == 0) {
    check_lens(a);
    for (int b = threadIdx.x; b <= c.batch; b += C::THREADS) a.plan[b] = s_first[b];
  }
  const int total = s_first[c.batch], runs = runs_of(a, total);
  const int begin = (int)blockIdx.x < runs ? run_begin(blockIdx.x, total, runs) : 0;
  const int end = (int)blockIdx.x < runs ? run_begin(blockIdx.x + 1, total, runs) : 0;

  if (warp == kProducer) {
    load_chunks<HD, F8, NST>(a, s_first, begin, end, map, sm + C::KV_OFF, sm + C::SCALE_OFF, s_pieces, k_full,
                             v_full, k_empty, v_empty);
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------------------- MMAs
    if (lane == 0) {
      constexpr uint32_t formats = F8 ? 0u : (1u << 7) | (1u << 10);
      constexpr uint32_t idesc = (1u << 4) | formats | (128u >> 4) << 24;
      constexpr uint32_t idesc_s = idesc | (uint32_t)(NQ >> 3) << 17;
      constexpr uint32_t idesc_o = idesc | (uint32_t)(C::OC >> 3) << 17 | 1u << 15 | 1u << 16;
      constexpr int STEP = 32 / C::EB;         // slots per MMA of P V
      auto mma = [](uint32_t d, uint64_t x, uint64_t y, uint32_t id, bool add) {
        if constexpr (F8) tc::umma_f8(d, x, y, id, add);
        else tc::umma_bf16(d, x, y, id, add);
      };
      // (a descriptor's low bits are its tile's address / 16: steps add to them)
      constexpr uint32_t next = C::NB > 1 ? C::BLOCK : 8 * C::BW;   // of V along M; head_dim 64: what the
                                               // second half of the M = 128 lanes reads and sums is not used
      const uint64_t desc_k = tc::desc_rows(sbase + C::KV_OFF, C::BW, 16);
      const uint64_t desc_q = tc::desc_rows(sbase + C::Q_OFF, C::BW, 16);
      const uint64_t desc_v = tc::desc_rows(sbase + C::KV_OFF + C::TILE, C::BW, next);
      const uint64_t desc_p = tc::desc_rows(sbase + C::P_OFF, C::RB, 16);
      auto s_mma = [&](int i) {                // S of chunk i
        const uint64_t k = desc_k + (uint32_t)(i % NST) * (2 * C::TILE / 16);
        const uint32_t d = tmem + (i & 1) * NQ;
#pragma unroll 1
        for (int p = C::QP - 1; p >= 0; --p)
#pragma unroll 1
          for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
            for (int x = 0; x < C::BW / 32; ++x)
              mma(d, k + (nb * C::BLOCK / 16 + 2 * x),
                  desc_q + ((uint32_t)(p * C::Q_PLANE + nb * NQ * C::BW) / 16 + 2 * x), idesc_s,
                  p < C::QP - 1 || nb + x > 0);
        tc::umma_commit(&s_full[i & 1]);
        tc::umma_commit(&k_empty[i % NST]);
      };
      auto pv = [&](int i) {                   // the P V of chunk i
        if (!tc::mbar_wait(&p_full, i & 1, a.status) ||
            !tc::mbar_wait(&v_full[i % NST], parity(i, NST), a.status))
          return false;
        tc::tc_fence_after();
        const uint64_t v = desc_v + (uint32_t)(i % NST) * (2 * C::TILE / 16);
#pragma unroll 1
        for (int p = C::PP - 1; p >= 0; --p)
#pragma unroll 4
          for (int k = 0; k < kKeys / STEP; ++k)
            mma(t_o, v + k * (STEP * C::BW / 16), desc_p + (p * C::P_TILE / 16 + k * (STEP * C::RB / 16)), idesc_o,
                k > 0 || p < C::PP - 1);
        tc::umma_commit(&p_empty);
        tc::umma_commit(&v_empty[i % NST]);
        return true;
      };
      // chunk i's S goes before chunk i - 1's P V, except that a new item's queries are staged only after
      // the last one's P V
      int it = 0, seg = 0;
      bool ok = true;
      for (int unit = begin; unit < end && ok; ++seg) {
        const Segment s = segment_at(a, s_first, unit, end);
        for (int ch = s.c0; ch <= s.c1; ++ch) {   // (one round more: the last chunk's P V)
          if (ch < s.c1) {
            ok = (ch > s.c0 || tc::mbar_wait(&q_full, seg & 1, a.status)) &&
                 tc::mbar_wait(&s_empty[it & 1], parity(it, 2) ^ 1, a.status) &&
                 tc::mbar_wait(&k_full[it % NST], parity(it, NST), a.status);
            if (!ok) break;
            tc::tc_fence_after();
            s_mma(it);
          }
          if (ch > s.c0 && !(ok = pv(it - 1))) break;
          if (ch < s.c1) ++it;
        }
        unit += s.c1 - s.c0;
      }
      // what was issued completes before the block's memory goes
      tc::umma_commit(&done);
      tc::mbar_wait(&done, 0, a.status);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------------------- softmax
    constexpr int CQ = C::CQ;
    const int tid = threadIdx.x;
    const int r = tid % kKeys;                 // slot of the chunk = TMEM lane; dimension of O^T
    const int c0 = tid / kKeys * CQ;           // this group's columns: c0 .. c0 + CQ - 1
    const int w4 = warp & 3;
    const uint32_t lane_base = (uint32_t)(w4 * 32) << 16;
    auto sync = [] { tc::named_barrier(1, kSoft); };
    const bool q_aligned = (reinterpret_cast<uintptr_t>(a.q) | (a.sq[0] | a.sq[1] | a.sq[2]) * 2) % 16 == 0;
    int it = 0;
    bool failed = false, gone = false;
    for (int unit = begin; unit < end && !gone;) {
      const Segment s = segment_at(a, s_first, unit, end);
      stage_queries<HD, NQ, F8, kSoft>(a, s, tid, q_aligned, sm + C::Q_OFF, [&](int v, const Vec& x, float qs, bool bad) {
        s_qs[v] = v < s.nq ? qs : 0.f;
        s_ref[v] = -INFINITY;
        s_bad[v] = bad;
        s_out[v] = s.b * a.so[0] + x.t * a.so[1] + x.h * a.so[2];
      });
      const int t0 = s.qb * NQ / a.G;          // the block's first node
      for (int i = tid; i < (NQ + 1) * kWords; i += kSoft) {
        const int t = t0 + i / kWords, w = i % kWords;
        s_mask[i / kWords][w] = t < s.nodes && w < a.W ? __ldg(a.mask + ((size_t)s.b * a.T + t) * a.W + w) : 0u;
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&q_full);
      sync();
      float l[CQ], o[CQ];
#pragma unroll
      for (int v = 0; v < CQ; ++v) l[v] = o[v] = 0.f;
      // a chunk's O^T (its P V complete) to the sums, with its factors
      auto add_o = [&](int i) {
        tc::tc_fence_after();
        if (r < HD) {                          // (whole warps)
#pragma unroll
          for (int g = 0; g < CQ; g += 16) {
            if (c0 + g >= s.nq) break;
            uint32_t x[16], y[16];
            tc::tmem_ld16_nowait(t_o + lane_base + c0 + g, x);
            if constexpr (F8) tc::tmem_ld16_nowait(t_o + lane_base + NQ + c0 + g, y);
            tc::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const float4 b = *reinterpret_cast<const float4*>(&s_bo[i & 1][c0 + g + e]);
              const float f[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float z = __uint_as_float(x[e + j]);
                if constexpr (F8) z += __uint_as_float(y[e + j]);
                o[g + e + j] = fmaf(z, f[j], o[g + e + j]);
              }
            }
          }
        }
        tc::tc_fence_before();
      };

      for (int ch = s.c0; ch < s.c1; ++ch, ++it) {
        const bool first = ch == s.c0;
        const int st = it % NST;
        // ---- this thread's slot: the scales, and which vectors see it (bit v of vis). Only chunks with slots
        //      of the tree or past the item's ask (a warp's branch).
        bool ok = tc::mbar_wait(&v_full[st], parity(it, NST), a.status);
        const int slot = ch * kKeys + r, node = slot - s.len;
        const bool valid = slot < s.keys && s_pieces[st] >> (r >> min(c.page_shift, 7)) & 1;
        const uint32_t kb = valid ? sm[C::SCALE_OFF + st * 2 * kKeys + r] : 127u;
        const uint32_t vb = valid ? sm[C::SCALE_OFF + (st * 2 + 1) * kKeys + r] : 0u;
        const float ks = scale_value(kb);
        const bool masked = __any_sync(0xffffffffu, !valid || node >= 0);
        uint32_t vis = ~0u;
        if (masked && (!valid || node >= 0)) {
          vis = 0;
          if (valid) {
            const uint64_t group = a.G < 64 ? (1ull << a.G) - 1 : ~0ull;
            const int first_t = (s.qb * NQ + c0) / a.G;
#pragma unroll 2
            for (int t = first_t, v = t * a.G - s.qb * NQ - c0; v < min(CQ, s.nq - c0); ++t, v += a.G)
              if (s_mask[t - t0][node >> 5] >> (node & 31) & 1)
                vis |= (uint32_t)(v < 0 ? group >> -v : group << v);
          }
        }
        // ---- scores, and their maxima over the warp's slots: lane v has column c0 + v's
        ok = ok && tc::mbar_wait(&s_full[it & 1], parity(it, 2), a.status);
        if (!__all_sync(0xffffffffu, ok)) failed = true;
        tc::tc_fence_after();
        float t[CQ], wm = -INFINITY;
#pragma unroll
        for (int g = 0; g < CQ; g += 16) {
          if (c0 + g >= s.nq) break;
          uint32_t x[16];
          tc::tmem_ld16_nowait(tmem + (it & 1) * NQ + lane_base + c0 + g, x);
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) t[g + e] = __uint_as_float(x[e]) * ks;
          if (masked) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!(vis >> (g + e) & 1)) t[g + e] = -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float top = warp_fmax(t[g + e]);
            if (lane == g + e) wm = top;
          }
        }
        tc::tc_fence_before();
        tc::mbar_arrive(&s_empty[it & 1]);
        if (lane < CQ) s_wmax[w4][c0 + lane] = wm;
        if (F8 && c0 == 0) {
          const int wv = __reduce_max_sync(0xffffffffu, vb == 255 ? 0 : (int)vb);
          if (lane == 0) s_wv[w4] = wv;
        }
        if (tc::named_barrier_or(1, kSoft, failed)) {
          gone = true;
          break;
        }
        // ---- the chunk's references: a thread per vector
        const int vref = F8 ? max(max(s_wv[0], s_wv[1]), max(s_wv[2], s_wv[3])) : 127;
        bool raise = false;
        if (tid < NQ) {
          const int v = tid;
          const float top = fmaxf(fmaxf(s_wmax[0][v], s_wmax[1][v]), fmaxf(s_wmax[2][v], s_wmax[3][v]));
          const float mq = top == -INFINITY ? 0.f : top * s_qs[v];
          float ref = s_ref[v], f = 1.f;
          if (top > -INFINITY && !(mq - ref <= kMargin)) {
            raise = ref > -INFINITY;
            f = raise ? ex2(ref - mq) : 1.f;   // (no reference: nothing seen so far, the sums are 0)
            s_ref[v] = ref = mq;
          }
          const float b = top == -INFINITY ? 0.f : ex2(mq - ref);
          s_mq[v] = mq;
          s_b[v] = b;
          s_f[v] = f;
          s_bo[it & 1][v] = F8 ? b * (1.f / (1 << kPShift)) * ex2((float)(vref - 127)) : b;
        }
        raise = tc::named_barrier_or(1, kSoft, raise);
        // ---- the chunk before's O^T; its P may be overwritten
        if (it > 0) {
          if (!__all_sync(0xffffffffu, tc::mbar_wait(&p_empty, (it - 1) & 1, a.status))) failed = true;
          else if (!first) add_o(it - 1);
        }
        if (raise) {
#pragma unroll
          for (int v = 0; v < CQ; ++v) {
            const float f = s_f[c0 + v];
            l[v] *= f;
            o[v] *= f;
          }
        }
        // ---- probabilities, their sums, V's scale on them
        const int ve = F8 ? (int)vb - vref + kPShift : 0;
        const float vf = !valid ? 0.f : ve < -126 ? 0.f : __uint_as_float((uint32_t)(ve + 127) << 23);
        const bool bad_v = __any_sync(0xffffffffu, vb == 255);
        uint8_t* const p = sm + C::P_OFF;
#pragma unroll
        for (int g = 0; g < CQ; g += 16) {
          if (c0 + g >= s.nq) break;
          float x[16];
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 qs = *reinterpret_cast<const float4*>(&s_qs[c0 + g + e]);
            const float4 mq = *reinterpret_cast<const float4*>(&s_mq[c0 + g + e]);
            const float4 b = *reinterpret_cast<const float4*>(&s_b[c0 + g + e]);
            x[e] = ex2(fmaf(t[g + e], qs.x, -mq.x));
            x[e + 1] = ex2(fmaf(t[g + e + 1], qs.y, -mq.y));
            x[e + 2] = ex2(fmaf(t[g + e + 2], qs.z, -mq.z));
            x[e + 3] = ex2(fmaf(t[g + e + 3], qs.w, -mq.w));
            l[g + e] = fmaf(x[e], b.x, l[g + e]);
            l[g + e + 1] = fmaf(x[e + 1], b.y, l[g + e + 1]);
            l[g + e + 2] = fmaf(x[e + 2], b.z, l[g + e + 2]);
            l[g + e + 3] = fmaf(x[e + 3], b.w, l[g + e + 3]);
          }
          if constexpr (F8) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= vf;
          }
          if (bad_v) {                         // a V that is not finite: NaN where it is seen
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (vb == 255) x[e] = vis >> (g + e) & 1 ? __uint_as_float(0x7fc00000u) : 0.f;
          }
          if constexpr (F8) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const __half2 z0 = __floats2half2_rn(x[4 * i], x[4 * i + 1]), z1 = __floats2half2_rn(x[4 * i + 2], x[4 * i + 3]);
              __half2 h0, h1;
              hi[i] = f8x4(z0, z1);
              f8x4_half(hi[i], &h0, &h1);
              lo[i] = f8x4(__hsub2(z0, h0), __hsub2(z1, h1));
            }
            *reinterpret_cast<uint4*>(p + tc::row_offset(r, (c0 + g) / 16, C::RB)) =
                make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(p + tc::row_offset(r, (NQ + c0 + g) / 16, C::RB)) =
                make_uint4(lo[0], lo[1], lo[2], lo[3]);
          } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float u = x[half * 8 + 2 * i], w = x[half * 8 + 2 * i + 1];
                const __nv_bfloat162 h = __floats2bfloat162_rn(u, w);
                const __nv_bfloat162 z = __floats2bfloat162_rn(u - __low2float(h), w - __high2float(h));
                hi[i] = *reinterpret_cast<const uint32_t*>(&h);
                lo[i] = *reinterpret_cast<const uint32_t*>(&z);
              }
              const uint32_t off = tc::row_offset(r, (c0 + g) / 8 + half, C::RB);
              *reinterpret_cast<uint4*>(p + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
              *reinterpret_cast<uint4*>(p + C::P_TILE + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
          }
        }
        if (!valid && c0 == 0) {               // nothing of its V row (page garbage, no copy) may reach the sums
          uint8_t* v = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + r * C::BW;
#pragma unroll
          for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
            for (int i = 0; i < C::BW; i += 16)
              *reinterpret_cast<uint4*>(v + nb * C::BLOCK + i) = make_uint4(0u, 0u, 0u, 0u);
        }
        tc::fence_proxy_async();
        tc::tc_fence_before();
        tc::mbar_arrive(&p_full);
      }
      if (gone) break;
      // ---- the last chunk's O^T, and the item's (or its part's) sums
      if (!__all_sync(0xffffffffu, tc::mbar_wait(&p_empty, (it - 1) & 1, a.status))) failed = true;
      if (tc::named_barrier_or(1, kSoft, failed)) {
        gone = true;
        break;
      }
      add_o(it - 1);
#pragma unroll
      for (int g = 0; g < CQ; g += 16) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = l[g + e];
        warp_sums<16>(x);
        if ((lane & 1) == 0) s_l[w4][c0 + g + (lane >> 1)] = x[0];
      }
      sync();
      // ---- a thread per vector: its sum (0: it saw nothing; of a query that is not finite: NaN)
      const bool whole = s.c0 == 0 && s.c1 == s.units;
      const size_t part = (size_t)blockIdx.x * 2 + (s.c0 == 0);
      const int live = min(NQ, a.T * a.G - s.qb * NQ);
      if (tid < live) {
        const int v = tid;
        float sum = 0.f;
        if (v < s.nq && s.keys > 0) sum = s_l[0][v] + s_l[1][v] + s_l[2][v] + s_l[3][v];
        const float m = sum == 0.f ? -INFINITY : s_ref[v] == -INFINITY ? 0.f : s_ref[v];   // (NaN scores: no maximum)
        if (sum != 0.f && s_bad[v]) sum = __uint_as_float(0x7fc00000u);
        if (whole) {
          s_inv[v] = sum == 0.f ? 0.f : 1.f / sum;
          store_lse(a, s.b, vector_of(a, s.h, s.qb, v), m, sum);
        } else {
          s_inv[v] = sum == 0.f ? 0.f : 1.f;
          a.part_ml[(part * 2) * NQ + v] = m;
          a.part_ml[(part * 2 + 1) * NQ + v] = sum;
        }
      }
      sync();
      if (r < HD) {
#pragma unroll
        for (int v = 0; v < CQ; ++v) {
          if (c0 + v >= live) break;
          const float inv = s_inv[c0 + v], x = inv == 0.f ? 0.f : o[v] * inv;
          if (whole) static_cast<__nv_bfloat16*>(a.out)[s_out[c0 + v] + r] = __float2bfloat16_rn(x);
          else a.part_o[(part * NQ + c0 + v) * HD + r] = x;
        }
      }
      sync();                                  // the statistics are read
      unit += s.c1 - s.c0;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) tc::tmem_dealloc(tmem, C::TMEM);
}

template <int HD, int NQ, bool F8>
cudaError_t launch(const TreeArgs& a, cudaStream_t s) {
  using C = Cfg<HD, NQ, F8>;
  CUtensorMap map;
  if (encode_cache_map<HD, F8>(a, &map)) return cudaErrorInvalidValue;
  auto k = k_tree_tc<HD, NQ, F8>;
  static const cudaError_t set =
      cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::smem(CDSL_TREE_MAX_BATCH));
  if (set != cudaSuccess) return set;
  return launch_pdl(k, dim3(a.blocks), dim3(C::THREADS), C::smem(a.c.batch), s, a, map);
}

template <typename F>
auto by_query_block(int NQ, F&& f) {
  return NQ == 16 ? f(std::integral_constant<int, 16>())
                  : NQ == 32 ? f(std::integral_constant<int, 32>()) : f(std::integral_constant<int, 64>());
}

}  // namespace

int tc_blocks_per_sm(const Cache& c, int NQ) {
  return by_query_block(NQ, [&](auto n) {
    if (c.hd == 128) return c.eb == 1 ? Cfg<128, n(), true>::CTAS : Cfg<128, n(), false>::CTAS;
    return c.eb == 1 ? Cfg<64, n(), true>::CTAS : Cfg<64, n(), false>::CTAS;
  });
}

cudaError_t launch_tree_tc(const TreeArgs& a, cudaStream_t s) {
  return by_query_block(a.NQ, [&](auto n) {
    if (a.c.hd == 128) return a.c.eb == 1 ? launch<128, n(), true>(a, s) : launch<128, n(), false>(a, s);
    return a.c.eb == 1 ? launch<64, n(), true>(a, s) : launch<64, n(), false>(a, s);
  });
}

}  // namespace tree
}  // namespace cdsl
