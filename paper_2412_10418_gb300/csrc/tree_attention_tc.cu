// tree_attention_tc.cu -- cdsl_tree_attention of bf16 queries with at most 32 query vectors per K/V head, on the
// 5th-generation tensor cores: cache slots are the MMA's M = 128.
//
// Codes go from HBM to the MMA as they are. A chunk of 128 slots is M and the query vectors are N (16 or
// 32; as M they would be padded to 128), so that the work follows the number of queries:
//   S^T = K Q^T     M = 128 slots, N = NQ vectors, K = head_dim    K tile K-major, as TMA lands it
//   O^T = V^T P^T   M = head_dim, N = NQ vectors, K = 128 slots    V tile MN-major, as TMA lands it
// An e4m3 cache takes kind::f8f6f4, twice the rate and half the shared memory of bf16 and no
// conversion of K and V at all. What is not e4m3 is split into two e4m3 planes instead, hi and the rest, each to 4
// bits: a query row, scaled by a power of two to at most 448 (together bf16's 8 bits, to 2^-18 of the row's
// largest), and the probabilities. A bf16 cache takes kind::f16 with Q as it is and
// P in two bf16 planes. The rows' power-of-two scales never touch the codes: K's multiplies the
// thread's scores, V's the thread's probabilities.
//
// e4m3 ends at a step of 2^-9, so what the two planes of P keep depends on V's scales, by which P is multiplied. The
// rest is stored times 2^kLoShift and has columns of O^T of its own (both planes are one MMA of twice the columns): a
// probability is held to 2^-8 of itself (2^-10 on average), or to a step of 2^-21 of the chunk's largest scale, if
// that is more. Where the chunk's V scales lie more than 2^kSpread apart, that could be all that a slot with a small scale
// has, next to one that has no weight, or is not seen: there the softmax threads multiply P and V themselves,
// in fp32 (the call below with every chunk so: 710 us).
//
// Every chunk's P is relative to that chunk's own column maxima and largest V scale, and its O^T starts
// anew in TMEM and is added to fp32 sums in registers with the factor that this takes, so that small
// probabilities keep their bits beside one large one chunks away, and no sum is a chain of the tensor
// core's truncating additions. The sums' own reference is raised only when a maximum passes it by
// more than 2^kMargin.
//
// Six warps. One loads the chunks by TMA into a ring (a box per page piece, the scale bytes with V), one issues
// the MMAs, the next chunk's S while this one's softmax runs (S has two buffers in TMEM), and four do the
// softmax: a thread owns a slot (a TMEM lane) of the chunk and walks the query vectors (columns), and later one
// dimension of O^T. Column maxima come from redux.sync over a warp and shared memory over the warps, the one
// barrier of a chunk; each warp then works out the columns' factors for itself. Each thread keeps its own
// slots' share of the sums l. Bound by HBM where a call fills the device: 64 sequences of up to 8,192 tokens, 8 heads of
// 128 in e4m3, four query heads each, one token: 130 to 137 us by inputs, 87 to 92 % of the copy bandwidth; by latency in
// small ones: one of 512 tokens in 9 us with the joining. The MMA's N is 16 or 32 by the number of vectors: 8 sequences of
// 16,384, 16 vectors: 54 us with 16, 67 with 32 (fewer blocks on an SM); 32 vectors: 70 us in one block, 92 as rows.
//
// Waits are bounded (by tc::kWaitLimitNs, the loading warp's by a number of tries): on expiry CDSL_ETIMEOUT is latched, the
// role winds down and the block frees its TMEM and exits.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "gemm.cuh"
#include "kernels.h"
#include "tree_attention.cuh"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {


constexpr float kMargin = 8.f;                 // base 2: a sum's reference is raised past it
constexpr int kPShift = 8;                     // e4m3 probabilities are stored times 2^kPShift <= 448, and
constexpr int kLoShift = 4;                    // what hi leaves of them, at most 2^(kPShift - 5), times 2^kLoShift more
constexpr int kSpread = 8;                     // octaves between V's scales in a chunk that P's two planes cover
constexpr int kSoft = kKeys;                   // softmax threads: one per slot of a chunk
constexpr int kThreads = kSoft + 64;
constexpr int kProducer = kSoft / 32, kIssuer = kProducer + 1;   // warps

template <int HD, int NQ, bool F8>
struct Cfg {
  static constexpr int EB = F8 ? 1 : 2;
  static constexpr int KROW = HD * EB;                     // bytes of a K or V row
  static constexpr int BW = KROW < 128 ? KROW : 128;       // of it per tile block
  static constexpr int NB = KROW / BW;                     // blocks
  static constexpr uint32_t BLOCK = kKeys * BW;            // bytes of a block of a chunk
  static constexpr uint32_t TILE = NB * BLOCK;             // K or V of a chunk
  static constexpr int QP = F8 ? 2 : 1;                    // planes of Q
  static constexpr uint32_t Q_PLANE = NQ * KROW;
  // P: a row per slot; e4m3: both planes in it; bf16: a tile per plane
  static constexpr int RB = 2 * NQ;
  static constexpr uint32_t P_TILE = kKeys * RB;
  static constexpr int OW = F8 ? 2 * NQ : NQ;              // columns of O^T: e4m3: of P's hi, then of the rest
  static constexpr uint32_t FIXED = QP * Q_PLANE + (F8 ? 1 : 2) * P_TILE;
  // two blocks per SM where two stages fit, else one
  static constexpr uint32_t LIMIT2 = 106 * 1024, LIMIT1 = 212 * 1024;
  static constexpr int CTAS = FIXED + 4 * TILE <= LIMIT2 ? 2 : 1;
  static constexpr int FIT = ((CTAS == 2 ? LIMIT2 : LIMIT1) - FIXED) / (2 * TILE);
  static constexpr int NST = FIT > 4 ? 4 : FIT;            // ring stages of K and V
  static_assert(NST >= 2, "stages");
  static constexpr uint32_t Q_OFF = 0;
  static constexpr uint32_t P_OFF = Q_OFF + QP * Q_PLANE;
  static constexpr uint32_t KV_OFF = (Q_OFF + FIXED + 1023) / 1024 * 1024;
  static constexpr uint32_t SCALE_OFF = KV_OFF + NST * 2 * TILE;   // a byte per slot, K and V
  static constexpr uint32_t PLAN_OFF = SCALE_OFF + NST * 2 * kKeys;
  static constexpr uint32_t TMEM = 4 * NQ;                 // S twice, O^T (a power of two)
  static constexpr size_t smem(int batch) { return 1024 + PLAN_OFF + plan_bytes(batch); }
};

template <int HD, int NQ, bool F8>
__global__ void __launch_bounds__(kThreads, Cfg<HD, NQ, F8>::CTAS)
    k_tree_tc(TreeArgs a, const __grid_constant__ CUtensorMap map) {
  using C = Cfg<HD, NQ, F8>;
  constexpr int NST = C::NST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const sm = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
  int* const s_first = reinterpret_cast<int*>(sm + C::PLAN_OFF);
  __shared__ __align__(8) uint64_t k_full[NST], v_full[NST], k_empty[NST], v_empty[NST];
  __shared__ __align__(8) uint64_t s_full[2], s_empty[2], p_full, p_empty, q_full, done;
  __shared__ uint32_t s_tmem;
  // per query vector: score factor (softmax scale and the row's own) and the end's 1 / l; the warps' maxima of two
  // chunks in turn; each warp's: the chunk's maximum in base 2, its factors to the sums of l, and of O^T with
  // V's scale (two chunks' in turn), and of a raise
  __shared__ __align__(16) float s_qs[NQ], s_inv[NQ], s_wmax[2][4][NQ];
  __shared__ __align__(16) float s_mq[4][NQ], s_b[4][NQ], s_bo[2][4][NQ], s_f[4][NQ];
  __shared__ float s_ref[NQ], s_l[4][NQ];
  __shared__ int s_bad[NQ];                    // the query is not finite
  __shared__ long long s_out[NQ];              // where its output begins
  __shared__ uint32_t s_mask[NQ + 1][kWords];  // of the block's nodes
  __shared__ uint32_t s_pieces[NST];           // pieces of a stage's chunk that hold slots, as bits
  __shared__ int s_wv[2][4];                   // V's largest and smallest scale byte in a warp's slots (smallest << 8)
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
  if (blockIdx.x == 0) check_lens(a);
  const int total = s_first[c.batch], runs = runs_of(a, total);
  const int begin = (int)blockIdx.x < runs ? run_begin(blockIdx.x, total, runs) : 0;
  const int end = (int)blockIdx.x < runs ? run_begin(blockIdx.x + 1, total, runs) : 0;

  if (warp == kProducer) {
    load_chunks<HD, F8, NST, false>(a, s_first, begin, end, map, sm + C::KV_OFF, sm + C::SCALE_OFF, s_pieces, k_full,
                             v_full, k_empty, v_empty);
  } else if (warp == kIssuer) {
    // ------------------------------------------------------------------------- MMAs
    if (lane == 0) {
      constexpr uint32_t formats = F8 ? 0u : (1u << 7) | (1u << 10);
      constexpr uint32_t idesc = (1u << 4) | formats | (128u >> 4) << 24;
      constexpr uint32_t idesc_s = idesc | (uint32_t)(NQ >> 3) << 17;
      constexpr uint32_t idesc_o = idesc | (uint32_t)(C::OW >> 3) << 17 | 1u << 15 | 1u << 16;
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
        for (int p = F8 ? 0 : 1; p >= 0; --p)
#pragma unroll 4
          for (int k = 0; k < kKeys / STEP; ++k)
            mma(t_o, v + k * (STEP * C::BW / 16), desc_p + (p * C::P_TILE / 16 + k * (STEP * C::RB / 16)), idesc_o,
                (!F8 && p < 1) || k > 0);
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
    const int r = threadIdx.x;                 // slot of the chunk = TMEM lane; dimension of O^T
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    auto sync = [] { tc::named_barrier(1, kSoft); };
    const bool q_aligned = (reinterpret_cast<uintptr_t>(a.q) | (a.sq[0] | a.sq[1] | a.sq[2]) * 2) % 16 == 0;
    int it = 0;
    bool failed = false, gone = false;
    for (int unit = begin; unit < end && !gone;) {
      const Segment s = segment_at(a, s_first, unit, end);
      stage_queries<HD, NQ, F8, kSoft, false>(a, s, r, q_aligned, sm + C::Q_OFF, [&](int v, const Vec& x, float qs, bool bad) {
        s_qs[v] = v < s.nq ? qs : 0.f;
        s_bad[v] = bad;
        s_out[v] = s.b * a.so[0] + x.t * a.so[1] + x.h * a.so[2];
      });
      const int t0 = s.qb * NQ / a.G;          // the block's first node
      stage_masks<kSoft>(a, s, t0, r, s_mask);
      tc::fence_proxy_async();
      tc::mbar_arrive(&q_full);
      sync();
      const float my_qs = lane < NQ ? s_qs[lane] : 0.f;   // of the lane's column
      float ref = -INFINITY;                   // and its sums' reference
      float l[NQ], o[NQ];
#pragma unroll
      for (int v = 0; v < NQ; ++v) l[v] = o[v] = 0.f;
      // a chunk's O^T (its P V complete) to the sums, with its factors
      auto add_o = [&](int i) {
        tc::tc_fence_after();
        if (r < HD) {                          // (whole warps)
#pragma unroll
          for (int g = 0; g < NQ; g += 16) {
            uint32_t hi[16], lo[16];
            tc::tmem_ld16_nowait(t_o + lane_base + g, hi);
            if constexpr (F8) tc::tmem_ld16_nowait(t_o + lane_base + NQ + g, lo);
            tc::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const float4 b = *reinterpret_cast<const float4*>(&s_bo[i & 1][warp][g + e]);
              auto add = [&](int v, float by) {
                float x = __uint_as_float(hi[v]);
                if constexpr (F8) x = fmaf(__uint_as_float(lo[v]), 1.f / (1 << kLoShift), x);
                o[g + v] = fmaf(x, by, o[g + v]);
              };
              add(e, b.x);
              add(e + 1, b.y);
              add(e + 2, b.z);
              add(e + 3, b.w);
            }
          }
        }
        tc::tc_fence_before();
      };

      for (int ch = s.c0; ch < s.c1 && !gone; ++ch, ++it) {
        const int st = it % NST;
        // ---- this thread's slot: its scales
        bool ok = tc::mbar_wait(&v_full[st], parity(it, NST), a.status);
        const int slot = ch * kKeys + r, node = slot - s.len;
        const bool valid = slot < s.keys && s_pieces[st] >> (r >> min(c.page_shift, 7)) & 1;
        const uint32_t kb = valid ? sm[C::SCALE_OFF + st * 2 * kKeys + r] : 127u;
        const uint32_t vb = valid ? sm[C::SCALE_OFF + (st * 2 + 1) * kKeys + r] : 0u;
        const float ks = scale_value(kb);
        ok = ok && tc::mbar_wait(&s_full[it & 1], parity(it, 2), a.status);
        failed = failed || !ok;
        tc::tc_fence_after();
        // A warp's chunk, with masks (slots of the tree or past the item's) or without. Code of its own for each: as
        // one, the compiler selects on every score, masked or not, which took as long as all else.
        auto chunk = [&](auto masked) {
          uint32_t vis = ~0u;                  // which vectors see the slot: bit v
          if constexpr (masked) {
            if (!valid || node >= 0) {
              vis = 0;
              if (valid) {
                const uint64_t group = a.G < 64 ? (1ull << a.G) - 1 : ~0ull;
#pragma unroll 2
                for (int t = t0, v = t0 * a.G - s.qb * NQ; v < s.nq; ++t, v += a.G)
                  if (s_mask[t - t0][node >> 5] >> (node & 31) & 1)
                    vis |= (uint32_t)(v < 0 ? group >> -v : group << v);
              }
            }
          }
          // ---- scores, and their maxima over the warp's slots
          float t[NQ];
          uint32_t x[NQ / 16][16];
#pragma unroll
          for (int g = 0; g < NQ / 16; ++g) tc::tmem_ld16_nowait(tmem + (it & 1) * NQ + lane_base + 16 * g, x[g]);
          tc::tmem_wait_ld();
          tc::tc_fence_before();
          tc::mbar_arrive(&s_empty[it & 1]);
#pragma unroll
          for (int v = 0; v < NQ; v += 4) {
            float top[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              t[v + e] = __uint_as_float(x[v / 16][v % 16 + e]) * ks;
              if constexpr (masked)
                if (!(vis >> (v + e) & 1)) t[v + e] = -INFINITY;
              top[e] = warp_fmax(t[v + e]);
            }
            if (lane == 0)
              *reinterpret_cast<float4*>(&s_wmax[it & 1][warp][v]) = make_float4(top[0], top[1], top[2], top[3]);
          }
          if constexpr (F8) {                  // (bytes 0, no scale, and 255, not finite, take no part)
            const int most = __reduce_max_sync(0xffffffffu, vb == 255 ? 0 : (int)vb);
            const int least = __reduce_min_sync(0xffffffffu, vb == 0 ? 255 : (int)vb);
            if (lane == 0) s_wv[it & 1][warp] = least << 8 | most;
          }
          if (tc::named_barrier_or(1, kSoft, failed)) {
            gone = true;
            return;
          }
          // ---- the chunk's references: a lane per column, each warp for itself
          int vref = 127;
          bool apart = false;                  // V's scales are (alike in all softmax threads)
          if constexpr (F8) {
            const int* const w = s_wv[it & 1];
            vref = max(max(w[0] & 255, w[1] & 255), max(w[2] & 255, w[3] & 255));
            apart = vref - (min(min(w[0], w[1]), min(w[2], w[3])) >> 8) > kSpread;
          }
          float f = 1.f;
          if (lane < NQ) {
            const float top = fmaxf(fmaxf(s_wmax[it & 1][0][lane], s_wmax[it & 1][1][lane]),
                                    fmaxf(s_wmax[it & 1][2][lane], s_wmax[it & 1][3][lane]));
            const float mq = top == -INFINITY ? 0.f : top * my_qs;
            if (top > -INFINITY && !(mq - ref <= kMargin)) {
              f = ref == -INFINITY ? 1.f : ex2(ref - mq);   // (no reference: nothing seen so far, the sums are 0)
              ref = mq;
            }
            const float b = top == -INFINITY ? 0.f : ex2(mq - ref);
            s_mq[warp][lane] = mq;
            s_b[warp][lane] = b;
            s_f[warp][lane] = f;
            s_bo[it & 1][warp][lane] = F8 ? b * (1.f / (1 << kPShift)) * ex2((float)(vref - 127)) : b;
          }
          const bool raise = __any_sync(0xffffffffu, f != 1.f);
          __syncwarp();
          // ---- the chunk before's O^T; its P may be overwritten
          if (it > 0) {
            if (!__all_sync(0xffffffffu, tc::mbar_wait(&p_empty, (it - 1) & 1, a.status))) failed = true;
            else if (ch > s.c0) add_o(it - 1);
          }
          if (raise) {
#pragma unroll
            for (int v = 0; v < NQ; ++v) {
              const float g = s_f[warp][v];
              l[v] *= g;
              o[v] *= g;
            }
          }
          if constexpr (masked) {
            if (!valid) {                      // nothing of its V row (page garbage, no copy) may reach the sums
              uint8_t* v = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + r * C::BW;
#pragma unroll
              for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll 1
                for (int i = 0; i < C::BW; i += 16)
                  *reinterpret_cast<uint4*>(v + nb * C::BLOCK + i) = make_uint4(0u, 0u, 0u, 0u);
            }
          }
          // ---- probabilities, their sums, V's scale on them
          if (F8 && apart) {
            // in fp32: P V of this thread's dimension, 64 slots at a time through P's tile, to the sums
            float* const p = reinterpret_cast<float*>(sm + C::P_OFF);
            static_assert(!F8 || C::P_TILE >= kKeys / 2 * NQ * 4);
            const float vf = scale_value(vb);
#pragma unroll
            for (int v = 0; v < NQ; ++v) {
              const float y = ex2(fmaf(t[v], s_qs[v], -s_mq[warp][v])) * s_b[warp][v];
              l[v] += y;
              t[v] = y * vf;
              if constexpr (masked)
                if (!(vis >> v & 1)) t[v] = 0.f;
            }
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              if (r / (kKeys / 2) == half)
#pragma unroll
                for (int v = 0; v < NQ; v += 4)
                  *reinterpret_cast<float4*>(&p[r % (kKeys / 2) * NQ + v]) = make_float4(t[v], t[v + 1], t[v + 2], t[v + 3]);
              sync();
              if (r < HD) {
#pragma unroll 1
                for (int k = 0; k < kKeys / 2; ++k) {
                  const uint32_t code = sm[C::KV_OFF + (st * 2 + 1) * C::TILE +
                                           tc::row_offset(half * (kKeys / 2) + k, r / 16, C::BW) + r % 16];
                  const float x = f8x2_to_f32(code).x;
#pragma unroll
                  for (int v = 0; v < NQ; v += 4) {
                    const float4 y = *reinterpret_cast<const float4*>(&p[k * NQ + v]);
                    o[v] = fmaf(y.x, x, o[v]);
                    o[v + 1] = fmaf(y.y, x, o[v + 1]);
                    o[v + 2] = fmaf(y.z, x, o[v + 2]);
                    o[v + 3] = fmaf(y.w, x, o[v + 3]);
                  }
                }
              }
              sync();
            }
            // (the chunk's P V adds zeros)
#pragma unroll
            for (int i = 0; i < C::RB; i += 16)
              *reinterpret_cast<uint4*>(sm + C::P_OFF + r * C::RB + i) = make_uint4(0u, 0u, 0u, 0u);
          } else {
            const int ve = F8 ? (int)vb - vref + kPShift + 127 : (int)vb;
            const float vf = vb == 255 ? __uint_as_float(0x7fc00000u)
                                       : !valid || ve < 1 ? 0.f : __uint_as_float((uint32_t)ve << 23);
            uint8_t* const p = sm + C::P_OFF;
#pragma unroll
            for (int g = 0; g < NQ; g += 16) {
              float y[16];
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const float4 qs = *reinterpret_cast<const float4*>(&s_qs[g + e]);
                const float4 mq = *reinterpret_cast<const float4*>(&s_mq[warp][g + e]);
                const float4 b = *reinterpret_cast<const float4*>(&s_b[warp][g + e]);
                y[e] = ex2(fmaf(t[g + e], qs.x, -mq.x));
                y[e + 1] = ex2(fmaf(t[g + e + 1], qs.y, -mq.y));
                y[e + 2] = ex2(fmaf(t[g + e + 2], qs.z, -mq.z));
                y[e + 3] = ex2(fmaf(t[g + e + 3], qs.w, -mq.w));
                l[g + e] = fmaf(y[e], b.x, l[g + e]);
                l[g + e + 1] = fmaf(y[e + 1], b.y, l[g + e + 1]);
                l[g + e + 2] = fmaf(y[e + 2], b.z, l[g + e + 2]);
                l[g + e + 3] = fmaf(y[e + 3], b.w, l[g + e + 3]);
              }
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                y[e] *= vf;
                if constexpr (masked)            // (0 * NaN of a V that the vector does not see)
                  if (!(vis >> (g + e) & 1)) y[e] = 0.f;
              }
              if constexpr (F8) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const __half2 z0 = __floats2half2_rn(y[4 * i], y[4 * i + 1]), z1 = __floats2half2_rn(y[4 * i + 2], y[4 * i + 3]);
                  __half2 h0, h1;
                  hi[i] = f8x4(z0, z1);
                  f8x4_half(hi[i], &h0, &h1);
                  const __half2 up = __float2half2_rn((float)(1 << kLoShift));
                  lo[i] = f8x4(__hmul2(__hsub2(z0, h0), up), __hmul2(__hsub2(z1, h1), up));
                }
                *reinterpret_cast<uint4*>(p + tc::row_offset(r, g / 16, C::RB)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4*>(p + tc::row_offset(r, (NQ + g) / 16, C::RB)) =
                    make_uint4(lo[0], lo[1], lo[2], lo[3]);
              } else {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  uint32_t hi[4], lo[4];
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const float u = y[half * 8 + 2 * i], w = y[half * 8 + 2 * i + 1];
                    const __nv_bfloat162 h = __floats2bfloat162_rn(u, w);
                    const __nv_bfloat162 z = __floats2bfloat162_rn(u - __low2float(h), w - __high2float(h));
                    hi[i] = *reinterpret_cast<const uint32_t*>(&h);
                    lo[i] = *reinterpret_cast<const uint32_t*>(&z);
                  }
                  const uint32_t off = tc::row_offset(r, g / 8 + half, C::RB);
                  *reinterpret_cast<uint4*>(p + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                  *reinterpret_cast<uint4*>(p + C::P_TILE + off) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
              }
            }
          }
          tc::fence_proxy_async();
          tc::tc_fence_before();
          tc::mbar_arrive(&p_full);
        };
        if (__any_sync(0xffffffffu, !valid || node >= 0)) chunk(std::true_type());
        else chunk(std::false_type());
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
      for (int g = 0; g < NQ; g += 16) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = l[g + e];
        warp_sums<16>(x);
        if ((lane & 1) == 0) s_l[warp][g + (lane >> 1)] = x[0];
      }
      if (warp == 0 && lane < NQ) s_ref[lane] = ref;
      sync();
      // ---- a thread per vector: its sum (0: it saw nothing; of a query that is not finite: NaN)
      const bool whole = s.c0 == 0 && s.c1 == s.units;
      const size_t part = (size_t)blockIdx.x * 2 + (s.c0 == 0);
      const int live = min(NQ, a.T * a.G - s.qb * NQ);
      if (r < live) {
        const int v = r;
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
        for (int v = 0; v < NQ; ++v) {
          if (v >= live) break;
          const float inv = s_inv[v], x = inv == 0.f ? 0.f : o[v] * inv;
          if (whole) static_cast<__nv_bfloat16*>(a.out)[s_out[v] + r] = __float2bfloat16_rn(x);
          else a.part_o[(part * NQ + v) * HD + r] = x;
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
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, k, C::smem(CDSL_TREE_MAX_BATCH))) return e;
  return launch_pdl(k, dim3(a.blocks), dim3(kThreads), C::smem(a.c.batch), s, a, map);
}

template <typename F>
auto by_query_block(int NQ, F&& f) {
  return NQ == 16 ? f(std::integral_constant<int, 16>()) : f(std::integral_constant<int, 32>());
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
