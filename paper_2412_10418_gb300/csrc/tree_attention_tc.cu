// tree_attention_tc.cu -- cdsl_tree_attention of bf16 queries on the 5th-generation tensor cores.
//
// Codes go from HBM to the MMA as they are. A chunk of 128 slots is the MMA's M = 128, the query vectors its
// N (16, 32 or 64: a tree has few of them, and as M they would be padded to 128), so that the work
// follows the number of queries:
//   S^T = K Q^T   M = 128 slots, N = NQ vectors, K = head_dim      K tile K-major, as TMA lands it
//   O^T += V^T P^T  M = head_dim, N = NQ (x planes), K = 128 slots   V tile MN-major, as TMA lands it
// An e4m3 cache takes kind::f8f6f4, twice the rate and half the shared memory of bf16 and no
// conversion of K and V at all. What is not e4m3 is split into e4m3 planes instead: a query row, scaled
// by a power of two to at most 448, is hi + lo, each to 4 bits, together bf16's 8 (to 2^-18 of the row's
// largest); a probability is hi + lo / 32 (to 2^-10 of itself), the planes side by side along N with
// sums of their own in TMEM. A bf16 cache takes kind::f16 with Q as it is and P in two bf16 planes.
// The rows' power-of-two scales never touch the codes: K's multiplies the thread's scores, V's the
// thread's probabilities (relative to the largest V scale so far, so that they use e4m3's range).
//
// Six warps. Warp 4 loads K and V chunks by TMA into a ring, a box per page piece; warp 5 issues
// the MMAs, the next chunk's S while this one's softmax runs (S has two buffers in TMEM). Warps 0-3 do the
// softmax: a thread owns a slot (a TMEM lane) and walks the query vectors (columns). Column maxima
// come from redux.sync over a warp; the running reference is raised only when some column's maximum passes
// it by more than kMargin (p <= 6.7: e4m3's 448 holds 64 p), which after the first chunk is rare, so a
// chunk costs one barrier among the four warps. Each thread keeps its own slots' share of the sums l.
//
// Waits are bounded (tc::kWaitLimitNs): on expiry CDSL_ETIMEOUT is latched, the role winds down and
// the block frees its TMEM and exits.
#include <cuda.h>

#include <algorithm>

#include "gemm.cuh"
#include "kernels.h"
#include "tree_attention.cuh"

namespace cdsl {
namespace tree {
namespace {

constexpr int kSoft = 128;                     // softmax threads: one per slot of a chunk
constexpr int kThreads = kSoft + 64;
constexpr int kProducer = 4, kIssuer = 5;      // warps
constexpr float kMargin = 2.75f;               // base 2: 2^2.75 * 64 < 448
constexpr int kPShift = 6;                     // probabilities are stored times 2^kPShift
constexpr float kLoScale = 32.f;               // of the second e4m3 plane

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
  static constexpr int RB = 2 * NQ;                        // bytes of a P row (slot): e4m3 both planes, bf16 one
  static constexpr int PP = F8 ? 1 : 2;                    // P tiles
  static constexpr uint32_t P_TILE = kKeys * RB;
  static constexpr uint32_t FIXED = QP * Q_PLANE + PP * P_TILE;
  // two blocks per SM where two stages fit, else one
  static constexpr uint32_t LIMIT2 = 110 * 1024, LIMIT1 = 220 * 1024;
  static constexpr int CTAS = FIXED + 4 * TILE <= LIMIT2 ? 2 : 1;
  static constexpr int FIT = ((CTAS == 2 ? LIMIT2 : LIMIT1) - FIXED) / (2 * TILE);
  static constexpr int NST = FIT > 4 ? 4 : FIT;            // ring stages of K and V
  static_assert(NST >= 2, "stages");
  static constexpr uint32_t Q_OFF = 0;
  static constexpr uint32_t P_OFF = Q_OFF + QP * Q_PLANE;
  static constexpr uint32_t KV_OFF = (P_OFF + PP * P_TILE + 1023) / 1024 * 1024;
  static constexpr uint32_t PLAN_OFF = KV_OFF + NST * 2 * TILE;
  static constexpr int OC = F8 ? 2 * NQ : NQ;              // TMEM columns of O^T
  static constexpr uint32_t TMEM = 4 * NQ;                 // S twice, O
  static constexpr size_t smem(int batch) { return 1024 + PLAN_OFF + (batch + 1) * 4; }
};

// Position in a sequence of phases: index and parity of the `n`-th use of one of `of` barriers.
__device__ __forceinline__ uint32_t parity(int n, int of) { return (n / of) & 1; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float warp_fmax(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// (a, b) to two e4m3 codes, a in the low byte, as a half2 (11 bits) would be rounded
__device__ __forceinline__ uint32_t f8x2(__half2 h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<uint32_t*>(&h)));
  return r;
}
__device__ __forceinline__ __half2 f8x2_half(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return *reinterpret_cast<__half2*>(&r);
}
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
  // per query vector: score factor (softmax scale and the row's own), reference in raw scores, what raises
  // it, reference in base 2; factors of a raise
  __shared__ __align__(16) float s_qs[NQ], s_mq[NQ], s_lim[NQ], s_alpha[NQ], s_beta[NQ], s_inv[NQ];
  __shared__ float s_ref[NQ], s_wmax[4][NQ], s_l[4][NQ];
  __shared__ int s_bad[NQ];                    // the query is not finite
  __shared__ long long s_out[NQ];              // where its output begins
  __shared__ uint32_t s_mask[NQ + 1][kWords];  // of the block's nodes
  __shared__ int s_vref, s_wv[4];
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
    for (int b = threadIdx.x; b <= c.batch; b += kThreads) a.plan[b] = s_first[b];
  }
  const int total = s_first[c.batch], runs = runs_of(a, total);
  const int begin = (int)blockIdx.x < runs ? run_begin(blockIdx.x, total, runs) : 0;
  const int end = (int)blockIdx.x < runs ? run_begin(blockIdx.x + 1, total, runs) : 0;
  const int P = 1 << c.page_shift;

  if (warp == kProducer) {
    // ------------------------------------------------------------------------- K and V chunks
    const int rows = min(P, kKeys), pieces = kKeys / rows;
    int it = 0, issued[2] = {0, 0};            // chunks, and copies of K and of V
    bool ok = true;
    for (int unit = begin; unit < end && ok;) {
      const Segment s = segment_at(a, s_first, unit, end);
      for (int ch = s.c0; ch < s.c1 && ok; ++ch, ++it) {
        const int st = it % NST;
        const int slot = ch * kKeys + lane * rows;
        int page = -1;
        if (lane < pieces && slot < s.keys) page = page_of(c, s.b, slot);
        const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, page >= 0)) * rows * C::KROW;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          uint64_t* full = kv ? &v_full[st] : &k_full[st];
          ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(kv ? &v_empty[st] : &k_empty[st],
                                                           parity(it, NST) ^ 1, a.status));
          if (!ok) break;
          if (lane == 0) tc::mbar_expect_tx(full, bytes);
          __syncwarp();
          if (page >= 0) {
            const int y = (int)row_of(c, 0, page, kv, s.h, slot & (P - 1));
            uint8_t* dst = sm + C::KV_OFF + (st * 2 + kv) * C::TILE + lane * rows * C::BW;
#pragma unroll
            for (int nb = 0; nb < C::NB; ++nb)
              tc::tma_load_2d(dst + nb * C::BLOCK, &map, nb * (C::BW / C::EB), y, full);
          }
          issued[kv] = it + 1;
        }
      }
      unit += s.c1 - s.c0;
    }
    // the block leaves only with its copies landed (where a role gave up, nothing may have waited for them)
    if (!ok)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        for (int i = max(0, issued[kv] - NST); i < issued[kv]; ++i)
          tc::mbar_wait(kv ? &v_full[i % NST] : &k_full[i % NST], parity(i, NST), a.status);
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
      auto pv = [&](int i, bool add) {         // the P V of chunk i
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
                add || k > 0 || p < C::PP - 1);
        tc::umma_commit(&p_empty);
        tc::umma_commit(&v_empty[i % NST]);
        return true;
      };
      // chunk i's S goes before chunk i - 1's P V, except that a new item's queries are staged only after
      // the last one's P V
      int it = 0, seg = 0;
      bool ok = true, add = false;             // add: chunk it - 1 is not its segment's first
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
          if (ch > s.c0 && !(ok = pv(it - 1, add))) break;
          add = ch > s.c0;
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
      // ---- scale bytes of the slots, loaded a chunk ahead and their page ids two
      auto page_at = [&](int ch) {
        const int slot = ch * kKeys + r;
        return ch < s.c1 && slot < s.keys ? page_of(c, s.b, slot) : -1;
      };
      struct Slot { int page; uint32_t ks, vs; };   // page -1: nothing to see
      auto slot_at = [&](int ch, int page) {
        Slot x = {page, 127, 127};
        if (page >= 0) {
          const size_t row = row_of(c, a.layer, page, 0, s.h, (ch * kKeys + r) & (P - 1));
          x.ks = __ldg(c.scale + row);
          x.vs = __ldg(c.scale + row + ((size_t)c.kvh << c.page_shift));
        }
        return x;
      };
      const int page0 = page_at(s.c0);
      int page_next = page_at(s.c0 + 1);
      Slot cur = slot_at(s.c0, page0);
      // ---- queries: eight threads a vector, HD / 8 values each
      sync();                                  // the item before is done with the statistics
      constexpr int QE = HD / 8;
#pragma unroll 1
      for (int v0 = 0; v0 < NQ; v0 += kSoft / 8) {
        const int v = v0 + r / 8, part = r % 8;
        const Vec x = vector_of(a, s.h, s.qb, v);
        uint32_t w[QE / 2];
#pragma unroll
        for (int i = 0; i < QE / 2; ++i) w[i] = 0u;
        if (v < s.nq) {
          const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + s.b * a.sq[0] + x.t * a.sq[1] +
                                   x.h * a.sq[2] + part * QE;
          if (q_aligned) {
#pragma unroll
            for (int i = 0; i < QE / 8; ++i) {
              const uint4 u = *reinterpret_cast<const uint4*>(q + 8 * i);
              w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
            }
          } else {
#pragma unroll
            for (int i = 0; i < QE; ++i)
              w[i / 2] |= (uint32_t)__bfloat16_as_ushort(q[i]) << (i % 2 * 16);
          }
        }
        uint32_t top = 0;                      // largest |x|, as bf16 bits
#pragma unroll
        for (int i = 0; i < QE / 2; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool bad = top >= 0x7f80u;
        float qs = a.scale;
        if constexpr (F8) {
          int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u);
          e = top == 0 || bad ? 0 : max(e, -126);
          const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
          qs *= __uint_as_float((uint32_t)(127 + e) << 23);
          uint32_t hi[QE / 4], lo[QE / 4];
#pragma unroll
          for (int i = 0; i < QE / 4; ++i) {
            float x[4] = {__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i] & 0xffff0000u),
                          __uint_as_float(w[2 * i + 1] << 16), __uint_as_float(w[2 * i + 1] & 0xffff0000u)};
            uint32_t hl[2], ll[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float2 y = make_float2(x[2 * j] * inv, x[2 * j + 1] * inv);
              hl[j] = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
              const float2 z = f8x2_to_f32(hl[j]);
              ll[j] = __nv_cvt_float2_to_fp8x2(make_float2(y.x - z.x, y.y - z.y), __NV_SATFINITE, __NV_E4M3);
            }
            hi[i] = bad ? 0u : hl[0] | hl[1] << 16;
            lo[i] = bad ? 0u : ll[0] | ll[1] << 16;
          }
          if constexpr (HD == 128) {
            const uint32_t off = C::Q_OFF + tc::row_offset(v, part, C::BW);
            *reinterpret_cast<uint4*>(sm + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(sm + off + C::Q_PLANE) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          } else {
            const uint32_t off = C::Q_OFF + tc::row_offset(v, part / 2, C::BW) + part % 2 * 8;
            *reinterpret_cast<uint2*>(sm + off) = make_uint2(hi[0], hi[1]);
            *reinterpret_cast<uint2*>(sm + off + C::Q_PLANE) = make_uint2(lo[0], lo[1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < QE / 8; ++i) {
            const int ch = part * (QE / 8) + i;   // 16-byte chunk of the row
            const uint32_t off = C::Q_OFF + ch / 8 * NQ * C::BW + tc::row_offset(v, ch % 8, C::BW);
            *reinterpret_cast<uint4*>(sm + off) =
                bad ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          }
        }
        if (part == 0) {
          s_qs[v] = v < s.nq ? qs : 0.f;
          s_ref[v] = s_lim[v] = -INFINITY;
          s_mq[v] = 0.f;
          s_bad[v] = v < s.nq && bad;
          s_out[v] = s.b * a.so[0] + x.t * a.so[1] + x.h * a.so[2];
        }
      }
      const int t0 = s.qb * NQ / a.G;          // the block's first node
      for (int i = r; i < (NQ + 1) * kWords; i += kSoft) {
        const int t = t0 + i / kWords, w = i % kWords;
        s_mask[i / kWords][w] = t < s.nodes && w < a.W ? __ldg(a.mask + ((size_t)s.b * a.T + t) * a.W + w) : 0u;
      }
      if (r == 0) s_vref = F8 ? -1 : 127;
      tc::fence_proxy_async();
      tc::mbar_arrive(&q_full);
      sync();
      float l[NQ];
#pragma unroll
      for (int v = 0; v < NQ; ++v) l[v] = 0.f;

      for (int ch = s.c0; ch < s.c1; ++ch, ++it) {
        const bool first = ch == s.c0;
        const uint32_t t_s = tmem + (it & 1) * NQ + lane_base;
        const Slot ahead = slot_at(ch + 1, page_next);
        page_next = page_at(ch + 2);
        const bool valid = cur.page >= 0;
        const int node = ch * kKeys + r - s.len;
        if (!valid && ch * kKeys + r < s.keys) set_status(a.status, CDSL_ERANGE);
        const float ks = scale_value(cur.ks);
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&s_full[it & 1], parity(it, 2), a.status))) failed = true;
        tc::tc_fence_after();
        // which vectors see this slot: bit v. Only chunks with slots of the tree or past the item's ask
        // (a warp's branch).
        const bool masked = __any_sync(0xffffffffu, !valid || node >= 0);
        uint64_t vis = ~0ull;
        if (masked && (!valid || node >= 0)) {
          vis = 0;
          const uint64_t group = a.G < 64 ? (1ull << a.G) - 1 : ~0ull;
          if (valid)
#pragma unroll 4
            for (int t = t0, v = t0 * a.G - s.qb * NQ; v < s.nq; ++t, v += a.G)
              if (s_mask[t - t0][node >> 5] >> (node & 31) & 1) vis |= v < 0 ? group >> -v : group << v;
        }
        // ---- scores; does any pass its column's limit?
        constexpr bool kKeep = NQ <= 32;       // scores stay in registers
        float t[kKeep ? NQ : 16];
        auto scores = [&](int g, float (&x)[16]) {
          tc::tmem_ld16(t_s + g, x);
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] *= ks;
          if (masked) {
            const uint32_t bits = (uint32_t)(vis >> g);
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (!(bits >> e & 1)) x[e] = -INFINITY;
          }
        };
        bool raise = F8 && valid && cur.vs != 255 && (int)cur.vs > s_vref;
#pragma unroll
        for (int g = 0; g < NQ; g += 16) {
          float x[16];
          scores(g, x);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 lim = *reinterpret_cast<const float4*>(&s_lim[g + e]);
            raise = raise || x[e] > lim.x || x[e + 1] > lim.y || x[e + 2] > lim.z || x[e + 3] > lim.w;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (kKeep) t[(kKeep ? g : 0) + e] = x[e];
        }
        bool waited = false;                   // for the chunk before's P V
        auto wait_pv = [&] {
          if (it > 0 && !waited &&
              !__all_sync(0xffffffffu, tc::mbar_wait(&p_empty, (it - 1) & 1, a.status)))
            failed = true;
          waited = true;
        };
        if (tc::named_barrier_or(1, kSoft, raise || failed)) {
          if (tc::named_barrier_or(1, kSoft, failed)) {
            gone = true;
            break;
          }
          // ---- raise every reference to its column's maximum so far
#pragma unroll 1
          for (int g = 0; g < NQ; g += 16) {
            float x[16], wm = 0.f;
            scores(g, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float top = warp_fmax(x[e]);
              if (lane == e) wm = top;
            }
            if (lane < 16) s_wmax[warp][g + lane] = wm;
          }
          const int wv = __reduce_max_sync(0xffffffffu, valid && cur.vs != 255 ? (int)cur.vs : -1);
          if (lane == 0) s_wv[warp] = wv;
          sync();
          const int v_old = s_vref;
          const int v_new = F8 ? max(max(v_old, max(s_wv[0], s_wv[1])), max(s_wv[2], s_wv[3])) : 127;
          for (int v = r; v < NQ; v += kSoft) {
            const float old = s_ref[v];
            const float top = fmaxf(fmaxf(s_wmax[0][v], s_wmax[1][v]), fmaxf(s_wmax[2][v], s_wmax[3][v]));
            const float now = fmaxf(old, top), qs = s_qs[v];
            const float alpha = old == -INFINITY ? (now == -INFINITY ? 1.f : 0.f) : ex2((old - now) * qs);
            s_alpha[v] = alpha;
            s_beta[v] = alpha * ex2((float)(v_old - v_new));
            s_ref[v] = now;
            s_lim[v] = now + kMargin / qs;
            s_mq[v] = now == -INFINITY ? 0.f : now * qs;
          }
          sync();
          if (r == 0) s_vref = v_new;          // (read again after the next chunk's barrier)
#pragma unroll
          for (int v = 0; v < NQ; ++v) l[v] *= s_alpha[v];
          if (!first) {
            wait_pv();
            tc::tc_fence_after();
#pragma unroll 1
            for (int g = 0; g < C::OC; g += 16) {
              float o[16];
              tc::tmem_ld16(t_o + lane_base + g, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] *= s_beta[(g + e) % NQ];
              tc::tmem_st16(t_o + lane_base + g, o);
            }
          }
          sync();                              // s_vref, and the factors are read
        }
        // ---- probabilities, their sums, and V's scale on them
        const int ve = F8 ? (int)cur.vs - s_vref + kPShift : 0;
        const float vf = cur.vs == 255 ? __uint_as_float(0x7fc00000u)
                                       : ve < -126 ? 0.f : __uint_as_float((uint32_t)(ve + 127) << 23);
        wait_pv();
#pragma unroll
        for (int g = 0; g < NQ; g += 16) {
          float x[16];
          if constexpr (kKeep) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = t[g + e];
          } else {
            scores(g, x);
          }
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 qs = *reinterpret_cast<const float4*>(&s_qs[g + e]);
            const float4 mq = *reinterpret_cast<const float4*>(&s_mq[g + e]);
            x[e] = ex2(fmaf(x[e], qs.x, -mq.x));
            x[e + 1] = ex2(fmaf(x[e + 1], qs.y, -mq.y));
            x[e + 2] = ex2(fmaf(x[e + 2], qs.z, -mq.z));
            x[e + 3] = ex2(fmaf(x[e + 3], qs.w, -mq.w));
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) l[g + e] += x[e];
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] *= vf;
          if (__any_sync(0xffffffffu, cur.vs == 255)) {   // a V that is not finite: NaN where it is seen
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (cur.vs == 255) x[e] = (uint32_t)(vis >> (g + e)) & 1 ? vf : 0.f;
          }
          uint8_t* const p = sm + C::P_OFF;
          if constexpr (F8) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              hi[i] = lo[i] = 0u;
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const __half2 h = __floats2half2_rn(x[4 * i + 2 * j], x[4 * i + 2 * j + 1]);
                const uint32_t y = f8x2(h);
                const __half2 rest = __hmul2(__hsub2(h, f8x2_half(y)), __float2half2_rn(kLoScale));
                hi[i] |= y << (16 * j);
                lo[i] |= f8x2(rest) << (16 * j);
              }
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
                const float u = x[half * 8 + 2 * i], w = x[half * 8 + 2 * i + 1];
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
        if (!valid) {                          // nothing of its V row (page garbage, no copy) may reach the sums
          const int st = it % NST;
          if (!tc::mbar_wait(&v_full[st], parity(it, NST), a.status)) failed = true;
          uint8_t* v = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + r * C::BW;
#pragma unroll
          for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
            for (int i = 0; i < C::BW; i += 16)
              *reinterpret_cast<uint4*>(v + nb * C::BLOCK + i) = make_uint4(0u, 0u, 0u, 0u);
        }
        tc::fence_proxy_async();
        tc::tc_fence_before();
        tc::mbar_arrive(&s_empty[it & 1]);
        tc::mbar_arrive(&p_full);
        cur = ahead;
      }
      if (gone) break;
      // ---- the item's (or its part's) sums and output
      if (!__all_sync(0xffffffffu, tc::mbar_wait(&p_empty, (it - 1) & 1, a.status))) failed = true;
      if (tc::named_barrier_or(1, kSoft, failed)) {
        gone = true;
        break;
      }
      tc::tc_fence_after();
#pragma unroll
      for (int g = 0; g < NQ; g += 16) {
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = l[g + e];
        warp_sums<16>(x);
        if ((lane & 1) == 0) s_l[warp][g + (lane >> 1)] = x[0];
      }
      sync();
      // ---- a thread per vector: its sum (0: it saw nothing; of a query that is not finite: NaN)
      const bool whole = s.c0 == 0 && s.c1 == s.units;
      const size_t slot = (size_t)blockIdx.x * 2 + (s.c0 == 0);
      const int live = min(NQ, a.T * a.G - s.qb * NQ);
      for (int v = r; v < live; v += kSoft) {
        float sum = 0.f;
        if (v < s.nq && s.keys > 0) sum = s_l[0][v] + s_l[1][v] + s_l[2][v] + s_l[3][v];
        const float m = sum == 0.f ? -INFINITY : s_mq[v];
        if (sum != 0.f && s_bad[v]) sum = __uint_as_float(0x7fc00000u);
        if (whole) {
          s_inv[v] = sum == 0.f ? 0.f : 1.f / sum;
          store_lse(a, s.b, vector_of(a, s.h, s.qb, v), m, sum);
        } else {
          s_inv[v] = sum == 0.f ? 0.f : 1.f;
          a.part_ml[(slot * 2) * NQ + v] = m;
          a.part_ml[(slot * 2 + 1) * NQ + v] = sum;
        }
      }
      sync();
      // O^T holds sums of p * 2^(V's scale - s_vref + kPShift)
      const float unscale = F8 ? ex2((float)(s_vref - 127)) : 1.f;
      if (r < HD) {                            // (whole warps)
#pragma unroll 1
        for (int g = 0; g < live; g += 16) {
          float o[16];
          tc::tmem_ld16(t_o + lane_base + g, o);
          if constexpr (F8) {
            float o2[16];
            tc::tmem_ld16(t_o + lane_base + NQ + g, o2);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = fmaf(o2[e], 1.f / kLoScale, o[e]) * (1.f / (1 << kPShift)) * unscale;
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (g + e >= live) break;
            const float inv = s_inv[g + e], x = inv == 0.f ? 0.f : o[e] * inv;
            if (whole) static_cast<__nv_bfloat16*>(a.out)[s_out[g + e] + r] = __float2bfloat16_rn(x);
            else a.part_o[(slot * NQ + g + e) * HD + r] = x;
          }
        }
      }
      tc::tc_fence_before();
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
  const Cache& c = a.c;
  const size_t rows = (size_t)c.n_pages * 2 * c.kvh << c.page_shift;
  const int e = encode_map(&map, F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, C::EB,
                           c.pool + (size_t)a.layer * rows * C::KROW, HD, rows, C::BW / C::EB,
                           std::min(1 << c.page_shift, kKeys),
                           C::BW == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
  if (e) return cudaErrorInvalidValue;
  auto k = k_tree_tc<HD, NQ, F8>;
  static const cudaError_t set =
      cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::smem(CDSL_TREE_MAX_BATCH));
  if (set != cudaSuccess) return set;
  return launch_pdl(k, dim3(a.blocks), dim3(kThreads), C::smem(c.batch), s, a, map);
}

template <typename F>
auto by_query_block(int NQ, F&& f) {
  return NQ == 16 ? f(std::integral_constant<int, 16>())
                  : NQ == 32 ? f(std::integral_constant<int, 32>()) : f(std::integral_constant<int, 64>());
}

}  // namespace

int tc_query_block(int vectors) { return vectors <= 16 ? 16 : vectors <= 32 ? 32 : 64; }

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
