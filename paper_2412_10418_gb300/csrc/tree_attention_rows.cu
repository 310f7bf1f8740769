// tree_attention_rows.cu -- cdsl_tree_attention of bf16 queries with more than 32 query vectors per K/V
// head, on the 5th-generation tensor cores: query vectors are the MMA's M = 128 rows.
//
//   S = Q K^T   M = 128 vectors, N = 128 slots, K = head_dim    Q and K tiles K-major in shared memory
//   O = P V     M = 128 vectors, N = head_dim, K = 128 slots    P in TMEM over S, V tile MN-major as it lands
//
// Codes, planes and scales are as in tree_attention_tc.cu, and so are the warps that load chunks and issue
// MMAs; another turns each chunk's scale bytes into factors. A softmax thread has a vector (a TMEM lane) and
// walks all the chunk's slots (columns): maximum, probabilities and their sum are its own, no value crosses
// lanes and no barrier stands in a chunk, whatever the number of vectors. What changes from slot to slot (scales,
// masks) is read from shared memory. That costs the same for 33 vectors as for 128, and reads K and V once
// for all of them.
//
// Two groups of four softmax warps take alternate chunks, each with its own S (P over it) and O in TMEM, so
// that one's conversions run beside the other's maxima; they keep nothing from chunk to chunk. Eight more warps
// hold the rows' sums (half of a row's O each): they take a chunk's maximum and sum from shared memory and its
// O, which starts anew, from TMEM. With all sixteen warps on one chunk, in the same phase behind a barrier, a
// chunk took 4,500 to 5,000 cycles. Bound by instruction issue: about nine instructions a score.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "tree_attention.cuh"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {

constexpr int kRows = 128;                     // query vectors per block
constexpr int kSoft = 2 * kRows;               // softmax threads: two groups
constexpr int kSum = 2 * kRows;                // threads that hold the sums: two per row
constexpr int kThreads = kSoft + kSum + 96;
constexpr int kSumWarp = kSoft / 32, kProducer = kSumWarp + kSum / 32, kIssuer = kProducer + 1,
              kScaler = kProducer + 2;         // warps
constexpr int kBuf = 3;                        // S (then P) buffers in TMEM; O has the rest
constexpr int kFlags = 4;                      // segments whose flags are held: the sums lag by less than three

template <int HD, bool F8>
struct Cfg {
  static constexpr int EB = F8 ? 1 : 2;
  static constexpr int KROW = HD * EB;                     // bytes of a K or V row
  static constexpr int BW = KROW < 128 ? KROW : 128;       // of it per tile block
  static constexpr int NB = KROW / BW;
  static constexpr uint32_t BLOCK = kKeys * BW;
  static constexpr uint32_t TILE = NB * BLOCK;             // K or V of a chunk
  static constexpr int QP = F8 ? 2 : 1;
  static constexpr uint32_t Q_PLANE = kRows * KROW;
  static constexpr uint32_t KV_OFF = QP * Q_PLANE;
  static constexpr int FIT = (208 * 1024 - KV_OFF) / (2 * TILE);
  static constexpr int NST = FIT > 4 ? 4 : FIT;
  static_assert(NST >= 2, "stages");
  static constexpr uint32_t SCALE_OFF = KV_OFF + NST * 2 * TILE;
  // K's scale of each slot, and V's relative to the chunk's largest, times 2^kPShift
  static constexpr uint32_t FACTOR_OFF = SCALE_OFF + NST * 2 * kKeys;
  static constexpr uint32_t PLAN_OFF = FACTOR_OFF + NST * 2 * kKeys * 4;
  static constexpr size_t smem(int batch) { return 1024 + PLAN_OFF + (batch + 1) * 4; }
};

template <int HD, bool F8>
__global__ void __launch_bounds__(kThreads, 1)
    k_tree_rows(TreeArgs a, const __grid_constant__ CUtensorMap map) {
  using C = Cfg<HD, F8>;
  constexpr int NST = C::NST;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const sm = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
  int* const s_first = reinterpret_cast<int*>(sm + C::PLAN_OFF);
  __shared__ __align__(8) uint64_t k_full[NST], v_full[NST], k_empty[NST], v_empty[NST];
  __shared__ __align__(8) uint64_t f_full[NST], s_full[kBuf], p_full[2], m_empty[2], o_full, o_empty, q_full, done;
  __shared__ uint32_t s_tmem;
  __shared__ __align__(16) uint32_t s_valid[NST][4];   // slots that there are, as bits
  __shared__ float s_o[NST];                   // factor of the chunk's O
  __shared__ float s_qs[kRows];                // score factors
  __shared__ float s_m[2][kRows], s_l[2][kRows], s_b[2];   // of a group's chunk: maxima, sums, factor of O
  __shared__ uint8_t s_bad[kFlags][kRows];     // the query is not finite
  __shared__ uint32_t s_mask[kRows + 1][kWords];
  __shared__ uint32_t s_pieces[NST];
  const Cache& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      tc::mbar_init(&k_full[i], 1);
      tc::mbar_init(&v_full[i], 1);
      tc::mbar_init(&k_empty[i], 1);
      tc::mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < NST; ++i) tc::mbar_init(&f_full[i], 32);
    for (int i = 0; i < kBuf; ++i) tc::mbar_init(&s_full[i], 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&p_full[i], kRows);
      tc::mbar_init(&m_empty[i], kSum);
    }
    tc::mbar_init(&o_full, 1);
    tc::mbar_init(&o_empty, kSum);
    tc::mbar_init(&q_full, kSoft);
    tc::mbar_init(&done, 1);
    tc::fence_mbar_init();
  }
  if (warp == kIssuer) tc::tmem_alloc(&s_tmem, 512);
  if (warp == kProducer && lane == 0) tc::tma_prefetch_map(&map);
  pdl_wait();
  pdl_launch_dependents();
  tc::tc_fence_before();
  build_plan(a, s_first);                      // (ends in a block barrier)
  tc::tc_fence_after();
  const uint32_t tmem = s_tmem;
  if (blockIdx.x == 0) {
    check_lens(a);
    for (int b = threadIdx.x; b <= c.batch; b += kThreads) a.plan[b] = s_first[b];
  }
  const int total = s_first[c.batch], runs = runs_of(a, total);
  const int begin = (int)blockIdx.x < runs ? run_begin(blockIdx.x, total, runs) : 0;
  const int end = (int)blockIdx.x < runs ? run_begin(blockIdx.x + 1, total, runs) : 0;
  const uint32_t t_o = tmem + kBuf * kKeys;

  if (warp == kProducer) {
    load_chunks<HD, F8, NST>(a, s_first, begin, end, map, sm + C::KV_OFF, sm + C::SCALE_OFF, s_pieces, k_full,
                             v_full, k_empty, v_empty);
  } else if (warp == kIssuer) {
    if (lane == 0) {
      constexpr uint32_t formats = F8 ? 0u : (1u << 7) | (1u << 10);
      constexpr uint32_t idesc = (1u << 4) | formats | (128u >> 4) << 24;
      constexpr uint32_t idesc_s = idesc | (uint32_t)(kKeys >> 3) << 17;
      constexpr uint32_t idesc_o = idesc | (uint32_t)(HD >> 3) << 17 | 1u << 16;
      const uint32_t sbase = tc::smem_u32(sm);
      const uint64_t desc_q = tc::desc_rows(sbase, C::BW, 16);
      const uint64_t desc_k = tc::desc_rows(sbase + C::KV_OFF, C::BW, 16);
      const uint64_t desc_v = tc::desc_rows(sbase + C::KV_OFF + C::TILE, C::BW, C::BLOCK);
      auto s_mma = [&](int i) {                // S of chunk i
        if (!tc::mbar_wait(&k_full[i % NST], parity(i, NST), a.status)) return false;
        tc::tc_fence_after();
        const uint64_t k = desc_k + (uint32_t)(i % NST) * (2 * C::TILE / 16);
#pragma unroll 1
        for (int p = C::QP - 1; p >= 0; --p)
#pragma unroll 1
          for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
            for (int x = 0; x < C::BW / 32; ++x) {
              const uint64_t q = desc_q + ((uint32_t)(p * C::Q_PLANE + nb * kRows * C::BW) / 16 + 2 * x);
              const uint64_t kk = k + (nb * C::BLOCK / 16 + 2 * x);
              const bool add = p < C::QP - 1 || nb + x > 0;
              if constexpr (F8) tc::umma_f8(tmem + i % kBuf * kKeys, q, kk, idesc_s, add);
              else tc::umma_bf16(tmem + i % kBuf * kKeys, q, kk, idesc_s, add);
            }
        tc::umma_commit(&s_full[i % kBuf]);
        tc::umma_commit(&k_empty[i % NST]);
        return true;
      };
      auto pv = [&](int i) {                   // P V of chunk i
        if (!tc::mbar_wait(&p_full[i & 1], parity(i, 2), a.status) ||
            !tc::mbar_wait(&o_empty, (i & 1) ^ 1, a.status) ||
            !tc::mbar_wait(&v_full[i % NST], parity(i, NST), a.status))
          return false;
        tc::tc_fence_after();
        const uint64_t v = desc_v + (uint32_t)(i % NST) * (2 * C::TILE / 16);
        constexpr int STEP = 32 / C::EB;       // slots of an MMA: 8 columns of P
        // P of 32 slots lies in the columns that held their S, hi then lo
        auto p_at = [](int k, int p) { return F8 ? k * 32 + p * 8 : k / 2 * 32 + p * 16 + k % 2 * 8; };
#pragma unroll 1
        for (int p = 1; p >= 0; --p)
#pragma unroll
          for (int k = 0; k < kKeys / STEP; ++k)
            tc::umma_tmem_a<F8>(t_o, tmem + i % kBuf * kKeys + p_at(k, p), v + k * (STEP * C::BW / 16), idesc_o,
                                p < 1 || k > 0);
        tc::umma_commit(&o_full);
        tc::umma_commit(&v_empty[i % NST]);
        return true;
      };
      bool ok = true;
      int it = 0, seg = 0;                     // chunks of the segments before
      for (int unit = begin; unit < end && ok; ++seg) {
        const Segment s = segment_at(a, s_first, unit, end);
        const int n = s.c1 - s.c0;
        ok = tc::mbar_wait(&q_full, seg & 1, a.status);
        // S as far ahead as it has buffers; one that overwrites a P follows the P V that reads it, in order
        for (int i = 0; i < n + kBuf && ok; ++i) {
          if (i >= kBuf) ok = pv(it + i - kBuf);
          if (ok && i < n) ok = s_mma(it + i);
        }
        it += n;
        unit += n;
      }
      tc::umma_commit(&done);                  // what was issued completes before the block's memory goes
      tc::mbar_wait(&done, 0, a.status);
    }
    __syncwarp();
  } else if (warp == kScaler) {
    // ------------------------------------------------------------------------- scale bytes to factors
    int it = 0;
    bool ok = true;
    for (int unit = begin; unit < end && ok;) {
      const Segment s = segment_at(a, s_first, unit, end);
      for (int ch = s.c0; ch < s.c1 && ok; ++ch, ++it) {
        const int st = it % NST;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&v_full[st], parity(it, NST), a.status));
        if (!ok) break;
        // a lane has slots 4 lane .. 4 lane + 3
        const uint8_t* from = sm + C::SCALE_OFF + st * 2 * kKeys + 4 * lane;
        const uint32_t kb = *reinterpret_cast<const uint32_t*>(from), vb = *reinterpret_cast<const uint32_t*>(from + kKeys);
        const int slot = ch * kKeys + 4 * lane;
        const bool piece = s_pieces[st] >> (4 * lane >> min(c.page_shift, 7)) & 1;
        const int n = piece ? min(max(s.keys - slot, 0), 4) : 0;   // of them that there are
        int vref = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = vb >> (8 * e) & 255;
          if (e < n && x != 255) vref = max(vref, x);
        }
        vref = __reduce_max_sync(0xffffffffu, vref);
        float kf[4], vf[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t k = kb >> (8 * e) & 255, v = vb >> (8 * e) & 255;
          const int x = F8 ? (int)v - vref + kPShift + 127 : 127;
          kf[e] = e < n ? scale_value(k) : 1.f;
          vf[e] = e >= n || x < 1 ? 0.f : v == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)x << 23);
        }
        float* to = reinterpret_cast<float*>(sm + C::FACTOR_OFF) + st * 2 * kKeys + 4 * lane;
        *reinterpret_cast<float4*>(to) = make_float4(kf[0], kf[1], kf[2], kf[3]);
        *reinterpret_cast<float4*>(to + kKeys) = make_float4(vf[0], vf[1], vf[2], vf[3]);
        uint32_t valid = ((1u << n) - 1) << (4 * (lane & 7));       // eight lanes a word
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) valid |= __shfl_xor_sync(0xffffffffu, valid, o);
        if ((lane & 7) == 0) s_valid[st][lane >> 3] = valid;
        if (lane == 0) s_o[st] = F8 ? (1.f / (1 << kPShift)) * ex2((float)(vref - 127)) : 1.f;
        if (n < 4) {                           // nothing of their V rows (page garbage, no copy) may reach the sums
#pragma unroll 1
          for (int e = n; e < 4; ++e) {
            uint8_t* v = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + (4 * lane + e) * C::BW;
#pragma unroll 1
            for (int x = 0; x < C::KROW; x += 16)
              *reinterpret_cast<uint4*>(v + x / C::BW * C::BLOCK + x % C::BW) = make_uint4(0u, 0u, 0u, 0u);
          }
          tc::fence_proxy_async();
        }
        tc::mbar_arrive(&f_full[st]);
      }
      unit += s.c1 - s.c0;
    }
    __syncwarp();
  } else if (warp < kSumWarp) {
    // ------------------------------------------------------------------------- softmax
    const int tid = threadIdx.x, grp = tid / kRows, r = tid % kRows, w4 = warp & 3;
    auto sync = [] { tc::named_barrier(1, kSoft); };
    const bool q_aligned = (reinterpret_cast<uintptr_t>(a.q) | (a.sq[0] | a.sq[1] | a.sq[2]) * 2) % 16 == 0;
    int it0 = 0, seg = 0;
    bool failed = false;
    for (int unit = begin; unit < end; ++seg) {
      const Segment s = segment_at(a, s_first, unit, end);
      stage_queries<HD, kRows, F8, kSoft>(a, s, tid, q_aligned, sm, [&](int v, const Vec&, float qs, bool bad) {
        s_qs[v] = v < s.nq ? qs : 0.f;
        s_bad[seg % kFlags][v] = bad;
      });
      const int t0 = s.qb * kRows / a.G;       // the block's first node
      for (int i = tid; i < (kRows + 1) * kWords; i += kSoft) {
        const int t = t0 + i / kWords, w = i % kWords;
        s_mask[i / kWords][w] = t < s.nodes && w < a.W ? __ldg(a.mask + ((size_t)s.b * a.T + t) * a.W + w) : 0u;
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&q_full);
      sync();
      const float qs = s_qs[r];
      const bool live = w4 * 32 < s.nq;        // (a warp's: its rows hold vectors)
      const uint32_t* const my_mask = s_mask[r < s.nq ? vector_of(a, s.h, s.qb, r).t - t0 : 0];
      const int n = s.c1 - s.c0;
      for (int i = (it0 & 1) ^ grp; i < n && !failed; i += 2) {   // chunks it with it % 2 == grp
        const int it = it0 + i, st = it % NST;
        const uint32_t t_s = tmem + it % kBuf * kKeys + ((uint32_t)(w4 * 32) << 16);
        const float* const kf = reinterpret_cast<const float*>(sm + C::FACTOR_OFF) + st * 2 * kKeys;
        bool ok = tc::mbar_wait(&f_full[st], parity(it, NST), a.status);
        ok = ok && tc::mbar_wait(&s_full[it % kBuf], parity(it, kBuf), a.status);
        tc::tc_fence_after();
        // a chunk with slots of the tree, past the item's, or without a page: each row has its mask
        const int node0 = (s.c0 + i) * kKeys - s.len;
        const uint4 valid = *reinterpret_cast<const uint4*>(s_valid[st]);
        const bool masked = node0 > -kKeys || (valid.x & valid.y & valid.z & valid.w) != ~0u;
        auto word = [&](int w) -> uint32_t {   // slots 32 w .. 32 w + 31 that this row sees
          const int first = node0 + 32 * w;    // the tree's node in the first of them
          uint32_t x;
          if (first <= -32) x = ~0u;
          else if (first < 0) x = ((1u << -first) - 1) | my_mask[0] << -first;
          else if (first >= 32 * kWords) x = 0u;
          else x = __funnelshift_r(my_mask[first >> 5], first >> 5 < kWords - 1 ? my_mask[(first >> 5) + 1] : 0u, first & 31);
          return r < s.nq ? x & s_valid[st][w] : 0u;
        };
        float mq = -INFINITY, sum = 0.f;
        // Code of its own for chunks with masks: as one, the compiler selects on every score, masked or not,
        // which took twice the time.
        auto softmax = [&](auto masked) {
          // slots 16 g .. as scores times K's scale, in pairs
          auto scores = [&](const uint32_t (&x)[16], int g, uint32_t seen, uint64_t (&t)[8]) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(kf + 16 * g + 2 * e);
              t[e] = mul2(pair(x[2 * e], x[2 * e + 1]), k.x);
              t[e + 1] = mul2(pair(x[2 * e + 2], x[2 * e + 3]), k.y);
            }
            if constexpr (masked) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 y = unpair(t[e]);
                t[e] = pair(seen >> (2 * e) & 1 ? y.x : -INFINITY, seen >> (2 * e + 1) & 1 ? y.y : -INFINITY);
              }
            }
          };
          // ---- the row's maximum
          float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t x[2][16];
            tc::tmem_ld16_nowait(t_s + 32 * w, x[0]);
            tc::tmem_ld16_nowait(t_s + 32 * w + 16, x[1]);
            const uint32_t seen = masked ? word(w) : ~0u;
            tc::tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint64_t t[8];
              scores(x[h], 2 * w + h, seen >> (16 * h), t);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 y = unpair(t[e]);
                m[e % 4] = fmaxf(fmaxf(y.x, y.y), m[e % 4]);
              }
            }
          }
          const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
          mq = top == -INFINITY ? -INFINITY : top * qs;
          const float off = top == -INFINITY ? 0.f : mq;
          // ---- probabilities, their sum, V's scale on them, P over S
          uint64_t add = 0ull;
          const uint64_t qs2 = pair(qs, qs), off2 = pair(-off, -off);
#pragma unroll 1
          for (int w = 0; w < 4; ++w) {
            uint32_t x[2][16];
            tc::tmem_ld16_nowait(t_s + 32 * w, x[0]);
            tc::tmem_ld16_nowait(t_s + 32 * w + 16, x[1]);
            const uint32_t seen = masked ? word(w) : ~0u;
            tc::tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint64_t t[8];
              scores(x[h], 2 * w + h, seen >> (16 * h), t);
              constexpr int W = F8 ? 4 : 8;
              uint32_t hi[W], lo[W];
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(kf + kKeys + 32 * w + 16 * h + e);
                float y[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  const float2 z = unpair(fma2(t[e / 2 + j], qs2, off2));
                  const uint64_t p = pair(ex2(z.x), ex2(z.y));
                  add = add2(add, p);
                  const float2 u = unpair(mul2(p, j ? v.y : v.x));
                  y[2 * j] = u.x;
                  y[2 * j + 1] = u.y;
                }
                if constexpr (masked) {        // (0 * NaN of a V that this row does not see)
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (!(seen >> (16 * h + e + j) & 1)) y[j] = 0.f;
                }
                if constexpr (F8) {            // four slots: a word of each plane
                  const __half2 z0 = __floats2half2_rn(y[0], y[1]), z1 = __floats2half2_rn(y[2], y[3]);
                  __half2 h0, h1;
                  hi[e / 4] = f8x4(z0, z1);
                  f8x4_half(hi[e / 4], &h0, &h1);
                  lo[e / 4] = f8x4(__hsub2(z0, h0), __hsub2(z1, h1));
                } else {
#pragma unroll
                  for (int j = 0; j < 2; ++j) {
                    const __nv_bfloat162 z = __floats2bfloat162_rn(y[2 * j], y[2 * j + 1]);
                    const __nv_bfloat162 d = __floats2bfloat162_rn(y[2 * j] - __low2float(z), y[2 * j + 1] - __high2float(z));
                    hi[e / 2 + j] = *reinterpret_cast<const uint32_t*>(&z);
                    lo[e / 2 + j] = *reinterpret_cast<const uint32_t*>(&d);
                  }
                }
              }
              const uint32_t to = t_s + 32 * w + h * W;
              tc::tmem_st_nowait(to, hi);
              tc::tmem_st_nowait(to + 2 * W, lo);
            }
          }
          const float2 two = unpair(add);
          sum = two.x + two.y;
          tc::tmem_wait_st();
        };
        if (live) {
          if (masked) softmax(std::true_type());
          else softmax(std::false_type());
        }
        // ---- for the sums, which have taken this group's chunk before
        ok = ok && tc::mbar_wait(&m_empty[grp], parity(it, 2) ^ 1, a.status);
        failed = !__all_sync(0xffffffffu, ok);   // (a warp gives up as one)
        s_m[grp][r] = mq;
        s_l[grp][r] = sum;
        if (r == 0) s_b[grp] = s_o[st];
        tc::tc_fence_before();
        tc::mbar_arrive(&p_full[grp]);
      }
      if (tc::named_barrier_or(1, kSoft, failed)) break;   // (and the queries and masks are free)
      it0 += n;
      unit += n;
    }
  } else {
    // ------------------------------------------------------------------------- sums
    const int tid = threadIdx.x - kSoft, half = tid / kRows, r = tid % kRows, w4 = warp & 3;
    constexpr int OD = HD / 2;                 // dimensions of O of a thread
    const uint32_t my_o = t_o + ((uint32_t)(w4 * 32) << 16) + half * OD;
    const bool o_aligned = (reinterpret_cast<uintptr_t>(a.out) | (a.so[0] | a.so[1] | a.so[2]) * 2) % 16 == 0;
    int it = 0, seg = 0;
    bool failed = false;
    for (int unit = begin; unit < end && !failed; ++seg) {
      const Segment s = segment_at(a, s_first, unit, end);
      const bool live = w4 * 32 < s.nq;
      float ref = -INFINITY, l = 0.f;
      uint64_t o[OD / 2];                      // in pairs
#pragma unroll
      for (int d = 0; d < OD / 2; ++d) o[d] = 0ull;
      for (int ch = s.c0; ch < s.c1 && !failed; ++ch, ++it) {
        const int g = it & 1;
        bool ok = tc::mbar_wait(&p_full[g], parity(it, 2), a.status);
        const float mq = s_m[g][r], add = s_l[g][r], scale = s_b[g];
        tc::mbar_arrive(&m_empty[g]);
        float f = 1.f;
        if (mq > -INFINITY && !(mq - ref <= kMargin)) {
          f = ref == -INFINITY ? 1.f : ex2(ref - mq);   // (no reference: the sums are 0)
          ref = mq;
        }
        float b = mq == -INFINITY ? 0.f : ex2(mq - ref);
        l = fmaf(l, f, add * b);
        b *= scale;
        if (__any_sync(0xffffffffu, f != 1.f)) {
          const uint64_t ff = pair(f, f);
#pragma unroll
          for (int d = 0; d < OD / 2; ++d) o[d] = mul2(o[d], ff);
        }
        ok = ok && tc::mbar_wait(&o_full, it & 1, a.status);
        failed = !__all_sync(0xffffffffu, ok);
        tc::tc_fence_after();
        if (live) {
          const uint64_t bb = pair(b, b);
#pragma unroll
          for (int d = 0; d < OD; d += 32) {
            uint32_t x[2][16];
            tc::tmem_ld16_nowait(my_o + d, x[0]);
            if (OD > 16) tc::tmem_ld16_nowait(my_o + d + 16, x[1]);
            tc::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; e += 2)
              if (d + e < OD)
                o[(d + e) / 2] = fma2(pair(x[e / 16][e % 16], x[e / 16][e % 16 + 1]), bb, o[(d + e) / 2]);
          }
        }
        tc::tc_fence_before();
        tc::mbar_arrive(&o_empty);
      }
      if (failed) break;
      const int rows = min(kRows, a.T * a.G - s.qb * kRows);
      if (r < rows) {
        if (r >= s.nq || s.keys == 0) l = 0.f;
        const float m = l == 0.f ? -INFINITY : ref == -INFINITY ? 0.f : ref;   // (NaN scores: no maximum)
        if (l != 0.f && s_bad[seg % kFlags][r]) l = __uint_as_float(0x7fc00000u);
        const Vec x = vector_of(a, s.h, s.qb, r);
        if (s.c0 == 0 && s.c1 == s.units) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          if (half == 0) store_lse(a, s.b, x, m, l);
          __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + s.b * a.so[0] + x.t * a.so[1] + x.h * a.so[2] +
                               half * OD;
#pragma unroll
          for (int d = 0; d < OD; d += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 y = unpair(o[d / 2 + e]);
              const __nv_bfloat162 z = __floats2bfloat162_rn(l == 0.f ? 0.f : y.x * inv, l == 0.f ? 0.f : y.y * inv);
              w[e] = *reinterpret_cast<const uint32_t*>(&z);
            }
            if (o_aligned) {
              *reinterpret_cast<uint4*>(out + d) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                out[d + e] = __ushort_as_bfloat16((unsigned short)(w[e / 2] >> (e % 2 * 16)));
            }
          }
        } else {
          const size_t part = (size_t)blockIdx.x * 2 + (s.c0 == 0);
          if (half == 0) {
            a.part_ml[(part * 2) * kRows + r] = m;
            a.part_ml[(part * 2 + 1) * kRows + r] = l;
          }
          float4* out = reinterpret_cast<float4*>(a.part_o + (part * kRows + r) * HD + half * OD);
#pragma unroll
          for (int d = 0; d < OD; d += 4) {
            const float2 y = unpair(o[d / 2]), z = unpair(o[d / 2 + 1]);
            out[d / 4] = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y.x, y.y, z.x, z.y);
          }
        }
      }
      unit += s.c1 - s.c0;
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) tc::tmem_dealloc(tmem, 512);
}

template <int HD, bool F8>
cudaError_t launch(const TreeArgs& a, cudaStream_t s) {
  using C = Cfg<HD, F8>;
  CUtensorMap map;
  if (encode_cache_map<HD, F8>(a, &map)) return cudaErrorInvalidValue;
  auto k = k_tree_rows<HD, F8>;
  static const cudaError_t set =
      cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::smem(CDSL_TREE_MAX_BATCH));
  if (set != cudaSuccess) return set;
  return launch_pdl(k, dim3(a.blocks), dim3(kThreads), C::smem(a.c.batch), s, a, map);
}

}  // namespace

cudaError_t launch_tree_rows(const TreeArgs& a, cudaStream_t s) {
  if (a.c.hd == 128) return a.c.eb == 1 ? launch<128, true>(a, s) : launch<128, false>(a, s);
  return a.c.eb == 1 ? launch<64, true>(a, s) : launch<64, false>(a, s);
}

}  // namespace tree
}  // namespace cdsl
