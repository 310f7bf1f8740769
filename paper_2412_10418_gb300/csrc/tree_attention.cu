// tree_attention.cu -- cdsl_tree_attention: the CUDA-core kernel (fp32 queries), the joining of
// partial results and the entry points.
//
// k_tree_simt: a warp has a run. Scores: a lane has four slots of the chunk and all of the block's eight query
// vectors; it reads its K rows 16 bytes at a time, and shared memory broadcasts the queries (fp32, scaled by
// softmax scale * log2 e), four vectors at a dimension: a broadcast serves eight FMAs of pairs. Softmax: maxima over the
// warp, a running maximum, and sums that each lane keeps of its own slots. P V: a lane has hd / 32 dimensions of all
// vectors and walks the chunk's V rows; a broadcast of a slot's four probabilities serves as many FMAs of pairs again
// (half where hd is 64). Blocks of one warp have no barrier, and those on an SM cover one another's loads. Bound by its
// fp32 FMAs where there are many vectors: 38 TFLOP/s, the FMA pipes 58 % busy, for a tree of 24 of 32 heads after
// 32,768 tokens, 350 us (a slot's scores by a thread, of 16 vectors, by blocks of four warps: 882 us); by latency
// where there are few: eight trees of 17 of 12 heads after 192 tokens in 19 us with the joining. Sixteen vectors a
// warp, with half the K and V loads: 344 and 30 us.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "tree_attention.cuh"
#include "tree_host.h"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {

// Four codes (1 or 2 words) to floats.
template <bool F8>
__device__ __forceinline__ void decode4(uint32_t u, uint32_t w, float (&x)[4]) {
  if constexpr (F8) {
    const float2 a = f8x2_to_f32(u & 0xffffu), b = f8x2_to_f32(u >> 16);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  } else {
    x[0] = __uint_as_float(u << 16);
    x[1] = __uint_as_float(u & 0xffff0000u);
    x[2] = __uint_as_float(w << 16);
    x[3] = __uint_as_float(w & 0xffff0000u);
  }
}

constexpr int SQ = 8;                          // query vectors per block
// Resident warps of an SM, by registers (16 of bf16 rows of 128 spill: 182 us where 12 take 143, four trees of 49 of 40 heads
// after 1024 tokens; e4m3: 46 us with 16, 59 with 12, a tree of 17 of 32 heads after 4096)
constexpr int simt_per_sm(int HD, bool F8) { return HD == 128 && !F8 ? 12 : 16; }

template <typename T, int HD, bool F8>
__global__ void __launch_bounds__(32, simt_per_sm(HD, F8)) k_tree_simt(TreeArgs a) {
  constexpr int EB = F8 ? 1 : 2, CPL = 16 / EB, LOADS = HD / CPL;   // codes in 16 bytes
  constexpr int DPL = HD / 32;                 // dimensions of a lane
  constexpr int AHEAD = DPL * EB > 4 ? 8 : 16; // V rows loaded together
  using VBits = std::conditional_t<DPL * EB == 8, uint2, std::conditional_t<DPL * EB == 4, uint32_t, uint16_t>>;
  extern __shared__ int s_first[];             // plan_bytes
  constexpr int ROW = SQ + 4;                  // floats (48 or 80 bytes: eight lanes' 16 bytes take all banks)
  __shared__ __align__(16) float s_q[HD][ROW];
  __shared__ __align__(16) float s_p[kKeys][ROW];   // slot k in row k % 4 * 32 + k / 4
  __shared__ float s_m[SQ];
  __shared__ uint32_t s_mask[SQ][kWords + 1];
  const int lane = threadIdx.x;
  const Cache& c = a.c;
  pdl_wait();
  pdl_launch_dependents();
  build_plan(a, s_first);
  if (blockIdx.x == 0) check_lens(a);
  const int total = s_first[c.batch], runs = runs_of(a, total);
  if ((int)blockIdx.x >= runs) return;
  const int end = run_begin(blockIdx.x + 1, total, runs);
  const size_t row0 = row_of(c, a.layer, 0, 0, 0, 0);
  for (int unit = run_begin(blockIdx.x, total, runs); unit < end;) {
    const Segment s = segment_at(a, s_first, unit, end);
    __syncwarp();                              // (the segment before is done with shared memory)
    {
      float x[SQ][DPL];
#pragma unroll
      for (int v = 0; v < SQ; ++v) {
        const Vec w = vector_of(a, s.h, s.qb, v);
        const T* const q = static_cast<const T*>(a.q) + s.b * a.sq[0] + w.t * a.sq[1] + w.h * a.sq[2] + lane;
#pragma unroll
        for (int i = 0; i < DPL; ++i) x[v][i] = v < s.nq ? to_f32<T>(q[i * 32]) * a.scale : 0.f;
      }
#pragma unroll
      for (int i = 0; i < DPL; ++i)
#pragma unroll
        for (int v = 0; v < SQ; v += 4)
          *reinterpret_cast<float4*>(&s_q[i * 32 + lane][v]) = make_float4(x[v][i], x[v + 1][i], x[v + 2][i], x[v + 3][i]);
    }
    for (int i = lane; i < SQ * (kWords + 1); i += 32) {
      const int v = i / (kWords + 1), w = i % (kWords + 1);
      s_mask[v][w] = v < s.nq && w < a.W
                         ? a.mask[((size_t)s.b * a.T + vector_of(a, s.h, s.qb, v).t) * a.W + w] : 0u;
    }
    if (lane < SQ) s_m[lane] = -INFINITY;
    __syncwarp();
    float l[SQ];
    uint64_t o[SQ / 2][DPL];                   // of two vectors each
#pragma unroll
    for (int v = 0; v < SQ; ++v) l[v] = 0.f;
#pragma unroll
    for (int v = 0; v < SQ / 2; ++v)
#pragma unroll
      for (int i = 0; i < DPL; ++i) o[v][i] = 0ull;
    for (int ch = s.c0; ch < s.c1; ++ch) {
      // ---- scores of this lane's slots (four of a page: pages have 16 at least)
      const int slot = ch * kKeys + 4 * lane;
      int n = min(max(s.keys - slot, 0), 4), page = -1;   // n: of them that there are
      if (n > 0) {
        page = page_of(c, s.b, slot);
        if (page < 0) {
          set_status(a.status, CDSL_ERANGE);
          n = 0;
        }
      }
      const int at = slot & ((1 << c.page_shift) - 1);
      const size_t row = page >= 0 ? row_of(c, a.layer, page, 0, s.h, at) : row0;
      const size_t vrow = page >= 0 ? row_of(c, a.layer, page, 1, s.h, at) : row0;
      const uint32_t ks4 = *reinterpret_cast<const uint32_t*>(c.scale + row);   // (slots past the item's: not used)
      const uint32_t vs4 = *reinterpret_cast<const uint32_t*>(c.scale + vrow);
      const uint8_t* const k = c.pool + row * HD * EB;
      uint64_t t[SQ / 2][4];
#pragma unroll
      for (int v = 0; v < SQ / 2; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) t[v][e] = 0ull;
      uint4 next[4];
      auto load_k = [&](int i) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          next[e] = e < n ? reinterpret_cast<const uint4*>(k + e * HD * EB)[i] : make_uint4(0u, 0u, 0u, 0u);
      };
      load_k(0);
#pragma unroll 1
      for (int i = 0; i < LOADS; ++i) {
        uint32_t raw[4][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          raw[e][0] = next[e].x; raw[e][1] = next[e].y; raw[e][2] = next[e].z; raw[e][3] = next[e].w;
        }
        if (i + 1 < LOADS) load_k(i + 1);
#pragma unroll
        for (int j = 0; j < 4; j += EB) {      // four dimensions
          float x[4][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) decode4<F8>(raw[e][j], raw[e][j + EB - 1], x[e]);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            uint64_t xx[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) xx[e] = pair(x[e][d], x[e][d]);
#pragma unroll
            for (int v = 0; v < SQ; v += 4) {
              const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&s_q[i * CPL + j * 4 / EB + d][v]);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                t[v / 2][e] = fma2(q.x, xx[e], t[v / 2][e]);
                t[v / 2 + 1][e] = fma2(q.y, xx[e], t[v / 2 + 1][e]);
              }
            }
          }
        }
      }
      // ---- masks, maxima, probabilities
      float ks[4], vs[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ks[e] = e < n ? scale_value(ks4 >> (8 * e) & 255) : 1.f;
        vs[e] = e < n ? scale_value(vs4 >> (8 * e) & 255) : 0.f;
      }
      const int node = slot - s.len;           // the tree's node in the first slot
      const bool masked = __any_sync(0xffffffffu, node > -4 || n < 4);
#pragma unroll
      for (int v4 = 0; v4 < SQ; v4 += 4) {
        float p[4][4];                         // [slot][vector]
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = v4 + u;
          uint32_t seen = 15u;
          if (masked) {
            if (node >= 0) {
              const int w = min(node >> 5, kWords - 1);
              seen = node < 32 * kWords ? __funnelshift_r(s_mask[v][w], s_mask[v][w + 1], node & 31) : 0u;
            } else if (node > -4) {
              seen = ((1u << -node) - 1) | s_mask[v][0] << -node;
            }
            seen &= (1u << n) - 1;
            if (v >= s.nq) seen = 0u;
          }
          float x[4], top = -INFINITY;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 two = unpair(t[v / 2][e]);
            x[e] = (u % 2 ? two.y : two.x) * ks[e];
            if (!masked || seen >> e & 1) top = fmaxf(top, x[e]);
          }
          const float m = s_m[v], mn = fmaxf(m, warp_fmax(top));
          float alpha = 1.f;
          if (mn != m) {                       // (alike in all lanes)
            alpha = m == -INFINITY ? 0.f : exp2f(m - mn);
            const uint64_t both = u % 2 ? pair(1.f, alpha) : pair(alpha, 1.f);
#pragma unroll
            for (int i = 0; i < DPL; ++i) o[v / 2][i] = mul2(o[v / 2][i], both);
            l[v] *= alpha;
            __syncwarp();
            if (lane == 0) s_m[v] = mn;
          }
          // NaN scores (a NaN row) survive: they are visible, and fmaxf left them out of the maximum
          const float off = mn == -INFINITY ? 0.f : mn;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool see = !masked || seen >> e & 1;
            const float y = see ? exp2f(x[e] - off) : 0.f;
            l[v] += y;
            p[e][u] = see ? y * vs[e] : 0.f;   // V's scale; what a row sees as NaN stays NaN
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<float4*>(&s_p[e * 32 + lane][v4]) = make_float4(p[e][0], p[e][1], p[e][2], p[e][3]);
      }
      __syncwarp();
      // ---- P V of this lane's dimensions (16 slots of a page at a time)
      const int kn = min(s.keys - ch * kKeys, kKeys);
      const uint32_t mine = page >= 0 ? (uint32_t)(vrow - row0) : ~0u;
      VBits ahead[AHEAD];
      auto load_v = [&](int k0) {
        const uint32_t first = __shfl_sync(0xffffffffu, mine, k0 / 4 & 31);
        const VBits* const v = reinterpret_cast<const VBits*>(c.pool + (row0 + first) * HD * EB) + lane;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e)
          ahead[e] = first != ~0u && k0 + e < kn ? v[e * 32] : VBits{};
      };
      load_v(0);
#pragma unroll 1
      for (int k0 = 0; k0 < kn; k0 += AHEAD) {
        VBits raw[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) raw[e] = ahead[e];
        if (k0 + AHEAD < kn) load_v(k0 + AHEAD);
#pragma unroll
        for (int e = 0; e < AHEAD; e += 4) {
          float x[4][DPL];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (DPL == 4 && F8) {
              decode4<true>(raw[e + i], 0u, x[i]);
            } else if constexpr (DPL == 4) {
              decode4<false>(raw[e + i].x, raw[e + i].y, x[i]);
            } else if constexpr (F8) {
              const float2 y = f8x2_to_f32(raw[e + i]);
              x[i][0] = y.x; x[i][1] = y.y;
            } else {
              x[i][0] = __uint_as_float(raw[e + i] << 16);
              x[i][1] = __uint_as_float(raw[e + i] & 0xffff0000u);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint64_t xx[DPL];
#pragma unroll
            for (int d = 0; d < DPL; ++d) xx[d] = pair(x[i][d], x[i][d]);
#pragma unroll
            for (int v = 0; v < SQ; v += 4) {
              const ulonglong2 p = *reinterpret_cast<const ulonglong2*>(&s_p[i * 32 + (k0 + e) / 4][v]);
#pragma unroll
              for (int d = 0; d < DPL; ++d) {
                o[v / 2][d] = fma2(p.x, xx[d], o[v / 2][d]);
                o[v / 2 + 1][d] = fma2(p.y, xx[d], o[v / 2 + 1][d]);
              }
            }
          }
        }
      }
      __syncwarp();
    }
    const bool whole = s.c0 == 0 && s.c1 == s.units;
    const size_t slot = (size_t)blockIdx.x * 2 + (s.c0 == 0);
    const int live = min(SQ, a.T * a.G - s.qb * SQ);
#pragma unroll
    for (int v = 0; v < SQ; ++v) {
      const bool any = v < s.nq;               // (a vector past the nodes: zeros)
      const float sum = any ? warp_sum(l[v]) : 0.f, m = any ? s_m[v] : -INFINITY;
      if (v < live) {
        float x[DPL];
#pragma unroll
        for (int i = 0; i < DPL; ++i) {
          const float2 two = unpair(o[v / 2][i]);
          x[i] = v % 2 ? two.y : two.x;
        }
        if (whole) {
          const Vec w = vector_of(a, s.h, s.qb, v);
#pragma unroll
          for (int i = 0; i < DPL; ++i) store_out<T>(a, s.b, w, lane * DPL + i, sum == 0.f ? 0.f : x[i] / sum);
          if (lane == 0) store_lse(a, s.b, w, m, sum);
        } else {
#pragma unroll
          for (int i = 0; i < DPL; ++i) a.part_o[(slot * SQ + v) * HD + lane * DPL + i] = any ? x[i] : 0.f;
          if (lane == 0) {
            a.part_ml[(slot * 2) * SQ + v] = m;
            a.part_ml[(slot * 2 + 1) * SQ + v] = sum;
          }
        }
      }
    }
    unit += s.c1 - s.c0;
  }
}

// Joins the parts of the items that several runs share: a warp per query vector, its lanes along
// head_dim. Grid: (items, blocks of kCombine vectors), or (bounds between runs, the same) where there are fewer of
// them: then the first bound inside an item stands for it. It is scheduled beside the pass and works out the item's runs
// from the lengths before it waits for the pass (whose blocks let it start after their own wait, so that what wrote the
// lengths has ended); then a vector's (m, l) and its first parts' values are loaded
// together. Bound by that one round trip to L2, on large passes by the parts' bytes, and with many short
// items by its blocks, most without anything to join: 33 trees of 48 of 32 heads after 115 tokens, 528 items, 152 runs:
// 27 us by items, 16 by bounds.
constexpr int kCombine = 4, kAhead = 8;
template <typename T, int HD, bool Bounds>
__global__ void __launch_bounds__(32 * kCombine) k_tree_combine(TreeArgs a) {
  constexpr int DPL = HD / 32;
  const int lane = threadIdx.x & 31;
  const int v = blockIdx.y * kCombine + (threadIdx.x >> 5);
  int qb = blockIdx.x % a.QB, h = blockIdx.x / a.QB % a.c.kvh, b = blockIdx.x / a.QB / a.c.kvh;
  if (!Bounds && (qb >= live_blocks(a, nodes_of(a, b)) || v >= min(a.NQ, a.T * a.G - qb * a.NQ))) return pdl_wait();
  int before = 0, total = 0;                   // units of the sequences before, and of all
  for (int x = lane; x < a.c.batch; x += 32) {
    const int w = units_of(a, len_of(a, x), nodes_of(a, x));
    total += w;
    if (!Bounds && x < b) before += w;
  }
  total = __reduce_add_sync(0xffffffffu, total);
  const int runs = runs_of(a, total);
  int x = 0;                                   // the bound, from the sequence's first unit
  if (Bounds) {
    const int bound = (int)blockIdx.x + 1;
    if (bound >= runs) return pdl_wait();
    x = run_begin(bound, total, runs);
    for (int b0 = 0; b0 < a.c.batch; b0 += 32) {   // the sequence that it lies in
      const int w = b0 + lane < a.c.batch ? units_of(a, len_of(a, b0 + lane), nodes_of(a, b0 + lane)) : 0;
      int upto = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, upto > x);
      if (past) {
        const int at = __ffs(past) - 1;
        const int skip = __shfl_sync(0xffffffffu, upto - w, at);
        b = b0 + at;
        before += skip;
        x -= skip;
        break;
      }
      const int all = __shfl_sync(0xffffffffu, upto, 31);
      before += all;
      x -= all;
    }
  } else {
    before = __reduce_add_sync(0xffffffffu, before);
  }
  const int n = nodes_of(a, b), live = live_blocks(a, n), u = item_units(a, len_of(a, b) + n);
  const int per_head = live * u + a.QB - live;
  if (Bounds) {
    h = x / per_head;
    const int y = x % per_head;
    qb = y / u;
    // (at an item's start; an item without queries, of one unit; past the block's vectors)
    if (y >= live * u || y % u == 0 || v >= min(a.NQ, a.T * a.G - qb * a.NQ)) return pdl_wait();
  }
  const int s = before + h * per_head + qb * u;
  const int r0 = run_of(s, total, runs), r1 = run_of(s + u - 1, total, runs);
  if (Bounds && r0 != (int)blockIdx.x) return pdl_wait();   // (not the item's first)
  pdl_wait();                                  // (no block ends before the pass has)
  if (r0 == r1) return;                        // whole: written
  auto slot = [&](int r) { return (size_t)r * 2 + (r == r0); };
  struct Values { float x[DPL]; };
  auto load = [&](int r) {
    Values z;
    const float* p = a.part_o + (slot(r) * a.NQ + v) * HD + lane * DPL;
    if constexpr (DPL == 4) {
      const float4 t = *reinterpret_cast<const float4*>(p);
      z.x[0] = t.x; z.x[1] = t.y; z.x[2] = t.z; z.x[3] = t.w;
    } else {
      const float2 t = *reinterpret_cast<const float2*>(p);
      z.x[0] = t.x; z.x[1] = t.y;
    }
    return z;
  };
  float M = -INFINITY, L = 0.f, acc[DPL];
#pragma unroll
  for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
  for (int rb = r0; rb <= r1; rb += 32) {      // 32 runs at a time: a lane has one's (m, l)
    const int cnt = min(32, r1 - rb + 1);
    float m = -INFINITY, l = 0.f;
    if (lane < cnt) {
      m = a.part_ml[slot(rb + lane) * 2 * a.NQ + v];
      l = a.part_ml[(slot(rb + lane) * 2 + 1) * a.NQ + v];
    }
    Values z[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      if (e < cnt) z[e] = load(rb + e);
    const float Mn = fmaxf(M, warp_max(m));
    const float keep = M == -INFINITY ? 0.f : exp2f(M - Mn);
    const float w = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(m - Mn);   // (l NaN: kept)
    L = L * keep + warp_sum(w * l);
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] *= keep;
    for (int r = 0; r < cnt; r += kAhead) {
      if (r > 0)
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
          if (r + e < cnt) z[e] = load(rb + r + e);
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const float wr = __shfl_sync(0xffffffffu, w, (r + e) & 31);
        if (r + e < cnt)
#pragma unroll
          for (int i = 0; i < DPL; ++i) acc[i] = fmaf(wr, z[e].x[i], acc[i]);
      }
    }
    M = Mn;
  }
  const Vec w = vector_of(a, h, qb, v);
#pragma unroll
  for (int i = 0; i < DPL; ++i) store_out<T>(a, b, w, lane * DPL + i, L == 0.f ? 0.f : acc[i] / L);
  if (lane == 0) store_lse(a, b, w, M, L);
}

// The same for items that many runs share (a 4-bit cache's, of a warp each): a block per vector, whose warps take parts in
// turn and join what they have through shared memory. Sequences of 16,384 tokens, one token of 32 heads over 8, the whole
// call, this way / the one above: 228 parts an item 17.1 / 33.7 us, 57 29.6 / 33.4, 33 42.7 / 44.4, 28 46.0 / 46.9, 23 56.7 /
// 56.5, 14 82.6 / 79.5; of four tokens (8 warps an SM) 38 parts 30.2 / 35.5, 19 73.3 / 69.9. From 32 on it is taken.
constexpr int kWide = 8;                       // warps
template <typename T, int HD>
__global__ void __launch_bounds__(32 * kWide) k_tree_combine_wide(TreeArgs a) {
  constexpr int DPL = HD / 32;
  __shared__ float s_m[kWide], s_l[kWide], s_o[kWide][HD];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int v = blockIdx.y, qb = blockIdx.x % a.QB, h = blockIdx.x / a.QB % a.c.kvh, b = blockIdx.x / a.QB / a.c.kvh;
  const int n = nodes_of(a, b), live = live_blocks(a, n), u = item_units(a, len_of(a, b) + n);
  if (qb >= live || v >= min(a.NQ, a.T * a.G - qb * a.NQ)) return pdl_wait();
  int before = 0, total = 0;                   // units of the sequences before, and of all
  for (int x = lane; x < a.c.batch; x += 32) {
    const int w = units_of(a, len_of(a, x), nodes_of(a, x));
    total += w;
    if (x < b) before += w;
  }
  total = __reduce_add_sync(0xffffffffu, total);
  before = __reduce_add_sync(0xffffffffu, before);
  const int runs = runs_of(a, total), s = before + h * (live * u + a.QB - live) + qb * u;
  const int r0 = run_of(s, total, runs), r1 = run_of(s + u - 1, total, runs);
  pdl_wait();                                  // (no block ends before the pass has)
  if (r0 == r1) return;                        // whole: written
  auto slot = [&](int r) { return (size_t)r * 2 + (r == r0); };
  float M = -INFINITY, L = 0.f, acc[DPL];
#pragma unroll
  for (int i = 0; i < DPL; ++i) acc[i] = 0.f;
  for (int rb = r0 + warp; rb <= r1; rb += 32 * kWide) {   // 32 of the warp's parts: a lane has one's (m, l)
    const int mine = rb + lane * kWide, cnt = min(32, (r1 - rb) / kWide + 1);
    float m = -INFINITY, l = 0.f;
    if (mine <= r1) {
      m = a.part_ml[slot(mine) * 2 * a.NQ + v];
      l = a.part_ml[(slot(mine) * 2 + 1) * a.NQ + v];
    }
    const float Mn = fmaxf(M, warp_max(m));
    const float keep = M == -INFINITY ? 0.f : exp2f(M - Mn);
    const float w = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : exp2f(m - Mn);   // (l NaN: kept)
    L = L * keep + warp_sum(w * l);
#pragma unroll
    for (int i = 0; i < DPL; ++i) acc[i] *= keep;
    for (int r = 0; r < cnt; r += kAhead) {
      float z[kAhead][DPL];
#pragma unroll
      for (int e = 0; e < kAhead; ++e)
        if (r + e < cnt) {
          const float* const p = a.part_o + (slot(rb + (r + e) * kWide) * a.NQ + v) * HD + lane * DPL;
          if constexpr (DPL == 4) {
            const float4 t = *reinterpret_cast<const float4*>(p);
            z[e][0] = t.x; z[e][1] = t.y; z[e][2] = t.z; z[e][3] = t.w;
          } else {
            const float2 t = *reinterpret_cast<const float2*>(p);
            z[e][0] = t.x; z[e][1] = t.y;
          }
        }
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const float wr = __shfl_sync(0xffffffffu, w, (r + e) & 31);
        if (r + e < cnt)
#pragma unroll
          for (int i = 0; i < DPL; ++i) acc[i] = fmaf(wr, z[e][i], acc[i]);
      }
    }
    M = Mn;
  }
  if (lane == 0) {
    s_m[warp] = M;
    s_l[warp] = L;
  }
#pragma unroll
  for (int i = 0; i < DPL; ++i) s_o[warp][lane * DPL + i] = acc[i];
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWide; ++w) top = fmaxf(top, s_m[w]);
  const Vec x = vector_of(a, h, qb, v);
  for (int d = threadIdx.x; d < HD; d += 32 * kWide) {
    float sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kWide; ++w) {
      const float f = s_m[w] == -INFINITY ? (s_l[w] == 0.f ? 0.f : 1.f) : exp2f(s_m[w] - top);
      sum = fmaf(f, s_l[w], sum);
      o = fmaf(f, s_o[w][d], o);
    }
    store_out<T>(a, b, x, d, sum == 0.f ? 0.f : o / sum);
    if (d == 0) store_lse(a, b, x, top, sum);
  }
}

// Sizes of a pass, the same at every length: runs and workspace.
struct Sizes {
  int NQ, QB, blocks;
  size_t o_off, bytes;
};
void bytes_of(const Cache& c, Sizes* z) {
  const size_t slots = (size_t)z->blocks * 2 * z->NQ;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  z->o_off = up(slots * 2 * sizeof(float));
  z->bytes = up(z->o_off + slots * c.hd * sizeof(float));
}
void sizes_of(const Cache& c, bool tc, int H, int T, Sizes* z) {   // tc: bf16 queries
  const int vectors = T * (H / c.kvh);
  if (c.format == kI4) {
    z->NQ = !tc ? 8 : vectors <= 4 ? 4 : vectors <= 8 ? 8 : vectors <= 16 ? 16 : kRowsBlock;
    z->QB = (vectors + z->NQ - 1) / z->NQ;
    z->blocks = kPlanSMs * (z->NQ == kRowsBlock ? 1 : i4_blocks_per_sm(c, z->NQ, !tc));
    return bytes_of(c, z);
  }
  z->NQ = !tc ? SQ : vectors <= 16 ? 16 : vectors <= 32 ? 32 : kRowsBlock;
  z->QB = (vectors + z->NQ - 1) / z->NQ;
  z->blocks = kPlanSMs * (!tc ? simt_per_sm(c.hd, c.format == kF8) : z->NQ == kRowsBlock ? 1 : tc_blocks_per_sm(c, z->NQ));
  bytes_of(c, z);
}

template <typename T, int HD>
cudaError_t launch_combine(const TreeArgs& a, cudaStream_t s) {
  const int items = a.c.batch * a.c.kvh * a.QB, bounds = std::max(a.blocks - 1, 1);
  if (a.c.format == kI4 && a.NQ < kRowsBlock && a.blocks >= 32 * items)   // (parts of an item, about: see there)
    return launch_pdl(k_tree_combine_wide<T, HD>, dim3(items, std::min(a.NQ, a.T * a.G)), dim3(32 * kWide), 0, s, a);
  const dim3 grid(std::min(items, bounds), (std::min(a.NQ, a.T * a.G) + kCombine - 1) / kCombine);
  return launch_pdl(bounds < items ? k_tree_combine<T, HD, true> : k_tree_combine<T, HD, false>, grid,
                    dim3(32 * kCombine), 0, s, a);
}

template <typename T, int HD, bool F8>
cudaError_t launch_simt(const TreeArgs& a, cudaStream_t s) {
  return launch_pdl(k_tree_simt<T, HD, F8>, dim3(a.blocks), dim3(32), plan_bytes(a.c.batch), s, a);
}

cudaError_t launch_pass(const TreeArgs& a, bool tc, bool split, cudaStream_t s) {
  const bool d128 = a.c.hd == 128, f8 = a.c.format == kF8, bf16 = a.dtype == CDSL_DTYPE_BF16;
  cudaError_t e;
  if (a.c.format == kI4 && a.NQ < kRowsBlock) e = launch_tree_i4(a, s);
  else if (tc) e = a.NQ == kRowsBlock ? launch_tree_rows(a, s) : launch_tree_tc(a, s);
  else if (d128) e = f8 ? launch_simt<float, 128, true>(a, s) : launch_simt<float, 128, false>(a, s);
  else e = f8 ? launch_simt<float, 64, true>(a, s) : launch_simt<float, 64, false>(a, s);
  if (e != cudaSuccess || !split) return e;
  if (bf16) return d128 ? launch_combine<__nv_bfloat16, 128>(a, s) : launch_combine<__nv_bfloat16, 64>(a, s);
  return d128 ? launch_combine<float, 128>(a, s) : launch_combine<float, 64>(a, s);
}

bool heads_ok(const Check& ck, const Cache& c, int n_heads) {
  if (n_heads < 1 || n_heads % c.kvh || n_heads / c.kvh > 64)
    return ck.no("n_heads must be a multiple of n_kv_heads, at most 64 to one");
  return true;
}

}  // namespace
}  // namespace tree
}  // namespace cdsl

using namespace cdsl;
using namespace cdsl::tree;

extern "C" int32_t cdsl_tree_mask(const int32_t* h_parents, int32_t T, uint32_t* h_mask,
                                  int32_t* h_depth) {
  Check ck("cdsl_tree_mask");
  if (!h_parents || !h_mask) return ck.fail("a required pointer is NULL");
  if (T < 1 || T > CDSL_TREE_MAX_NODES) return ck.fail("T must be 1 .. 128 nodes");
  for (int i = 1; i < T; ++i)
    if (h_parents[i] < 0 || h_parents[i] >= i) return ck.fail("a node's parent must have a smaller index");
  const int W = (T + 31) / 32;
  for (int i = 0; i < T; ++i) {
    for (int w = 0; w < W; ++w) h_mask[i * W + w] = i ? h_mask[h_parents[i] * W + w] : 0u;
    h_mask[i * W + i / 32] |= 1u << (i % 32);
    if (h_depth) h_depth[i] = i ? h_depth[h_parents[i]] + 1 : 0;
  }
  return CDSL_OK;
}

extern "C" int32_t cdsl_tree_attention_workspace(const cdsl_kv_cache* cache, int32_t n_heads, int32_t T,
                                                 size_t* bytes) {
  Check ck("cdsl_tree_attention_workspace");
  Cache c;
  if (!ck.cache(cache, &c, false) || !ck.nodes(c, T) || !heads_ok(ck, c, n_heads)) return CDSL_EINVAL;
  if (!bytes) return ck.fail("bytes is NULL");
  Sizes z[2];
  sizes_of(c, false, n_heads, T, &z[0]);
  sizes_of(c, true, n_heads, T, &z[1]);
  *bytes = std::max(z[0].bytes, z[1].bytes);
  return CDSL_OK;
}

extern "C" int32_t cdsl_tree_attention(const cdsl_kv_cache* cache, int32_t layer, const void* d_q,
                                       int32_t dtype, int32_t n_heads, int32_t T,
                                       const int64_t* h_strides, const int32_t* d_lens,
                                       const int32_t* d_nodes, const uint32_t* d_mask, float scale,
                                       int32_t max_len, void* d_out, float* d_lse, void* d_workspace,
                                       size_t workspace_bytes, int32_t* d_status, void* stream) {
  Check ck("cdsl_tree_attention");
  Cache c;
  if (!ck.cache(cache, &c) || !ck.layers(c, layer, 1) || !ck.value_type(dtype) || !ck.nodes(c, T) ||
      !heads_ok(ck, c, n_heads))
    return CDSL_EINVAL;
  if (!d_q || !d_out || !h_strides || !d_lens || !d_mask || !d_workspace)
    return ck.fail("a required pointer is NULL");
  if (!(scale > 0.f) || scale > 1e30f) return ck.fail("scale must be positive and finite");
  if (max_len < 0 || (long long)max_len + T > ((long long)c.max_pages << c.page_shift))
    return ck.fail("max_len must be 0 .. max_pages * page_size - T");
  const int eb = dtype == CDSL_DTYPE_BF16 ? 2 : 4;
  if (!ck.aligned(d_q, eb) || !ck.aligned(d_out, eb)) return ck.fail("q and out must be aligned to their type");
  const int64_t* const so = h_strides + 3;
  if ((c.batch > 1 && so[0] == 0) || (T > 1 && so[1] == 0) || (n_heads > 1 && so[2] == 0))
    return ck.fail("out must not have a stride of 0 between sequences, tokens or heads");
  const bool tc = dtype == CDSL_DTYPE_BF16;
  Sizes z;
  sizes_of(c, tc, n_heads, T, &z);
  if (!ck.aligned(d_workspace, 256) || workspace_bytes < z.bytes)
    return ck.fail("the workspace must be 256-byte aligned and hold cdsl_tree_attention_workspace bytes",
                   workspace_bytes < z.bytes ? CDSL_ENOMEM : CDSL_EINVAL);
  const int unit_shift = c.format == kI4 && z.NQ < kRowsBlock ? 6 : 7;
  static_assert(kKeys == 1 << 7);
  const long long chunks = ((long long)max_len + T + (1 << unit_shift) - 1) >> unit_shift;
  const long long units = chunks * c.batch * c.kvh * z.QB;   // at most
  if (units >= (1LL << 31)) return ck.fail("the pass is beyond the limit (2^31 chunks of 128 slots, 64 in 4 bits)");
  TreeArgs a = {};
  a.c = c;
  a.dtype = dtype;
  a.unit_shift = unit_shift;
  a.layer = layer; a.T = T; a.H = n_heads; a.G = n_heads / c.kvh; a.W = (T + 31) / 32;
  a.NQ = z.NQ; a.QB = z.QB;
  a.q = d_q; a.out = d_out; a.lse = d_lse;
  for (int i = 0; i < 3; ++i) { a.sq[i] = h_strides[i]; a.so[i] = h_strides[3 + i]; }
  a.lens = d_lens; a.nodes = d_nodes; a.mask = d_mask;
  a.scale = scale * kLog2e;
  a.max_len = max_len;
  a.blocks = (int)std::min<long long>(z.blocks, units);
  char* ws = static_cast<char*>(d_workspace);
  a.part_ml = reinterpret_cast<float*>(ws);
  a.part_o = reinterpret_cast<float*>(ws + z.o_off);
  a.status = d_status;
  const bool split = chunks > 1;               // one chunk: every item is whole
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return ck.launched(launch_pass(a, tc, split, s));
}
