// tree_attention.cu -- cdsl_tree_attention: the CUDA-core kernel (fp32 queries), the joining of
// partial results and the entry points.
//
// k_tree_simt: 128 threads. Scores: a thread owns a slot of the chunk, reads its K row 16 bytes at a time
// and multiplies it by the block's 16 query vectors, which shared memory broadcasts (fp32, scaled by
// softmax scale * log2 e). Softmax: maxima over the warps, a running maximum and a sum that each thread
// keeps of its own slots. P V: a thread owns a dimension (head_dim 64: of half the slots) and walks
// the chunk's V rows. Bound by its fp32 FMAs and shared-memory broadcasts: 2 * 16 * head_dim products a
// slot.
#include <cuda.h>

#include <algorithm>

#include "tree_attention.cuh"
#include "tree_host.h"

namespace cdsl {
namespace tree {
namespace {

constexpr int SQ = 16;                         // query vectors per block
constexpr int kThreads = kKeys;
constexpr int kWarps = kThreads / 32;

// 16 bytes of codes to floats.
template <bool F8>
__device__ __forceinline__ void decode16(const uint4& u, float (&x)[F8 ? 16 : 8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F8) {
      const float2 a = f8x2_to_f32(w[i] & 0xffffu), b = f8x2_to_f32(w[i] >> 16);
      x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = b.x; x[4 * i + 3] = b.y;
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

template <typename T, int HD, bool F8>
__global__ void __launch_bounds__(kThreads) k_tree_simt(TreeArgs a) {
  extern __shared__ int s_first[];             // [batch + 1]
  __shared__ __align__(16) float s_q[SQ][HD], s_p[SQ][kKeys];
  __shared__ float s_max[kWarps][SQ], s_sum[kWarps][SQ];
  __shared__ uint32_t s_mask[SQ][kWords];
  __shared__ uint32_t s_row[kKeys];            // V row of each slot of the chunk, ~0: none
  constexpr int CPL = F8 ? 16 : 8;             // codes per 16 bytes
  constexpr int SPLIT = kThreads / HD;         // threads per dimension
  const int tid = threadIdx.x, warp = tid >> 5;
  const Cache& c = a.c;
  pdl_wait();
  pdl_launch_dependents();
  build_plan(a, s_first);
  if (blockIdx.x == 0) check_lens(a);
  const int total = s_first[c.batch], runs = runs_of(a, total);
  if ((int)blockIdx.x >= runs) return;
  const int end = run_begin(blockIdx.x + 1, total, runs);
  for (int unit = run_begin(blockIdx.x, total, runs); unit < end;) {
    const Segment s = segment_at(a, s_first, unit, end);
    __syncthreads();                           // (the segment before is done with shared memory)
    for (int i = tid; i < SQ * HD; i += kThreads) {
      const int v = i / HD, d = i % HD;
      float x = 0.f;
      if (v < s.nq) {
        const Vec w = vector_of(a, s.h, s.qb, v);
        x = to_f32<T>(static_cast<const T*>(a.q)[s.b * a.sq[0] + w.t * a.sq[1] + w.h * a.sq[2] + d]) * a.scale;
      }
      s_q[v][d] = x;
    }
    for (int i = tid; i < SQ * kWords; i += kThreads) {
      const int v = i / kWords, w = i % kWords;
      s_mask[v][w] = v < s.nq && w < a.W
                         ? __ldg(a.mask + ((size_t)s.b * a.T + vector_of(a, s.h, s.qb, v).t) * a.W + w) : 0u;
    }
    __syncthreads();
    float m[SQ], l[SQ], o[SQ];
#pragma unroll
    for (int v = 0; v < SQ; ++v) { m[v] = -INFINITY; l[v] = o[v] = 0.f; }
    for (int ch = s.c0; ch < s.c1; ++ch) {
      const int slot = ch * kKeys + tid;
      // ---- scores of this thread's slot
      int page = -1;
      if (slot < s.keys) {
        page = page_of(c, s.b, slot);
        if (page < 0) set_status(a.status, CDSL_ERANGE);
      }
      float t[SQ], vs = 0.f;
#pragma unroll
      for (int v = 0; v < SQ; ++v) t[v] = 0.f;
      s_row[tid] = ~0u;
      if (page >= 0) {
        const int at = slot & ((1 << c.page_shift) - 1);
        const size_t row = row_of(c, a.layer, page, 0, s.h, at);
        const size_t vrow = row_of(c, a.layer, page, 1, s.h, at);
        s_row[tid] = (uint32_t)(vrow - row_of(c, a.layer, 0, 0, 0, 0));
        const uint4* k = reinterpret_cast<const uint4*>(c.pool + row * HD * (F8 ? 1 : 2));
        constexpr int LOADS = HD / CPL, AHEAD = LOADS < 8 ? LOADS : 8;   // in flight together
#pragma unroll 1
        for (int i0 = 0; i0 < LOADS; i0 += AHEAD) {
          uint4 raw[AHEAD];
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) raw[i] = __ldg(k + i0 + i);
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) {
            float x[CPL];
            decode16<F8>(raw[i], x);
#pragma unroll
            for (int v = 0; v < SQ; ++v)
#pragma unroll
              for (int e = 0; e < CPL; e += 4) {
                const float4 q = *reinterpret_cast<const float4*>(&s_q[v][(i0 + i) * CPL + e]);
                t[v] = fmaf(q.x, x[e], fmaf(q.y, x[e + 1], fmaf(q.z, x[e + 2], fmaf(q.w, x[e + 3], t[v]))));
              }
          }
        }
        const float ks = scale_value(c.scale[row]);
        vs = scale_value(c.scale[vrow]);
#pragma unroll
        for (int v = 0; v < SQ; ++v) t[v] *= ks;
      }
      // ---- masks, maxima
      const int node = slot - s.len;
      uint32_t vis = 0;
#pragma unroll
      for (int v = 0; v < SQ; ++v) {
        const bool ok = page >= 0 && v < s.nq && (node < 0 || (s_mask[v][node >> 5] >> (node & 31) & 1));
        vis |= (uint32_t)ok << v;
        const float wm = warp_max(ok ? t[v] : -INFINITY);
        if ((tid & 31) == 0) s_max[warp][v] = wm;
      }
      __syncthreads();
#pragma unroll
      for (int v = 0; v < SQ; ++v) {
        float mn = m[v];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mn = fmaxf(mn, s_max[w][v]);
        const float alpha = m[v] == -INFINITY ? 0.f : exp2f(m[v] - mn);
        m[v] = mn;
        // NaN scores (a NaN row) survive: they are visible, and fmaxf left them out of the maximum
        const float p = vis >> v & 1 ? exp2f(t[v] - (mn == -INFINITY ? 0.f : mn)) : 0.f;
        l[v] = l[v] * alpha + p;
        o[v] *= alpha;
        s_p[v][tid] = vis >> v & 1 ? p * vs : 0.f;   // V's scale; what a row sees as NaN stays NaN
      }
      __syncthreads();
      // ---- P V of this thread's dimension (and share of the slots)
      const int d = tid % HD, k0 = tid / HD * (kKeys / SPLIT);
      const int kn = min(s.keys - ch * kKeys, k0 + kKeys / SPLIT);
      const uint8_t* const pool = c.pool + row_of(c, a.layer, 0, 0, 0, 0) * HD * (F8 ? 1 : 2);
#pragma unroll 1
      for (int k = k0; k < kn; k += 16) {      // 16 slots' loads in flight
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint32_t row = s_row[k + e];
          x[e] = 0.f;
          if (k + e < kn && row != ~0u) {
            const uint8_t* v = pool + (size_t)row * HD * (F8 ? 1 : 2);
            x[e] = F8 ? f8x2_to_f32(__ldg(v + d)).x
                      : __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(v) + d) << 16);
          }
        }
#pragma unroll
        for (int v = 0; v < SQ; ++v)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const float4 p = *reinterpret_cast<const float4*>(&s_p[v][k + e]);
            o[v] = fmaf(p.x, x[e], fmaf(p.y, x[e + 1], fmaf(p.z, x[e + 2], fmaf(p.w, x[e + 3], o[v]))));
          }
      }
      __syncthreads();
    }
    // ---- the threads' sums, and the halves' outputs of a dimension
#pragma unroll
    for (int v = 0; v < SQ; ++v) {
      const float ws = warp_sum(l[v]);
      if ((tid & 31) == 0) s_sum[warp][v] = ws;
      if (SPLIT > 1) s_p[v][tid] = o[v];
    }
    __syncthreads();
    const bool whole = s.c0 == 0 && s.c1 == s.units;
    const size_t slot = (size_t)blockIdx.x * 2 + (s.c0 == 0);
    const int live = min(SQ, a.T * a.G - s.qb * SQ);
#pragma unroll
    for (int v = 0; v < SQ; ++v) {
      if (v >= live || tid >= HD) break;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += s_sum[w][v];
      float x = o[v];
      if (SPLIT > 1) x += s_p[v][tid + HD];
      if (whole) {
        const Vec w = vector_of(a, s.h, s.qb, v);
        store_out<T>(a, s.b, w, tid, sum == 0.f ? 0.f : x / sum);
        if (tid == 0) store_lse(a, s.b, w, m[v], sum);
      } else {
        a.part_o[(slot * SQ + v) * HD + tid] = x;
        if (tid == 0) {
          a.part_ml[(slot * 2) * SQ + v] = m[v];
          a.part_ml[(slot * 2 + 1) * SQ + v] = sum;
        }
      }
    }
    unit += s.c1 - s.c0;
  }
}

// Joins the parts of the items that several runs share: a warp per query vector, its lanes along
// head_dim. Grid: (items, blocks of kCombine vectors). It is scheduled beside the pass and works out the item's runs
// from the lengths before it waits for them; then a vector's (m, l) and its first parts' values are loaded
// together. Bound by that one round trip to L2, and on large passes by the parts' bytes.
constexpr int kCombine = 4, kAhead = 8;
template <typename T, int HD>
__global__ void __launch_bounds__(32 * kCombine) k_tree_combine(TreeArgs a) {
  constexpr int DPL = HD / 32;
  const int lane = threadIdx.x & 31;
  const int item = blockIdx.x;
  const int qb = item % a.QB, h = item / a.QB % a.c.kvh, b = item / a.QB / a.c.kvh;
  const int v = blockIdx.y * kCombine + (threadIdx.x >> 5);
  const int n = nodes_of(a, b), live = live_blocks(a, n);
  if (qb >= live || v >= min(a.NQ, a.T * a.G - qb * a.NQ)) return pdl_wait();
  int before = 0, total = 0;                   // units of the sequences before, and of all
  for (int x = lane; x < a.c.batch; x += 32) {
    const int w = units_of(a, x);
    total += w;
    if (x < b) before += w;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  total = __reduce_add_sync(0xffffffffu, total);
  const int u = item_units(len_of(a, b) + n);
  const int s = before + h * (live * u + a.QB - live) + qb * u;
  const int runs = runs_of(a, total), r0 = run_of(s, total, runs), r1 = run_of(s + u - 1, total, runs);
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

// Sizes of a pass, the same at every length: runs and workspace.
struct Sizes {
  int NQ, QB, blocks;
  size_t o_off, bytes;
};
constexpr int kSimtPerSM = 4;                  // resident k_tree_simt blocks per SM

void sizes_of(const Cache& c, bool tc, int H, int T, Sizes* z) {
  const int vectors = T * (H / c.kvh);
  z->NQ = !tc ? SQ : vectors <= 16 ? 16 : vectors <= 32 ? 32 : kRowsBlock;
  z->QB = (vectors + z->NQ - 1) / z->NQ;
  z->blocks = kPlanSMs * (!tc ? kSimtPerSM : z->NQ == kRowsBlock ? 1 : tc_blocks_per_sm(c, z->NQ));
  const size_t slots = (size_t)z->blocks * 2 * z->NQ;
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  z->o_off = up(slots * 2 * sizeof(float));
  z->bytes = up(z->o_off + slots * c.hd * sizeof(float));
}

template <typename T, int HD>
cudaError_t launch_combine(const TreeArgs& a, cudaStream_t s) {
  const dim3 grid(a.c.batch * a.c.kvh * a.QB, (std::min(a.NQ, a.T * a.G) + kCombine - 1) / kCombine);
  return launch_pdl(k_tree_combine<T, HD>, grid, dim3(32 * kCombine), 0, s, a);
}

template <typename T, int HD, bool F8>
cudaError_t launch_simt(const TreeArgs& a, cudaStream_t s) {
  return launch_pdl(k_tree_simt<T, HD, F8>, dim3(a.blocks), dim3(kThreads), (a.c.batch + 1) * 4, s, a);
}

cudaError_t launch_pass(const TreeArgs& a, bool tc, bool split, cudaStream_t s) {
  const bool d128 = a.c.hd == 128, f8 = a.c.eb == 1;
  cudaError_t e;
  if (tc) e = a.NQ == kRowsBlock ? launch_tree_rows(a, s) : launch_tree_tc(a, s);
  else if (d128) e = f8 ? launch_simt<float, 128, true>(a, s) : launch_simt<float, 128, false>(a, s);
  else e = f8 ? launch_simt<float, 64, true>(a, s) : launch_simt<float, 64, false>(a, s);
  if (e != cudaSuccess || !split) return e;
  if (tc) return d128 ? launch_combine<__nv_bfloat16, 128>(a, s) : launch_combine<__nv_bfloat16, 64>(a, s);
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
  const bool tc = dtype == CDSL_DTYPE_BF16;
  Sizes z;
  sizes_of(c, tc, n_heads, T, &z);
  if (!ck.aligned(d_workspace, 256) || workspace_bytes < z.bytes)
    return ck.fail("the workspace must be 256-byte aligned and hold cdsl_tree_attention_workspace bytes",
                   workspace_bytes < z.bytes ? CDSL_ENOMEM : CDSL_EINVAL);
  const long long chunks = ((long long)max_len + T + kKeys - 1) / kKeys;
  const long long units = chunks * c.batch * c.kvh * z.QB;   // at most
  if (units >= (1LL << 31)) return ck.fail("the pass is beyond the limit (2^31 chunks of 128 slots)");
  TreeArgs a = {};
  a.c = c;
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
