// tree_verify.cu -- cdsl_tree_verify: which drafted path the target takes, and the next token.
//
// Only the rows on the way are read. At a node: the row's maximum, the sum of its weights, the children's
// decisions, and where none is taken the token at a position of the weights' running sum. Weights are summed as
// whole numbers, so that neither the decisions nor the token depend on the order of any sum.
//
// k_tree_walk: a cluster of up to eight blocks walks a sequence's tree, each with its part of the row in registers
// (J values a thread, 16 bytes a load where rows are aligned). A reduction is one cluster barrier: each warp's value
// goes to every block's shared memory, where each warp reduces all of them for itself; the children's decisions are
// then made alike by every thread. Bound by latency and, with drafts, by the exponentials: a level of 32,000 bf16
// tokens with drafts in four blocks is 12,000 cycles (loads 3,400, exponentials 2,900, two reductions of 1,500 each,
// the decisions 1,600 and more with rejections). 32 sequences of 49 sampled nodes, the longest path 8: 47 us; one of
// 17 chosen nodes, fp32: 10 us. (A value a load, and keys of 64 bits in the maximum: 18,500 cycles a level, 82 us.) A
// block of more than 8,192 tokens has up to 40 values a thread, which do not fit its 128 registers (350 bytes of stack): 64
// sequences of 16 nodes and 32,000 tokens with drafts, two blocks each, 109 us, 32 sequences 33; 8 of 17 and 128,256 tokens 81. Rows
// of more than the cluster's registers hold (163,840 tokens) take k_tree_verify, a block per sequence that
// reads a row several times: one sequence of 262,144 tokens, a root without a taken child, 301 us, of 163,840 tokens 14.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "tc_ptx.cuh"
#include "tree_host.h"

namespace cdsl {
namespace tree {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxT = CDSL_TREE_MAX_NODES;
constexpr float kTwo31 = 2147483648.f;
typedef unsigned long long u64;

struct VerifyArgs {
  int T, V;
  const void* logits;
  const void* draft;
  long long sl[2], sd[2];
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* nodes;
  const float* u;
  const float* u_last;
  float inv_t;                         // 0: greedy
  int32_t* path;
  int32_t* n_path;
  int32_t* emitted;
  int32_t* status;
};

// floor(2^31 x), 0 <= x <= 1
__device__ __forceinline__ uint32_t units_of(float x) { return __float2uint_rz(x * kTwo31); }
// floor(k Z / 2^24), k = floor(2^24 u)
__device__ __forceinline__ u64 share_of(float u, u64 Z) {
  const u64 k = (u64)__float2uint_rz(fminf(fmaxf(u, 0.f), 0.99999994f) * 16777216.f);
  return k * (Z >> 24) + (k * (Z & 0xffffffull) >> 24);
}

template <typename T>
struct Row {                           // exp((l_v - top) / temperature)
  const T* p;
  float top, inv_t;
  __device__ __forceinline__ float logit(int v) const { return to_f32<T>(p[v]); }
  __device__ __forceinline__ float weight(int v) const { return expf(__fmul_rn(__fsub_rn(logit(v), top), inv_t)); }
};

__device__ __forceinline__ u64 block_sum(u64 x, u64* s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  u64 t = 0;
  for (int w = 0; w < kWarps; ++w) t += s[w];
  return t;
}

// Largest logit of a row and its lowest index; bad: a NaN, +inf or nothing finite.
template <typename T>
__device__ u64 row_max(const T* p, int V, u64* s, bool* bad) {
  u64 best = 0;
  bool nan = false;
  for (int v = threadIdx.x; v < V; v += kThreads) {
    const float x = to_f32<T>(p[v]);
    if (!(x < INFINITY)) nan = true;
    else if (x > -INFINITY) best = max(best, argmax_key(x + 0.f, v));
  }
  best = warp_max_u64(best);
  *bad = __syncthreads_or(nan) != 0;
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = best;
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) best = max(best, s[w]);
  __syncthreads();
  if (best == 0) *bad = true;
  return best;
}
__device__ __forceinline__ float key_value(u64 key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_tree_verify(VerifyArgs a) {
  __shared__ u64 s_red[kWarps];
  __shared__ int s_tok[kMaxT], s_par[kMaxT];
  __shared__ float s_inv[kMaxT];       // of the distributions after each rejection
  __shared__ int s_out[kMaxT];         // tokens that left the distribution
  __shared__ int s_last;
  const int b = blockIdx.x, tid = threadIdx.x, V = a.V;
  pdl_wait();
  pdl_launch_dependents();
  const int n = a.nodes ? min(max(a.nodes[b], 0), a.T) : a.T;
  for (int i = tid; i < a.T; i += kThreads) {
    s_tok[i] = a.tokens[(size_t)b * a.T + i];
    s_par[i] = a.parents[(size_t)b * a.T + i];
    a.path[(size_t)b * a.T + i] = a.emitted[(size_t)b * a.T + i] = -1;
  }
  __syncthreads();
  if (n == 0) {
    if (tid == 0) a.n_path[b] = 0;
    return;
  }
  int cur = 0, m = 0, last = -1;
  for (;;) {
    if (tid == 0) {
      a.path[(size_t)b * a.T + m] = cur;
      if (m) a.emitted[(size_t)b * a.T + m - 1] = s_tok[cur];
    }
    ++m;
    bool bad;
    Row<T> p = {static_cast<const T*>(a.logits) + b * a.sl[0] + cur * a.sl[1], 0.f, a.inv_t};
    const u64 best = row_max(p.p, V, s_red, &bad);
    if (bad) {
      if (tid == 0) set_status(a.status, CDSL_ENONFINITE);
      last = -1;                       // (greedy: not the row's before)
      break;
    }
    p.top = key_value(best);
    int next = -1;
    if (a.inv_t == 0.f) {
      last = argmax_key_index(best);
      for (int i = cur + 1; i < n && next < 0; ++i) {
        if (s_par[i] != cur) continue;
        if (s_tok[i] == last) next = i;
        else if ((unsigned)s_tok[i] >= (unsigned)V && tid == 0) set_status(a.status, CDSL_ERANGE);
      }
      if (next < 0) break;
      cur = next;
      continue;
    }
    u64 z = 0;
    for (int v = tid; v < V; v += kThreads) z += units_of(p.weight(v));
    u64 Z = block_sum(z, s_red);
    const float inv0 = __fdiv_rn(1.f, __fmul_rn(__ull2float_rn(Z), 1.f / kTwo31));
    Row<T> q = {nullptr, 0.f, a.inv_t};
    float invq = 0.f;
    bool kids = false;                 // (nothing was sampled from the draft's row of a leaf)
    for (int i = cur + 1; i < n; ++i) kids = kids || s_par[i] == cur;
    if (a.draft && kids) {
      q.p = static_cast<const T*>(a.draft) + b * a.sd[0] + cur * a.sd[1];
      q.top = key_value(row_max(q.p, V, s_red, &bad));
      if (bad) {
        if (tid == 0) set_status(a.status, CDSL_ENONFINITE);
        break;
      }
      u64 zq = 0;
      for (int v = tid; v < V; v += kThreads) zq += units_of(q.weight(v));
      invq = __fdiv_rn(1.f, __fmul_rn(__ull2float_rn(block_sum(zq, s_red)), 1.f / kTwo31));
    }
    int rejected = 0;                  // entries of s_out / s_inv
    // the distribution after `rounds` rejections, the last one's normalisation done or not
    auto residual = [&](int v, int rounds, bool normalised) {
      float x = __fmul_rn(p.weight(v), inv0);
      const float y = __fmul_rn(q.weight(v), invq);
      for (int r = 0; r < rounds; ++r) {
        x = fmaxf(__fsub_rn(x, y), 0.f);
        if (normalised || r + 1 < rounds) x = __fmul_rn(x, s_inv[r]);
      }
      return x;
    };
    auto unit = [&](int v) -> uint32_t {
      if (a.draft && rejected) return units_of(residual(v, rejected, false));
      const uint32_t w = units_of(p.weight(v));
      if (!a.draft)
        for (int r = 0; r < rejected; ++r)
          if (s_out[r] == v) return 0u;
      return w;
    };
    for (int i = cur + 1; i < n && next < 0; ++i) {
      if (s_par[i] != cur) continue;
      const int x = s_tok[i];
      if ((unsigned)x >= (unsigned)V) {
        if (tid == 0) set_status(a.status, CDSL_ERANGE);
        continue;
      }
      const float u = a.u[(size_t)b * a.T + i];
      if (!a.draft) {
        const uint32_t w = unit(x);
        if (share_of(u, Z) < w) { next = i; break; }
        Z -= w;
        __syncthreads();
        if (tid == 0) s_out[rejected] = x;
        ++rejected;
        __syncthreads();
      } else {
        if (__fmul_rn(u, __fmul_rn(q.weight(x), invq)) < residual(x, rejected, true)) { next = i; break; }
        u64 zr = 0;
        for (int v = tid; v < V; v += kThreads) zr += units_of(residual(v, rejected + 1, false));
        zr = block_sum(zr, s_red);
        if (zr) {
          Z = zr;
          if (tid == 0) s_inv[rejected] = __fdiv_rn(1.f, __fmul_rn(__ull2float_rn(zr), 1.f / kTwo31));
          ++rejected;
          __syncthreads();
        }
      }
    }
    if (next >= 0) {
      cur = next;
      continue;
    }
    // ---- the first token whose running sum passes the draw: block-wide sums of kThreads tokens
    const u64 want = share_of(a.u_last[b], Z);
    if (tid == 0) s_last = -1;
    u64 before = 0;
    for (int v0 = 0; v0 < V; v0 += kThreads) {
      const u64 w = v0 + tid < V ? unit(v0 + tid) : 0u;
      u64 scan = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, scan, o);
        if ((tid & 31) >= o) scan += t;
      }
      __syncthreads();
      if ((tid & 31) == 31) s_red[tid >> 5] = scan;
      __syncthreads();
      u64 all = 0;
      for (int q2 = 0; q2 < kWarps; ++q2) {
        if (q2 == (tid >> 5)) scan += all;
        all += s_red[q2];
      }
      if (before + scan > want && before + scan - w <= want) s_last = v0 + tid;
      before += all;
      if (before > want) break;
    }
    __syncthreads();
    last = s_last;
    break;
  }
  if (tid == 0) {
    a.n_path[b] = m;
    a.emitted[(size_t)b * a.T + m - 1] = last;
  }
}


// ------------------------------------------------------------------------------------- the walk in registers
constexpr int kWalk = 512;             // threads of a block
constexpr int kWalkWarps = kWalk / 32;
constexpr int kMaxCluster = 8;
constexpr int kPrefetch = 4;           // children whose rows are fetched into L2 ahead

// Values of all warps of the cluster, two at a time, two reductions' in turn.
struct Slots {
  u64 v[2][2][kMaxCluster * kWalkWarps];
};

// Over a warp, in two 32-bit reductions each. Sums: of 2^51 at most a lane.
__device__ __forceinline__ u64 warp_sum(u64 x) {
  const uint32_t lo = __reduce_add_sync(0xffffffffu, (uint32_t)x & 0xffffffu);
  return ((u64)__reduce_add_sync(0xffffffffu, (uint32_t)(x >> 24)) << 24) + lo;
}
__device__ __forceinline__ u64 warp_most(u64 x) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(x >> 32));
  return (u64)hi << 32 | __reduce_max_sync(0xffffffffu, (uint32_t)(x >> 32) == hi ? (uint32_t)x : 0u);
}

// a and b of every thread of the cluster, their sums or their maxima; C: blocks. One cluster barrier. Afterwards
// s.v[turn][.] holds the warps' values, block by block.
template <bool Sum>
__device__ __forceinline__ void reduce_cluster(u64& a, u64& b, bool both, Slots& s, int& turn, int C, int rank) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const auto over_warp = [](u64 x) { return Sum ? warp_sum(x) : warp_most(x); };
  a = over_warp(a);
  if (both) b = over_warp(b);
  turn ^= 1;
  const int at = rank * kWalkWarps + warp;
  if (C > 1) {
    if (lane < C) {
      const uint32_t to = tc::map_cluster_rank(tc::smem_u32(&s.v[turn][0][at]), lane);
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(a) : "memory");
      if (both)
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to + (uint32_t)sizeof(s.v[0][0])), "l"(b) : "memory");
    }
    tc::cluster_arrive();
    tc::cluster_wait();
  } else {
    if (lane == 0) {
      s.v[turn][0][at] = a;
      if (both) s.v[turn][1][at] = b;
    }
    __syncthreads();
  }
  a = b = 0;                           // (neutral to both operations: keys and sums are not negative)
  for (int i = lane; i < C * kWalkWarps; i += 32) {
    const u64 x = s.v[turn][0][i], y = both ? s.v[turn][1][i] : 0;
    a = Sum ? a + x : max(a, x);
    b = Sum ? b + y : max(b, y);
  }
  a = over_warp(a);
  if (both) b = over_warp(b);
}

// E values from p, in one load.
template <int E, typename T>
__device__ __forceinline__ void load_values(const T* p, float* out) {
  if constexpr (E == 1) {
    out[0] = to_f32<T>(*p);
  } else {
    using Bits = std::conditional_t<E * sizeof(T) == 16, uint4, uint2>;
    const Bits x = *reinterpret_cast<const Bits*>(p);
    const T* const v = reinterpret_cast<const T*>(&x);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = to_f32<T>(v[e]);
  }
}

// J values a thread, E of them next to one another: value k is token (k / E * kWalk + tid) * E + k % E of the block's.
template <typename T, int J, int E>
__global__ void __launch_bounds__(kWalk) k_tree_walk(VerifyArgs a) {
  __shared__ Slots s_slots;
  __shared__ int s_tok[kMaxT];
  __shared__ uint32_t s_child[kMaxT][kMaxT / 32];   // a node's children, by bits
  __shared__ float s_u[kMaxT];
  __shared__ float s_lx[kMaxT], s_qx[kMaxT];   // a node's children's logits, the target's and the draft's
  __shared__ float s_inv[kMaxT];
  constexpr int kSums = J / E * kWalkWarps;
  __shared__ u64 s_sum[kSums];                 // a block's weights by 32 E tokens, in their order
  __shared__ int s_at;
  __shared__ u64 s_before;
  const int C = (int)gridDim.x, rank = (int)blockIdx.x, b = blockIdx.y, tid = threadIdx.x, V = a.V;
  const int lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const int n = a.nodes ? min(max(a.nodes[b], 0), a.T) : a.T;
  if (C > 1) tc::cluster_arrive();     // (before any store to another block's memory: that all have started)
  for (int i = tid; i < kMaxT * kMaxT / 32; i += kWalk) s_child[0][i] = 0u;
  __syncthreads();
  for (int i = tid; i < a.T; i += kWalk) {
    const int parent = a.parents[(size_t)b * a.T + i];
    if (i > 0 && i < n && parent >= 0 && parent < i) atomicOr(&s_child[parent][i >> 5], 1u << (i & 31));
    s_tok[i] = a.tokens[(size_t)b * a.T + i];
    if (a.inv_t != 0.f) s_u[i] = a.u[(size_t)b * a.T + i];
    if (rank == 0) a.path[(size_t)b * a.T + i] = a.emitted[(size_t)b * a.T + i] = -1;
  }
  const float u_last = a.inv_t != 0.f ? a.u_last[b] : 0.f;
  const bool greedy = a.inv_t == 0.f, given = a.draft != nullptr;
  const int size = ((V + C - 1) / C + E - 1) / E * E, base = rank * size, top = min(V, base + size);   // this block's tokens
  int turn = 0;
  if (C > 1) tc::cluster_wait();
  __syncthreads();
  if (n == 0) {
    if (rank == 0 && tid == 0) a.n_path[b] = 0;
    return;
  }
  const T* const rows = static_cast<const T*>(a.logits) + b * a.sl[0];
  const T* const draft_rows = static_cast<const T*>(a.draft) + b * a.sd[0];
  auto weight = [&](float l, float m) { return expf(__fmul_rn(__fsub_rn(l, m), a.inv_t)); };
  auto inverse = [](u64 Z) { return __fdiv_rn(1.f, __fmul_rn(__ull2float_rn(Z), 1.f / kTwo31)); };
  int cur = 0, m = 0, last = -1;
  const auto child = [&](int i) {      // the node's first child after i, kMaxT: none
    for (++i; i < kMaxT; i = (i | 31) + 1)
      if (const uint32_t x = s_child[cur][i >> 5] >> (i & 31)) return i + __ffs(x) - 1;
    return kMaxT;
  };
  for (;;) {
    if (rank == 0 && tid == 0) {
      a.path[(size_t)b * a.T + m] = cur;
      if (m) a.emitted[(size_t)b * a.T + m - 1] = s_tok[cur];
    }
    ++m;
    bool drafts = false;               // (nothing was sampled from the draft's row of a leaf)
    if (given) drafts = (s_child[cur][0] | s_child[cur][1] | s_child[cur][2] | s_child[cur][3]) != 0u;
    // ---- the row, the children's logits, and the likely next rows into L2
    float l[J], q[J];
    const T* const row = rows + cur * a.sl[1];
    const T* const draft_row = draft_rows + cur * a.sd[1];
    const auto load = [&](const T* from, float (&x)[J]) {
#pragma unroll
      for (int j = 0; j < J; j += E) {
        const int v = base + (j / E * kWalk + tid) * E;
        if (v + E <= top) {
          load_values<E>(from + v, x + j);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) x[j + e] = v + e < top ? to_f32<T>(from[v + e]) : -INFINITY;
        }
      }
    };
    load(row, l);
    if (drafts) load(draft_row, q);
    if (tid < n && s_child[cur][tid >> 5] >> (tid & 31) & 1 && (unsigned)s_tok[tid] < (unsigned)V) {
      s_lx[tid] = to_f32<T>(row[s_tok[tid]]);
      if (drafts) s_qx[tid] = to_f32<T>(draft_row[s_tok[tid]]);
    }
    for (int i = child(cur), ahead = 0; i < kMaxT && ahead < kPrefetch; i = child(i), ++ahead) {
      constexpr int kLine = 128 / sizeof(T);
      for (int v = base + tid * kLine; v < top; v += kWalk * kLine) {
        asm volatile("prefetch.global.L2 [%0];" ::"l"(rows + i * a.sl[1] + v));
        if (drafts) asm volatile("prefetch.global.L2 [%0];" ::"l"(draft_rows + i * a.sd[1] + v));
      }
    }
    // ---- maxima (all ones: a row that cannot be drawn from)
    const auto most = [&](const float (&x)[J]) {
      float m = -INFINITY;
      int k = 0;
      bool bad = false;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        bad |= !(x[j] < INFINITY);
        k = x[j] > m ? j : k;
        m = fmaxf(x[j], m);
      }
      return bad ? ~0ull : m > -INFINITY ? argmax_key(m + 0.f, base + (k / E * kWalk + tid) * E + k % E) : 0ull;
    };
    u64 best = most(l), best_q = drafts ? most(q) : 0ull;
    reduce_cluster<false>(best, best_q, drafts, s_slots, turn, C, rank);
    if (best == 0 || best == ~0ull || (drafts && (best_q == 0 || best_q == ~0ull))) {
      if (rank == 0 && tid == 0) set_status(a.status, CDSL_ENONFINITE);
      last = -1;                       // (greedy: not the row's before)
      break;
    }
    int next = -1;
    if (greedy) {
      last = argmax_key_index(best);
      for (int i = child(cur); i < kMaxT && next < 0; i = child(i)) {
        if (s_tok[i] == last) next = i;
        else if ((unsigned)s_tok[i] >= (unsigned)V && tid == 0) set_status(a.status, CDSL_ERANGE);
      }
      if (next < 0) break;
      cur = next;
      __syncthreads();                 // (s_lx of the next node)
      continue;
    }
    // ---- weights, as whole numbers and their sums
    const float lm = key_value(best), qm = key_value(best_q);
    uint32_t W[J];
    u64 Z = 0, Zq = 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      l[j] = weight(l[j], lm);
      W[j] = units_of(l[j]);
      Z += W[j];
      if (drafts) {
        q[j] = weight(q[j], qm);
        Zq += units_of(q[j]);
      }
    }
    reduce_cluster<true>(Z, Zq, drafts, s_slots, turn, C, rank);
    float inv0 = 0.f, invq = 0.f;
    if (drafts) {                      // the distributions p and q
      inv0 = inverse(Z);
      invq = inverse(Zq);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        l[j] = __fmul_rn(l[j], inv0);
        q[j] = __fmul_rn(q[j], invq);
      }
    }
    int rejected = 0;
    bool changed = false;              // the weights are no longer those of the last reduction
    for (int i = child(cur); i < kMaxT && next < 0; i = child(i)) {
      const int x = s_tok[i];
      if ((unsigned)x >= (unsigned)V) {
        if (rank == 0 && tid == 0) set_status(a.status, CDSL_ERANGE);
        continue;
      }
      if (!drafts) {
        uint32_t w = units_of(weight(s_lx[i], lm));
        for (int r = child(cur); r < i; r = child(r))   // (a sibling's token has left the distribution)
          if (s_tok[r] == x) w = 0;
        if (share_of(s_u[i], Z) < w) { next = i; break; }
        Z -= w;
        changed = true;
        const int at = x - base;       // it leaves the distribution
        if (x >= base && x < top && at / E % kWalk == tid)
#pragma unroll
          for (int j = 0; j < J; ++j)
            if (j == at / E / kWalk * E + at % E) W[j] = 0;
      } else {
        const float qx = __fmul_rn(weight(s_qx[i], qm), invq);
        float px = __fmul_rn(weight(s_lx[i], lm), inv0);
        for (int r = 0; r < rejected; ++r) px = __fmul_rn(fmaxf(__fsub_rn(px, qx), 0.f), s_inv[r]);
        if (__fmul_rn(s_u[i], qx) < px) { next = i; break; }
        // the rest of p: it stays p where that is nothing
        u64 zr = 0, none = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) zr += units_of(fmaxf(__fsub_rn(l[j], q[j]), 0.f));
        reduce_cluster<true>(zr, none, false, s_slots, turn, C, rank);
        if (zr) {
          const float inv = inverse(zr);
          Z = zr;
          changed = false;
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const float r = fmaxf(__fsub_rn(l[j], q[j]), 0.f);
            W[j] = units_of(r);
            l[j] = __fmul_rn(r, inv);
          }
          if (tid == 0) s_inv[rejected] = inv;
          ++rejected;
          __syncthreads();
        } else {
          changed = true;
        }
      }
    }
    if (next >= 0) {
      cur = next;
      __syncthreads();                 // (s_lx and s_inv of the next node)
      continue;
    }
    // ---- the first token whose running sum passes the draw: the block, the 32 tokens, the token
    if (changed) {
      u64 z = 0, none = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) z += W[j];
      reduce_cluster<true>(z, none, false, s_slots, turn, C, rank);
    }
    u64 before = 0, mine = 0;
    for (int i = lane; i < (rank + 1) * kWalkWarps; i += 32)
      (i < rank * kWalkWarps ? before : mine) += s_slots.v[turn][0][i];
    mine = warp_sum(mine);
    const u64 want = share_of(u_last, Z) - warp_sum(before);   // (wraps past 0: not this block's)
    if ((long long)want < 0 || want >= mine) return;
#pragma unroll
    for (int j = 0; j < J; j += E) {
      u64 z = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) z += W[j + e];
      z = warp_sum(z);
      if (lane == 0) s_sum[j / E * kWalkWarps + warp] = z;
    }
    __syncthreads();
    const auto scan = [&](u64 x) {     // the sum of the lanes' up to this one
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 t = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += t;
      }
      return x;
    };
    if (warp == 0) {                   // a few sums a lane, in order
      constexpr int PER = (kSums + 31) / 32;
      u64 own = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) own += lane * PER + i < kSums ? s_sum[lane * PER + i] : 0;
      const u64 upto = scan(own);
      u64 at = upto - own;
      if (upto > want && at <= want) {
        int i = lane * PER;
        while (at + s_sum[i] <= want) at += s_sum[i++];
        s_at = i;
        s_before = at;
      }
    }
    __syncthreads();
    if (warp == s_at % kWalkWarps) {
      const int jj = s_at / kWalkWarps;
      uint32_t w[E];
      u64 own = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        w[e] = 0;
#pragma unroll
        for (int j = 0; j < J; j += E)
          if (j / E == jj) w[e] = W[j + e];
        own += w[e];
      }
      u64 upto = scan(own) + s_before, at = upto - own;
      if (upto > want && at <= want) {
        int v = base + (jj * kWalk + tid) * E;
#pragma unroll
        for (int e = 0; e < E - 1; ++e)
          if ((at += w[e]) <= want) ++v;
          else at = upto;
        a.n_path[b] = m;
        a.emitted[(size_t)b * a.T + m - 1] = v;
      }
    }
    return;
  }
  if (rank == 0 && tid == 0) {
    a.n_path[b] = m;
    a.emitted[(size_t)b * a.T + m - 1] = last;
  }
}

template <typename T>
cudaError_t launch_verify(const VerifyArgs& a, int batch, cudaStream_t s) {
  // As many blocks to a sequence as leave every SM at most one, while a thread has two values to hold at
  // least; more where the row does not fit otherwise.
  int C = 1;
  while (C < kMaxCluster && ((2 * C * batch <= kPlanSMs && 8 * C * kWalk <= 2 * a.V) || a.V > C * kWalk * 40)) C *= 2;
  const int J = ((a.V + C - 1) / C + kWalk - 1) / kWalk;
  const dim3 grid(C, batch), block(kWalk);
  auto go = [&](auto k) {
    return C == 1 ? launch_pdl(k, grid, block, 0, s, a) : launch_pdl_cluster(k, grid, block, 0, C, s, a);
  };
  // 16 bytes a load where every row starts at 16
  constexpr int E = 16 / sizeof(T);
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.draft)) % 16 == 0 &&
                   (a.sl[0] | a.sl[1] | (a.draft ? a.sd[0] | a.sd[1] : 0)) % E == 0;
  if (J <= 4) return vec ? go(k_tree_walk<T, 4, 4>) : go(k_tree_walk<T, 4, 1>);
  if (J <= 8) return vec ? go(k_tree_walk<T, 8, E>) : go(k_tree_walk<T, 8, 1>);
  if (J <= 16) return vec ? go(k_tree_walk<T, 16, E>) : go(k_tree_walk<T, 16, 1>);
  if (J <= 40) return vec ? go(k_tree_walk<T, 40, E>) : go(k_tree_walk<T, 40, 1>);
  return launch_pdl(k_tree_verify<T>, dim3(batch), dim3(kThreads), 0, s, a);
}

}  // namespace
}  // namespace tree
}  // namespace cdsl

using namespace cdsl;
using namespace cdsl::tree;

extern "C" int32_t cdsl_tree_verify(int32_t batch, int32_t T, int32_t vocab, const void* d_logits,
                                    const void* d_draft_logits, int32_t dtype, const int64_t* h_strides,
                                    const int32_t* d_tokens, const int32_t* d_parents,
                                    const int32_t* d_nodes, const float* d_u, const float* d_u_last,
                                    float temperature, int32_t* d_path, int32_t* d_n_path,
                                    int32_t* d_emitted, int32_t* d_status, void* stream) {
  Check ck("cdsl_tree_verify");
  if (batch < 1 || batch > CDSL_TREE_MAX_BATCH || T < 1 || T > CDSL_TREE_MAX_NODES || vocab < 1 ||
      vocab > CDSL_TREE_MAX_VOCAB)
    return ck.fail("sizes: need 1 <= batch <= 1024, 1 <= T <= 128, 1 <= vocab <= 2^20");
  if (!ck.value_type(dtype)) return CDSL_EINVAL;
  if (!d_logits || !h_strides || !d_tokens || !d_parents || !d_u || !d_u_last || !d_path || !d_n_path ||
      !d_emitted)
    return ck.fail("a required pointer is NULL");
  if (!(temperature >= 0.f) || temperature > 1e30f || (temperature > 0.f && temperature < 1e-30f))
    return ck.fail("temperature must be 0, or positive and finite");
  const int eb = dtype == CDSL_DTYPE_BF16 ? 2 : 4;
  if (!ck.aligned(d_logits, eb) || !ck.aligned(d_draft_logits, eb))
    return ck.fail("logits must be aligned to their type");
  VerifyArgs a = {T, vocab, d_logits, temperature > 0.f ? d_draft_logits : nullptr,
                  {h_strides[0], h_strides[1]}, {h_strides[2], h_strides[3]}, d_tokens, d_parents, d_nodes,
                  d_u, d_u_last, temperature > 0.f ? 1.f / temperature : 0.f, d_path, d_n_path, d_emitted,
                  d_status};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return ck.launched(dtype == CDSL_DTYPE_BF16 ? launch_verify<__nv_bfloat16>(a, batch, s)
                                              : launch_verify<float>(a, batch, s));
}
