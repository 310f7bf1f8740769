// tree_verify.cu -- cdsl_tree_verify: which drafted path the target takes, and the next token.
//
// A block per sequence walks its tree. Only the rows on the way are read: at a node the row's
// maximum, the sum of its weights, the children's decisions, and where none is taken the token at
// a position of the weights' running sum. Weights are summed as whole numbers, so that neither the
// decisions nor the token depend on the order of any sum.
#include <cuda.h>

#include <algorithm>

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
    if (a.draft) {
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
  auto k = dtype == CDSL_DTYPE_BF16 ? k_tree_verify<__nv_bfloat16> : k_tree_verify<float>;
  return ck.launched(launch_pdl(k, dim3(batch), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a));
}
