// rope.cu -- cdsl_rope, cdsl_rope_turns: rotary positions.
//
// Pair i of a head's first `rot` dimensions, (a, b), turns by pos * f_i: (a cos - b sin, b cos + a sin). An angle
// in fp32 loses its fraction of a turn at far positions (at 10^6 radians it is off by 0.03), so frequencies are kept
// in turns, as 64-bit fractions of one: pos * turns modulo 2^64 is the fraction exactly, with no range to reduce.
// Its nearest quarter is taken off in whole numbers and the rest, at most an eighth of a turn, goes through sincospif.
//
// Bound by HBM on large calls, where the sines, once for all heads of a token, go beside the loads, and by the launch on
// a decoding step's.
#include <cuda.h>

#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "tree_host.h"

namespace cdsl {
namespace tree {
namespace {

constexpr int kThreads = 256;

struct RopeArgs {
  const uint64_t* turns;
  int half;                            // pairs
  int hd, T, heads[2];                 // of q, k (0: none)
  float magnitude, sign;               // sign: of the sine
  const void* x[2];
  void* y[2];
  long long sx[2][3], sy[2][3];        // strides of sequences, tokens, heads
  const int32_t* start;
  const int32_t* offset;
};

// A pair, turned; written out, so that every variant rounds alike.
__device__ __forceinline__ float2 turn(float p, float q, float2 cs) {
  return make_float2(fmaf(p, cs.x, -__fmul_rn(q, cs.y)), fmaf(q, cs.x, __fmul_rn(p, cs.y)));
}

// V values of a head.
template <typename T, int V> struct alignas(sizeof(T) * V) Values { T x[V]; };

// Grid: (tokens, batch). A thread has V values of a head: both sides of V pairs (halves: V values of each; neighbours: V / 2
// pairs), or V values that are not turned.
template <typename T, int V, bool PAIRS>
__global__ void __launch_bounds__(kThreads) k_rope(RopeArgs a) {
  extern __shared__ float2 s_cs[];             // cosine and sine, times the magnitude
  pdl_wait();
  pdl_launch_dependents();
  const int t = blockIdx.x, b = blockIdx.y;
  const long long pos = (long long)a.start[b] + (a.offset ? a.offset[(size_t)b * a.T + t] : t);
  for (int i = threadIdx.x; i < a.half; i += kThreads) {
    const uint64_t turn = (uint64_t)pos * a.turns[i];
    const uint32_t top = (uint32_t)(turn >> 32);
    const uint32_t quarter = (top + (1u << 29)) >> 30;           // the nearest (4: 0)
    const float rest = (float)(int32_t)(top - (quarter << 30)) * 0x1p-31f;   // of half a turn
    float s, c;
    sincospif(rest, &s, &c);
    const float cs = quarter & 1 ? -s : c, sn = quarter & 1 ? c : s;
    const float flip = quarter & 2 ? -a.magnitude : a.magnitude;
    s_cs[i] = make_float2(cs * flip, sn * flip * a.sign);
  }
  __syncthreads();
  using Vec = Values<T, V>;
  const int turned = PAIRS ? 2 * a.half / V : a.half / V, per = turned + (a.hd - 2 * a.half) / V;   // parts of a head
  const int all = (a.heads[0] + a.heads[1]) * per;
  for (int i = threadIdx.x; i < all; i += kThreads) {
    int h = i / per;
    const int part = i - h * per, w = h >= a.heads[0];
    if (w) h -= a.heads[0];
    const T* const x = static_cast<const T*>(a.x[w]) + b * a.sx[w][0] + t * a.sx[w][1] + h * a.sx[w][2];
    T* const y = static_cast<T*>(a.y[w]) + b * a.sy[w][0] + t * a.sy[w][1] + h * a.sy[w][2];
    if (part >= turned) {
      const int d = 2 * a.half + (part - turned) * V;
      *reinterpret_cast<Vec*>(y + d) = *reinterpret_cast<const Vec*>(x + d);
    } else if constexpr (PAIRS && V > 1) {
      const int d = part * V;
      Vec u = *reinterpret_cast<const Vec*>(x + d);
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 cs = s_cs[(d + e) / 2];
        const float2 z = turn(to_f32<T>(u.x[e]), to_f32<T>(u.x[e + 1]), cs);
        u.x[e] = from_f32<T>(z.x);
        u.x[e + 1] = from_f32<T>(z.y);
      }
      *reinterpret_cast<Vec*>(y + d) = u;
    } else if constexpr (PAIRS) {              // (one value at a time: the thread of a pair's first has both)
      if (part % 2) continue;
      const float2 cs = s_cs[part / 2];
      const float2 z = turn(to_f32<T>(x[part]), to_f32<T>(x[part + 1]), cs);
      y[part] = from_f32<T>(z.x);
      y[part + 1] = from_f32<T>(z.y);
    } else {
      const int d = part * V;
      Vec u = *reinterpret_cast<const Vec*>(x + d), v = *reinterpret_cast<const Vec*>(x + a.half + d);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 cs = s_cs[d + e];
        const float2 z = turn(to_f32<T>(u.x[e]), to_f32<T>(v.x[e]), cs);
        u.x[e] = from_f32<T>(z.x);
        v.x[e] = from_f32<T>(z.y);
      }
      *reinterpret_cast<Vec*>(y + d) = u;
      *reinterpret_cast<Vec*>(y + a.half + d) = v;
    }
  }
}

template <typename T>
cudaError_t launch(const RopeArgs& a, int batch, bool pairs, bool wide, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const auto k = pairs ? (wide ? k_rope<T, V, true> : k_rope<T, 1, true>) : (wide ? k_rope<T, V, false> : k_rope<T, 1, false>);
  return launch_pdl(k, dim3(a.T, batch), dim3(kThreads), a.half * sizeof(float2), s, a);
}

}  // namespace
}  // namespace tree
}  // namespace cdsl

using namespace cdsl;
using namespace cdsl::tree;

extern "C" int32_t cdsl_rope_turns(int32_t rot, double theta, double factor, int32_t original_len, double low, double high,
                                   uint64_t* h_turns) {
  Check ck("cdsl_rope_turns");
  if (!h_turns) return ck.fail("a required pointer is NULL");
  if (rot < 2 || rot % 2 || rot > CDSL_ROPE_MAX_DIM) return ck.fail("rot must be even, 2 .. 1024");
  if (!(theta >= 1.0) || !std::isfinite(theta)) return ck.fail("theta must be finite and 1 at least");
  if (!(factor > 0.0) || !std::isfinite(factor)) return ck.fail("factor must be positive and finite");
  if (factor != 1.0 && (original_len < 1 || !(high > low) || !std::isfinite(low) || !std::isfinite(high)))
    return ck.fail("scaled positions need original_len >= 1 and low < high, finite");
  const double two_pi = 6.283185307179586476925286766559;
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / rot);                  // radians a position
    if (factor != 1.0) {
      const double kept = std::min(1.0, std::max(0.0, (original_len * f / two_pi - low) / (high - low)));
      f = f * kept + f / factor * (1.0 - kept);
    }
    double turn = f / two_pi;
    turn -= std::floor(turn);                                    // (a factor below 1: whole turns say nothing)
    const double scaled = std::ldexp(turn, 64);
    h_turns[i] = scaled >= 18446744073709551615.0 ? 0 : (uint64_t)scaled;
  }
  return CDSL_OK;
}

extern "C" int32_t cdsl_rope(const uint64_t* d_turns, int32_t rot, int32_t interleaved, int32_t inverse, float magnitude,
                             int32_t dtype, int32_t batch, int32_t T, int32_t head_dim, const void* d_q, void* d_q_out,
                             int32_t n_heads, const void* d_k, void* d_k_out, int32_t n_kv_heads, const int64_t* h_strides,
                             const int32_t* d_start, const int32_t* d_offset, void* stream) {
  Check ck("cdsl_rope");
  if (!ck.value_type(dtype)) return CDSL_EINVAL;
  if (!d_turns || !d_q || !d_q_out || !h_strides || !d_start) return ck.fail("a required pointer is NULL");
  if (!d_k != !d_k_out) return ck.fail("k and k's output go together");
  if (head_dim < 2 || head_dim > CDSL_ROPE_MAX_DIM) return ck.fail("head_dim must be 2 .. 1024");
  if (rot < 2 || rot % 2 || rot > head_dim) return ck.fail("rot must be even, 2 .. head_dim");
  if (batch < 1 || batch > 65535 || T < 1 || n_heads < 1 || n_heads > (1 << 16) || (d_k && (n_kv_heads < 1 || n_kv_heads > (1 << 16))))
    return ck.fail("sizes: need 1 <= batch <= 65535, T >= 1, 1 .. 65536 heads");
  if (!(magnitude > 0.f) || !std::isfinite(magnitude)) return ck.fail("magnitude must be positive and finite");
  const int eb = dtype == CDSL_DTYPE_BF16 ? 2 : 4, V = 16 / eb;
  RopeArgs a = {};
  a.turns = d_turns;
  a.half = rot / 2;
  a.hd = head_dim;
  a.T = T;
  a.heads[0] = n_heads;
  a.heads[1] = d_k ? n_kv_heads : 0;
  a.magnitude = magnitude;
  a.sign = inverse ? -1.f : 1.f;
  a.x[0] = d_q; a.x[1] = d_k;
  a.y[0] = d_q_out; a.y[1] = d_k_out;
  a.start = d_start;
  a.offset = d_offset;
  // 16 bytes at a time where every part of a head begins at a multiple of them
  bool wide = (interleaved ? rot : a.half) % V == 0 && (head_dim - rot) % V == 0;
  for (int w = 0; w < (d_k ? 2 : 1); ++w) {
    if (!ck.aligned(a.x[w], eb) || !ck.aligned(a.y[w], eb)) return ck.fail("tensors must be aligned to their type");
    wide = wide && ck.aligned(a.x[w], 16) && ck.aligned(a.y[w], 16);
    for (int i = 0; i < 3; ++i) {
      a.sx[w][i] = h_strides[6 * w + i];
      a.sy[w][i] = h_strides[6 * w + 3 + i];
      if (a.sx[w][i] % V || a.sy[w][i] % V) wide = false;
    }
    const long long* const so = a.sy[w];
    if ((batch > 1 && so[0] == 0) || (T > 1 && so[1] == 0) || (a.heads[w] > 1 && so[2] == 0))
      return ck.fail("an output must not have a stride of 0 between sequences, tokens or heads");
    if (a.x[w] == a.y[w] && !std::equal(a.sx[w], a.sx[w] + 3, a.sy[w]))
      return ck.fail("an output in its input's place must have its strides");
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return ck.launched(dtype == CDSL_DTYPE_BF16 ? launch<__nv_bfloat16>(a, batch, interleaved, wide, s)
                                              : launch<float>(a, batch, interleaved, wide, s));
}
