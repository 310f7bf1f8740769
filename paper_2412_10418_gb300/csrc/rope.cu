// rope.cu -- cdsl_rope, cdsl_rope_turns: rotary positions.
//
// Pair i of a head's first `rot` dimensions, (a, b), turns by pos * f_i: (a cos - b sin, b cos + a sin). An angle
// in fp32 loses its fraction of a turn at far positions (at 10^6 radians it is off by 0.03), so frequencies are kept
// in turns, as 64-bit fractions of one: pos * turns modulo 2^64 is the fraction exactly, with no range to reduce.
// Its nearest quarter is taken off in whole numbers and the rest, at most an eighth of a turn, goes through sincospif.
//
// Bound by HBM on large calls and by the launch on a decoding step's: 4 x 4093 tokens of 48 heads of 128 in bf16, 96 of them
// turned, and their gradients (two calls, 805 MB): 128 us as neighbours, 93 % of the copy bandwidth; halves of whole heads 137, 87 %;
// one token 2.4 us in a graph. What counts there is instructions, of which 16 bytes have room for some fifty: a token by a
// block, with the sines through shared memory and each address worked out, took 167 us; heads' addresses worked out in a
// warp's loop 235; blocks of 256 threads 150; eight heads loaded together 179; halves by 16 bytes of each side, with as
// many angles in registers, 240.
#include <cuda.h>

#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "tree_host.h"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {

constexpr int kHalves = 4;                     // values of each side (8 of bf16 are as many angles, and take their registers)
constexpr int kThreads = 128, kBlocks = 6;     // of an SM, by registers

struct RopeArgs {
  const uint64_t* turns;
  int half;                            // pairs
  int hd, batch, T, heads[2];          // of q, k (0: none)
  int slices;
  float magnitude, sign;               // sign: of the sine
  const void* x[2];
  void* y[2];
  long long sx[2][3], sy[2][3];        // strides of sequences, tokens, heads
  const int32_t* start;
  const int32_t* offset;
};

// Pairs (p, q), turned, by twos: the products of every variant are these, so that all round alike.
__device__ __forceinline__ void turn(uint64_t& p, uint64_t& q, uint64_t cos2, uint64_t sin2, uint64_t minus2) {
  const uint64_t z = fma2(p, cos2, mul2(q, minus2));
  q = fma2(q, cos2, mul2(p, sin2));
  p = z;
}

// V values of a head.
template <typename T, int V> struct alignas(sizeof(T) * V) Values { T x[V]; };

// A warp has a token's heads, or a share of them: `slices` warps a token. A lane has the same part of every head it
// turns, V values (halves: V of both sides; neighbours: V / 2 pairs, of single values a pair) or V that are not turned, so
// that it needs its sines once, in registers; a head's parts are side by side in the lanes, several heads' where a head
// has fewer than 32. Four heads are loaded together.
template <typename T, int V, bool PAIRS>
__global__ void __launch_bounds__(kThreads, kBlocks) k_rope(const __grid_constant__ RopeArgs a) {
  constexpr int STEP = PAIRS && V == 1 ? 2 : V;          // values of a turned part's first side
  constexpr int ANGLES = PAIRS ? STEP / 2 : V;
  constexpr int AHEAD = 4;
  using Vec = Values<T, STEP>;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long warp = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const long long token = warp / a.slices;
  if (token >= (long long)a.batch * a.T) return;
  const int slice = (int)(warp % a.slices), b = (int)(token / a.T), t = (int)(token % a.T);
  // parts of a head (halves: what is not turned goes by two sides as well, of which the second may be one shorter)
  const int turned = PAIRS ? 2 * a.half / STEP : a.half / V, rest = a.hd - 2 * a.half, side = PAIRS ? 0 : (rest + 1) / 2;
  const int per = turned + (PAIRS ? rest : side) / V;
  const int together = max(1, 32 / per), sub = per < 32 ? lane / per : 0;   // heads that a warp has at once
  const int heads = a.heads[0] + a.heads[1], share = (heads + a.slices - 1) / a.slices;
  const int end = min(heads, (slice + 1) * share);
  const long long pos = (long long)a.start[b] + (a.offset ? a.offset[(size_t)b * a.T + t] : t);
#pragma unroll 1
  for (int p0 = 0; p0 < per; p0 += 32) {
    const int part = per < 32 ? lane % per : p0 + lane;
    if (part >= per || sub >= together) continue;
    const bool turns = part < turned;
    const int d = turns ? part * STEP : 2 * a.half + (part - turned) * V;   // the part's first value
    const int other = turns ? a.half : side;   // halves: the second side, from the first
    const bool both = !PAIRS && (turns || d + side + V <= a.hd);
    float2 cs[ANGLES];
    if (turns) {
#pragma unroll
      for (int i = 0; i < ANGLES; ++i) {
        const uint64_t turn = (uint64_t)pos * a.turns[PAIRS ? d / 2 + i : d + i];
        const uint32_t top = (uint32_t)(turn >> 32);
        const uint32_t quarter = (top + (1u << 29)) >> 30;           // the nearest (4: 0)
        const float rest = (float)(int32_t)(top - (quarter << 30)) * 0x1p-31f;   // of half a turn
        float s, c;
        if constexpr (sizeof(T) == 2) __sincosf(rest * 3.14159265f, &s, &c);   // (off by 2^-21: bf16's rounding is 2^-9)
        else sincospif(rest, &s, &c);
        const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
        const float flip = quarter & 2 ? -a.magnitude : a.magnitude;
        cs[i] = make_float2(x * flip, y * flip * a.sign);
      }
    }
    uint64_t c2[(ANGLES + 1) / 2], s2[(ANGLES + 1) / 2], m2[(ANGLES + 1) / 2];   // of two angles
#pragma unroll
    for (int i = 0; i < (ANGLES + 1) / 2; ++i) {
      const float2 x = cs[2 * i], y = cs[min(2 * i + 1, ANGLES - 1)];
      c2[i] = pair(x.x, y.x);
      s2[i] = pair(x.y, y.y);
      m2[i] = pair(-x.y, -y.y);
    }
    const auto turn_part = [&](Vec& u, Vec& v) {
#pragma unroll
      for (int i = 0; i < ANGLES; i += 2) {
        const int j = min(i + 1, ANGLES - 1);
        T& p0 = u.x[PAIRS ? 2 * i : i], & p1 = u.x[PAIRS ? 2 * j : j];
        T& q0 = PAIRS ? u.x[PAIRS ? 2 * i + 1 : 0] : v.x[PAIRS ? 0 : i], & q1 = PAIRS ? u.x[PAIRS ? 2 * j + 1 : 0] : v.x[PAIRS ? 0 : j];
        uint64_t p = pair(to_f32<T>(p0), to_f32<T>(p1)), q = pair(to_f32<T>(q0), to_f32<T>(q1));
        turn(p, q, c2[i / 2], s2[i / 2], m2[i / 2]);
        const float2 y = unpair(p), z = unpair(q);
        p1 = from_f32<T>(y.y);
        q1 = from_f32<T>(z.y);
        p0 = from_f32<T>(y.x);
        q0 = from_f32<T>(z.x);
      }
    };
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {              // q, k
      const int first = w ? max(slice * share - a.heads[0], 0) : slice * share;
      const int last = w ? end - a.heads[0] : min(end, a.heads[0]);
      int h = first + sub;
      if (h >= last) continue;
      const T* x = static_cast<const T*>(a.x[w]) + b * a.sx[w][0] + t * a.sx[w][1] + h * a.sx[w][2] + d;
      T* y = static_cast<T*>(a.y[w]) + b * a.sy[w][0] + t * a.sy[w][1] + h * a.sy[w][2] + d;
      const long long dx = together * a.sx[w][2], dy = together * a.sy[w][2];
      const auto load = [&](const T* x, Vec& u, Vec& v) {
        if constexpr (STEP == V) {
          u = *reinterpret_cast<const Vec*>(x);
          if (both) v = *reinterpret_cast<const Vec*>(x + other);
        } else {                               // (single values need not be aligned in twos)
          u.x[0] = x[0];
          if (turns) u.x[1] = x[1];
        }
      };
      const auto store = [&](T* y, Vec& u, Vec& v) {
        if (turns) turn_part(u, v);
        if constexpr (STEP == V) {
          *reinterpret_cast<Vec*>(y) = u;
          if (both) *reinterpret_cast<Vec*>(y + other) = v;
        } else {
          y[0] = u.x[0];
          if (turns) y[1] = u.x[1];
        }
      };
#pragma unroll 1
      for (; h + (AHEAD - 1) * together < last; h += AHEAD * together) {
        Vec u[AHEAD], v[AHEAD];
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
          load(x, u[e], v[e]);
          x += dx;
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
          store(y, u[e], v[e]);
          y += dy;
        }
      }
#pragma unroll 1
      for (; h < last; h += together) {
        Vec u, v;
        load(x, u, v);
        x += dx;
        store(y, u, v);
        y += dy;
      }
    }
  }
}

template <typename T>
cudaError_t launch(RopeArgs& a, bool pairs, bool wide, cudaStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const auto k = pairs ? (wide ? k_rope<T, V, true> : k_rope<T, 1, true>) : (wide ? k_rope<T, kHalves, false> : k_rope<T, 1, false>);
  // a token's heads among warps where tokens alone do not fill the device
  const long long tokens = (long long)a.batch * a.T, want = (long long)kPlanSMs * 16;
  a.slices = (int)std::min<long long>(a.heads[0] + a.heads[1], (want + tokens - 1) / tokens);
  const long long blocks = (tokens * a.slices + kThreads / 32 - 1) / (kThreads / 32);
  return launch_pdl(k, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
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
    if (!std::isfinite(f)) return ck.fail("factor is too small: a frequency over it is not finite");
    double turn = f / two_pi;
    turn -= std::floor(turn);                                    // (a factor below 1: whole turns say nothing)
    const double scaled = std::ldexp(turn, 64);
    h_turns[i] = scaled >= 18446744073709551615.0 ? 0 : (uint64_t)scaled;
  }
  return CDSL_OK;
}

extern "C" int32_t cdsl_rope(const cdsl_rope_cfg* rope, int32_t inverse, const cdsl_rope_rows* rows, const void* d_q,
                             void* d_q_out, const void* d_k, void* d_k_out, const int32_t* d_start, const int32_t* d_offset,
                             void* stream) {
  Check ck("cdsl_rope");
  if (!rope || !rows || !rope->d_turns || !d_q || !d_q_out || !d_start) return ck.fail("a required pointer is NULL");
  const cdsl_rope_rows& z = *rows;
  if (!ck.value_type(z.dtype)) return CDSL_EINVAL;
  if (!d_k != !d_k_out) return ck.fail("k and k's output go together");
  if (z.head_dim < 2 || z.head_dim > CDSL_ROPE_MAX_DIM) return ck.fail("head_dim must be 2 .. 1024");
  if (rope->rot < 2 || rope->rot % 2 || rope->rot > z.head_dim) return ck.fail("rot must be even, 2 .. head_dim");
  if (z.batch < 1 || z.T < 1 || (long long)z.batch * z.T > (1 << 26) || z.n_heads < 1 || z.n_heads > (1 << 16) ||
      (d_k && (z.n_kv_heads < 1 || z.n_kv_heads > (1 << 16))))
    return ck.fail("sizes: need batch, T >= 1, at most 2^26 tokens, 1 .. 65536 heads");
  if (!(rope->magnitude > 0.f) || !std::isfinite(rope->magnitude)) return ck.fail("magnitude must be positive and finite");
  const int eb = z.dtype == CDSL_DTYPE_BF16 ? 2 : 4, V = 16 / eb;
  RopeArgs a = {};
  a.turns = rope->d_turns;
  a.half = rope->rot / 2;
  a.hd = z.head_dim;
  a.batch = z.batch;
  a.T = z.T;
  a.heads[0] = z.n_heads;
  a.heads[1] = d_k ? z.n_kv_heads : 0;
  a.magnitude = rope->magnitude;
  a.sign = inverse ? -1.f : 1.f;
  a.x[0] = d_q; a.x[1] = d_k;
  a.y[0] = d_q_out; a.y[1] = d_k_out;
  a.start = d_start;
  a.offset = d_offset;
  // 16 bytes at a time where every part of a head begins at a multiple of them
  bool wide = rope->interleaved ? rope->rot % V == 0 && (z.head_dim - rope->rot) % V == 0
                                : a.half % kHalves == 0 && (z.head_dim - rope->rot) % (2 * kHalves) == 0;
  for (int w = 0; w < (d_k ? 2 : 1); ++w) {
    if (!ck.aligned(a.x[w], eb) || !ck.aligned(a.y[w], eb)) return ck.fail("tensors must be aligned to their type");
    wide = wide && ck.aligned(a.x[w], 16) && ck.aligned(a.y[w], 16);
    for (int i = 0; i < 3; ++i) {
      a.sx[w][i] = z.strides[6 * w + i];
      a.sy[w][i] = z.strides[6 * w + 3 + i];
      if (a.sx[w][i] % V || a.sy[w][i] % V) wide = false;
    }
    const long long* const so = a.sy[w];
    if ((z.batch > 1 && so[0] == 0) || (z.T > 1 && so[1] == 0) || (a.heads[w] > 1 && so[2] == 0))
      return ck.fail("an output must not have a stride of 0 between sequences, tokens or heads");
    if (a.x[w] == a.y[w] && !std::equal(a.sx[w], a.sx[w] + 3, a.sy[w]))
      return ck.fail("an output in its input's place must have its strides");
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool pairs = rope->interleaved != 0;
  return ck.launched(z.dtype == CDSL_DTYPE_BF16 ? launch<__nv_bfloat16>(a, pairs, wide, s)
                                                : launch<float>(a, pairs, wide, s));
}
