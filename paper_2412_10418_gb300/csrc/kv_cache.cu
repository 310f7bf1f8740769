// kv_cache.cu -- the quantised paged cache: cdsl_kv_write, cdsl_kv_read, cdsl_kv_commit.
//
// A cache row is one head's K or V of one token: head_dim codes and a scale byte. The scale is a
// power of two, because a float code loses nothing to it (the spacing of e4m3 values is relative, so a
// finer scale moves the values between the same 16 steps per octave) and multiplying by it is exact:
// a code's value is the same in bf16, fp32 and 64 bits, and the attention folds it into scores and
// probabilities without a rounding.
//
// Codes of 4 bits are whole numbers, -7 .. 7, which have no steps of their own to follow small values with: 32 values
// share a scale, and it is not a power of two but the group's largest over 7, kept to 4 significant bits. With the code's
// three that makes 7 bits, so a value is exact in bf16 all the same. (A bf16 scale as it comes has 8 bits, and every
// product with a code would be rounded on its way to a tensor core.) 4.5 bits a value.
//
// All three are bound by HBM on large calls and by one launch on a decoding step's few rows. A lane of the first
// two has 16 values, so that a row's few dependent loads (its start, its page, its values) are waited for half as often
// as with 8: rows of 4 prompts of 1031 tokens, 8 heads of 128, bf16 to e4m3: 8.6 us written (25 MB, 10.1 with 8
// values), 9.3 us read; a tree of 17 nodes 3.5 us in a graph. In 4 bits 9.9 and 9.3 us (16 MB and 20; the dependent
// loads); 40 layers of 32 sequences' last pages read back, 377 MB, 61 us with a thread for several layers, 70 with one each.
#include <cuda.h>

#include <algorithm>
#include <string>

#include "kernels.h"
#include "tree.cuh"
#include "tree_host.h"

namespace cdsl {
namespace tree {
namespace {

constexpr int kThreads = 256;
constexpr int EPL = 16;                // values per lane: a row is head_dim / 16 lanes

struct RowsArgs {
  Cache c;
  int layer, T;
  const int32_t* start;
  const int32_t* count;
  int32_t* status;
};

// EPL values of a row, element type T. Unaligned rows (a base or a stride off 16 bytes) by single values.
template <typename T>
__device__ __forceinline__ void load_values(const T* p, bool aligned, float (&x)[EPL]) {
  if (aligned) {
    constexpr int N = 16 / sizeof(T);  // 16 bytes at a time
#pragma unroll
    for (int j = 0; j < EPL; j += N) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + j);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (N == 8) {
          x[j + 2 * i] = __uint_as_float(w[i] << 16);
          x[j + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
          x[j + i] = __uint_as_float(w[i]);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = to_f32<T>(p[i]);
  }
}
// EPL values as bf16 to an address that is a multiple of 16 bytes; zeros: zeros in their place.
__device__ __forceinline__ void store_bf16(void* p, const float (&x)[EPL], bool zeros) {
#pragma unroll
  for (int j = 0; j < EPL; j += 8) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 y = __floats2bfloat162_rn(x[j + 2 * i], x[j + 2 * i + 1]);
      w[i] = zeros ? 0u : *reinterpret_cast<const uint32_t*>(&y);
    }
    reinterpret_cast<uint4*>(p)[j / 8] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

struct WriteArgs {
  RowsArgs r;
  const void* k;
  const void* v;
  long long sk[3], sv[3];              // strides of sequences, tokens, heads
  bool aligned;
};

// Grid: (rows of a sequence over blocks, batch). LPR = head_dim / 16 lanes work on a row.
template <typename T, int LPR, bool F8>
__global__ void __launch_bounds__(kThreads) k_kv_write(WriteArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const Cache& c = a.r.c;
  const int b = blockIdx.y;
  const unsigned row = (blockIdx.x * kThreads + threadIdx.x) / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned h = row % c.kvh, kv = row / c.kvh & 1, t = row / c.kvh / 2;
  const int n = a.r.count ? min(a.r.count[b], a.r.T) : a.r.T;
  if ((int)t >= n) return;             // (a row's lanes return together)
  const T* base = static_cast<const T*>(kv ? a.v : a.k);
  const long long* st = kv ? a.sv : a.sk;
  float x[EPL];
  load_values<T>(base + b * st[0] + t * st[1] + h * st[2] + part * EPL, a.aligned, x);
  const int page = page_of(c, b, (long long)a.r.start[b] + t);
  const int at = (a.r.start[b] + (int)t) & ((1 << c.page_shift) - 1);
  // largest |x| over the row, as bits: they order like the values, and 0x7f800000 on is not finite
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  const unsigned lanes = ((1u << LPR) - 1) << ((threadIdx.x & 31) / LPR * LPR);   // of this row
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(lanes, top, o));
  if (page < 0) {
    if (part == 0) set_status(a.r.status, CDSL_ERANGE);
    return;
  }
  const bool bad = top >= (F8 ? 0x7f800000u : 0x7f7f8000u);   // (not finite, or bf16 rounds it to infinity)
  const size_t r = row_of(c, a.r.layer, page, kv, h, at);
  if constexpr (F8) {
    // smallest E with top <= 448 * 2^E = 1.75 * 2^(E + 8)
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u);
    e = top == 0 || bad ? 0 : max(e, -126);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[EPL / 4];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * inv, x[4 * i + 1] * inv),
                                                   __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * inv, x[4 * i + 3] * inv),
                                                   __NV_SATFINITE, __NV_E4M3);
      w[i] = bad ? 0u : lo | hi << 16;
    }
    *reinterpret_cast<uint4*>(c.pool + r * c.hd + part * EPL) = make_uint4(w[0], w[1], w[2], w[3]);
    if (part == 0) c.scale[r] = (uint8_t)(bad ? 255 : e + 127);
  } else {
    store_bf16(c.pool + (r * c.hd + part * EPL) * 2, x, bad);
    if (part == 0) c.scale[r] = (uint8_t)(bad ? 255 : 127);
  }
}

struct ReadArgs {
  RowsArgs r;
  void* k;
  void* v;
};

// Grid: (rows of a sequence over blocks, batch, layers).
template <typename T, int LPR, bool F8>
__global__ void __launch_bounds__(kThreads) k_kv_read(ReadArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const Cache& c = a.r.c;
  const int b = blockIdx.y, layer = blockIdx.z;
  const unsigned row = (blockIdx.x * kThreads + threadIdx.x) / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned h = row % c.kvh, kv = row / c.kvh & 1, t = row / c.kvh / 2;
  if ((int)t >= a.r.T) return;
  const int n = a.r.count ? a.r.count[b] : a.r.T;
  float x[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) x[i] = 0.f;
  if ((int)t < n) {
    const int page = page_of(c, b, (long long)a.r.start[b] + t);
    if (page < 0) {
      if (part == 0) set_status(a.r.status, CDSL_ERANGE);
    } else {
      const int at = (a.r.start[b] + (int)t) & ((1 << c.page_shift) - 1);
      const size_t r = row_of(c, a.r.layer + layer, page, kv, h, at);
      const float s = scale_value(c.scale[r]);
      if constexpr (F8) {
        const uint4 u = *reinterpret_cast<const uint4*>(c.pool + r * c.hd + part * EPL);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = f8x2_to_f32(w[i / 2] >> (16 * (i % 2)) & 0xffffu);
          x[2 * i] = f.x * s;
          x[2 * i + 1] = f.y * s;
        }
      } else {
        load_values(reinterpret_cast<const __nv_bfloat16*>(c.pool) + r * c.hd + part * EPL, true, x);
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] *= s;
      }
    }
  }
  T* out = static_cast<T*>(kv ? a.v : a.k) +
           ((((size_t)layer * c.batch + b) * a.r.T + t) * c.kvh + h) * c.hd + part * EPL;
  if constexpr (sizeof(T) == 2) {
    store_bf16(out, x, false);
  } else {
#pragma unroll
    for (int j = 0; j < EPL; j += 4)
      reinterpret_cast<float4*>(out)[j / 4] = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
  }
}

// ---- 4 bits. A lane has 8 bytes of a row, 16 codes: pieces of four of one group each. Its values are 8 or 16 bytes of each
// group (pieces 4 part .. of number j * G + g: G = 4: dimensions 32 g + 4 part .., G = 2: 32 g + 8 part ..), so that a row's
// lanes take whole sectors and no value changes lanes.

__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Codes of 8 values, x[i] / step rounded to nearest, ties to even, as nibbles; step has 4 significant bits. A product with
// the reciprocal is off by 2^-20 at most, which only a quotient on or next to a tie notices. Of bfloat16 values (8 bits)
// one that is not a tie is 2^-11 away from it: rounded to 2^-15 first, ties are ties. Of float32 values the remainder
// decides where it is close.
template <typename T>
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], const float (&steps)[2]) {   // of four values each
  const float invs[2] = {rcp(steps[0]), rcp(steps[1])};
  int c[8];
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = __float_as_int(fmaf(x[i], invs[i / 4], 384.f) + (12582912.f - 384.f));   // 1.5 * 2^8, 1.5 * 2^23
  } else {
    bool close = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float y = fmaf(x[i], invs[i / 4], 12582912.f);
      close = close || fabsf(fmaf(12582912.f - y, steps[i / 4], x[i])) > steps[i / 4] * 0.4999f;
      c[i] = __float_as_int(y);
    }
    if (close)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float rem = fmaf(12582912.f - __int_as_float(c[i]), steps[i / 4], x[i]), away = fabsf(rem), half = steps[i / 4] * 0.5f;
        if (away > half || (away == half && (c[i] & 1))) c[i] += rem > 0.f ? 1 : -1;
      }
  }
  // sum of (c_i + 8) 16^i, the constants' own bits taken off (modulo 2^32), then two's complement
  uint32_t all = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i) all = all * 16 + (uint32_t)c[i];
  return (all + 0x88888888u - 0x4b400000u * 0x11111111u) ^ 0x88888888u;
}

// Grid: (rows of a sequence over blocks, batch). LPR = head_dim / 16 lanes work on a row.
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads) k_kv_write4(WriteArgs a) {
  constexpr int G = LPR / 2, N = 16 / G;       // values of a group
  pdl_wait();
  pdl_launch_dependents();
  const Cache& c = a.r.c;
  const int b = blockIdx.y;
  const unsigned row = (blockIdx.x * kThreads + threadIdx.x) / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned h = row % c.kvh, kv = row / c.kvh & 1, t = row / c.kvh / 2;
  const int n = a.r.count ? min(a.r.count[b], a.r.T) : a.r.T;
  if ((int)t >= n) return;             // (a row's lanes return together)
  const long long* st = kv ? a.sv : a.sk;
  const T* const from = static_cast<const T*>(kv ? a.v : a.k) + b * st[0] + t * st[1] + h * st[2] + part * N;
  float x[G][N];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const T* const p = from + g * kGroup;
    if (a.aligned) {
      constexpr int W = N * sizeof(T) / 8;     // 8 bytes at a time
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const uint2 u = reinterpret_cast<const uint2*>(p)[i];
        if constexpr (sizeof(T) == 2) {
          x[g][4 * i] = bf16_at(u.x, 0); x[g][4 * i + 1] = bf16_at(u.x, 1);
          x[g][4 * i + 2] = bf16_at(u.y, 0); x[g][4 * i + 3] = bf16_at(u.y, 1);
        } else {
          x[g][2 * i] = __uint_as_float(u.x); x[g][2 * i + 1] = __uint_as_float(u.y);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[g][i] = to_f32<T>(p[i]);
    }
  }
  const int page = page_of(c, b, (long long)a.r.start[b] + t);
  const int at = (a.r.start[b] + (int)t) & ((1 << c.page_shift) - 1);
  // the groups' largest |x| as bits (they order like the values): lane part gets group part % G's
  uint32_t top[G];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    top[g] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top[g] = max(top[g], __float_as_uint(x[g][i]) & 0x7fffffffu);
  }
  const unsigned lanes = ((1u << LPR) - 1) << ((threadIdx.x & 31) / LPR * LPR);   // of this row
  uint32_t mine;
  if constexpr (G == 4) {
    uint32_t two[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {              // bit 1 of the lane keeps groups 2, 3
      const uint32_t keep = part & 2 ? top[2 + i] : top[i], give = part & 2 ? top[i] : top[2 + i];
      two[i] = max(keep, __shfl_xor_sync(lanes, give, 2));
    }
    const uint32_t keep = part & 1 ? two[1] : two[0], give = part & 1 ? two[0] : two[1];
    mine = max(keep, __shfl_xor_sync(lanes, give, 1));
    mine = max(mine, __shfl_xor_sync(lanes, mine, 4));
  } else {
    const uint32_t keep = part & 1 ? top[1] : top[0], give = part & 1 ? top[0] : top[1];
    mine = max(keep, __shfl_xor_sync(lanes, give, 1));
    mine = max(mine, __shfl_xor_sync(lanes, mine, 2));
  }
  // its scale: top / 7 to 4 significant bits, nearest, ties to even; 2^-120 at least. (Not finite, or 2^120 and more, beyond
  // which codes times 8 would not fit: NaN.)
  uint32_t s = __float_as_uint(__fdiv_rn(__uint_as_float(mine), 7.f));
  s = max((s + 0x7ffffu + (s >> 20 & 1)) & 0xfff00000u, 0x03800000u);
  if (mine >= 0x7b800000u) s = 0x7fc00000u;
  float step[G];
  bool bad = false;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    step[g] = __uint_as_float(__shfl_sync(lanes, s, g, LPR));
    bad = bad || step[g] != step[g];
  }
  if (page < 0) {
    if (part == 0) set_status(a.r.status, CDSL_ERANGE);
    return;
  }
  const size_t r = row_of(c, a.r.layer, page, kv, h, at);
  // pieces in the order of their numbers: the groups of 4 j, then of the next j
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[(2 * i + e / 4) % G][(2 * i + e / 4) / G * 4 + e % 4];
    const float steps[2] = {step[2 * i % G], step[(2 * i + 1) % G]};
    w[i] = bad ? 0u : codes_of<T>(y, steps);
  }
  *reinterpret_cast<uint2*>(c.pool + r * c.row + part * 8) = make_uint2(w[0], w[1]);
  if (part < G) reinterpret_cast<uint16_t*>(c.scale + r * c.srow)[part] = (uint16_t)(bad ? 0x7fc0u : s >> 16);
}

// Grid: (rows of a sequence over blocks, batch, layers or fewer): a thread has its row of every gridDim.z-th layer, kLayers
// of them at a time: where it lies takes three dependent loads, which a layer of one's own would wait for each time.
constexpr int kLayers = 4;
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads) k_kv_read4(ReadArgs a, int n_layers) {
  constexpr int G = LPR / 2, N = 16 / G;       // values of a group
  pdl_wait();
  pdl_launch_dependents();
  const Cache& c = a.r.c;
  const int b = blockIdx.y;
  const unsigned row = (blockIdx.x * kThreads + threadIdx.x) / LPR;
  const int part = threadIdx.x % LPR;
  const unsigned h = row % c.kvh, kv = row / c.kvh & 1, t = row / c.kvh / 2;
  if ((int)t >= a.r.T) return;
  const int n = a.r.count ? a.r.count[b] : a.r.T;
  int page = -1;
  if ((int)t < n) {
    page = page_of(c, b, (long long)a.r.start[b] + t);
    if (page < 0 && part == 0) set_status(a.r.status, CDSL_ERANGE);
  }
  const int at = (a.r.start[b] + (int)t) & ((1 << c.page_shift) - 1);
#pragma unroll 1
  for (int l0 = blockIdx.z; l0 < n_layers; l0 += kLayers * gridDim.z) {
    uint2 u[kLayers];                          // codes
    uint32_t s[kLayers][G / 2];                // scales
#pragma unroll
    for (int l = 0; l < kLayers; ++l) {
      const int layer = l0 + l * gridDim.z;
      u[l] = make_uint2(0u, 0u);
#pragma unroll
      for (int i = 0; i < G / 2; ++i) s[l][i] = 0u;
      if (page >= 0 && layer < n_layers) {
        const size_t r = row_of(c, a.r.layer + layer, page, kv, h, at);
        u[l] = *reinterpret_cast<const uint2*>(c.pool + r * c.row + part * 8);
        const uint32_t* const sp = reinterpret_cast<const uint32_t*>(c.scale + r * c.srow);
#pragma unroll
        for (int i = 0; i < G / 2; ++i) s[l][i] = sp[i];
      }
    }
#pragma unroll
    for (int l = 0; l < kLayers; ++l) {
      const int layer = l0 + l * gridDim.z;
      if (layer >= n_layers) break;
      // (one scale that is not finite: the row's all count as NaN)
      if (i4_not_finite(make_uint2(s[l][0], s[l][G / 2 - 1]), G))
#pragma unroll
        for (int i = 0; i < G / 2; ++i) s[l][i] = 0x7fc07fc0u;
      T* const out = static_cast<T*>(kv ? a.v : a.k) +
                     ((((size_t)layer * c.batch + b) * a.r.T + t) * c.kvh + h) * c.hd + part * N;
      const uint32_t w[2] = {u[l].x, u[l].y};
      float x[G][N];
#pragma unroll
      for (int i = 0; i < 4; ++i) {            // pieces
        const int g = i % G;
        float y[4];
        i4x4_to_f32(w[i / 2] >> (i % 2 * 16), bf16_at(s[l][g / 2], g % 2), y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[g][i / G * 4 + e] = y[e];
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < N; i += 4)
            *reinterpret_cast<float4*>(out + g * kGroup + i) = make_float4(x[g][i], x[g][i + 1], x[g][i + 2], x[g][i + 3]);
        } else {
          uint32_t two[N / 2];
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(x[g][2 * i], x[g][2 * i + 1]);
            two[i] = *reinterpret_cast<const uint32_t*>(&z);
          }
          if constexpr (N == 4) *reinterpret_cast<uint2*>(out + g * kGroup) = make_uint2(two[0], two[1]);
          else *reinterpret_cast<uint4*>(out + g * kGroup) = make_uint4(two[0], two[1], two[2], two[3]);
        }
      }
    }
  }
}

struct CommitArgs {
  Cache c;
  const int32_t* lens;
  const int32_t* path;
  const int32_t* n_path;
  int T;
  int32_t* new_lens;
  int32_t* status;
};

constexpr int kMoves = 8;              // rows that a thread holds at a time

// Grid: (layer, K or V, sequence). A thread moves 16 bytes of a head's row (or its scales) for
// path entries 1, 2, .. in order, kMoves reads before their writes. In order is enough: the path is
// strictly increasing from 0, so entry i's target i is below the sources of all later entries. Blocks have a thread a
// part, so that one wave takes a served batch: 40 layers of 16 trees of 49 nodes in 7.7 us, 3 us less than with 256
// threads a block; 16 rows in place of 8 a thread, 1.5 us more.
template <typename S>
__global__ void __launch_bounds__(kThreads) k_kv_commit(CommitArgs a) {   // S: a row's scales
  __shared__ int s_from[CDSL_TREE_MAX_NODES], s_to[CDSL_TREE_MAX_NODES];   // page << 8 | place, -1
  pdl_wait();
  pdl_launch_dependents();
  const Cache& c = a.c;
  const int layer = blockIdx.x, kv = blockIdx.y, b = blockIdx.z;
  const int len = a.lens[b], n = a.n_path[b];
  const int32_t* path = a.path + (size_t)b * a.T;
  int err = n < 0 || n > a.T ? CDSL_EINVAL : 0;
  if (!err)
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
      const int p = path[i];
      if (i == 0 ? p != 0 : p <= path[i - 1] || p >= a.T) err = CDSL_EINVAL;
      const long long from = (long long)len + p, to = (long long)len + i;
      const int fp = page_of(c, b, from), tp = page_of(c, b, to);
      if (!err && (fp < 0 || tp < 0)) err = CDSL_ERANGE;
      s_from[i] = (int)(from & ((1 << c.page_shift) - 1));
      s_to[i] = (int)(to & ((1 << c.page_shift) - 1));
      if (fp >= 0) s_from[i] |= fp << 8;
      if (tp >= 0) s_to[i] |= tp << 8;
    }
  if (err) set_status(a.status, err);
  const bool bad = __syncthreads_or(err != 0);
  if (layer == 0 && kv == 0 && threadIdx.x == 0 && a.new_lens) a.new_lens[b] = bad ? len : len + n;
  if (bad) return;
  auto row = [&](int x, int head) { return row_of(c, layer, x >> 8, kv, head, x & 255); };
  auto move = [&](auto* base, size_t pitch, int head) {
    using E = std::remove_reference_t<decltype(*base)>;
    for (int i0 = 1; i0 < n; i0 += kMoves) {
      E x[kMoves];
#pragma unroll
      for (int i = 0; i < kMoves; ++i)
        if (i0 + i < n) x[i] = base[row(s_from[i0 + i], head) * pitch];
#pragma unroll
      for (int i = 0; i < kMoves; ++i)
        if (i0 + i < n && s_from[i0 + i] != s_to[i0 + i]) base[row(s_to[i0 + i], head) * pitch] = x[i];
    }
  };
  const int per = c.row / 16, codes = c.kvh * per;   // 16-byte parts of a row, of all heads
  for (int q = threadIdx.x; q < codes + c.kvh; q += blockDim.x) {
    if (q < codes) move(reinterpret_cast<uint4*>(c.pool) + q % per, per, q / per);
    else move(reinterpret_cast<S*>(c.scale), 1, q - codes);
  }
}

template <typename F>
int by_shape(const Cache& c, int dtype, F&& f) {   // f(element type tag, lanes per row, e4m3?)
  auto g = [&](auto t) {
    if (c.hd == 128)
      return c.format == kF8 ? f(t, std::integral_constant<int, 8>(), std::true_type())
                       : f(t, std::integral_constant<int, 8>(), std::false_type());
    return c.format == kF8 ? f(t, std::integral_constant<int, 4>(), std::true_type())
                     : f(t, std::integral_constant<int, 4>(), std::false_type());
  };
  return dtype == CDSL_DTYPE_BF16 ? g(__nv_bfloat16()) : g(float());
}

// Blocks for T tokens' rows of a sequence.
unsigned row_blocks(const Cache& c, int T) {
  const size_t threads = (size_t)T * 2 * c.kvh * (c.hd / EPL);
  return (unsigned)((threads + kThreads - 1) / kThreads);
}

}  // namespace
}  // namespace tree
}  // namespace cdsl

using namespace cdsl;
using namespace cdsl::tree;

extern "C" int32_t cdsl_kv_write(const cdsl_kv_cache* cache, int32_t layer, const void* d_k,
                                 const void* d_v, int32_t dtype, int32_t T, const int64_t* h_strides,
                                 const int32_t* d_start, const int32_t* d_count, int32_t* d_status,
                                 void* stream) {
  Check ck("cdsl_kv_write");
  Cache c;
  if (!ck.cache(cache, &c) || !ck.layers(c, layer, 1) || !ck.value_type(dtype) || !ck.tokens(c, T))
    return CDSL_EINVAL;
  if (!d_k || !d_v || !h_strides || !d_start) return ck.fail("a required pointer is NULL");
  const int eb = dtype == CDSL_DTYPE_BF16 ? 2 : 4;
  if (!ck.aligned(d_k, eb) || !ck.aligned(d_v, eb)) return ck.fail("k and v must be aligned to their type");
  WriteArgs a;
  a.r = {c, layer, T, d_start, d_count, d_status};
  a.k = d_k;
  a.v = d_v;
  a.aligned = ck.aligned(d_k, 16) && ck.aligned(d_v, 16);
  for (int i = 0; i < 3; ++i) {
    a.sk[i] = h_strides[i];
    a.sv[i] = h_strides[3 + i];
    if (a.sk[i] * eb % 16 || a.sv[i] * eb % 16) a.aligned = false;
  }
  const dim3 grid(row_blocks(c, T), c.batch);
  return by_shape(c, dtype, [&](auto t, auto lpr, auto f8) {
    const auto k = c.format == kI4 ? k_kv_write4<decltype(t), lpr()> : k_kv_write<decltype(t), lpr(), f8()>;
    return ck.launched(launch_pdl(k, grid, dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a));
  });
}

extern "C" int32_t cdsl_kv_read(const cdsl_kv_cache* cache, int32_t layer, int32_t n_layers, void* d_k,
                                void* d_v, int32_t dtype, int32_t T, const int32_t* d_start,
                                const int32_t* d_count, int32_t* d_status, void* stream) {
  Check ck("cdsl_kv_read");
  Cache c;
  if (!ck.cache(cache, &c) || !ck.layers(c, layer, n_layers) || !ck.value_type(dtype) || !ck.tokens(c, T))
    return CDSL_EINVAL;
  if (!d_k || !d_v || !d_start) return ck.fail("a required pointer is NULL");
  if (!ck.aligned(d_k, 16) || !ck.aligned(d_v, 16)) return ck.fail("k and v must be 16-byte aligned");
  ReadArgs a;
  a.r = {c, layer, T, d_start, d_count, d_status};
  a.k = d_k;
  a.v = d_v;
  const dim3 grid(row_blocks(c, T), c.batch, n_layers);
  return by_shape(c, dtype, [&](auto t, auto lpr, auto f8) {
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (c.format == kI4) {
      // (several layers a thread where there are blocks enough)
      const long long each = (long long)grid.x * grid.y, want = (long long)kPlanSMs * 16;
      const int z = (int)std::min<long long>(n_layers, std::max<long long>((n_layers + 2 * kLayers - 1) / (2 * kLayers), (want + each - 1) / each));
      return ck.launched(launch_pdl(k_kv_read4<decltype(t), lpr()>, dim3(grid.x, grid.y, z), dim3(kThreads), 0, s, a, n_layers));
    }
    return ck.launched(launch_pdl(k_kv_read<decltype(t), lpr(), f8()>, grid, dim3(kThreads), 0, s, a));
  });
}

extern "C" int32_t cdsl_kv_commit(const cdsl_kv_cache* cache, const int32_t* d_lens,
                                  const int32_t* d_path, const int32_t* d_n_path, int32_t T,
                                  int32_t* d_new_lens, int32_t* d_status, void* stream) {
  Check ck("cdsl_kv_commit");
  Cache c;
  if (!ck.cache(cache, &c) || !ck.nodes(c, T)) return CDSL_EINVAL;
  if (!d_lens || !d_path || !d_n_path) return ck.fail("a required pointer is NULL");
  if (d_new_lens == d_lens) return ck.fail("d_new_lens must not be d_lens");
  const CommitArgs a = {c, d_lens, d_path, d_n_path, T, d_new_lens, d_status};
  const int parts = c.kvh * (c.row / 16 + 1);   // a token's, scales last: a thread each
  const auto k = c.srow == 1 ? k_kv_commit<uint8_t> : c.srow == 4 ? k_kv_commit<uint32_t> : k_kv_commit<uint2>;
  return ck.launched(launch_pdl(k, dim3(c.n_layers, 2, c.batch), dim3(std::min(kThreads, (parts + 31) / 32 * 32)), 0,
                                static_cast<cudaStream_t>(stream), a));
}
