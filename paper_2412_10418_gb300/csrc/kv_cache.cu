// kv_cache.cu -- the quantised paged cache: cdsl_kv_write, cdsl_kv_read, cdsl_kv_commit.
//
// A cache row is one head's K or V of one token: head_dim codes and a scale byte. The scale is a
// power of two, because a float code loses nothing to it (the spacing of e4m3 values is relative, so a
// finer scale moves the values between the same 16 steps per octave) and multiplying by it is exact:
// a code's value is the same in bf16, fp32 and 64 bits, and the attention folds it into scores and
// probabilities without a rounding.
//
// All three are bound by HBM on large calls and by one launch on a decoding step's few rows. A lane of the first
// two has 16 values, so that a row's few dependent loads (its start, its page, its values) are waited for half as often
// as with 8: rows of 4 prompts of 1031 tokens, 8 heads of 128, bf16 to e4m3: 8.6 us written (25 MB, 10.1 with 8
// values), 9.3 us read; a tree of 17 nodes 3.5 us in a graph.
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

// Grid: (layer, K or V, sequence). A thread moves 16 bytes of a head's row (or its scale byte) for
// path entries 1, 2, .. in order, kMoves reads before their writes. In order is enough: the path is
// strictly increasing from 0, so entry i's target i is below the sources of all later entries. Blocks have a thread a
// part, so that one wave takes a served batch: 40 layers of 16 trees of 49 nodes in 7.7 us, 3 us less than with 256
// threads a block; 16 rows in place of 8 a thread, 1.5 us more.
__global__ void __launch_bounds__(kThreads) k_kv_commit(CommitArgs a) {
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
  const int per = c.hd * c.eb / 16, codes = c.kvh * per;   // 16-byte parts of a row, of all heads
  for (int q = threadIdx.x; q < codes + c.kvh; q += blockDim.x) {
    if (q < codes) move(reinterpret_cast<uint4*>(c.pool) + q % per, per, q / per);
    else move(c.scale, 1, q - codes);
  }
}

template <typename F>
int by_shape(const Cache& c, int dtype, F&& f) {   // f(element type tag, lanes per row, e4m3?)
  auto g = [&](auto t) {
    if (c.hd == 128)
      return c.eb == 1 ? f(t, std::integral_constant<int, 8>(), std::true_type())
                       : f(t, std::integral_constant<int, 8>(), std::false_type());
    return c.eb == 1 ? f(t, std::integral_constant<int, 4>(), std::true_type())
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
    return ck.launched(launch_pdl(k_kv_write<decltype(t), lpr(), f8()>, grid, dim3(kThreads), 0,
                                  static_cast<cudaStream_t>(stream), a));
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
    return ck.launched(launch_pdl(k_kv_read<decltype(t), lpr(), f8()>, grid, dim3(kThreads), 0,
                                  static_cast<cudaStream_t>(stream), a));
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
  const int parts = c.kvh * (c.hd * c.eb / 16 + 1);   // a token's, scales last: a thread each
  return ck.launched(launch_pdl(k_kv_commit, dim3(c.n_layers, 2, c.batch), dim3(std::min(kThreads, (parts + 31) / 32 * 32)), 0,
                                static_cast<cudaStream_t>(stream), a));
}
