// tree.cuh -- the quantised paged cache (cdsl_kv_cache) on the device, and how a tree attention
// pass is dealt to blocks.
#pragma once

#include <cuda_fp8.h>

#include "../../include/cdsl_tree.h"
#include "common.cuh"

namespace cdsl {
namespace tree {

enum Format { kF8, kBF16, kI4 };
constexpr int kGroup = 32;                     // I4: values that share a scale

struct Cache {
  uint8_t* pool;          // rows of hd codes
  uint8_t* scale;         // a byte per row; I4: a bf16 per group of a row
  const int32_t* table;
  int32_t n_layers, n_pages, kvh, page_shift, hd, batch, max_pages;
  int32_t format, row, srow /* bytes of a row's codes, and of its scales */;
};

// Row (one head's codes of one slot) of the pool and of the scale bytes. 64 bits: a cache of a few
// thousand pages and tens of layers has more than 2^31 codes.
__host__ __device__ inline size_t row_of(const Cache& c, int layer, int page, int kv, int head, int at) {
  return ((((size_t)layer * c.n_pages + page) * 2 + kv) * c.kvh + head << c.page_shift) + at;
}

// Page of a sequence's slot, -1 where the slot or the page is out of range.
__device__ __forceinline__ int page_of(const Cache& c, int b, long long slot) {
  const long long col = slot >> c.page_shift;
  if (slot < 0 || col >= c.max_pages) return -1;
  const int page = c.table[(size_t)b * c.max_pages + col];
  return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

// 2^(byte - 127), NaN for 255. (Byte 0, which no row written by cdsl_kv_write has, stands for 0.)
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 255 ? 0x7fc00000u : byte << 23);
}

// I4. A row's codes are two's complement nibbles, its groups taking turns by four: nibble (j * G + g) * 4 + i is value
// 32 g + 4 j + i, G = hd / 32. So each 16 bits lie in one group, and 8, 16 or 64 bytes hold as many of every group.
// Four codes (16 bits) to floats times a scale, exactly: 2^23 + (code + 8) as a float's bits.
__device__ __forceinline__ void i4x4_to_f32(uint32_t four, float scale, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = (__uint_as_float((four >> (4 * i) & 15u) ^ 0x4b000008u) - 8388616.f) * scale;
}
// A row's scales (in a uint2 or the low word of one): is any of them not finite?
__device__ __forceinline__ bool i4_not_finite(uint2 s, int groups) {
  const auto bad = [](uint32_t two) { return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u; };
  return bad(s.x) || (groups > 2 && bad(s.y));
}
__device__ __forceinline__ float bf16_at(uint32_t two, int high) {
  return __uint_as_float(high ? two & 0xffff0000u : two << 16);
}

// Two e4m3 codes to floats (exact).
__device__ __forceinline__ float2 f8x2_to_f32(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

}  // namespace tree
}  // namespace cdsl
