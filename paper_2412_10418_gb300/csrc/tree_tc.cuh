// tree_tc.cuh -- pieces that the tensor-core kernels of the tree attention share.
#pragma once

#include <algorithm>

#include "kernels.h"
#include "once.h"
#include "tree_attention.cuh"

namespace cdsl {
namespace tree {

// Position in a sequence of phases: index and parity of the `n`-th use of one of `of` barriers.
__device__ __forceinline__ uint32_t parity(int n, int of) { return (n / of) & 1; }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Waits for the phase of parity `parity` to complete; false (and CDSL_ETIMEOUT latched) if it has not after kTries
// suspended tries, a second or more. (Tries are counted, not timed: there are some twenty waits in a kernel, and their
// code in the instruction cache counts.)
constexpr int kTries = 1 << 19;
__device__ __forceinline__ bool wait_for(uint64_t* m, uint32_t parity, int32_t* status) {
#pragma unroll 1
  for (int i = 0; i < kTries; ++i)
    if (tc::mbar_try_wait_sleep(m, parity)) return true;
  set_status(status, CDSL_ETIMEOUT);
  return false;
}
// Pairs of fp32 values in a 64-bit register.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair(uint32_t a, uint32_t b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ float warp_fmax(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
// Four e4m3 codes, a's low half in the low byte; two codes to a half2 (exact).
__device__ __forceinline__ uint32_t f8x4(__half2 a, __half2 b) {
  uint32_t r;
  asm("{\n\t.reg .b16 x, y;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 x, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 y, %2;\n\t"
      "mov.b32 %0, {x, y};\n\t}"
      : "=r"(r)
      : "r"(*reinterpret_cast<uint32_t*>(&a)), "r"(*reinterpret_cast<uint32_t*>(&b)));
  return r;
}
// The half2 pairs of four codes.
__device__ __forceinline__ void f8x4_half(uint32_t four, __half2* a, __half2* b) {
  asm("{\n\t.reg .b16 x, y;\n\t"
      "mov.b32 {x, y}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, x;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, y;\n\t}"
      : "=r"(*reinterpret_cast<uint32_t*>(a)), "=r"(*reinterpret_cast<uint32_t*>(b))
      : "r"(four));
}
// (x & mask) ^ c in one instruction, of which only one operand may be a constant: masks come from registers.
__device__ __forceinline__ uint32_t and_xor(uint32_t x, uint32_t mask, uint32_t c) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(d) : "r"(x), "r"(mask), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 4-bit code I of both halves of x, times their scales, exactly: (128 + 8 (code + 8)) scale / 8 - 24 scale in bf16, of
// mask = 0x00780078, s8 = (scale / 8) and m24 = (-24 scale) of the two.
template <int I>
__device__ __forceinline__ uint32_t value_bf16(uint32_t x, uint32_t mask, uint32_t s8, uint32_t m24) {
  const uint32_t t = I == 0 ? x << 3 : x >> (4 * I - 3);
  return fma_bf16x2(and_xor(t, mask, 0x43404340u), s8, m24);
}

// Queries of a segment's block to shared memory, by NT threads, eight a vector: K-major tiles of NQ rows in
// blocks of at most 128 bytes. F8: two e4m3 planes of q / 2^e, hi = e4m3(q / 2^e) and lo the rest, e the
// smallest with which the row's largest value is at most 448; else bf16 as they are. A row that is not finite, and
// rows past the block's, become zeros. put(v, where, factor of the scores, not finite) once per vector. LIVE: groups
// of NT / 8 vectors that are all past the block's are left out. I4: bf16 with a row's dimensions in the order in which a
// 4-bit cache's words give them: 16 bytes W are those of codes 8 W .., one of each of two groups in turn.
template <int HD, int NQ, bool F8, int NT, bool LIVE, bool I4 = false, typename F>
__device__ __forceinline__ void stage_queries(const TreeArgs& a, const Segment& s, int tid, bool q_aligned,
                                              uint8_t* q_smem, F&& put) {
  constexpr int QE = HD / 8;                   // values per thread
  constexpr int KROW = HD * (F8 ? 1 : 2), BW = KROW < 128 ? KROW : 128;
  constexpr uint32_t PLANE = NQ * KROW;
  const int rounds = LIVE ? (s.nq + NT / 8 - 1) / (NT / 8) : NQ * 8 / NT;
  uint32_t next[QE / 2];
#pragma unroll 1
  for (int n = -1; n < rounds; ++n) {          // (the next round's loads before this one's work; one copy of the code)
    uint32_t w[QE / 2];
#pragma unroll
    for (int i = 0; i < QE / 2; ++i) {
      w[i] = next[i];
      next[i] = 0u;
    }
    int v = (n + 1) * (NT / 8) + tid / 8;
    if (v < s.nq) {
      const Vec x = vector_of(a, s.h, s.qb, v);
      const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + s.b * a.sq[0] + x.t * a.sq[1] +
                               x.h * a.sq[2] + (I4 ? 0 : tid % 8 * QE);
      if constexpr (I4) {
        constexpr int PAIRS = HD / kGroup / 2; // of groups
#pragma unroll
        for (int i = 0; i < QE / 8; ++i) {
          const int W = tid % 8 * (QE / 8) + i;
          const __nv_bfloat16* const lo = q + W % PAIRS * 2 * kGroup + W / PAIRS * 4;
          uint32_t l[2], h[2];                 // four dimensions of each group
          if (q_aligned) {
            const uint2 u = *reinterpret_cast<const uint2*>(lo), z = *reinterpret_cast<const uint2*>(lo + kGroup);
            l[0] = u.x; l[1] = u.y; h[0] = z.x; h[1] = z.y;
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              l[e] = __bfloat16_as_ushort(lo[2 * e]) | (uint32_t)__bfloat16_as_ushort(lo[2 * e + 1]) << 16;
              h[e] = __bfloat16_as_ushort(lo[kGroup + 2 * e]) | (uint32_t)__bfloat16_as_ushort(lo[kGroup + 2 * e + 1]) << 16;
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) next[4 * i + e] = __byte_perm(l[e / 2], h[e / 2], e % 2 ? 0x7632 : 0x5410);
        }
      } else if (q_aligned) {
#pragma unroll
        for (int i = 0; i < QE / 8; ++i) {
          const uint4 u = *reinterpret_cast<const uint4*>(q + 8 * i);
          next[4 * i] = u.x; next[4 * i + 1] = u.y; next[4 * i + 2] = u.z; next[4 * i + 3] = u.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < QE; ++i)
          next[i / 2] |= (uint32_t)__bfloat16_as_ushort(q[i]) << (i % 2 * 16);
      }
    }
    if (n < 0) continue;
    v -= NT / 8;
    const int part = tid % 8;
    uint32_t top = 0;                      // largest |x|, as bf16 bits
#pragma unroll
    for (int i = 0; i < QE / 2; ++i) top = max(top, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool bad = top >= 0x7f80u;
    float qs = a.scale;
    if constexpr (F8) {
      int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u);
      e = top == 0 || bad ? 0 : max(e, -126);
      const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
      qs *= __uint_as_float((uint32_t)(127 + e) << 23);
      uint32_t hi[QE / 4], lo[QE / 4];
#pragma unroll
      for (int i = 0; i < QE / 4; ++i) {
        const float y[4] = {__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i] & 0xffff0000u),
                            __uint_as_float(w[2 * i + 1] << 16), __uint_as_float(w[2 * i + 1] & 0xffff0000u)};
        uint32_t hl[2], ll[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 u = make_float2(y[2 * j] * inv, y[2 * j + 1] * inv);
          hl[j] = __nv_cvt_float2_to_fp8x2(u, __NV_SATFINITE, __NV_E4M3);
          const float2 z = f8x2_to_f32(hl[j]);
          ll[j] = __nv_cvt_float2_to_fp8x2(make_float2(u.x - z.x, u.y - z.y), __NV_SATFINITE, __NV_E4M3);
        }
        hi[i] = bad ? 0u : hl[0] | hl[1] << 16;
        lo[i] = bad ? 0u : ll[0] | ll[1] << 16;
      }
      if constexpr (HD == 128) {
        const uint32_t off = tc::row_offset(v, part, BW);
        *reinterpret_cast<uint4*>(q_smem + off) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(q_smem + off + PLANE) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      } else {
        const uint32_t off = tc::row_offset(v, part / 2, BW) + part % 2 * 8;
        *reinterpret_cast<uint2*>(q_smem + off) = make_uint2(hi[0], hi[1]);
        *reinterpret_cast<uint2*>(q_smem + off + PLANE) = make_uint2(lo[0], lo[1]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < QE / 8; ++i) {
        const int ch = part * (QE / 8) + i;   // 16-byte chunk of the row
        const uint32_t off = ch / 8 * NQ * BW + tc::row_offset(v, ch % 8, BW);
        *reinterpret_cast<uint4*>(q_smem + off) =
            bad ? make_uint4(0u, 0u, 0u, 0u) : make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
    }
    if (part == 0) put(v, vector_of(a, s.h, s.qb, v), qs, v < s.nq && bad);
  }
}

// The masks of the block's nodes to shared memory, s_mask[t - t0], by NT threads; of a part of an item without slots
// of the tree, none. (Words past a.W stay as they are: no slot has such a node.)
template <int NT>
__device__ __forceinline__ void stage_masks(const TreeArgs& a, const Segment& s, int t0, int tid, uint32_t (*s_mask)[kWords]) {
  if (s.c1 * kKeys <= s.len) return;
  const int n = (min(s.nodes, t0 + (s.nq + a.G - 1) / a.G + 1) - t0) * a.W;
  for (int i = tid; i < n; i += NT)
    s_mask[i / a.W][i % a.W] = a.mask[((size_t)s.b * a.T + t0) * a.W + i];
}

// The loading warp: K and V chunks of a run's segments into a ring of NST stages (tiles of kKeys rows in blocks
// of at most 128 bytes, swizzled as their rows are wide), a box per page piece, and the slots' scale bytes and which
// pieces there are, with V; EARLY: with K, and K a chunk ahead of V, whose stage comes free later. Waits are bounded; on
// expiry it returns with its copies landed.
template <int HD, bool F8, int NST, bool EARLY>
__device__ __forceinline__ void load_chunks(const TreeArgs& a, const int* first, int begin, int end,
                                            const CUtensorMap& map, uint8_t* ring, uint8_t* scales,
                                            uint32_t* s_pieces, uint64_t* k_full, uint64_t* v_full,
                                            uint64_t* k_empty, uint64_t* v_empty) {
  constexpr int EB = F8 ? 1 : 2, KROW = HD * EB, BW = KROW < 128 ? KROW : 128, NB = KROW / BW;
  constexpr uint32_t BLOCK = kKeys * BW, TILE = NB * BLOCK;
  const Cache& c = a.c;
  const int lane = threadIdx.x & 31, P = 1 << c.page_shift;
  const int rows = min(P, kKeys), pieces = kKeys / rows;
  struct Chunk {
    int page, h, at;                           // this lane's piece
    uint32_t live;
  };
  int issued_k = 0, issued_v = 0;              // copies
  auto issue = [&](int kv, int it, const Chunk& x) {
    const int st = it % NST;
    uint64_t* full = kv ? &v_full[st] : &k_full[st];
    if (!__all_sync(0xffffffffu, wait_for(kv ? &v_empty[st] : &k_empty[st], parity(it, NST) ^ 1, a.status)))
      return false;
    const bool bytes = kv == (EARLY ? 0 : 1);  // both scale bytes too
    if (lane == 0) {
      if (bytes) s_pieces[st] = x.live;
      tc::mbar_expect_tx(full, __popc(x.live) * rows * (KROW + (bytes ? 2 : 0)));
    }
    __syncwarp();
    if (x.page >= 0) {
      const int y = (int)row_of(c, 0, x.page, kv, x.h, x.at);
      uint8_t* dst = ring + (st * 2 + kv) * TILE + lane * rows * BW;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) tc::tma_load_2d(dst + nb * BLOCK, &map, nb * (BW / EB), y, full);
      if (bytes) {
        const uint8_t* from = c.scale + row_of(c, a.layer, x.page, 0, x.h, x.at);
        uint8_t* to = scales + st * 2 * kKeys + lane * rows;
        tc::bulk_load(to, from, rows, full);
        tc::bulk_load(to + kKeys, from + ((size_t)c.kvh << c.page_shift), rows, full);
      }
    }
    if (kv) issued_v = it + 1;
    else issued_k = it + 1;
    return true;
  };
  int it = 0;                                  // chunks
  bool ok = true;
  Chunk before = {};
#pragma unroll 1
  for (int unit = begin; unit < end && ok;) {
    const Segment s = segment_at(a, first, unit, end);
#pragma unroll 1
    for (int ch = s.c0; ch < s.c1 && ok; ++ch, ++it) {
      const int slot = ch * kKeys + lane * rows;
      Chunk x = {-1, s.h, slot & (P - 1), 0u};
      if (lane < pieces && slot < s.keys) {
        x.page = page_of(c, s.b, slot);
        if (x.page < 0) set_status(a.status, CDSL_ERANGE);
      }
      x.live = __ballot_sync(0xffffffffu, x.page >= 0);
      ok = issue(0, it, x);
      if (EARLY) {
        if (it > 0) ok = ok && issue(1, it - 1, before);
        before = x;
      } else {
        ok = ok && issue(1, it, x);
      }
    }
    unit += s.c1 - s.c0;
  }
  if (EARLY && it > 0) ok = ok && issue(1, it - 1, before);
  // where a role gave up, nothing may have waited for the copies
  if (!ok)
#pragma unroll 1
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll 1
      for (int n = kv ? issued_v : issued_k, i = max(0, n - NST); i < n; ++i)
        wait_for(kv ? &v_full[i % NST] : &k_full[i % NST], parity(i, NST), a.status);
}

// 32 bytes to an address that is a multiple of 32 (a whole sector: two stores of 16 bytes take two).
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// Dynamic shared memory beyond 48 KB for `kernel` on the current device; once: the kernel's.
template <typename K>
cudaError_t allow_shared(OncePerDevice& once, K kernel, size_t bytes) {
  int device = 0;
  if (const cudaError_t e = cudaGetDevice(&device)) return e;
  return once(device, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); });
}

// The tensor map of a layer's rows for load_chunks.
template <int HD, bool F8>
int encode_cache_map(const TreeArgs& a, CUtensorMap* map) {
  constexpr int EB = F8 ? 1 : 2, KROW = HD * EB, BW = KROW < 128 ? KROW : 128;
  const Cache& c = a.c;
  const size_t rows = (size_t)c.n_pages * 2 * c.kvh << c.page_shift;
  return encode_map(map, F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, EB,
                    c.pool + (size_t)a.layer * rows * KROW, HD, rows, BW / EB, std::min(1 << c.page_shift, kKeys),
                    BW == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

}  // namespace tree
}  // namespace cdsl
