// tree_host.h -- argument checks shared by the tree speculation entry points.
#pragma once

#include <cuda_runtime.h>

#include <cstdio>
#include <type_traits>

#include "kernels.h"
#include "tree.cuh"

namespace cdsl {
namespace tree {

// One entry point's checks. A failed one sets the thread's error message (no exception leaves an
// entry point: a message that cannot be stored is dropped).
struct Check {
  const char* fn;
  explicit Check(const char* name) : fn(name) {}

  int fail(const char* why, int code = CDSL_EINVAL) const noexcept {
    char buf[256];
    snprintf(buf, sizeof buf, "%s: %s", fn, why);
    try {
      set_thread_error(buf);
    } catch (...) {
    }
    return code;
  }
  bool no(const char* why) const { fail(why); return false; }

  static bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

  // A cache's sizes (pointers: whether they are looked at too).
  bool cache(const cdsl_kv_cache* k, Cache* c, bool pointers = true) const {
    if (!k) return no("cache is NULL");
    if (pointers && (!k->d_pool || !k->d_scale || !k->d_page_table)) return no("a cache pointer is NULL");
    if (pointers && (!aligned(k->d_pool, 16) || !aligned(k->d_scale, 16)))
      return no("the cache's pool and scale must be 16-byte aligned");
    if (k->head_dim != 64 && k->head_dim != 128) return no("head_dim must be 64 or 128");
    if (k->page_size < 16 || k->page_size > 256 || (k->page_size & (k->page_size - 1)))
      return no("page_size must be a power of two, 16..256");
    if (k->dtype != CDSL_DTYPE_F8E4M3 && k->dtype != CDSL_DTYPE_BF16)
      return no("the cache's dtype must be e4m3 or bfloat16");
    if (k->n_layers < 1 || k->n_layers > 65535 || k->n_pages < 1 || k->n_kv_heads < 1 || k->max_pages < 1 ||
        k->batch < 1 || k->batch > CDSL_TREE_MAX_BATCH)
      return no("cache sizes: need n_layers, n_pages, n_kv_heads, max_pages >= 1, 1 <= batch <= 1024");
    // a layer's rows are numbered in 31 bits, pages in 23
    if ((long long)k->n_pages * 2 * k->n_kv_heads * k->page_size >= (1LL << 31) || k->n_pages >= (1 << 23) ||
        (long long)k->max_pages * k->page_size >= (1LL << 30) || k->n_kv_heads > 1024)
      return no("cache sizes beyond the limits (2^31 rows per layer, 2^23 pages, 2^30 slots per sequence, "
                "1024 heads)");
    int shift = 4;
    while ((1 << shift) < k->page_size) ++shift;
    *c = {static_cast<uint8_t*>(k->d_pool), k->d_scale, k->d_page_table, k->n_layers, k->n_pages,
          k->n_kv_heads, shift, k->head_dim, k->dtype == CDSL_DTYPE_BF16 ? 2 : 1, k->batch, k->max_pages};
    return true;
  }
  bool layers(const Cache& c, int layer, int n) const {
    if (layer < 0 || n < 1 || layer > c.n_layers - n) return no("layers outside the cache's");
    return true;
  }
  bool value_type(int dtype) const {
    if (dtype != CDSL_DTYPE_F32 && dtype != CDSL_DTYPE_BF16) return no("dtype must be float32 or bfloat16");
    return true;
  }
  bool tokens(const Cache& c, int T) const {
    if (T < 1 || (long long)T > ((long long)c.max_pages << c.page_shift))
      return no("T must be 1 .. max_pages * page_size");
    if ((long long)T * 2 * c.kvh * 16 >= (1LL << 31)) return no("T rows of all heads beyond the limit (2^26)");
    return true;
  }
  bool nodes(const Cache& c, int T) const {
    if (T < 1 || T > CDSL_TREE_MAX_NODES) return no("T must be 1 .. 128 nodes");
    return tokens(c, T);
  }
  int launched(cudaError_t e) const {
    if (e == cudaSuccess) return CDSL_OK;
    cudaGetLastError();
    return fail(cudaGetErrorString(e), CDSL_ECUDA);
  }
};

}  // namespace tree
}  // namespace cdsl
