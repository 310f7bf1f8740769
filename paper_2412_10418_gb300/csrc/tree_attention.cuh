// tree_attention.cuh -- how a tree attention pass is dealt to blocks, and the masks and partial results
// that its kernels share.
//
// Work: an item is (sequence, K/V head, block of NQ query vectors), its units the chunks of kKeys
// slots that its queries may see. The units of all items, in order, are cut into as many equal runs as
// there are blocks, so that ragged lengths and any batch keep every block equally long at work. A
// run covers parts of at most two items and any number of whole ones. A whole item's output is written
// at once; of a part the block leaves (m, l, o) in the workspace, and k_tree_combine adds the parts
// up in order (deterministic).
#pragma once

#include "tc_ptx.cuh"
#include "tree.cuh"

namespace cdsl {
namespace tree {

constexpr int kKeys = 128;                     // slots per chunk
constexpr int kWords = CDSL_TREE_MAX_NODES / 32;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;

struct TreeArgs {
  Cache c;
  int layer, T, H, G, W, NQ, QB;               // W: mask words; QB: query blocks per head
  const void* q;
  void* out;
  float* lse;
  long long sq[3], so[3];
  const int32_t* lens;
  const int32_t* nodes;
  const uint32_t* mask;
  float scale;                                 // softmax scale * log2(e): scores in base 2
  int max_len;
  int blocks;                                  // launched: runs at most
  float* part_ml;                              // workspace: [blocks][2][2][NQ]: m, l
  float* part_o;                               // [blocks][2][NQ][hd]
  int32_t* status;
};

// Runs of a pass: none is empty (a block beyond them has nothing to do).
__device__ __forceinline__ int runs_of(const TreeArgs& a, int total) { return min(a.blocks, total); }
// The runs' bounds (products below 2^63: both factors are below 2^31).
__device__ __forceinline__ int run_begin(int run, int total, int runs) {
  return (int)((long long)run * total / runs);
}
__device__ __forceinline__ int run_of(int unit, int total, int runs) {
  return (int)((((long long)unit + 1) * runs - 1) / total);
}

__device__ __forceinline__ int len_of(const TreeArgs& a, int b) {
  return min(max(a.lens[b], 0), a.max_len);
}
__device__ __forceinline__ int nodes_of(const TreeArgs& a, int b) {
  return a.nodes ? min(max(a.nodes[b], 0), a.T) : a.T;
}
// Units of a block of queries (an item without anything to see has one, which writes its zeros), of those
// that hold nodes, and how many blocks hold some.
__device__ __forceinline__ int item_units(int keys) { return max(1, (keys + kKeys - 1) / kKeys); }
__device__ __forceinline__ int live_blocks(const TreeArgs& a, int nodes) {
  return (nodes * a.G + a.NQ - 1) / a.NQ;
}

// of a sequence of `len` cached slots and n nodes
__device__ __forceinline__ int units_of(const TreeArgs& a, int len, int n) {
  const int live = live_blocks(a, n);
  return a.c.kvh * (live * item_units(len + n) + (a.QB - live));
}

// first[b], b <= batch: the units before sequence b's; behind them the sequences' lengths and nodes. The whole block
// calls; first is in shared memory, plan_bytes of it.
constexpr int plan_bytes(int batch) { return (3 * batch + 1) * 4; }
__device__ __forceinline__ void build_plan(const TreeArgs& a, int* first) {
  if (threadIdx.x < 32) {
    int sum = 0;
    for (int b0 = 0; b0 < a.c.batch; b0 += 32) {
      const int b = b0 + (int)threadIdx.x;
      const int len = b < a.c.batch ? len_of(a, b) : 0, n = b < a.c.batch ? nodes_of(a, b) : 0;
      const int v = b < a.c.batch ? units_of(a, len, n) : 0;
      int s = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, s, o);
        if ((int)threadIdx.x >= o) s += w;
      }
      if (b < a.c.batch) {
        first[b] = sum + s - v;
        first[a.c.batch + 1 + b] = len;
        first[2 * a.c.batch + 1 + b] = n;
      }
      sum += __shfl_sync(0xffffffffu, s, 31);
    }
    if (threadIdx.x == 0) first[a.c.batch] = sum;
  }
  __syncthreads();
}

// One item's part that a run covers.
struct Segment {
  int b, h, qb;
  int len, nodes, keys;     // cached slots, tree slots after them, both (0 of an item without queries)
  int c0, c1, units;        // chunks [c0, c1) of the item's
  int nq;                   // its query vectors (0 without any)
};
__device__ __forceinline__ Segment segment_at(const TreeArgs& a, const int* first, int unit, int end) {
  int lo = 0, hi = a.c.batch - 1;              // the last sequence whose first unit is not after `unit`
#pragma unroll 1
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (first[mid] <= unit) lo = mid; else hi = mid - 1;
  }
  Segment s;
  s.b = lo;
  s.len = first[a.c.batch + 1 + lo];
  s.nodes = first[2 * a.c.batch + 1 + lo];
  const int live = live_blocks(a, s.nodes), u = item_units(s.len + s.nodes);
  const int per_head = live * u + (a.QB - live);
  const int x = unit - first[lo];
  s.h = x / per_head;
  const int y = x % per_head;
  if (y < live * u) {
    s.qb = y / u;
    s.c0 = y % u;
    s.units = u;
    s.keys = s.len + s.nodes;
    s.nq = min(a.NQ, s.nodes * a.G - s.qb * a.NQ);
  } else {
    s.qb = live + (y - live * u);
    s.c0 = 0;
    s.units = 1;
    s.keys = 0;
    s.nq = 0;
  }
  s.c1 = min(s.units, s.c0 + (end - unit));
  return s;
}

// Where query vector v (of the item's block) is: node t, head of the K/V head's group.
struct Vec { int t, h; };
__device__ __forceinline__ Vec vector_of(const TreeArgs& a, int h, int qb, int v) {
  const int x = qb * a.NQ + v;
  return {x / a.G, h * a.G + x % a.G};
}

template <typename T>
__device__ __forceinline__ void store_out(const TreeArgs& a, int b, const Vec& v, int d, float x) {
  static_cast<T*>(a.out)[b * a.so[0] + v.t * a.so[1] + v.h * a.so[2] + d] = from_f32<T>(x);
}
__device__ __forceinline__ void store_lse(const TreeArgs& a, int b, const Vec& v, float m, float l) {
  if (a.lse)
    a.lse[((size_t)b * a.T + v.t) * a.H + v.h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Lengths outside 0 .. max_len are latched (they count as the nearer bound).
__device__ __forceinline__ void check_lens(const TreeArgs& a) {
  for (int b = threadIdx.x; b < a.c.batch; b += blockDim.x)
    if (a.lens[b] < 0 || a.lens[b] > a.max_len) set_status(a.status, CDSL_ERANGE);
}

// The tensor-core kernels: slots as M, up to 32 query vectors per block (tree_attention_tc.cu), and vectors as
// M, up to 128 (tree_attention_rows.cu).
constexpr int kRowsBlock = 128;
int tc_blocks_per_sm(const Cache& c, int NQ);
cudaError_t launch_tree_tc(const TreeArgs& a, cudaStream_t s);
cudaError_t launch_tree_rows(const TreeArgs& a, cudaStream_t s);

}  // namespace tree
}  // namespace cdsl
