// kv_pages.cu -- which sequence has which pages: cdsl_kv_fork, cdsl_kv_resize, cdsl_kv_compact.
//
// A pool's state is a page table and a count of holders for every page (0: free). Every call makes new tables
// and counts from old ones, so that nothing depends on the order of threads: the counts are sums of whole numbers, and
// free pages are dealt lowest first, in order of sequences and columns. One block plans, as a decoding step's tables
// are small and all of it hangs on prefix sums over the pages; the rows to be copied are a list for a second kernel,
// over the whole device, whose blocks are scheduled beside the plan. Bound by the latency of the plan on small calls (a fork of
// 32 beams 8.4 us, a resize 5.0 to 5.6, a compaction's plan 5.3 to 6.4, by ncu) and by HBM where many layers' pages move: a third of a pool
// in 8 layers, 700 MB, 113 us, 91 % of the copy bandwidth with the plan apart (119 to 122 as calls; parts of 4 KB a warp 124).
#include <cuda.h>

#include <algorithm>
#include <climits>

#include "kernels.h"
#include "tree.cuh"
#include "tree_host.h"

namespace cdsl {
namespace tree {
namespace {

constexpr int kPlan = 1024;                    // threads of the planning block
constexpr int kCopy = 256;

struct Move { int from, to, rows, pad; };      // pages, and how many rows of each head

struct PagesArgs {
  Cache c;
  const int32_t* refs;
  const int32_t* src;                          // fork: the sequence that each new one comes from
  const int32_t* lens;                         // fork: cached tokens; resize: slots
  int new_batch;
  int32_t* new_table;
  int32_t* new_lens;
  int32_t* new_refs;
  int32_t* page_map;
  int32_t* n_live;
  int32_t* status;
  // workspace
  int* n_moves;
  Move* moves;
  int32_t* free_pages;
  int32_t* entries;                            // compact: of each page, in the free pages' place
};

// Sum of x over the block's threads before this one, and over all.
__device__ __forceinline__ int scan(int x, int* all) {
  __shared__ int s_sum[kPlan / 32], s_all;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
  if (warp == 0) {
    const int w = s_sum[lane];
    int t = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += y;
    }
    s_sum[lane] = t - w;
    if (lane == 31) s_all = t;
  }
  __syncthreads();
  const int before = s_sum[warp] + upto - x;
  *all = s_all;
  __syncthreads();                             // (the sums may be overwritten)
  return before;
}

// The `want` lowest pages whose count is 0 (fewer where there are no more: the number comes back) to `to`. The counts are
// read from L2, where the block's atomics are.
__device__ int find_free(const int32_t* refs, int n_pages, int want, int32_t* to) {
  int found = 0;
  for (int p0 = 0; p0 < n_pages && found < want; p0 += 4 * kPlan) {
    const int p = p0 + 4 * (int)threadIdx.x;
    int free[4], n = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      free[e] = p + e < n_pages && __ldcg(refs + p + e) == 0;
      n += free[e];
    }
    int at = found + scan(n, &all);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (free[e]) {
        if (at < want) to[at] = p + e;
        ++at;
      }
    found += all;
  }
  __syncthreads();
  return min(found, want);
}

__device__ __forceinline__ bool is_page(const Cache& c, int page) { return (unsigned)page < (unsigned)c.n_pages; }

// The counts without the table's entries, to new_refs (the holders beyond it), and whether one of them is below 0, to the whole
// block: then the counts are not the table's, which settle() latches, and has them count from 0. Every entry is taken off
// before any is kept, so that nothing depends on which thread comes first.
__device__ bool take_off(const PagesArgs& a) {
  constexpr int AHEAD = 4;                     // entries whose counts are waited for together
  const Cache& c = a.c;
  const int tid = threadIdx.x;
  bool low = false;
  for (int p = tid; p < c.n_pages; p += kPlan) {
    const int r = a.refs[p];
    low = low || r < 0;
    if (a.new_refs != a.refs) a.new_refs[p] = r;
  }
  __syncthreads();
  const long long n = (long long)c.batch * c.max_pages;
  for (long long i0 = tid; i0 < n; i0 += AHEAD * kPlan) {
    int page[AHEAD], had[AHEAD];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) page[e] = i0 + e * kPlan < n ? c.table[i0 + e * kPlan] : -1;
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) had[e] = is_page(c, page[e]) ? atomicSub(a.new_refs + page[e], 1) : 1;
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) low = low || had[e] < 1;
  }
  return __syncthreads_or(low);
}
__device__ void settle(const PagesArgs& a) {
  if (threadIdx.x == 0) set_status(a.status, CDSL_EINVAL);
  for (int p = threadIdx.x; p < a.c.n_pages; p += kPlan)
    if (__ldcg(a.new_refs + p) < 0) a.new_refs[p] = 0;
  __syncthreads();
}

__global__ void __launch_bounds__(kPlan) k_fork_plan(PagesArgs a) {
  __shared__ int s_first[CDSL_TREE_MAX_BATCH]; // the first of a sequence's children
  __shared__ int s_free[CDSL_TREE_MAX_BATCH];
  const Cache& c = a.c;
  const int tid = threadIdx.x, P = 1 << c.page_shift;
  pdl_wait();
  pdl_launch_dependents();
  for (int b = tid; b < c.batch; b += kPlan) s_first[b] = INT_MAX;
  __syncthreads();
  // a new sequence per thread
  int parent = -1, len = 0;
  if (tid < a.new_batch) {
    parent = a.src[tid];
    if ((unsigned)parent >= (unsigned)c.batch) {
      set_status(a.status, CDSL_ERANGE);
      parent = -1;
    } else {
      const long long most = (long long)c.max_pages << c.page_shift;
      len = a.lens[parent];
      if (len < 0 || len > most) {
        set_status(a.status, CDSL_ERANGE);
        len = len < 0 ? 0 : (int)most;
      }
      atomicMin(&s_first[parent], tid);
    }
  }
  // every old sequence gives its pages up
  const bool low = take_off(a);
  // its last page, if partly filled, is the first child's if nobody else has it, and copied for others
  const int full = len >> c.page_shift, rest = len & (P - 1);
  int part = rest ? c.table[(size_t)parent * c.max_pages + full] : -1;
  const bool is = is_page(c, part);
  // (one entry, and the count that belongs to it)
  const bool copies = is && (s_first[parent] != tid || a.refs[part] != 1 || __ldcg(a.new_refs + part) != 0);
  __syncthreads();
  if (low) settle(a);
  if (is) atomicAdd(a.new_refs + part, 1);     // (kept; or, until the free pages are dealt, read from)
  if (rest && !is) {
    set_status(a.status, CDSL_ERANGE);
    part = -1;
  }
  // whole pages are shared
  for (long long i = tid; i < (long long)a.new_batch * c.max_pages; i += kPlan) {
    const int b = (int)(i / c.max_pages), col = (int)(i % c.max_pages);
    const int from = a.src[b];
    int page = -1;
    if ((unsigned)from < (unsigned)c.batch) {
      const long long most = (long long)c.max_pages << c.page_shift;
      const int n = (int)min((long long)max(a.lens[from], 0), most) >> c.page_shift;
      if (col < n) {
        page = c.table[(size_t)from * c.max_pages + col];
        if (is_page(c, page)) atomicAdd(a.new_refs + page, 1);
        else {
          set_status(a.status, CDSL_ERANGE);
          page = -1;
        }
      }
    }
    a.new_table[i] = page;
  }
  int want;
  const int rank = scan(copies, &want);        // (a block barrier: the counts and the table are written)
  const int found = find_free(a.new_refs, c.n_pages, want, s_free);
  if (copies) {
    atomicSub(a.new_refs + part, 1);
    int to = -1;
    if (rank < found) {
      to = s_free[rank];
      atomicAdd(a.new_refs + to, 1);
      a.moves[rank] = {part, to, rest, 0};
    } else {
      set_status(a.status, CDSL_ENOMEM);
    }
    part = to;
  }
  if (rest) a.new_table[(size_t)tid * c.max_pages + full] = part;
  if (tid < a.new_batch) a.new_lens[tid] = rest && part < 0 ? full << c.page_shift : len;
  if (tid == 0) *a.n_moves = found;
}

__global__ void __launch_bounds__(kPlan) k_resize(PagesArgs a) {
  const Cache& c = a.c;
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  const long long n = (long long)c.batch * c.max_pages;
  const auto columns = [&](int b) {            // that sequence b is to have
    const long long most = (long long)c.max_pages << c.page_shift;
    const long long s = min(max((long long)a.lens[b], 0ll), most);
    return (int)((s + (1 << c.page_shift) - 1) >> c.page_shift);
  };
  for (int b = tid; b < c.batch; b += kPlan)
    if (a.lens[b] < 0 || a.lens[b] > (long long)c.max_pages << c.page_shift) set_status(a.status, CDSL_ERANGE);
  if (take_off(a)) settle(a);
  int missing = 0;
  for (long long i = tid; i < n; i += kPlan) { // (in its place each entry is read before it is written)
    int page = c.table[i];
    const bool is = is_page(c, page);
    if (!is && page != -1) set_status(a.status, CDSL_ERANGE);
    if (i % c.max_pages >= columns((int)(i / c.max_pages))) {
      page = -1;
    } else if (is) {
      atomicAdd(a.new_refs + page, 1);         // (kept)
    } else {
      ++missing;
      page = -2;
    }
    a.new_table[i] = page;
  }
  int want;
  scan(missing, &want);                        // (a block barrier)
  const int found = find_free(a.new_refs, c.n_pages, want, a.free_pages);
  if (found < want && tid == 0) set_status(a.status, CDSL_ENOMEM);
  int before = 0;
  for (long long i0 = 0; i0 < n && before < want; i0 += kPlan) {
    const long long i = i0 + tid;
    const bool miss = i < n && a.new_table[i] == -2;
    int all;
    const int at = before + scan(miss, &all);
    if (miss) {
      const int page = at < found ? a.free_pages[at] : -1;
      a.new_table[i] = page;
      if (page >= 0) atomicAdd(a.new_refs + page, 1);
    }
    before += all;
  }
}

__global__ void __launch_bounds__(kPlan) k_compact_plan(PagesArgs a) {
  const Cache& c = a.c;
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  int mine = 0, live;
  bool low = false;                            // counts that are not the table's
  for (int p = tid; p < c.n_pages; p += kPlan) {
    const int r = a.refs[p];
    low = low || r < 0;
    mine += r > 0;
    a.entries[p] = 0;
  }
  scan(mine, &live);
  // the k-th hole below `live`, and the k-th page in use from there on, belong together
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += kPlan) {
    const int p = p0 + tid;
    const int r = p < c.n_pages ? a.refs[p] : 0;
    const bool front = p < live, hole = front && r <= 0, mover = !front && r > 0;
    int h, m;
    const int hk = holes + scan(hole, &h), mk = movers + scan(mover, &m);
    if (hole) a.moves[hk].to = p;
    if (mover) a.moves[mk].from = p;
    holes += h;
    movers += m;
    if (p < c.n_pages) {
      a.page_map[p] = r > 0 ? p : -1;          // (of movers below)
      a.new_refs[p] = max(r, 0);
    }
  }
  __syncthreads();
  for (int k = tid; k < movers; k += kPlan) {
    Move& m = a.moves[k];
    m.rows = 1 << c.page_shift;
    const int r = a.new_refs[m.from];
    a.page_map[m.from] = m.to;
    a.new_refs[m.to] = r;
    a.new_refs[m.from] = 0;
  }
  __syncthreads();
  for (long long i = tid; i < (long long)c.batch * c.max_pages; i += kPlan) {
    const int page = c.table[i];
    const bool is = is_page(c, page);
    if (!is && page != -1) set_status(a.status, CDSL_ERANGE);
    const int to = is ? a.page_map[page] : -1; // (-1 of a page whose count is 0)
    if (is) low = low || atomicAdd(a.entries + page, 1) >= (to < 0 ? 0 : a.new_refs[to]);
    a.new_table[i] = to;
  }
  if (__syncthreads_or(low) && tid == 0) set_status(a.status, CDSL_EINVAL);
  if (tid == 0) {
    *a.n_moves = movers;
    *a.n_live = live;
  }
}

// Copies the listed pages' rows in every layer. A warp has a part of at most kPart bytes of one head's codes or its scales,
// kAhead loads before their stores. Sources and targets are apart: a target was free, a source was not.
constexpr int kAhead = 8, kPart = 2 * kAhead * 32 * 16;
__global__ void __launch_bounds__(kCopy) k_copy_pages(Cache c, const int* n_moves, const Move* moves) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int page_bytes = c.row << c.page_shift, parts = (page_bytes + kPart - 1) / kPart;   // of a head's codes
  const int heads = c.n_layers * 2 * c.kvh;
  const long long items = (long long)*n_moves * heads * (parts + 1);
  const long long step = (long long)gridDim.x * (kCopy / 32);
  for (long long i = (long long)blockIdx.x * (kCopy / 32) + (threadIdx.x >> 5); i < items; i += step) {
    const int part = (int)(i % (parts + 1));
    const long long j = i / (parts + 1);
    const int h = (int)(j % heads);
    const Move m = moves[j / heads];
    const int layer = h / (2 * c.kvh), kv = h / c.kvh % 2, head = h % c.kvh;
    const size_t from = row_of(c, layer, m.from, kv, head, 0), to = row_of(c, layer, m.to, kv, head, 0);
    const bool codes = part < parts;
    const size_t pitch = codes ? c.row : c.srow;
    // (in whole 16 bytes: a page's scales have so many)
    const int bytes = m.rows * (int)pitch, first = codes ? part * kPart : 0, end = codes ? min(bytes, first + kPart) : bytes;
    const uint8_t* const base = codes ? c.pool : c.scale;
    const uint4* const x = reinterpret_cast<const uint4*>(base + from * pitch);
    uint4* const y = reinterpret_cast<uint4*>(const_cast<uint8_t*>(base) + to * pitch);
    for (int q0 = first / 16 + lane; q0 * 16 < end; q0 += 32 * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int e = 0; e < kAhead; ++e)
        if ((q0 + 32 * e) * 16 < end) v[e] = x[q0 + 32 * e];
#pragma unroll
      for (int e = 0; e < kAhead; ++e)
        if ((q0 + 32 * e) * 16 < end) y[q0 + 32 * e] = v[e];
    }
  }
}

cudaError_t launch_copies(const Cache& c, const PagesArgs& a, long long most, cudaStream_t s) {
  const long long parts = ((c.row << c.page_shift) + kPart - 1) / kPart + 1;
  const long long warps = most * c.n_layers * 2 * c.kvh * parts;
  const int blocks = (int)std::min<long long>((warps + kCopy / 32 - 1) / (kCopy / 32), kPlanSMs * 16);
  return launch_pdl(k_copy_pages, dim3(blocks), dim3(kCopy), 0, s, c, (const int*)a.n_moves, (const Move*)a.moves);
}

// Workspace: the moves' number, the moves, the free pages (or the entries of each).
struct Sizes { size_t moves, free_pages, bytes; };
Sizes sizes_of(const Cache& c, int new_batch) {
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  Sizes z;
  z.moves = 256;
  z.free_pages = z.moves + up(sizeof(Move) * std::max<size_t>(c.n_pages, new_batch));
  z.bytes = z.free_pages + up(sizeof(int32_t) * c.n_pages);
  return z;
}

bool workspace(const Check& ck, PagesArgs* a, int new_batch, void* ws, size_t bytes, int* code) {
  const Sizes z = sizes_of(a->c, new_batch);
  *code = bytes < z.bytes ? CDSL_ENOMEM : CDSL_EINVAL;
  if (!ws || !ck.aligned(ws, 256) || bytes < z.bytes) {
    ck.fail("the workspace must be 256-byte aligned and hold cdsl_kv_pages_workspace bytes", *code);
    return false;
  }
  char* const p = static_cast<char*>(ws);
  a->n_moves = reinterpret_cast<int*>(p);
  a->moves = reinterpret_cast<Move*>(p + z.moves);
  a->free_pages = a->entries = reinterpret_cast<int32_t*>(p + z.free_pages);
  return true;
}

bool table_ok(const Check& ck, const Cache& c) {
  if ((long long)c.batch * c.max_pages >= (1LL << 30)) return ck.no("the page table is beyond the limit (2^30 entries)");
  return true;
}

}  // namespace
}  // namespace tree
}  // namespace cdsl

using namespace cdsl;
using namespace cdsl::tree;

extern "C" int32_t cdsl_kv_pages_workspace(const cdsl_kv_cache* cache, int32_t new_batch, size_t* bytes) {
  Check ck("cdsl_kv_pages_workspace");
  Cache c;
  if (!ck.cache(cache, &c, false)) return CDSL_EINVAL;
  if (new_batch < 1 || new_batch > CDSL_TREE_MAX_BATCH) return ck.fail("new_batch must be 1 .. 1024");
  if (!bytes) return ck.fail("bytes is NULL");
  *bytes = sizes_of(c, new_batch).bytes;
  return CDSL_OK;
}

extern "C" int32_t cdsl_kv_fork(const cdsl_kv_cache* cache, const int32_t* d_refs, const int32_t* d_src,
                                const int32_t* d_lens, int32_t new_batch, int32_t* d_new_table, int32_t* d_new_lens,
                                int32_t* d_new_refs, void* d_workspace, size_t workspace_bytes, int32_t* d_status,
                                void* stream) {
  Check ck("cdsl_kv_fork");
  PagesArgs a = {};
  int code;
  if (!ck.cache(cache, &a.c) || !table_ok(ck, a.c)) return CDSL_EINVAL;
  if (new_batch < 1 || new_batch > CDSL_TREE_MAX_BATCH) return ck.fail("new_batch must be 1 .. 1024");
  if ((long long)new_batch * a.c.max_pages >= (1LL << 30)) return ck.fail("the new page table is beyond the limit (2^30 entries)");
  if (!d_refs || !d_src || !d_lens || !d_new_table || !d_new_lens || !d_new_refs) return ck.fail("a required pointer is NULL");
  if (d_new_refs == d_refs || d_new_table == a.c.table || d_new_lens == d_lens || d_new_lens == d_src)
    return ck.fail("the new table, lengths and counts must not be the old ones");
  if (!workspace(ck, &a, new_batch, d_workspace, workspace_bytes, &code)) return code;
  a.refs = d_refs; a.src = d_src; a.lens = d_lens; a.new_batch = new_batch;
  a.new_table = d_new_table; a.new_lens = d_new_lens; a.new_refs = d_new_refs;
  a.status = d_status;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (const cudaError_t e = launch_pdl(k_fork_plan, dim3(1), dim3(kPlan), 0, s, a)) return ck.launched(e);
  return ck.launched(launch_copies(a.c, a, new_batch, s));
}

extern "C" int32_t cdsl_kv_resize(const cdsl_kv_cache* cache, const int32_t* d_refs, const int32_t* d_slots,
                                  int32_t* d_new_table, int32_t* d_new_refs, void* d_workspace, size_t workspace_bytes,
                                  int32_t* d_status, void* stream) {
  Check ck("cdsl_kv_resize");
  PagesArgs a = {};
  int code;
  if (!ck.cache(cache, &a.c) || !table_ok(ck, a.c)) return CDSL_EINVAL;
  if (!d_refs || !d_slots || !d_new_table || !d_new_refs) return ck.fail("a required pointer is NULL");
  if (!workspace(ck, &a, a.c.batch, d_workspace, workspace_bytes, &code)) return code;
  a.refs = d_refs; a.lens = d_slots;
  a.new_table = d_new_table; a.new_refs = d_new_refs;
  a.status = d_status;
  return ck.launched(launch_pdl(k_resize, dim3(1), dim3(kPlan), 0, static_cast<cudaStream_t>(stream), a));
}

extern "C" int32_t cdsl_kv_compact(const cdsl_kv_cache* cache, const int32_t* d_refs, int32_t* d_new_table,
                                   int32_t* d_new_refs, int32_t* d_page_map, int32_t* d_n_live, void* d_workspace,
                                   size_t workspace_bytes, int32_t* d_status, void* stream) {
  Check ck("cdsl_kv_compact");
  PagesArgs a = {};
  int code;
  if (!ck.cache(cache, &a.c) || !table_ok(ck, a.c)) return CDSL_EINVAL;
  if (!d_refs || !d_new_table || !d_new_refs || !d_page_map || !d_n_live) return ck.fail("a required pointer is NULL");
  if (d_page_map == d_refs || d_page_map == d_new_refs) return ck.fail("the page map must not be the counts");
  if (!workspace(ck, &a, a.c.batch, d_workspace, workspace_bytes, &code)) return code;
  a.refs = d_refs;
  a.new_table = d_new_table; a.new_refs = d_new_refs; a.page_map = d_page_map; a.n_live = d_n_live;
  a.status = d_status;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (const cudaError_t e = launch_pdl(k_compact_plan, dim3(1), dim3(kPlan), 0, s, a)) return ck.launched(e);
  return ck.launched(launch_copies(a.c, a, a.c.n_pages, s));
}
