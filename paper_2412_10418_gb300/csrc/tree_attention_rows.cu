// tree_attention_rows.cu -- cdsl_tree_attention of bf16 queries with more than 32 query vectors per K/V
// head (a 4-bit cache: more than 16), on the 5th-generation tensor cores: query vectors are the MMA's M = 128 rows.
//
//   S = Q K^T   M = 128 vectors, N = 128 slots, K = head_dim    Q and K tiles K-major in shared memory
//   O = P V     M = 128 vectors, N = head_dim, K = 128 slots    P in TMEM over S, V tile MN-major as it lands
//
// S of an e4m3 cache is taken as in tree_attention_tc.cu, from the codes and two e4m3 planes of Q. P V is not:
// turning a pair of probabilities into two e4m3 planes takes 14 cycles of a quarter of an SM (four
// conversions at 2 or 4 and a difference, measured), 7 a score, where its exponential takes 4. Here the chunk's V is
// turned into fp16 once for all rows instead, with its power-of-two scales multiplied in relative to a reference (the
// largest of the first chunk, raised when one passes it by more than 2^kVRoom), and P into
// fp16 by one conversion a pair: 2^-12 of itself down to 2^-21 of a row's reference, and 2^-32 of that below, which is nothing
// beside a V of much the same size. V is exact for scales down to 2^-kVBelow of the reference. From a chunk with a
// smaller one on, to the end of what the block has of the item, V is in bf16, exact over fp32's range, and P in two bf16 planes
// (2^-17), as a bf16 cache's are with its V as it is: the slot with that V may be the one whose weight is the reference, and those
// below 2^-32 of it, chunks later, all that the row has. (Of that chunk alone, as it was: 1,000 tokens of 2^-33 each behind one
// with a V of 2^-40 counted for nothing.)
//
// A softmax thread has a vector (a TMEM lane) and walks all the chunk's slots (columns): maximum, reference,
// probabilities and their sum are its own, no value crosses lanes and no barrier stands in a chunk, whatever
// the number of vectors. What changes from slot to slot (K's scales, masks) is read from shared memory. That
// costs the same for 33 vectors as for 128, and reads K and V once for all of them.
//
// Two groups of four softmax warps take alternate chunks, so that one's exponentials run beside the other's
// maxima; S, which P then overwrites, has three buffers in TMEM, so that neither waits for its next one (with two,
// and an O for each group, half of a chunk's time was waiting). O is one chain over the chunks: fp16's range
// leaves P exact enough under a reference that is raised only when a maximum passes it by more than 2^kMargin,
// which after the first chunk is rare; then the thread multiplies its O. A row's reference goes from chunk to chunk, and
// so from group to group, through shared memory. (O started anew in every chunk and was added up in registers before:
// eight more warps, and a chain of waits through them that held a chunk to 3,500 cycles.) Four warps convert V, one
// loads, one issues MMAs, one turns scale bytes into factors. A bf16 cache has shared memory for two stages only:
// there K and the scale bytes are loaded a chunk ahead of V, or S would wait for the V of a chunk before (36 vectors,
// 8 sequences of 16,384 tokens, 8 heads: 191 -> 123 us, 125 now; with three stages of e4m3 it loses 5 %).
//
// Between two items the next one's queries and masks are staged as soon as the last S has read this one's, beside
// the last P V (33 trees of 48 after 115 tokens: 7 % less).
//
// Measured: 8 trees of 25 nodes, 100 vectors a K/V head, up to 32,768 tokens of 8 heads of 128 in e4m3: 150 us, 400
// TFLOP/s, 40 % of the copy bandwidth (16,384 tokens each 111 us; with V's scales far apart from the first chunk on 174). A
// chunk takes 3,000 cycles, of which its MMAs need 1,024; a softmax thread spends 1,500 on the maxima, 2,000 on the
// probabilities and the rest waiting. What holds it is latency (166 cycles a TMEM load), shared memory, which operands,
// conversion and factors keep busy for 1,900, and instruction fetches: the roles together are about as large as the instruction cache, and the same kernel took 150 to 190 us
// with the sizes of its loops (0.4 to 1.6 million misses a call), which are kept rolled for that. A third group of
// softmax warps: 177 us. At 36 vectors 8 sequences of 16,384 take 99.5 us, two blocks of 32 on
// tree_attention_tc.cu 117. At 32, 70 there and 92 here. A block has 128 rows whatever it holds: 8 trees of 32 nodes of four
// heads each after 4096 tokens take 50.5 us, of 33 nodes, whose 132 vectors take two blocks, 75.
//
// A 4-bit cache's rows land packed, and eight warps turn them into tiles with their scales multiplied in: K into bf16, in which
// a value is exact (4 bits of scale by 3 of code), with Q as it is; V as e4m3's is, into fp16 under a reference from
// 2^kVRoom4 above it to 2^-kVBelow4 below, and into bf16 from a chunk with smaller scales on (a group of zeros
// has 2^-120). A tile's dimensions are in the order in
// which a row's words give them (one of each of two groups in turn), so that a word is 16 bytes of it and takes no byte moves; Q is
// staged, and O written, in that order. V's factors come from the scaling warp. Measured: 8 trees of 25 nodes after up to 32,768
// tokens (243 MB): 152 to 160 us by inputs, where e4m3 takes 150; 8 sequences of 16,384 of 20 / 36 / 100
// vectors 97 / 102 / 115 (of 16: 70 by tree_attention_i4.cu). Of the 97, conversions are some 20, softmax 15, an empty
// pipeline 60 (20 of them whatever the length). Steps and trials, the trees among other calls: both conversions by four warps 174,
// loops unrolled twice 184, four times 236; eight warps 164; factors by the scaling warp 161; and one after another, from 174
// there: MMAs by an elected lane 172, factors by integer moves 167, stages loaded as they become free 163.
//
// Waits are bounded by a number of tries (wait_for): on expiry CDSL_ETIMEOUT is latched, the role winds down and the block
// frees its TMEM and exits.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "tree_attention.cuh"
#include "tree_tc.cuh"

namespace cdsl {
namespace tree {
namespace {

constexpr int kRows = 128;                     // query vectors per block
constexpr int kSoft = 2 * kRows;               // softmax threads: two groups
constexpr int kConv = 128;                     // threads that convert V, and as many K of 4 bits
constexpr int kConvWarp = kSoft / 32;          // warps: softmax, conversion, loading, MMAs, scales
constexpr float kMargin = 7.f;                 // base 2: probabilities are at most 2^kMargin of a reference, and
constexpr float kUp = 7.f;                     // stored times 2^kUp: below fp16's largest
constexpr int kBuf = 3;                        // S (then P) buffers in TMEM; O has the rest
constexpr int kVRoom = 6;                      // octaves that V's scales may pass their reference by: 448 * 2^6 in fp16,
constexpr int kVBelow = 15;                    // and lie below it: 2^-9 * 2^-15
// (So in fp16 V's scales lie within 21 octaves of one another, 4 bits: 16, and a probability of less than 2^-32, which is nothing
// there, leaves out 2^-11, or 2^-16, of what the reference's slot gives, each.) V of 4 bits is held 2^kVUp4 larger: a factor
// that is 2^-4 of a scale is a normal fp16 number down to 14 below.
constexpr int kVRoom4 = 4, kVBelow4 = 12, kVUp4 = 4;

template <int HD, int FORMAT>
struct Cfg {
  static constexpr bool F8 = FORMAT == kF8, I4 = FORMAT == kI4;
  static constexpr bool TURNED = FORMAT != kBF16;          // V is turned into 16 bits
  static constexpr int CONV = I4 ? 2 * kConv : kConv, THREADS = kSoft + CONV + 96;
  static constexpr int PRODUCER = kConvWarp + CONV / 32, ISSUER = PRODUCER + 1, SCALER = PRODUCER + 2;   // warps
  static constexpr int EB = F8 ? 1 : 2;                    // I4: of K's tile
  static constexpr int KROW = HD * EB;                     // bytes of a K or V row
  static constexpr int BW = KROW < 128 ? KROW : 128;       // of it per tile block
  static constexpr int NB = KROW / BW;
  static constexpr uint32_t BLOCK = kKeys * BW;
  static constexpr uint32_t TILE = NB * BLOCK;             // K or V of a chunk
  static constexpr int QP = F8 ? 2 : 1;
  static constexpr uint32_t Q_PLANE = kRows * KROW;
  // e4m3 and 4 bits: V of two chunks in fp16, in blocks of 64 dimensions
  static constexpr uint32_t H_BLOCK = kKeys * 128, H_TILE = TURNED ? HD / 64 * H_BLOCK : 0;
  static constexpr uint32_t H_OFF = QP * Q_PLANE;
  // 4 bits: K of two chunks in bf16
  static constexpr uint32_t KT_OFF = H_OFF + 2 * H_TILE;
  static constexpr uint32_t KV_OFF = KT_OFF + (I4 ? 2 * TILE : 0);
  // the ring: K's and V's rows; 4 bits: with their scales
  static constexpr int RB = HD / 2, SB = HD / kGroup * 2;
  static constexpr uint32_t PACKED = kKeys * (RB + SB), HALF = I4 ? PACKED : TILE;
  static constexpr int FIT = (208 * 1024 - KV_OFF) / (2 * HALF);
  static constexpr int NST = FIT > 4 ? 4 : FIT;
  static_assert(NST >= 2, "stages");
  static constexpr uint32_t SCALE_OFF = KV_OFF + NST * 2 * HALF;
  // K's scale of each slot, and V's, e4m3: relative to its reference (0: nothing, or not finite). 4 bits: V's by two groups,
  // the two factors of its fma (0: the same)
  static constexpr uint32_t FACTOR_OFF = SCALE_OFF + (I4 ? 0 : NST * 2 * kKeys);
  static constexpr uint32_t FACTORS = I4 ? kKeys * HD / kGroup * 4 : 2 * kKeys * 4;
  static constexpr uint32_t PLAN_OFF = FACTOR_OFF + NST * FACTORS;
  static constexpr size_t smem(int batch) { return 1024 + PLAN_OFF + plan_bytes(batch); }
};

constexpr int kLoadTries = 1 << 24;            // of the loading warp's, some 0.1 us each, without a stage becoming free

// Has the phase of `parity` completed? (An answer at once; the whole warp's.)
__device__ __forceinline__ bool is_done(uint64_t* m, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(tc::smem_u32(m)), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, ok != 0);
}

// The loading warp of a 4-bit cache: plain bulk copies, a page piece's codes and scales each, scales behind the codes. K's and V's
// stages are filled as either becomes free, since K is turned as many chunks ahead as S has buffers, V when P V is at it: with
// K's loads behind V's, 8 sequences of 16,384 with 20 vectors took 100 us for 98. (V's scales loaded ahead of both, into a ring
// of four of their own: 107.)
template <int HD, int NST>
__device__ __forceinline__ void load_packed(const TreeArgs& a, const int* first, int begin, int end, uint8_t* ring,
                                            uint32_t* s_pieces, uint64_t* k_full, uint64_t* v_full, uint64_t* k_empty,
                                            uint64_t* v_empty) {
  using C = Cfg<HD, kI4>;
  const Cache& c = a.c;
  const int lane = threadIdx.x & 31, P = 1 << c.page_shift;
  const int rows = min(P, kKeys), pieces = kKeys / rows, n = end - begin;   // (a unit is a chunk)
  const size_t page_rows = (size_t)2 * c.kvh << c.page_shift, layer_row = row_of(c, a.layer, 0, 0, 0, 0);
  struct Chunk {
    int page, row;                             // this lane's piece (-1: none), and K's row in the page
  };
  Segment s = {};
  int ch = 0, unit = begin;
  const auto look = [&] {                      // the run's next chunk
    if (unit == begin || ch + 1 == s.c1) {
      s = segment_at(a, first, unit, end);
      ch = s.c0;
    } else {
      ++ch;
    }
    ++unit;
    const int slot = ch * kKeys + lane * rows;
    Chunk x = {-1, (s.h << c.page_shift) + (slot & (P - 1))};
    if (lane < pieces && slot < s.keys) {
      x.page = page_of(c, s.b, slot);
      if (x.page < 0) set_status(a.status, CDSL_ERANGE);
    }
    return x;
  };
  const auto load = [&](const Chunk& x, int st, int kv) {
    uint64_t* const full = kv ? &v_full[st] : &k_full[st];
    const uint32_t live = __ballot_sync(0xffffffffu, x.page >= 0);
    if (lane == 0) {
      if (kv) s_pieces[st] = live;
      tc::mbar_expect_tx(full, __popc(live) * rows * (C::RB + C::SB));
    }
    __syncwarp();
    if (x.page >= 0) {
      const size_t row = layer_row + x.page * page_rows + x.row + (kv ? (size_t)c.kvh << c.page_shift : 0);
      uint8_t* const to = ring + (st * 2 + kv) * C::PACKED;
      tc::bulk_load(to + lane * rows * C::RB, c.pool + row * C::RB, rows * C::RB, full);
      tc::bulk_load(to + kKeys * C::RB + lane * rows * C::SB, c.scale + row * C::SB, rows * C::SB, full);
    }
  };
  Chunk chunks[NST];                           // whose V is to come
  int ik = 0, iv = 0, tries = 0;               // chunks whose K and V have been asked for
  Chunk next = {};
  if (n > 0) next = look();
#pragma unroll 1
  while (iv < n) {
    bool moved = false;
    if (ik < n && ik - iv < NST && is_done(&k_empty[ik % NST], parity(ik, NST) ^ 1)) {
      load(next, ik % NST, 0);
#pragma unroll
      for (int i = 0; i < NST; ++i)
        if (i == ik % NST) chunks[i] = next;
      if (++ik < n) next = look();
      moved = true;
    }
    if (iv < ik && is_done(&v_empty[iv % NST], parity(iv, NST) ^ 1)) {
      Chunk x = chunks[0];
#pragma unroll
      for (int i = 1; i < NST; ++i)
        if (i == iv % NST) x = chunks[i];
      load(x, iv % NST, 1);
      ++iv;
      moved = true;
    }
    if (moved) {
      tries = 0;
    } else {
      if (++tries > kLoadTries) {
        set_status(a.status, CDSL_ETIMEOUT);
        break;
      }
      __nanosleep(20);
    }
  }
  // where a role gave up, nothing may have waited for the copies
  if (iv < n) {
#pragma unroll 1
    for (int i = max(0, ik - NST); i < ik; ++i) wait_for(&k_full[i % NST], parity(i, NST), a.status);
#pragma unroll 1
    for (int i = max(0, iv - NST); i < iv; ++i) wait_for(&v_full[i % NST], parity(i, NST), a.status);
  }
}

// 4-bit code I of both halves of w, times their scales, exactly: (1024 + 16 (code + 8)) scale / 16 - 72 scale in fp16, of mask =
// 0x00f000f0.
template <int I>
__device__ __forceinline__ uint32_t value_f16(uint32_t w, uint32_t mask, uint32_t s16, uint32_t m72) {
  const uint32_t t = I == 0 ? w << 4 : w >> (4 * I - 4);
  const uint32_t x = and_xor(t, mask, 0x64806480u);
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(s16), "r"(m72));
  return d;
}

// MMAs of a warp that is at one place, of which an elected lane issues them: the operands, which the compiler knows to be the
// warp's (shuffled from one lane), stay in uniform registers. Issued by a lane on a branch of its own each took 80 cycles, 120
// beside the other roles, where a tensor core takes 64.
template <bool F8>
__device__ __forceinline__ void warp_umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  if constexpr (F8)
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}
__device__ __forceinline__ void warp_umma_tmem_a(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void warp_commit(uint64_t* mbar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(tc::smem_u32(mbar))
      : "memory");
}

template <int HD, int FORMAT>
__global__ void __launch_bounds__((Cfg<HD, FORMAT>::THREADS), 1)
    k_tree_rows(TreeArgs a, const __grid_constant__ CUtensorMap map) {
  using C = Cfg<HD, FORMAT>;
  constexpr bool F8 = C::F8, I4 = C::I4, TURNED = C::TURNED;
  constexpr int NST = C::NST, kProducer = C::PRODUCER, kIssuer = C::ISSUER, kScaler = C::SCALER;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const sm = smem_raw + ((1024 - (tc::smem_u32(smem_raw) & 1023)) & 1023);
  int* const s_first = reinterpret_cast<int*>(sm + C::PLAN_OFF);
  __shared__ __align__(8) uint64_t k_full[NST], v_full[NST], k_empty[NST], v_empty[NST];
  __shared__ __align__(8) uint64_t f_full[NST], f_empty[NST], h_full[2];
  __shared__ __align__(8) uint64_t s_full[kBuf], p_full[kBuf], r_full[kBuf], pv_done[2], q_full, done;
  __shared__ __align__(8) uint64_t kt_full[2], kt_empty[2];   // 4 bits: K's tiles
  __shared__ uint32_t s_tmem;
  __shared__ __align__(16) uint32_t s_valid[NST][4], s_nan[NST][4];   // slots that there are, whose V is not finite
  __shared__ int s_kind[NST], s_h_far[2];      // a chunk's: bit 0 has masks, 1 V's scales far apart (bf16: not 1); V's buffers'
  __shared__ int s_vref[NST], s_vstep[NST];    // V's reference in the chunk, and that of the chunk before less it
  __shared__ float s_qs[2][kRows];             // score factors, of this segment's queries and the next one's
  __shared__ int s_v;                          // V's reference at the end
  __shared__ float s_ref[kRows], s_l[2][kRows];   // the rows' references; the groups' sums
  __shared__ uint8_t s_bad[2][kRows];          // the query is not finite
  __shared__ uint32_t s_mask[2][kRows + 1][kWords];
  __shared__ uint32_t s_pieces[NST], s_masks[2];
  const Cache& c = a.c;
  const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // (the warp's, to the compiler)

  if (threadIdx.x == 0) {
    s_masks[0] = 0x00780078u;
    s_masks[1] = 0x00f000f0u;
    for (int i = 0; i < NST; ++i) {
      tc::mbar_init(&k_full[i], 1);
      tc::mbar_init(&v_full[i], 1);
      tc::mbar_init(&k_empty[i], I4 ? kConv : F8 ? 1 : 2);   // (the scale bytes' reader arrives where they came)
      tc::mbar_init(&v_empty[i], TURNED ? kConv + 1 : 1);
      tc::mbar_init(&f_full[i], 32);
      tc::mbar_init(&f_empty[i], kRows);
    }
    // (P and references by buffers of S: a warp can be at its group's next chunk, two on, before the others have
    // finished this one, but not at the chunk that takes the same buffer)
    for (int i = 0; i < kBuf; ++i) {
      tc::mbar_init(&s_full[i], 1);
      tc::mbar_init(&p_full[i], kRows);
      tc::mbar_init(&r_full[i], kRows);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&h_full[i], kConv);
      tc::mbar_init(&kt_full[i], kConv);
      tc::mbar_init(&kt_empty[i], 1);
      tc::mbar_init(&pv_done[i], 1);
    }
    tc::mbar_init(&q_full, kSoft);
    tc::mbar_init(&done, 1);
    tc::fence_mbar_init();
  }
  if (warp == kIssuer) tc::tmem_alloc(&s_tmem, 512);
  if (!I4 && warp == kProducer && lane == 0) tc::tma_prefetch_map(&map);
  pdl_wait();
  pdl_launch_dependents();
  tc::tc_fence_before();
  build_plan(a, s_first);                      // (ends in a block barrier)
  tc::tc_fence_after();
  const uint32_t tmem = s_tmem;
  if (blockIdx.x == 0) check_lens(a);
  const int total = s_first[c.batch], runs = runs_of(a, total);
  const int begin = (int)blockIdx.x < runs ? run_begin(blockIdx.x, total, runs) : 0;
  const int end = (int)blockIdx.x < runs ? run_begin(blockIdx.x + 1, total, runs) : 0;
  const uint32_t t_o = tmem + kBuf * kKeys;

  if (warp == kProducer) {
    if constexpr (I4)
      load_packed<HD, NST>(a, s_first, begin, end, sm + C::KV_OFF, s_pieces, k_full, v_full, k_empty, v_empty);
    else
      load_chunks<HD, F8, NST, !F8>(a, s_first, begin, end, map, sm + C::KV_OFF, sm + C::SCALE_OFF, s_pieces, k_full,
                                    v_full, k_empty, v_empty);
  } else if (warp == kIssuer) {
    // (the whole warp is here: see warp_umma)
    const auto uniform = [](uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); };
    const uint32_t tmem = uniform(s_tmem), t_o = tmem + kBuf * kKeys;
    constexpr uint32_t formats = F8 ? 0u : (1u << 7) | (1u << 10);
    constexpr uint32_t idesc = (1u << 4) | formats | (128u >> 4) << 24;
    constexpr uint32_t idesc_s = idesc | (uint32_t)(kKeys >> 3) << 17;
    // P V in 16 bits: fp16 (format 0) or bf16
    constexpr uint32_t idesc_half = (1u << 4) | (128u >> 4) << 24 | (uint32_t)(HD >> 3) << 17 | 1u << 16;
    constexpr uint32_t idesc_bf16 = idesc_half | (1u << 7) | (1u << 10);
    const uint32_t sbase = uniform(tc::smem_u32(sm));
    const uint64_t desc_q = tc::desc_rows(sbase, C::BW, 16);
    const uint64_t desc_k = tc::desc_rows(sbase + (I4 ? C::KT_OFF : C::KV_OFF), C::BW, 16);
    const uint64_t desc_v = TURNED ? tc::desc_rows(sbase + C::H_OFF, 128, C::H_BLOCK)
                               : tc::desc_rows(sbase + C::KV_OFF + C::TILE, C::BW, C::BLOCK);
    auto s_mma = [&](int i) {                // S of chunk i
      if (!__all_sync(0xffffffffu, I4 ? wait_for(&kt_full[i & 1], parity(i, 2), a.status)
                                      : wait_for(&k_full[i % NST], parity(i, NST), a.status)))
        return false;
      tc::tc_fence_after();
      const uint64_t k = desc_k + (I4 ? (uint32_t)(i & 1) * (C::TILE / 16) : (uint32_t)(i % NST) * (2 * C::TILE / 16));
#pragma unroll 1
      for (int p = C::QP - 1; p >= 0; --p)
#pragma unroll 1
        for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
          for (int x = 0; x < C::BW / 32; ++x) {
            const uint64_t q = desc_q + ((uint32_t)(p * C::Q_PLANE + nb * kRows * C::BW) / 16 + 2 * x);
            const uint64_t kk = k + (nb * C::BLOCK / 16 + 2 * x);
            const bool add = p < C::QP - 1 || nb + x > 0;
            warp_umma<F8>(tmem + i % kBuf * kKeys, q, kk, idesc_s, add);
          }
      warp_commit(&s_full[i % kBuf]);
      warp_commit(I4 ? &kt_empty[i & 1] : &k_empty[i % NST]);
      return true;
    };
    auto pv = [&](int i, bool add) {         // P V of chunk i
      if (!__all_sync(0xffffffffu, TURNED ? wait_for(&h_full[i & 1], parity(i, 2), a.status)
                                          : wait_for(&v_full[i % NST], parity(i, NST), a.status)))
        return false;
      const bool planes = !TURNED || uniform(s_h_far[i & 1]);
      if (!__all_sync(0xffffffffu, wait_for(&p_full[i % kBuf], parity(i, kBuf), a.status))) return false;
      tc::tc_fence_after();
      const uint64_t v = desc_v + (TURNED ? (uint32_t)(i & 1) * (C::H_TILE / 16) : (uint32_t)(i % NST) * (2 * C::TILE / 16));
      // 16 slots an MMA: 8 columns of P, 16 rows of 128 bytes of V. P of 32 slots lies in the columns that held
      // their S, bf16 hi then lo.
      const auto plane = [&](int p, uint32_t idesc, bool add) {
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          warp_umma_tmem_a(t_o, tmem + i % kBuf * kKeys + k / 2 * 32 + p * 16 + k % 2 * 8, v + k * (16 * 128 / 16), idesc,
                          add || k > 0);
      };
      if (!planes) {
        plane(0, idesc_half, add);
      } else {
#pragma unroll 1
        for (int p = 1; p >= 0; --p) plane(p, idesc_bf16, add || p < 1);
      }
      warp_commit(&pv_done[i & 1]);
      if (!TURNED) warp_commit(&v_empty[i % NST]);
      return true;
    };
    bool ok = true;
    int it = 0, seg = 0;                     // chunks of the segments before
    const int last = (int)uniform(end);
    for (int unit = (int)uniform(begin); unit < last && ok; ++seg) {
      const Segment s = segment_at(a, s_first, unit, last);
      const int n = (int)uniform(s.c1 - s.c0);
      ok = __all_sync(0xffffffffu, wait_for(&q_full, seg & 1, a.status));
      // S as far ahead as it has buffers; it overwrites a P after the P V that reads it, in order
      for (int i = 0; i < n + kBuf && ok; ++i) {
        if (i >= kBuf) ok = pv(it + i - kBuf, i > kBuf);
        if (ok && i < n) ok = s_mma(it + i);
      }
      it += n;
      unit += n;
    }
    warp_commit(&done);                  // what was issued completes before the block's memory goes
    wait_for(&done, 0, a.status);
  } else if (warp == kScaler) {
    // ------------------------------------------------------------------------- scale bytes to factors
    int it = 0;
    bool ok = true;
    for (int unit = begin; unit < end && ok;) {
      const Segment s = segment_at(a, s_first, unit, end);
      int vref = 0, vlow = 255;                // V's reference, and its smallest exponent so far (e4m3: of the lane's slots)
      for (int ch = s.c0; ch < s.c1 && ok; ++ch, ++it) {
        const int st = it % NST;
        ok = __all_sync(0xffffffffu, wait_for(TURNED ? &v_full[st] : &k_full[st], parity(it, NST), a.status) &&
                                         wait_for(&f_empty[st], parity(it, NST) ^ 1, a.status));
        if (!ok) break;
        if constexpr (I4) {
          // a lane has slots lane, lane + 32 ..: their scales, two groups a word, of whose exponents (bits 7 .. 14; all set: not
          // finite, to which 0x80 carries into bit 15) it takes the largest and the smallest (a negative scale's: below 0)
          constexpr int G2 = HD / kGroup / 2;
          const uint32_t* const from = reinterpret_cast<const uint32_t*>(sm + C::KV_OFF + (st * 2 + 1) * C::PACKED + kKeys * C::RB);
          const uint32_t pieces = s_pieces[st];
          const int before = vref;
          uint32_t z[4][G2], most = 0u, least = 0x7fff7fffu;
          bool there[4], nan[4], masks = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = 32 * e + lane, slot = ch * kKeys + row;
#pragma unroll
            for (int i = 0; i < G2; ++i) z[e][i] = from[row * G2 + i];
            const uint32_t x = z[e][0] & 0x7f807f80u, y = z[e][G2 - 1] & 0x7f807f80u;
            there[e] = slot < s.keys && pieces >> (row >> min(c.page_shift, 7)) & 1;
            nan[e] = there[e] && (((x + 0x00800080u) | (y + 0x00800080u)) & 0x80008000u) != 0;
            masks = masks || !there[e] || slot >= s.len || nan[e];
            if (there[e] && !nan[e]) {
              most = __vmaxu2(most, __vmaxu2(x, y));
              least = __vmins2(least, __vmins2(z[e][0], z[e][G2 - 1]));
            }
          }
          const int vmax = __reduce_max_sync(0xffffffffu, max(most >> 23, most >> 7 & 0xff));
          vlow = min(vlow, __reduce_min_sync(0xffffffffu, min((int)least >> 23, (int)(least << 16) >> 23)));
          masks = __any_sync(0xffffffffu, masks);
          if (vref == 0 || vmax > vref + kVRoom4) vref = vmax;
          const bool far = vlow < max(vref - kVBelow4, 1);
          uint32_t* const to = reinterpret_cast<uint32_t*>(sm + C::FACTOR_OFF + st * C::FACTORS) + lane * (2 * G2);
          const auto put = [&](auto factors) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t y[2 * G2];
#pragma unroll
              for (int i = 0; i < G2; ++i) factors(z[e][i], there[e] && !nan[e], &y[2 * i]);
              if constexpr (G2 == 2) *reinterpret_cast<uint4*>(to + e * (64 * G2)) = make_uint4(y[0], y[1], y[2], y[3]);
              else *reinterpret_cast<uint2*>(to + e * (64 * G2)) = make_uint2(y[0], y[1]);
            }
          };
          if (far) {
            const uint32_t rel = (uint32_t)min(max(254 + kVUp4 - vref, 1), 254) * 0x00800080u;   // 2^(kVUp4 - reference)
            put([&](uint32_t x, bool some, uint32_t* y) {
              y[0] = some ? mul_bf16x2(mul_bf16x2(x, rel), 0x3e003e00u) : 0u;   // 1 / 8
              y[1] = mul_bf16x2(y[0], 0xc340c340u);                             // -192
            });
          } else {
            // bf16 to fp16, 2^-4 of it: the exponents moved (3 at least is left of one, so that no half borrows of the other), then
            // all bits by three
            const uint32_t move = (uint32_t)(vref - 15) * (128u * 0x00010001u);
            put([&](uint32_t x, bool some, uint32_t* y) {
              y[0] = some ? (x - move) * 8u : 0u;
              const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&y[0]), __float2half2_rn(-1152.f));
              y[1] = *reinterpret_cast<const uint32_t*>(&h);
            });
          }
          if (masks || far)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t v = __ballot_sync(0xffffffffu, there[e]), w = __ballot_sync(0xffffffffu, nan[e]);
              if (lane == e) {
                s_valid[st][e] = v;
                s_nan[st][e] = w;
              }
            }
          if (lane == 0) {
            s_vref[st] = vref;
            s_vstep[st] = before ? before - vref : 0;
            s_kind[st] = masks | far << 1;
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&v_empty[st]);   // (the scales are read)
          tc::mbar_arrive(&f_full[st]);
          continue;
        }
        // a lane has slots 4 lane .. 4 lane + 3
        const int slot = ch * kKeys + 4 * lane;
        const bool piece = s_pieces[st] >> (4 * lane >> min(c.page_shift, 7)) & 1;
        const int n = piece ? min(max(s.keys - slot, 0), 4) : 0;   // of them that there are
        const int before = vref;
        float kf[4], vf[4];
        uint32_t nan = 0;
        bool far = false, masks = n < 4 || slot + 3 >= s.len;   // slots past the item's, without a page or of the tree
        const uint8_t* from = sm + C::SCALE_OFF + st * 2 * kKeys + 4 * lane;
        const uint32_t kb = *reinterpret_cast<const uint32_t*>(from), vb = *reinterpret_cast<const uint32_t*>(from + kKeys);
        int vmax = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = vb >> (8 * e) & 255;
          if (e < n && x != 255) vmax = max(vmax, x);
        }
        vmax = __reduce_max_sync(0xffffffffu, vmax);
        if (vref == 0 || vmax > vref + kVRoom) vref = vmax;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t k = kb >> (8 * e) & 255, v = vb >> (8 * e) & 255;
          const int x = F8 ? (int)v - vref + 127 : (int)v;
          kf[e] = e < n ? scale_value(k) : 1.f;
          vf[e] = e >= n || v == 255 || x < 1 ? 0.f : __uint_as_float((uint32_t)x << 23);
          nan |= (uint32_t)(e < n && v == 255) << e;
          masks = masks || (e < n && v == 255);
          if (F8 && e < n && v != 255 && v > 0) vlow = min(vlow, (int)v);
          far = far || (!F8 && e < n && v != 255 && v != 127);
        }
        if (F8) far = vlow < vref - kVBelow;
        far = __any_sync(0xffffffffu, far);
        masks = __any_sync(0xffffffffu, masks);
        if constexpr (!I4) {
          float* to = reinterpret_cast<float*>(sm + C::FACTOR_OFF) + st * 2 * kKeys + 4 * lane;
          *reinterpret_cast<float4*>(to) = make_float4(kf[0], kf[1], kf[2], kf[3]);
          *reinterpret_cast<float4*>(to + kKeys) = make_float4(vf[0], vf[1], vf[2], vf[3]);
        }
        uint32_t valid = ((1u << n) - 1) << (4 * (lane & 7));       // eight lanes a word
        nan <<= 4 * (lane & 7);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) {
          valid |= __shfl_xor_sync(0xffffffffu, valid, o);
          nan |= __shfl_xor_sync(0xffffffffu, nan, o);
        }
        if ((lane & 7) == 0) {
          s_valid[st][lane >> 3] = valid;
          s_nan[st][lane >> 3] = nan;
        }
        if (lane == 0) {
          s_vref[st] = TURNED ? vref : 127;
          s_vstep[st] = TURNED && before ? before - vref : 0;
          s_kind[st] = masks | far << 1;
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(TURNED ? &v_empty[st] : &k_empty[st]);   // (the scale bytes are read)
        if (!TURNED && __any_sync(0xffffffffu, n < 4))
          ok = __all_sync(0xffffffffu, wait_for(&v_full[st], parity(it, NST), a.status));
        if (!ok) break;
        if (!TURNED && n < 4) {                    // nothing of their V rows (page garbage, no copy) may reach the sums
#pragma unroll 1
          for (int e = n; e < 4; ++e) {
            uint8_t* v = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + (4 * lane + e) * C::BW;
#pragma unroll 1
            for (int x = 0; x < C::KROW; x += 16)
              *reinterpret_cast<uint4*>(v + x / C::BW * C::BLOCK + x % C::BW) = make_uint4(0u, 0u, 0u, 0u);
          }
          tc::fence_proxy_async();
        }
        tc::mbar_arrive(&f_full[st]);
      }
      unit += s.c1 - s.c0;
    }
    __syncwarp();
  } else if (warp < kConvWarp) {
    // ------------------------------------------------------------------------- softmax
    const int tid = threadIdx.x, grp = tid / kRows, r = tid % kRows, w4 = warp & 3;
    auto sync = [] { tc::named_barrier(1, kSoft); };
    const bool q_aligned = (reinterpret_cast<uintptr_t>(a.q) | (a.sq[0] | a.sq[1] | a.sq[2]) * 2) % 16 == 0;
    const bool o_aligned = (reinterpret_cast<uintptr_t>(a.out) | (a.so[0] | a.so[1] | a.so[2]) * 2) % 16 == 0;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    int it0 = 0, buf = 0;
    bool failed = false;
    const auto stage = [&](const Segment& s, int to) {   // a segment's queries and masks
      stage_queries<HD, kRows, F8, kSoft, true, I4>(a, s, tid, q_aligned, sm, [&](int v, const Vec&, float qs, bool bad) {
        s_qs[to][v] = v < s.nq ? qs : 0.f;
        s_bad[to][v] = bad;
      });
      stage_masks<kSoft>(a, s, s.qb * kRows / a.G, tid, s_mask[to]);
      tc::fence_proxy_async();
      tc::mbar_arrive(&q_full);
    };
    Segment s;
    if (begin < end) {
      s = segment_at(a, s_first, begin, end);
      stage(s, 0);
      sync();
    }
    for (int unit = begin; unit < end; buf ^= 1) {
      const int t0 = s.qb * kRows / a.G;       // the block's first node
      const float qs = s_qs[buf][r];
      const bool live = w4 * 32 < s.nq;        // (a warp's: its rows hold vectors)
      const uint32_t* const my_mask = s_mask[buf][r < s.nq ? vector_of(a, s.h, s.qb, r).t - t0 : 0];
      const int n = s.c1 - s.c0;
      float ref = -INFINITY, l = 0.f;          // the row's reference at the group's last chunk, and its sum
      int vref = 127;                          // V's reference in O
      for (int i = (it0 & 1) ^ grp; i < n && !failed; i += 2) {   // chunks it with it % 2 == grp
        const int it = it0 + i, st = it % NST;
        const uint32_t t_s = tmem + it % kBuf * kKeys + lanes;
        const float* const kf = reinterpret_cast<const float*>(sm + C::FACTOR_OFF) + st * 2 * kKeys;
        bool ok = wait_for(&f_full[st], parity(it, NST), a.status);
        ok = ok && wait_for(&s_full[it % kBuf], parity(it, kBuf), a.status);
        failed = !__all_sync(0xffffffffu, ok);   // (a warp gives up as one)
        tc::tc_fence_after();
        const int node0 = (s.c0 + i) * kKeys - s.len;
        auto word = [&](int w) -> uint32_t {   // slots 32 w .. 32 w + 31 that this row sees
          const int first = node0 + 32 * w;    // the tree's node in the first of them
          uint32_t x;
          if (first <= -32) x = ~0u;
          else if (first < 0) x = ((1u << -first) - 1) | my_mask[0] << -first;
          else if (first >= 32 * kWords) x = 0u;
          else x = __funnelshift_r(my_mask[first >> 5], first >> 5 < kWords - 1 ? my_mask[(first >> 5) + 1] : 0u, first & 31);
          return r < s.nq ? x & s_valid[st][w] : 0u;
        };
        // Code of its own for chunks with slots of the tree, past the item's, without a page or with a V that is not finite,
        // where each row has its mask: as one, the compiler selects on every score, masked or not, which took twice
        // the time; and for those with V's scales far apart.
        auto softmax = [&](auto masked, auto far) {
          // slots 16 g .. as scores times K's scale, in pairs
          auto scores = [&](const uint32_t (&x)[16], int g, uint32_t seen, uint64_t (&t)[8]) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
              if constexpr (I4) {              // (K's tile has the scales)
                t[e] = pair(x[2 * e], x[2 * e + 1]);
                t[e + 1] = pair(x[2 * e + 2], x[2 * e + 3]);
                continue;
              }
              const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(kf + 16 * g + 2 * e);
              t[e] = mul2(pair(x[2 * e], x[2 * e + 1]), k.x);
              t[e + 1] = mul2(pair(x[2 * e + 2], x[2 * e + 3]), k.y);
            }
            if constexpr (masked) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 y = unpair(t[e]);
                t[e] = pair(seen >> (2 * e) & 1 ? y.x : -INFINITY, seen >> (2 * e + 1) & 1 ? y.y : -INFINITY);
              }
            }
          };
          // ---- the row's maximum
          float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
          for (int w = 0; w < 4; ++w) {
            uint32_t x[2][16];
            tc::tmem_ld16_nowait(t_s + 32 * w, x[0]);
            tc::tmem_ld16_nowait(t_s + 32 * w + 16, x[1]);
            const uint32_t seen = masked ? word(w) : ~0u;
            tc::tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint64_t t[8];
              scores(x[h], 2 * w + h, seen >> (16 * h), t);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 y = unpair(t[e]);
                m[e % 4] = fmaxf(fmaxf(y.x, y.y), m[e % 4]);
              }
            }
          }
          const float top = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
          // ---- the row's reference: the chunk before's, raised where the maximum asks for it
          float was = -INFINITY;
          if (i > 0) {
            ok = wait_for(&r_full[(it - 1) % kBuf], parity(it - 1, kBuf), a.status);
            was = s_ref[r];
          }
          const float mq = top * qs, now = top > -INFINITY && !(mq - was <= kMargin) ? mq : was;
          s_ref[r] = now;
          tc::mbar_arrive(&r_full[it % kBuf]);
          if (ref != now) l *= ref == -INFINITY ? 1.f : ex2(ref - now);   // (no reference: the sums are 0)
          ref = now;
          float f = was == now || was == -INFINITY ? 1.f : ex2(was - now);
          if (TURNED) f *= ex2((float)s_vstep[st]);
          if (i > 0 && __any_sync(0xffffffffu, f != 1.f)) {
            ok = ok && wait_for(&pv_done[1 - grp], parity(it - 1, 2), a.status);
            tc::tc_fence_after();
#pragma unroll 1
            for (int d = 0; d < HD; d += 16) {
              float o[16];
              tc::tmem_ld16(t_o + lanes + d, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] *= f;
              tc::tmem_st16(t_o + lanes + d, o);
            }
          }
          const float off = ref == -INFINITY ? 0.f : ref - kUp;
          // ---- probabilities, their sum, P over S
          uint64_t add = 0ull;
          const uint64_t qs2 = pair(qs, qs), off2 = pair(-off, -off);
#pragma unroll 1
          for (int w = 0; w < 4; ++w) {
            uint32_t x[2][16];
            tc::tmem_ld16_nowait(t_s + 32 * w, x[0]);
            tc::tmem_ld16_nowait(t_s + 32 * w + 16, x[1]);
            const uint32_t seen = masked ? word(w) : ~0u;
            tc::tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint64_t t[8];
              scores(x[h], 2 * w + h, seen >> (16 * h), t);
              uint32_t hi[8], lo[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float2 z = unpair(fma2(t[e], qs2, off2));
                float2 y = make_float2(ex2(z.x), ex2(z.y));
                add = add2(add, pair(y.x, y.y));
                if constexpr (far && !TURNED) {      // (V as it is: its scales, 1 in other chunks)
                  const float2 f = *reinterpret_cast<const float2*>(kf + kKeys + 16 * (2 * w + h) + 2 * e);
                  y = make_float2(y.x * f.x, y.y * f.y);
                }
                if constexpr (masked) {        // a V that is not finite: NaN in the rows that see it
                  const uint32_t m = (seen & s_nan[st][w]) >> (16 * h + 2 * e);
                  if (m & 1) y.x = __uint_as_float(0x7fc00000u);
                  if (m & 2) y.y = __uint_as_float(0x7fc00000u);
                }
                if constexpr (TURNED && !far) {
                  const __half2 p = __floats2half2_rn(y.x, y.y);
                  hi[e] = *reinterpret_cast<const uint32_t*>(&p);
                } else {
                  const __nv_bfloat162 p = __floats2bfloat162_rn(y.x, y.y);
                  const __nv_bfloat162 d = __floats2bfloat162_rn(y.x - __low2float(p), y.y - __high2float(p));
                  hi[e] = *reinterpret_cast<const uint32_t*>(&p);
                  lo[e] = *reinterpret_cast<const uint32_t*>(&d);
                }
              }
              const uint32_t to = t_s + 32 * w + h * 8;
              tc::tmem_st_nowait(to, hi);
              if (!TURNED || far) tc::tmem_st_nowait(to + 16, lo);
            }
          }
          const float2 two = unpair(add);
          l += two.x + two.y;
          tc::tmem_wait_st();
        };
        if (live) {
          const int kind = s_kind[st];
          if (kind == 0) softmax(std::false_type(), std::false_type());
          else if (kind == 1) softmax(std::true_type(), std::false_type());
          else softmax(std::true_type(), std::true_type());
          failed = !__all_sync(0xffffffffu, ok);
        } else {
          tc::mbar_arrive(&r_full[it % kBuf]);
        }
        vref = s_vref[st];
        tc::tc_fence_before();
        tc::mbar_arrive(&p_full[it % kBuf]);
        tc::mbar_arrive(&f_empty[st]);
      }
      // ---- the groups' sums: each thread finishes half of its row's dimensions
      // the next segment's queries, as soon as the last S has read this one's, beside the last P V
      const int last = it0 + n - 1;
      unit += n;
      const Segment now = s;
      if (unit < end) {
        if (!failed) failed = !__all_sync(0xffffffffu, wait_for(&s_full[last % kBuf], parity(last, kBuf), a.status));
        s = segment_at(a, s_first, unit, end);
        if (!failed) stage(s, buf ^ 1);
      }
      if (!failed)
        failed = !__all_sync(0xffffffffu, wait_for(&pv_done[last & 1], parity(last, 2), a.status));
      if (tc::named_barrier_or(1, kSoft, failed)) break;
      tc::tc_fence_after();
      const int rows = min(kRows, a.T * a.G - now.qb * kRows);
      {
        float m = live ? s_ref[r] : -INFINITY;   // the last chunk's
        if (ref != m) l *= ref == -INFINITY ? 1.f : ex2(ref - m);
        s_l[grp][r] = l;
        if (grp == (last & 1) && r == 0) s_v = vref;
        sync();
        l = s_l[0][r] + s_l[1][r];
        if (m == -INFINITY) m = 0.f;           // (nothing seen, or NaN scores alone)
        if (r >= now.nq || now.keys == 0) l = 0.f;
        if (l != 0.f && s_bad[buf][r]) l = __uint_as_float(0x7fc00000u);
        m = l == 0.f ? -INFINITY : m - kUp;
        const bool whole = now.c0 == 0 && now.c1 == now.units;
        const float inv = l == 0.f ? 0.f : whole ? 1.f / l : 1.f;
        const float unscale = TURNED ? ex2((float)(s_v - 127 - (I4 ? kVUp4 : 0))) : 1.f;
        const Vec x = vector_of(a, now.h, now.qb, r);
        const size_t part = (size_t)blockIdx.x * 2 + (now.c0 == 0);
        if (grp == 0 && r < rows) {
          if (whole) {
            store_lse(a, now.b, x, m, l);
          } else {
            a.part_ml[(part * 2) * kRows + r] = m;
            a.part_ml[(part * 2 + 1) * kRows + r] = l;
          }
        }
        __nv_bfloat16* const out =
            static_cast<__nv_bfloat16*>(a.out) + now.b * a.so[0] + x.t * a.so[1] + x.h * a.so[2];
        float* const part_o = a.part_o + (part * kRows + r) * HD;
#pragma unroll 1
        for (int d = grp * (HD / 2); d < (grp + 1) * (HD / 2); d += 16) {
          float o[16];
          tc::tmem_ld16(t_o + lanes + d, o);
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = inv == 0.f ? 0.f : o[e] * unscale * inv;
          if (I4 && r < rows) {
            // (columns d + 8 w + 2 i + h are dimension 4 j + i of one of two groups)
            constexpr int PAIRS = HD / kGroup / 2;
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int W = d / 8 + w, to = (W % PAIRS * 2 + h) * kGroup + W / PAIRS * 4;
                const float y[4] = {o[8 * w + h], o[8 * w + 2 + h], o[8 * w + 4 + h], o[8 * w + 6 + h]};
                if (!whole) {
                  *reinterpret_cast<float4*>(part_o + to) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
                  const __nv_bfloat162 z0 = __floats2bfloat162_rn(y[0], y[1]), z1 = __floats2bfloat162_rn(y[2], y[3]);
                  if (o_aligned) {
                    *reinterpret_cast<uint2*>(out + to) =
                        make_uint2(*reinterpret_cast<const uint32_t*>(&z0), *reinterpret_cast<const uint32_t*>(&z1));
                  } else {
                    out[to] = z0.x;
                    out[to + 1] = z0.y;
                    out[to + 2] = z1.x;
                    out[to + 3] = z1.y;
                  }
                }
              }
          } else if (r < rows) {
            if (!whole) {
#pragma unroll
              for (int e = 0; e < 16; e += 8) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(o[e + j]);
                store32(part_o + d + e, w);
              }
            } else {
              uint32_t w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const __nv_bfloat162 z = __floats2bfloat162_rn(o[2 * e], o[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t*>(&z);
              }
              if (o_aligned) {
                *reinterpret_cast<uint4*>(out + d) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(out + d + 8) = make_uint4(w[4], w[5], w[6], w[7]);
              } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  out[d + e] = __ushort_as_bfloat16((unsigned short)(w[e / 2] >> (e % 2 * 16)));
              }
            }
          }
        }
      }
      tc::tc_fence_before();
      sync();                                  // queries, masks, sums and O are free
      it0 += n;
    }
  } else if constexpr (I4) {
    // ------------------------------------------------------------------------- K to bf16, V to 16 bits
    // 16 bytes of a row at a time, 8 values of every group, a word (one of each of two groups in turn) to 16 bytes of a
    // tile; exactly, with the scales. Four warps have K, four V.
    constexpr int G2 = HD / kGroup / 2, PER = C::RB / 16, kRowsAt = kConv / PER;
    const int tid = (threadIdx.x - kSoft) % kConv, row0 = tid / PER, part = tid % PER;
    // (words 2, 3 first in the second block of 64 dimensions: eight lanes' stores then meet no bank twice)
    const int flip = part >> 1 & 1;
    uint32_t to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int W = 4 * part + (i ^ flip << 1);
      to[i] = W / 8 * C::H_BLOCK + tc::row_offset(row0, W % 8, 128);
    }
    static_assert(C::BLOCK == C::H_BLOCK && C::BW == 128);
    // (through shared memory, or the compiler knows them as constants and takes two instructions)
    const volatile uint32_t* const masks = s_masks;
    const uint32_t mb = masks[0], mh = masks[1];
    const auto words = [&](const uint8_t* half, int k, uint32_t (&w)[4]) {
      const uint4 u = *reinterpret_cast<const uint4*>(half + (row0 + k * kRowsAt) * C::RB + part * 16);
      w[0] = flip ? u.z : u.x; w[1] = flip ? u.w : u.y; w[2] = flip ? u.x : u.z; w[3] = flip ? u.y : u.w;
    };
    const auto bf16_words = [&](uint8_t* tile, const uint32_t (&w)[4], const uint32_t (&s8)[G2], const uint32_t (&m24)[G2]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint4*>(tile + to[i]) =
            make_uint4(value_bf16<0>(w[i], mb, s8[i % G2], m24[i % G2]), value_bf16<1>(w[i], mb, s8[i % G2], m24[i % G2]),
                       value_bf16<2>(w[i], mb, s8[i % G2], m24[i % G2]), value_bf16<3>(w[i], mb, s8[i % G2], m24[i % G2]));
    };
    const auto turn_k = [&](int i) {
      const int st = i % NST;
      if (!__all_sync(0xffffffffu, wait_for(&k_full[st], parity(i, NST), a.status) &&
                                       wait_for(&kt_empty[i & 1], parity(i, 2) ^ 1, a.status)))
        return false;
      const uint8_t* const from = sm + C::KV_OFF + st * 2 * C::PACKED;
#pragma unroll 1
      for (int k = 0; k < kKeys / kRowsAt; ++k) {
        uint32_t w[4], s8[G2], m24[G2];
        words(from, k, w);
        const uint32_t* const z = reinterpret_cast<const uint32_t*>(from + kKeys * C::RB + (row0 + k * kRowsAt) * C::SB);
#pragma unroll
        for (int e = 0; e < G2; ++e) {
          s8[e] = mul_bf16x2(z[e], 0x3e003e00u);                 // 1 / 8
          m24[e] = mul_bf16x2(s8[e], 0xc340c340u);               // -192
        }
        bf16_words(sm + C::KT_OFF + (i & 1) * C::TILE + k * (kRowsAt * 128), w, s8, m24);
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&kt_full[i & 1]);
      tc::mbar_arrive(&k_empty[st]);
      return true;
    };
    const int n = end - begin;
    bool ok = true;
    if (warp >= kConvWarp + kConv / 32) {      // K
      for (int i = 0; i < n && ok; ++i) ok = turn_k(i);
      ok = false;
    }
    for (int i = 0; i < n && ok; ++i) {
      const int st = i % NST;
      ok = wait_for(&f_full[st], parity(i, NST), a.status) && wait_for(&v_full[st], parity(i, NST), a.status) &&
           wait_for(&pv_done[i & 1], parity(i, 2) ^ 1, a.status);   // (chunk i - 2's: the buffer is free)
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const bool far = s_kind[st] >> 1;
      if (threadIdx.x == kSoft) s_h_far[i & 1] = far;
      const uint8_t* const from = sm + C::KV_OFF + (st * 2 + 1) * C::PACKED;
      uint8_t* const tile = sm + C::H_OFF + (i & 1) * C::H_TILE;
      const uint32_t* const factors = reinterpret_cast<const uint32_t*>(sm + C::FACTOR_OFF + st * C::FACTORS);
#pragma unroll 1
      for (int k = 0; k < kKeys / kRowsAt; ++k) {
        uint32_t w[4], x[G2], y[G2];
        words(from, k, w);
        const uint32_t* const z = factors + (row0 + k * kRowsAt) * (2 * G2);
        if constexpr (G2 == 2) {
          const uint4 u = *reinterpret_cast<const uint4*>(z);
          x[0] = u.x; y[0] = u.y; x[1] = u.z; y[1] = u.w;
        } else {
          const uint2 u = *reinterpret_cast<const uint2*>(z);
          x[0] = u.x; y[0] = u.y;
        }
        uint8_t* const at = tile + k * (kRowsAt * 128);
        if (far) {
          bf16_words(at, w, x, y);
          continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint4*>(at + to[e]) =
              make_uint4(value_f16<0>(w[e], mh, x[e % G2], y[e % G2]), value_f16<1>(w[e], mh, x[e % G2], y[e % G2]),
                         value_f16<2>(w[e], mh, x[e % G2], y[e % G2]), value_f16<3>(w[e], mh, x[e % G2], y[e % G2]));
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&h_full[i & 1]);
      tc::mbar_arrive(&v_empty[st]);
    }
  } else if constexpr (F8) {
    // ------------------------------------------------------------------------- V to 16 bits
    // 16 codes at a time, exactly, with the rows' scales; rows that there are not become zeros. fp16, which two
    // instructions a pair give; where V's scales are far apart bf16, in which no scale is too small.
    constexpr int kRowsAt = kConv / (HD / 16);
    const int row0 = (threadIdx.x - kSoft) / (HD / 16), part = (threadIdx.x - kSoft) % (HD / 16);
    // (the other half first in the second block of 64 dimensions: eight lanes' stores then meet no bank twice)
    const int flip = part >> 2 & 1;
    const uint32_t to0 = part / 4 * C::H_BLOCK + tc::row_offset(row0, part % 4 * 2 + flip, 128);
    const uint32_t to1 = part / 4 * C::H_BLOCK + tc::row_offset(row0, part % 4 * 2 + 1 - flip, 128);
    bool ok = true;
    for (int i = 0; i < end - begin && ok; ++i) {   // (a unit of the run is a chunk)
      const int st = i % NST;
      ok = wait_for(&f_full[st], parity(i, NST), a.status) &&
           wait_for(&v_full[st], parity(i, NST), a.status) &&
           wait_for(&pv_done[i & 1], parity(i, 2) ^ 1, a.status);   // (chunk i - 2's: the buffer is free)
      ok = __all_sync(0xffffffffu, ok);
      const float* vf = reinterpret_cast<const float*>(sm + C::FACTOR_OFF) + (st * 2 + 1) * kKeys;
      const bool far = s_kind[st] >> 1;
      if (threadIdx.x == kSoft) s_h_far[i & 1] = far;
      const uint8_t* from = sm + C::KV_OFF + (st * 2 + 1) * C::TILE + tc::row_offset(row0, part, C::BW);
      uint8_t* to = sm + C::H_OFF + (i & 1) * C::H_TILE;
      const auto store = [&](int k, const uint32_t (&h)[8]) {   // (rows that many apart lie alike in their tiles)
        const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
        *reinterpret_cast<uint4*>(to + k * (kRowsAt * 128) + to0) = flip ? hi : lo;
        *reinterpret_cast<uint4*>(to + k * (kRowsAt * 128) + to1) = flip ? lo : hi;
      };
      if (!far) {
#pragma unroll 1
        for (int k = 0; k < kKeys / kRowsAt; ++k) {
          const uint4 u = *reinterpret_cast<const uint4*>(from + k * kRowsAt * C::BW);
          const float f = vf[row0 + k * kRowsAt];
          const __half2 f2 = __float2half2_rn(f);
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __half2 p, q;
            f8x4_half(f == 0.f ? 0u : w[e], &p, &q);   // (a row that there is not holds anything)
            p = __hmul2(p, f2);
            q = __hmul2(q, f2);
            h[2 * e] = *reinterpret_cast<const uint32_t*>(&p);
            h[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&q);
          }
          store(k, h);
        }
      } else {
#pragma unroll 1
        for (int k = 0; k < kKeys / kRowsAt; ++k) {
          const uint4 u = *reinterpret_cast<const uint4*>(from + k * kRowsAt * C::BW);
          const float f = vf[row0 + k * kRowsAt];
          const uint32_t w[4] = {u.x, u.y, u.z, u.w};
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __half2 p, q;
            f8x4_half(f == 0.f ? 0u : w[e], &p, &q);
            const float2 x = __half22float2(p), y = __half22float2(q);
            const __nv_bfloat162 a2 = __floats2bfloat162_rn(x.x * f, x.y * f), b2 = __floats2bfloat162_rn(y.x * f, y.y * f);
            h[2 * e] = *reinterpret_cast<const uint32_t*>(&a2);
            h[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&b2);
          }
          store(k, h);
        }
      }
      tc::fence_proxy_async();
      tc::mbar_arrive(&h_full[i & 1]);
      tc::mbar_arrive(&v_empty[st]);
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) tc::tmem_dealloc(tmem, 512);
}

template <int HD, int FORMAT>
cudaError_t launch(const TreeArgs& a, cudaStream_t s) {
  using C = Cfg<HD, FORMAT>;
  CUtensorMap map = {};
  if constexpr (!C::I4)
    if (encode_cache_map<HD, C::F8>(a, &map)) return cudaErrorInvalidValue;
  auto k = k_tree_rows<HD, FORMAT>;
  static OncePerDevice once;
  if (const cudaError_t e = allow_shared(once, k, C::smem(CDSL_TREE_MAX_BATCH))) return e;
  return launch_pdl(k, dim3(a.blocks), dim3(C::THREADS), C::smem(a.c.batch), s, a, map);
}

}  // namespace

cudaError_t launch_tree_rows(const TreeArgs& a, cudaStream_t s) {
  if (a.c.format == kI4) return a.c.hd == 128 ? launch<128, kI4>(a, s) : launch<64, kI4>(a, s);
  if (a.c.hd == 128) return a.c.format == kF8 ? launch<128, kF8>(a, s) : launch<128, kBF16>(a, s);
  return a.c.format == kF8 ? launch<64, kF8>(a, s) : launch<64, kBF16>(a, s);
}

}  // namespace tree
}  // namespace cdsl
