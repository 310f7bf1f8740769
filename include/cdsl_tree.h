/*
 * cdsl_tree.h -- C ABI of tree speculation over a quantised paged cache.
 *
 * The CDSL step (cdsl.h) drafts k chains and keeps fp32 K/V of its own. These calls serve a program
 * that runs its own model and drafts a tree of tokens (Sec. 2.2's speculative decoding with several
 * candidates per position): the cache in 8 or 16 bits, the attention of the tree over it, the
 * validation of the drafts by M_p with the random numbers given (Sec. 3.2.2), and the move of the
 * taken path's K/V to their places. One decoding step is, for every layer, cdsl_kv_write and
 * cdsl_tree_attention, then cdsl_tree_verify and cdsl_kv_commit:
 *
 *   nodes      0 .. n_b - 1 of sequence b; node 0 is the newest token, whose K/V are not yet cached;
 *              every other node is a drafted token whose parent has a smaller index
 *   slots      node i's K/V go to slot len_b + i of the sequence, len_b the tokens cached so far
 *   a path     0 = i_0 < i_1 < ... < i_(m-1): after the step len_b grows by m, and the token that
 *              cdsl_tree_verify drew is the next step's node 0
 *
 * Conventions are those of cdsl.h: calls are asynchronous on `stream` (a cudaStream_t, NULL: the
 * legacy default stream) and allocate nothing; d_ pointers are device pointers on the current
 * device, h_ pointers host pointers read before the call returns; arguments are checked on the host
 * before anything is launched, with the message in cdsl_last_error(NULL). What only the device can
 * see (an index in device memory that is out of range, a logits row without a finite value) is
 * latched as a cdsl_status in *d_status, first error wins, if d_status is not NULL; the caller sets
 * it to 0. CDSL_ETIMEOUT there means that a wait inside a kernel of cdsl_tree_attention has run out,
 * after a second or more, and that its output is not complete. Calls can be captured into CUDA graphs,
 * and calls on different streams may overlap unless they share a workspace or one writes what another
 * reads.
 */
#ifndef CDSL_TREE_H
#define CDSL_TREE_H

#include "cdsl.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CDSL_DTYPE_F8E4M3 = 2 };          /* of a cache only */
enum { CDSL_TREE_MAX_NODES = 128, CDSL_TREE_MAX_BATCH = 1024, CDSL_TREE_MAX_VOCAB = 1 << 20 };

/* A paged cache of `batch` sequences, all memory the caller's.
 *   d_pool   [n_layers][n_pages][2 (K, V)][n_kv_heads][page_size][head_dim], e4m3 or bfloat16, 16-byte
 *            aligned
 *   d_scale  [n_layers][n_pages][2][n_kv_heads][page_size] bytes, 16-byte aligned: row (token and head) values are
 *            code * 2^(byte - 127). Byte 255: the row held a value that is not finite (in the cache's type); its
 *            codes are zeros and it stands for NaN. (A caller's own codes are finite.)
 *   d_page_table [batch][max_pages]: the page of slots [i * page_size, (i + 1) * page_size) of each
 *            sequence, any page ids in any order; entries beyond the cached slots are not read.
 * The pool needs no initial values. page_size: a power of two, 16..256. head_dim: 64 or 128. */
typedef struct cdsl_kv_cache {
  void* d_pool;
  uint8_t* d_scale;
  const int32_t* d_page_table;
  int32_t n_layers, n_pages, n_kv_heads, page_size, head_dim;
  int32_t dtype;                          /* CDSL_DTYPE_F8E4M3 or CDSL_DTYPE_BF16 */
  int32_t batch, max_pages;
} cdsl_kv_cache;

/* Write rows i < d_count[b] (NULL: all T) of k and v [batch, T, n_kv_heads, head_dim] into slots
 * d_start[b] + i of `layer`. dtype: of k and v, CDSL_DTYPE_F32 or CDSL_DTYPE_BF16. h_strides[6]:
 * elements between sequences, tokens and heads of k, then of v (a head's values are contiguous).
 * e4m3: the scale is the smallest power of two (2^-126 at least) with which the row's largest
 * absolute value is at most 448, 1 for a row of zeros; codes are value / scale rounded to nearest
 * even. bfloat16: rounded to nearest even, scale 1. A slot beyond the page table, or a page id
 * outside [0, n_pages), latches CDSL_ERANGE and its rows are not written. */
CDSL_API int32_t cdsl_kv_write(const cdsl_kv_cache* cache, int32_t layer, const void* d_k,
                               const void* d_v, int32_t dtype, int32_t T, const int64_t* h_strides,
                               const int32_t* d_start, const int32_t* d_count, int32_t* d_status,
                               void* stream);

/* Read slots d_start[b] + i, i < d_count[b] (NULL: all T), of layers layer .. layer + n_layers - 1
 * back as values: d_k, d_v [n_layers, batch, T, n_kv_heads, head_dim] contiguous, 16-byte aligned,
 * of `dtype` (exact in either type for an e4m3 cache, but for values above the type's largest or below
 * its smallest). Rows i >= d_count[b], and rows whose slot or page is out of range (which latches
 * CDSL_ERANGE), are zeros. */
CDSL_API int32_t cdsl_kv_read(const cdsl_kv_cache* cache, int32_t layer, int32_t n_layers, void* d_k,
                              void* d_v, int32_t dtype, int32_t T, const int32_t* d_start,
                              const int32_t* d_count, int32_t* d_status, void* stream);

/* Move the taken path's rows, in every layer: slot d_lens[b] + d_path[b, i] to slot d_lens[b] + i,
 * 1 <= i < d_n_path[b]. d_path [batch, T], d_n_path [batch] as cdsl_tree_verify writes them: strictly
 * increasing from 0 (anything else latches CDSL_EINVAL and moves nothing of that sequence; a slot
 * or page out of range latches CDSL_ERANGE and does the same). d_new_lens [batch], if not NULL, is set
 * to d_lens + d_n_path (to d_lens where nothing was moved for such a reason); it must not be d_lens. */
CDSL_API int32_t cdsl_kv_commit(const cdsl_kv_cache* cache, const int32_t* d_lens,
                                const int32_t* d_path, const int32_t* d_n_path, int32_t T,
                                int32_t* d_new_lens, int32_t* d_status, void* stream);

/* Host helper: the attention mask of a tree from its parents (h_parents[i] < i for i >= 1; [0] is
 * ignored): h_mask [T][(T + 31) / 32] words, bit j of row i set when node j is node i or one of its
 * ancestors, and h_depth [T] (NULL: not wanted) the number of ancestors, so that node i's position is
 * len_b + h_depth[i]. */
CDSL_API int32_t cdsl_tree_mask(const int32_t* h_parents, int32_t T, uint32_t* h_mask,
                                int32_t* h_depth);

/* Bytes of d_workspace that cdsl_tree_attention needs for trees of up to T nodes and n_heads query
 * heads over this cache (its sizes; no pointer of it is read). */
CDSL_API int32_t cdsl_tree_attention_workspace(const cdsl_kv_cache* cache, int32_t n_heads, int32_t T,
                                               size_t* bytes);

/* Attention of each sequence's tree over its cached tokens and the tree itself:
 *   out[b, t, h] = sum_j p_j v_j,  p = softmax over the visible slots j of scale * q[b, t, h] . k_j
 * with head h reading K/V head h / (n_heads / n_kv_heads). Node t < d_nodes[b] (NULL: T) sees the slots
 * j < d_lens[b], and slot d_lens[b] + i, i < d_nodes[b], where bit i of d_mask[b, t]
 * ([batch, T, (T + 31) / 32] words, as cdsl_tree_mask writes them; any bits are allowed) is set. A node
 * that sees nothing, and nodes t >= d_nodes[b], give zeros (lse -inf). T = 1 is plain decoding.
 *   d_q, d_out [batch, T, n_heads, head_dim] of `dtype` (CDSL_DTYPE_F32 or CDSL_DTYPE_BF16);
 *   h_strides[6]: elements between sequences, tokens and heads of q, then of out (whose places must not coincide: a 0
 *   between two of them is refused). d_lse
 *   [batch, T, n_heads] float32 or NULL: log of the sum of exp(scale * q . k_j).
 *   max_len: an upper bound of d_lens (0 .. max_pages * page_size - T); a length outside 0 .. max_len
 *   latches CDSL_ERANGE and counts as the nearer bound. It sets the launch size alone, so a captured
 *   call may be replayed while the lengths stay below it. Pages out of range latch CDSL_ERANGE and
 *   their slots count as not visible.
 * bfloat16 queries run on the tensor cores with fp32 sums and softmax. Over an e4m3 cache queries are
 * held to 2^-18 of a row's largest value and probabilities to 2^-8 of themselves (2^-10 on average) for
 * up to 32 query vectors per K/V head, to 2^-12 for more; small V rows count beside large ones by their
 * scales, which for that are to be the smallest ones, as cdsl_kv_write makes them. Over a bfloat16 cache
 * probabilities are held to 2^-17. float32 queries run on the CUDA cores in fp32.
 * d_workspace: cdsl_tree_attention_workspace bytes, 256-byte aligned, in any state; it
 * holds nothing between calls. */
CDSL_API int32_t cdsl_tree_attention(const cdsl_kv_cache* cache, int32_t layer, const void* d_q,
                                     int32_t dtype, int32_t n_heads, int32_t T,
                                     const int64_t* h_strides, const int32_t* d_lens,
                                     const int32_t* d_nodes, const uint32_t* d_mask, float scale,
                                     int32_t max_len, void* d_out, float* d_lse, void* d_workspace,
                                     size_t workspace_bytes, int32_t* d_status, void* stream);

/* Validation of each sequence's tree by M_p (Sec. 3.2.2): walk from node 0 to a child that M_p takes,
 * and so on; at the node where no child is taken (or there is none) draw the next token. Row
 * d_logits[b, i] gives the distribution p of the token after node i, exp((l - max l) / temperature)
 * over its sum.
 *   Drafts that were chosen, not sampled (d_draft_logits NULL; M_q's best tokens, Sec. 3.2.1): the
 *   children of a node are tried in order of index; child c with token x is taken with probability p(x),
 *   and if it is not, x leaves the distribution. Weights are whole numbers
 *   W_v = floor(2^31 exp((l_v - max l) / temperature)), Z their sum: c is taken when
 *   floor(k Z / 2^24) < W_x, k = floor(2^24 u[b, c]).
 *   Drafts sampled from M_q (d_draft_logits[b, i] the row that node i's children were sampled from,
 *   independently, at the same temperature; not read where node i has none): c is taken when u[b, c] q(x) < p(x), and if it is not, p
 *   becomes max(p - q, 0) over its sum (p stays where that is nothing); W_v = floor(2^31 max(p - q, 0)).
 *   The drawn token is the first v with W_0 + .. + W_v > floor(k Z / 2^24), k = floor(2^24
 *   u_last[b]): both procedures draw from p exactly, to the weights' resolution. Whole numbers make it
 *   independent of the order of the sums.
 *   temperature 0: the child whose token is the argmax is taken, and the last token is the argmax, lower
 *   index first on ties; the random numbers and draft logits are not read.
 * d_logits, d_draft_logits [batch, T, vocab] of `dtype` (CDSL_DTYPE_F32 or CDSL_DTYPE_BF16), h_strides[4]:
 * elements between sequences and nodes of the logits, then of the draft's. d_tokens, d_parents
 * [batch, T] (entry 0 of d_parents is ignored; a parent outside 0 .. i - 1 leaves node i out);
 * d_nodes [batch] or NULL (T); d_u [batch, T] and d_u_last [batch] float32 in [0, 1). -inf logits
 * are tokens that cannot be drawn. A row with NaN, +inf or nothing finite latches CDSL_ENONFINITE, and the
 * walk ends at its node without a token; a token outside the vocabulary latches CDSL_ERANGE and is not
 * taken.
 * Outputs, int32: d_n_path [batch] the nodes on the path (0 for a sequence without nodes), d_path
 * [batch, T] the path, d_emitted [batch, T] the d_n_path - 1 drafted tokens on it and then the drawn
 * one (-1 where there is none); both filled up with -1. */
CDSL_API int32_t cdsl_tree_verify(int32_t batch, int32_t T, int32_t vocab, const void* d_logits,
                                  const void* d_draft_logits, int32_t dtype, const int64_t* h_strides,
                                  const int32_t* d_tokens, const int32_t* d_parents,
                                  const int32_t* d_nodes, const float* d_u, const float* d_u_last,
                                  float temperature, int32_t* d_path, int32_t* d_n_path,
                                  int32_t* d_emitted, int32_t* d_status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CDSL_TREE_H */
