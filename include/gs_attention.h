/*
 * gs_attention.h -- C ABI of softmax attention on the MI355X (gfx950), the
 * normalised companion of the Gauss sums of gauss_sum.h: for queries q, keys k
 * (D wide), values v (C wide) and a scale,
 *
 *     out_m = sum_n w_mn v_n / sum_n w_mn ,   w_mn = exp(scale <q_m, k_n>) ,
 *     lse_m = log sum_n w_mn ,
 *
 * over the keys n that row m sees, its gradients, and the same over keys and
 * values kept in the pages of a cache.  Status codes and dtypes are those of
 * gauss_sum.h.
 *
 * Heads.  Query head h reads key head h / (Hq / Hkv); Hq is a multiple of Hkv.
 *
 * Sequences.  A call holds B independent ones, laid out in one of two ways:
 *   dense   M query rows and N keys a sequence; q_index / k_index are NULL or B
 *           lengths (32-bit, on the device): the rows from the length on belong
 *           to no sequence.
 *   packed  M query rows and N keys in all, one sequence behind the other;
 *           q_index and k_index are B + 1 offsets (32-bit, on the device), from 0
 *           on and not decreasing.
 * Lengths and offsets are brought into the arrays' range where they are not in
 * it, so that no value of theirs leads outside an array.
 *
 * Rows see:  all keys of their sequence; with `causal`, row i of qn sees keys
 * j <= i + kn - qn (the last row sees every key), and with window > 0 only the
 * last `window` of those.  A row that sees nothing gives out = 0, lse = -inf and
 * no gradient.  (One that sees keys whose scores are all -inf is another matter:
 * out is 0 / 0 = NaN, lse log 0 = -inf.)
 *
 * Memory and ownership
 *   - Data pointers are DEVICE pointers owned by the caller.  Arrays are given by
 *     gs_attention_array: element (sequence b, row i, head h, column c) lies at
 *     data + b*batch_stride + i*row_stride + h*head_stride + c (elements; the
 *     batch stride is not used where arrays are packed).  Columns are contiguous.
 *     Strides are >= 0; inputs may have strides of 0 (broadcast), the elements of
 *     an output are distinct.  Rows that are 16-byte aligned (outputs: 8) and a
 *     multiple of 8 (4) elements wide are moved in wide accesses; any other
 *     alignment to the element size is accepted and slower.
 *   - The address range of an output must not overlap that of an input, the
 *     workspace or another output.  (The pages of keys and of values may
 *     interleave in one allocation.)
 *   - lse is fp32: B x Hq x M (dense) or Hq x M (packed), contiguous.
 *   - Rows of outputs that belong to no sequence are left as they were, or, as
 *     `zero_rest` asks, written as 0 (out and gradients) and -inf (lse).
 *   - The library allocates nothing; the workspace (256-byte aligned, its
 *     contents ignored and left undefined) is the caller's.  Calls that may
 *     overlap in time need workspaces of their own.  That of the backward pass
 *     holds 8 bytes a query row and head, and, where few keys leave the query heads
 *     of a key head to s workgroups (s at most Hq / Hkv), s sums of 8 max(D, C)
 *     bytes a key and key head: 268 MB for 8192 tokens, 32 heads over 8, D = 128,
 *     causal.
 *
 * Execution: as in gauss_sum.h.  All work is enqueued on `stream`, arguments are
 * validated before anything is enqueued, nothing synchronises, the calls may be
 * captured into a graph, and results are bitwise reproducible for equal arguments
 * and lengths.
 *
 * Precision.  q, k, v, out, dout and gradients share one dtype, fp16 or bf16.
 * Products run on the matrix cores with fp32 sums; scores, exponentials, their sums
 * and lse are fp32.  Weights (relative to the row's maximum), and P and dS of the
 * backward pass, are rounded once to the inputs' type before they are contracted,
 * and results once at the end; in fp16 P and dS enter times powers of two, dS times
 * one of each row's (dK: key's) own.  Sums of weights (below 2^15) times values are
 * fp32, so bf16 values beyond 2^112 may overflow.  NaN and Inf propagate to the rows
 * that see them and to no other.
 */
#ifndef GS_ATTENTION_H
#define GS_ATTENTION_H

#include "gauss_sum.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GS_ATTENTION_REST_OUT 1 /* rows of no sequence: out and gradients 0 */
#define GS_ATTENTION_REST_LSE 2 /* rows of no sequence: lse -inf */

typedef struct {
  int64_t B, M, N, Hq, Hkv; /* 0 <= B <= 2^20; 0 <= M, N <= 2^30; 1 <= Hkv <= Hq <= 2^14 */
  int64_t D, C;             /* 1 .. 256 */
  int64_t window;           /* 0, or with causal the number of keys a row sees at most */
  int32_t dtype;            /* GS_F16 or GS_BF16 */
  int32_t packed, causal;   /* 0 or 1 */
  int32_t zero_rest;        /* GS_ATTENTION_REST_* flags */
  float scale;              /* finite, also times log2 e */
} gs_attention_problem;

typedef struct {
  void* data; /* not written where it is an input */
  int64_t batch_stride, row_stride, head_stride;
} gs_attention_array;

/* Keys and values in pages: row (position p of sequence b, head h) lies in page
 * table[b * table_width + p / page_size] at row p % page_size of it, page x of
 * the keys at k.data + x * k.batch_stride.  lens: keys of each sequence, those of
 * the call's own tokens included.  A key on a page whose number is outside
 * [0, pages) reads as NaN and is not written; positions from table_width *
 * page_size on do not exist (they are not written and not seen; the tokens of a
 * longer sequence keep their places), nor does any in a cache of 0 pages. */
typedef struct {
  gs_attention_array k, v;
  int64_t pages, page_size, table_width;
  const int32_t* table;
  const int32_t* lens;
} gs_attention_cache;

/* All calls: GS_ERR_BAD_SHAPE also where a launch would need more than 2^24 - 1
 * workgroups (tiles of rows times heads and sequences).
 *
 * out and (unless NULL) lse of every row.  low (unless NULL): what the rounding
 * of out leaves, out - rounded, itself rounded to the dtype, for the backward
 * pass.  M == 0, or B == 0 in the dense layout, is a no-op.
 * Workspace: gs_attention_fwd_workspace_size(p) bytes (which may be 0). */
gs_status gs_attention_fwd(const gs_attention_problem* p, const gs_attention_array* q,
                           const gs_attention_array* k, const gs_attention_array* v,
                           const int32_t* q_index, const int32_t* k_index,
                           const gs_attention_array* out, const gs_attention_array* low, float* lse,
                           void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t gs_attention_fwd_workspace_size(const gs_attention_problem* p);

/* Gradients of L = sum <dout, out>, any of dq, dk, dv NULL where not wanted (one
 * at least is), from the forward call's out, lse and (or NULL) low: the rows'
 * <dout, out> is subtracted from every dP, and rows of few keys gain from the part
 * that out lost to its rounding.  dk and dv are summed over the query heads that
 * share a key head. */
gs_status gs_attention_bwd(const gs_attention_problem* p, const gs_attention_array* q,
                           const gs_attention_array* k, const gs_attention_array* v,
                           const int32_t* q_index, const int32_t* k_index,
                           const gs_attention_array* out, const gs_attention_array* low,
                           const float* lse, const gs_attention_array* dout, const gs_attention_array* dq,
                           const gs_attention_array* dk, const gs_attention_array* dv, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
size_t gs_attention_bwd_workspace_size(const gs_attention_problem* p, int want_dq, int want_dk,
                                       int want_dv);

/* A chunk of new tokens, or one, of every sequence over a paged cache that holds
 * their keys and values already (gs_attention_append): token i of qn sees the
 * keys up to its own position lens[b] - qn + i (causal has to be 1; N is not
 * used).  q and out: packed, or dense with M tokens of every sequence (q_index
 * NULL).  lse: Hq x (rows of all sequences), or NULL.  M == 0, or B == 0 in the
 * dense layout, is a no-op. */
gs_status gs_attention_paged(const gs_attention_problem* p, const gs_attention_array* q,
                             const gs_attention_cache* cache, const int32_t* q_index,
                             const gs_attention_array* out, float* lse, void* workspace,
                             size_t workspace_bytes, hipStream_t stream);
size_t gs_attention_paged_workspace_size(const gs_attention_problem* p, const gs_attention_cache* cache);

/* Keys k and values v of the new tokens (rows as the queries of
 * gs_attention_paged) into the pages, at positions lens[b] - qn + i.  Two tokens of
 * one call must not share a place (sequences share pages only before their new
 * tokens). */
gs_status gs_attention_append(const gs_attention_problem* p, const gs_attention_array* k,
                              const gs_attention_array* v, const gs_attention_cache* cache,
                              const int32_t* q_index, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* GS_ATTENTION_H */
