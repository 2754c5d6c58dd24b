/* llm42_mx4.h -- the fast path in 4 bits: matrices and a paged KV cache held in
 * MXFP4, and a decoding step that runs on them.
 *
 * The fast path proposes, the verifier decides [paper Section 4.1, 4.2]: what the
 * candidates were computed with changes how many of them are reproduced, never the
 * released stream.  So the fast path may read a copy of the weights and of the
 * cache that takes 4.25 bits a value instead of 16.
 *
 * Format.  32 consecutive values of a row (of a matrix; of the features of one
 * token's kv head, in a cache) are a block.  They share the scale 2^E, with
 * E = floor(log2(largest magnitude)) - 2 within -127 .. 127, held as the byte E + 127;
 * each value is held in 4 bits as its sign and the index of the nearest of
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 to its magnitude / 2^E (ties to the even index, 6 beyond 6).
 * The last block of a row is filled up with zeros.  A block that holds a NaN or an
 * infinity has the byte 255 and stands for NaN throughout.  (This is the OCP
 * microscaling format of that name, with its conversion from wider types.)
 *
 * The conventions of llm42.h hold here too: "dev" pointers are device addresses on the current
 * device, calls enqueue on `hip_stream`, allocate nothing (but llm42_mx4_model_create),
 * never synchronise, never read device memory on the host, and may be captured into a
 * graph; nothing in a workspace has to start at zero.  A workspace belongs to one call at a time: calls (and replays of
 * captured ones) that share one follow each other on a stream.  Calls of these functions are
 * deterministic, but not independent of the batch as the verifier's are.
 */
#ifndef LLM42_MX4_H_
#define LLM42_MX4_H_

#include "llm42.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of plain arrays. */
#define LLM42_BF16 0
#define LLM42_F32  1

/* ---- matrices ------------------------------------------------------------------------------------------ */

/* Bytes of a rows x cols matrix in MXFP4, rows 1 .. 2^30 and cols 1 .. 2^26.  The layout inside is the library's own (tiles of 16 rows x
 * 256 columns, padded with zeros: about 4.25 bits a value where cols is a multiple of 256).  A call takes matrices of up to
 * 2^26 - 4 tiles: LLM42_EINVAL beyond. */
llm42_status llm42_mx4_bytes(int32_t rows, int32_t cols, size_t* out_bytes);

/* src[r][c] at src + r * src_stride + c elements of type src_type; blocks run along c.  dst: 16-byte aligned,
 * llm42_mx4_bytes(rows, cols) or more (LLM42_EWORKSPACE if dst_bytes is less). */
llm42_status llm42_mx4_quantize(
    const void* src,               /* dev                                                 */
    int32_t     src_type,          /* LLM42_BF16 or LLM42_F32                             */
    int64_t     src_stride,        /* elements from a row to the next, >= cols            */
    int32_t     rows,
    int32_t     cols,
    void*       dst,               /* dev                                                 */
    size_t      dst_bytes,
    void*       hip_stream);

/* The values that the matrix stands for (every one of them is a bf16): dst[r][c] at dst + r * dst_stride + c.  What lies
 * between the rows of dst is left as it was. */
llm42_status llm42_mx4_dequantize(
    const void* src,               /* dev                                                 */
    size_t      src_bytes,
    int32_t     rows,
    int32_t     cols,
    void*       dst,               /* dev                                                 */
    int32_t     dst_type,
    int64_t     dst_stride,
    void*       hip_stream);

/* out[i][j] = sum over c of x[i][c] * w[j][c], w an n x k matrix in MXFP4, x bf16: the products are exact (a 4-bit value is
 * a bf16), summed in fp32 in an order that depends on the sizes; out is rounded once.  x[i] at x + i * x_stride elements and
 * out[i] at out + i * out_stride; what lies between the rows of out is left as it was.  out must not overlap x or w.
 * workspace: llm42_mx4_matmul_workspace_bytes(rows, n, k) bytes, 256-byte aligned.  Rows that are not 4-byte aligned need it, and so do
 * more than 16 that are not 16-byte aligned, are more than 2^26 elements apart or whose k is not a multiple of 32 (LLM42_EWORKSPACE).
 * Otherwise the call does with less, or NULL, but then sums over k in one piece, which takes longer where rows and n are few (and
 * gives other low bits).  LLM42_EINVAL where rows * n (past 2^28), or rows * k of rows that need the workspace (about 2^35), ask for more
 * threads than one launch takes (2^32). */
llm42_status llm42_mx4_matmul_workspace_bytes(int32_t rows, int32_t n, int32_t k, size_t* out_bytes);
llm42_status llm42_mx4_matmul(
    const void* w,                 /* dev                                                 */
    size_t      w_bytes,
    int32_t     n,
    int32_t     k,
    const void* x,                 /* dev bf16                                            */
    int64_t     x_stride,          /* >= k                                                */
    int32_t     rows,              /* 1 .. LLM42_MAX_ROWS                                 */
    void*       out,               /* dev                                                 */
    int32_t     out_type,
    int64_t     out_stride,        /* >= n                                                */
    void*       workspace,         /* dev or NULL                                         */
    size_t      workspace_bytes,
    void*       hip_stream);

/* ---- the 4-bit cache ------------------------------------------------------------------------------------ */

/* A 4-bit cache is described by the same llm42_kv_cache as the bf16 one: kv_base (16-byte aligned) holds
 * llm42_kv4_bytes(model, num_blocks) bytes, [layer][block][kv head] records of 17 * head_dim bytes, block_table says where the
 * blocks of 16 positions of a sequence lie.  It may be the bf16 cache's table (a mirror of it) or one of its own.
 * Nothing in a fresh cache has to be initialised: no call reads a position that was not stored before. */
llm42_status llm42_kv4_bytes(const llm42_model* model, int64_t num_blocks, size_t* out_bytes);

/* K and V of positions first[s] .. first[s] + count[s] - 1 of every sequence, all layers, from the bf16 cache into the 4-bit
 * one.  Behind a verifier pass and its commit: first = the length before, count = the committed tokens; behind a prefill: 0 and
 * the length.  No other position is written.  No two sequences of a call may have positions in the same 4-bit block, unless both cover all
 * 16 of it from the same K and V (a shared prefix: they write the same bytes).
 * first[s] < 0, positions beyond a table's capacity, count[s] outside 0 .. max_count: LLM42_SEQ_BAD_LENGTH; a needed entry of either
 * table out of range: LLM42_SEQ_BAD_BLOCK; nothing of such a sequence is stored.  LLM42_EINVAL where num_seqs times the blocks that
 * max_count positions can touch, times a quarter of the kv heads, rounded up, exceeds 2^31 - 1. */
llm42_status llm42_kv4_store(
    const llm42_model*    model,
    const llm42_kv_cache* kv_cache,    /* bf16                                            */
    const llm42_kv_cache* kv4_cache,
    const int32_t*        first,       /* dev [num_seqs]                                  */
    const int32_t*        count,       /* dev [num_seqs]                                  */
    int32_t               num_seqs,
    int32_t               max_count,   /* host: >= every count                            */
    int32_t*              seq_status,  /* dev [num_seqs] or NULL                          */
    void*                 hip_stream);

/* What the 4-bit cache stands for at such positions: out_k and out_v are bf16
 * [n_layers][num_seqs][max_count][n_kv_heads][head_dim] (16-byte aligned); entries at count[s] and beyond, and those of a
 * flagged sequence, are left as they were.  Checks and status as for llm42_kv4_store. */
llm42_status llm42_kv4_read(
    const llm42_model*    model,
    const llm42_kv_cache* kv4_cache,
    const int32_t*        first,       /* dev [num_seqs]                                  */
    const int32_t*        count,       /* dev [num_seqs]                                  */
    int32_t               num_seqs,
    int32_t               max_count,
    void*                 out_k,       /* dev                                             */
    void*                 out_v,       /* dev                                             */
    int32_t*              seq_status,  /* dev [num_seqs] or NULL                          */
    void*                 hip_stream);

/* Attention of one layer over the 4-bit cache.  Row (s, i), i < n_valid[s], is the query at position seq_lens[s] + i and sees
 * positions 0 .. seq_lens[s] + i, all of which must have been stored; its head h uses kv head h / (n_q_heads / n_kv_heads):
 * out = softmax(q . k / sqrt(head_dim)) v.  Weights are rounded to bf16 before they multiply V; sums are fp32, of weights up to 2^8,
 * so that magnitudes of V up to about 2^119 / max_context stay in range (and those below 2^-110 may count as zero).
 * q and out: bf16 rows of n_q_heads * head_dim, row (s, i) at (s * window + i) * stride elements; both 16-byte aligned, strides
 * multiples of 8 and at least that long.  Rows that take no part (i >= n_valid[s]; a sequence whose status is not
 * LLM42_SEQ_OK; n_valid[s] may be 0) are left as they were.  max_context: as in llm42_verify_window, up to 2^30.
 * workspace: llm42_kv4_attention_workspace_bytes, 256-byte aligned. */
llm42_status llm42_kv4_attention_workspace_bytes(const llm42_model* model, int32_t num_seqs, int32_t window, int32_t max_context,
                                                 size_t* out_bytes);
llm42_status llm42_kv4_attention(
    const llm42_model*    model,
    int32_t               layer,           /* of the cache: 0 .. n_layers - 1             */
    const llm42_kv_cache* kv4_cache,
    const void*           q,               /* dev bf16                                    */
    int64_t               q_stride,
    const int32_t*        seq_lens,        /* dev [num_seqs]                              */
    int32_t               window,          /* 1 .. LLM42_MAX_WINDOW                       */
    const int32_t*        n_valid,         /* dev [num_seqs] or NULL (= window)           */
    int32_t               num_seqs,        /* num_seqs * window <= LLM42_MAX_ROWS         */
    int32_t               max_context,
    void*                 out,             /* dev bf16                                    */
    int64_t               out_stride,
    int32_t*              seq_status,      /* dev [num_seqs] or NULL                      */
    void*                 workspace,
    size_t                workspace_bytes,
    void*                 hip_stream);

/* ---- the fast path -------------------------------------------------------------------------------------- */

/* A 4-bit copy of every matrix of a model but the embedding, made on the model's device (which must be the current one)
 * from the weights that the model holds.  The copy uses the model's norms, embedding and rotary table: destroy it before the model.
 * Synchronises once. */
typedef struct llm42_mx4_model llm42_mx4_model;
llm42_status llm42_mx4_model_create(const llm42_model* model, llm42_mx4_model** out);
void         llm42_mx4_model_destroy(llm42_mx4_model* mx4);

/* llm42_decode_step_sampled by the 4-bit copy: the same arguments, effects, errors and status.  K and V of the input tokens are
 * written to the bf16 cache as there.  workspace: llm42_decode_step_mx4_workspace_bytes, 256-byte aligned.
 * kv4_cache NULL: attention over the bf16 cache.  Else they are stored into the 4-bit cache as well, and attention reads that: positions
 * 0 .. seq_lens[s] - 1 must have been stored, and its block table needs entries for position seq_lens[s] too (a block that no other
 * sequence of the call has; max_context up to 2^30).  The verifier overwrites the window's entries of the bf16 cache; those of the
 * 4-bit cache are overwritten by llm42_kv4_store behind the commit. */
llm42_status llm42_decode_step_mx4_workspace_bytes(const llm42_mx4_model* mx4, int32_t max_seqs, int32_t max_context,
                                                   size_t* out_bytes);
llm42_status llm42_decode_step_mx4(
    const llm42_mx4_model* mx4,
    const llm42_kv_cache*  kv_cache,
    const llm42_kv_cache*  kv4_cache,       /* or NULL                                     */
    const int32_t*         seq_lens,        /* dev [num_seqs]                              */
    const int32_t*         tokens,          /* dev [num_seqs]                              */
    int32_t                num_seqs,
    int32_t                max_context,
    int32_t*               out_tokens,      /* dev [num_seqs]                              */
    int32_t*               seq_status,      /* dev [num_seqs] or NULL                      */
    void* workspace, size_t workspace_bytes, void* hip_stream,
    const llm42_sampling*  sampling);       /* or NULL                                     */

#ifdef __cplusplus
}
#endif
#endif /* LLM42_MX4_H_ */
