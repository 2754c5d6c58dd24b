/* llm42_paged.h -- operators around the paged bf16 KV cache of llm42.h: appending to it with head
 * norms and rotary positions, attention over selected blocks of it, and a decoding step that uses that.
 *
 * The fast path proposes, the verifier decides [paper Section 4.1, 4.2]: what the fast path leaves
 * out of a long context changes how many of its candidates are reproduced, never the released stream.
 * A candidate's attention over a few blocks that a cheap score selects reads a fraction of the cache.
 *
 * The conventions of llm42.h hold here too: "dev" pointers are device addresses on the current
 * device, calls enqueue on `hip_stream`, allocate nothing (but llm42_rope_create), never synchronise, never
 * read device memory on the host, and may be captured into a graph; nothing in a workspace has to start
 * at zero.  A workspace belongs to one call at a time: calls (and replays of captured ones) that share
 * one follow each other on a stream.  Calls of these functions are deterministic.
 *
 * Rows.  Row (s, i), i < n_valid[s], is token seq_lens[s] + i of sequence s; a call has num_seqs * window rows,
 * 1 <= window <= LLM42_MAX_WINDOW, at most LLM42_MAX_ROWS; n_valid[s] may be 0, and NULL stands for window everywhere.
 * A plain array of rows holds row (s, i) at (s * window + i) * stride elements, its heads side by side; it is 16-byte aligned
 * and so are its rows.  Rows that take no part (i >= n_valid[s]; a sequence whose status is not LLM42_SEQ_OK) are left
 * as they were in every output (llm42_kv_sparse_attention looks at a row and kv head at a time, see there).  max_context (host, 1 .. 2^30) bounds seq_lens[s] + n_valid[s]: LLM42_ECAPACITY if it exceeds what
 * the block table or the rotary table holds.
 * Status of a sequence, where asked for: LLM42_SEQ_BAD_LENGTH if seq_lens[s] < 0, n_valid[s] is outside 0 .. window or their sum
 * exceeds max_context; LLM42_SEQ_BAD_BLOCK if a block-table entry that the call needs is < 0 or >= num_blocks.
 */
#ifndef LLM42_PAGED_H_
#define LLM42_PAGED_H_

#include "llm42.h"
#include "llm42_mx4.h"   /* LLM42_BF16, LLM42_F32 */

#ifdef __cplusplus
extern "C" {
#endif

/* The heads of an attention layer and the layers of a cache (caller-owned POD).  head_dim 64 or 128; n_q_heads 1 .. 16 times n_kv_heads, at most
 * 1024; n_layers at most 65535.  The layout of the cache is that of llm42_kv_cache (a cache of a model with the same numbers is such a cache). */
typedef struct {
  int32_t n_layers, n_q_heads, n_kv_heads, head_dim;
} llm42_heads;

/* Bytes of a bf16 cache of num_blocks blocks (all layers, K and V). */
llm42_status llm42_heads_kv_bytes(const llm42_heads* heads, int64_t num_blocks, size_t* out_bytes);

/* A model's numbers as llm42_heads: those of the operators on its cache.  (Other numbers can give the same bytes of cache, in another layout.) */
llm42_status llm42_model_heads(const llm42_model* model, llm42_heads* out);

/* ---- rotary positions ----------------------------------------------------------------------------------- */

#define LLM42_ROPE_HALF        0   /* pairs (j, j + rot_dim / 2)                                           */
#define LLM42_ROPE_INTERLEAVED 1   /* pairs (2 j, 2 j + 1)                                                 */

#define LLM42_ROPE_NONE   0        /* f_j = theta^(-2 j / rot_dim)                                         */
#define LLM42_ROPE_LINEAR 1        /* f_j / factor                                                         */
#define LLM42_ROPE_LLAMA3 2        /* in bands: a frequency that turns t = original_max_position f_j / (2 pi) times keeps the part
                                      x = clamp((t - low_freq_factor) / (high_freq_factor - low_freq_factor), 0, 1) of itself: f_j (x + (1 - x) / factor) */
#define LLM42_ROPE_YARN   3        /* f_j (1 - r) + f_j / factor * r, r = clamp((j - lo) / (hi - lo), 0, 1), lo and hi where a frequency turns
                                      beta_fast and beta_slow times: at(t) = rot_dim ln(original_max_position / (2 pi t)) / (2 ln theta),
                                      lo = max(0, floor(at(beta_fast))), hi = min(rot_dim - 1, ceil(at(beta_slow))), 0.001 more if they are equal */

/* Pair (a, b) of a row at position p becomes attention_factor * (a cos - b sin, b cos + a sin), angle p * (scaled f_j); features from
 * rot_dim on pass unchanged.  attention_factor 0 stands for 0.1 ln(factor) + 1 with LLM42_ROPE_YARN and for 1 without. */
typedef struct {
  int32_t rot_dim;                  /* even, 2 .. 128                                       */
  int32_t layout;                   /* LLM42_ROPE_HALF or LLM42_ROPE_INTERLEAVED            */
  int32_t scaling;                  /* LLM42_ROPE_NONE .. LLM42_ROPE_YARN                   */
  int32_t max_position;             /* positions 0 .. max_position - 1 are usable, at most 2^24 */
  int32_t original_max_position;    /* LLAMA3, YARN: >= 1                                   */
  double  theta;                    /* > 1                                                  */
  double  factor;                   /* LINEAR, LLAMA3, YARN: >= 1                           */
  double  low_freq_factor, high_freq_factor;   /* LLAMA3: 0 < low < high                    */
  double  beta_fast, beta_slow;     /* YARN: beta_fast >= beta_slow > 0                     */
  double  attention_factor;         /* >= 0                                                 */
} llm42_rope_config;

/* A table of cos and sin for every position (angles in 64 bits, held in fp32: 4 rot_dim bytes a position) on the current device.
 * Allocates it and synchronises once; belongs to the caller until llm42_rope_destroy, which waits for no work that still reads it. */
typedef struct llm42_rope llm42_rope;
llm42_status llm42_rope_create(const llm42_rope_config* cfg, llm42_rope** out);
void         llm42_rope_destroy(llm42_rope* rope);

/* ---- appending to the cache ----------------------------------------------------------------------------- */

/* Q, K and V of the call's rows: each head of Q and K divided by sqrt(mean of its squares + norm_eps) and multiplied by the gains q_norm / k_norm
 * (NULL: not), then rotated to its position (rope NULL: not); Q into q_out, K and V into the layer's cache at positions seq_lens[s] + i, overwriting
 * what was there.  Arithmetic is fp32, rounded once to bf16.  No other position is written; entries of the block table are needed for the
 * rows' own positions only.  No two sequences of a call may have positions in the same block.
 * kv_bounds (or NULL): the bounds of every block that becomes whole with the call are written as llm42_kv_bounds_store writes them; the block's earlier
 * positions must have been stored.
 * LLM42_EINVAL where num_seqs * (window / 16 + 2) * n_kv_heads exceeds 2^24.
 * q and q_out NULL: K and V alone.  q_out may be q where that is bf16 and the strides are the same; else outputs must not overlap inputs. */
llm42_status llm42_kv_append(
    const llm42_heads*    heads,
    int32_t               layer,           /* 0 .. n_layers - 1                            */
    const llm42_kv_cache* kv_cache,
    void*                 kv_bounds,       /* dev, 16-byte aligned, or NULL                */
    const void*           q,               /* dev rows of n_q_heads * head_dim, or NULL    */
    int64_t               q_stride,
    const void*           k,               /* dev rows of n_kv_heads * head_dim            */
    int64_t               k_stride,
    const void*           v,               /* dev rows of n_kv_heads * head_dim            */
    int64_t               v_stride,
    int32_t               type,            /* of q, k and v: LLM42_BF16 or LLM42_F32       */
    const void*           q_norm,          /* dev bf16 [head_dim] or NULL, 16-byte aligned */
    const void*           k_norm,          /* dev bf16 [head_dim] or NULL, 16-byte aligned */
    float                 norm_eps,        /* >= 0                                         */
    const llm42_rope*     rope,            /* of the current device, or NULL               */
    const int32_t*        seq_lens,        /* dev [num_seqs]                               */
    int32_t               window,
    const int32_t*        n_valid,         /* dev [num_seqs] or NULL                       */
    int32_t               num_seqs,
    int32_t               max_context,
    void*                 q_out,           /* dev bf16 rows of n_q_heads * head_dim, or NULL */
    int64_t               q_out_stride,
    int32_t*              seq_status,      /* dev [num_seqs] or NULL                       */
    void*                 hip_stream);

/* ---- bounds of the cached keys -------------------------------------------------------------------------- */

/* For each layer, block of 16 positions and kv head a record of 2 * head_dim + 16 bytes ([layer][block][kv head], blocks numbered as in the bf16 cache and
 * found by its block table): 2^e is the smallest power of two, e >= -40, with every |key| <= 127 * 2^e; byte f is the largest key of
 * feature f divided by 2^e and rounded up, byte head_dim + f the smallest, rounded down (signed), byte 2 * head_dim is e + 64.  A block with a NaN, an infinity or
 * a magnitude beyond 127 * 2^40 has 255 there and zeros before: it stands for -infinity .. infinity.  Nothing in fresh bounds has to
 * be initialised: no call reads those of a block that was not whole when they were stored. */
llm42_status llm42_kv_bounds_bytes(const llm42_heads* heads, int64_t num_blocks, size_t* out_bytes);

/* Bounds of every block that holds one of the positions first[s] .. first[s] + count[s] - 1 and is whole with them (all its positions are below
 * first[s] + count[s], and have been stored), of one layer or (layer -1) all.  Behind a verifier pass and its commit: first = the length before, count = the
 * committed tokens; behind a prefill: 0 and the length.  Two sequences may share blocks.  first[s] < 0, positions beyond the table's
 * capacity, count[s] outside 0 .. max_count: LLM42_SEQ_BAD_LENGTH; an entry of the table for one of those blocks out of
 * range: LLM42_SEQ_BAD_BLOCK; nothing of such a sequence is written.  LLM42_EINVAL where num_seqs times the blocks that max_count positions can touch,
 * (max_count + 14) / 16 + 1, times n_kv_heads is 2^26 or more. */
llm42_status llm42_kv_bounds_store(
    const llm42_heads*    heads,
    int32_t               layer,           /* or -1: all                                   */
    const llm42_kv_cache* kv_cache,
    void*                 kv_bounds,       /* dev, 16-byte aligned                         */
    const int32_t*        first,           /* dev [num_seqs]                               */
    const int32_t*        count,           /* dev [num_seqs]                               */
    int32_t               num_seqs,
    int32_t               max_count,       /* host: >= every count                         */
    int32_t*              seq_status,      /* dev [num_seqs] or NULL                       */
    void*                 hip_stream);

/* What the bounds of the physical blocks block_ids[j] stand for, all layers (each value is a bf16): out_lo and out_hi are bf16
 * [n_layers][num_ids][n_kv_heads][head_dim], 16-byte aligned; an id out of range gives zeros. */
llm42_status llm42_kv_bounds_read(
    const llm42_heads*    heads,
    const void*           kv_bounds,       /* dev                                          */
    int64_t               num_blocks,
    const int32_t*        block_ids,       /* dev [num_ids]                                */
    int32_t               num_ids,         /* >= 0, times n_kv_heads at most 2^27          */
    void*                 out_lo,          /* dev                                          */
    void*                 out_hi,          /* dev                                          */
    void*                 hip_stream);

/* ---- attention over selected blocks --------------------------------------------------------------------- */

#define LLM42_MAX_SELECTED 4096

/* Which blocks each row reads.  Row (s, i) sees the blocks 0 .. own, own = (seq_lens[s] + i) / 16.  For each kv head it gets all of them where they are no more than
 * `budget`; else the first `sink` and the last `recent` (its own is the last), and of those between the ones with the highest
 * scores, the lowest block on ties, so that they are `budget` together.
 * Score: a query head is rounded to whole multiples of a power of two of its own, as the bounds are (2^e, e >= -40, every |q| <= 127 * 2^e; ties to even; a head with a
 * NaN, an infinity or a magnitude beyond 127 * 2^40 counts as zeros); a block's score is the largest, over the query heads of the kv head, of
 * sum over f of max(q_f hi_f, q_f lo_f) - an upper bound of the rounded query's products with the block's keys, exact in fp32, so the selection does not
 * depend on an order of summation.  A block whose bounds are infinite comes first.
 * The bounds of blocks sink .. own - recent must have been stored; other blocks' are not read.  Block-table entries are needed for
 * all positions of the sequence.
 * selected[s][i][kv head][0 .. budget - 1]: the blocks, ascending, -1 behind them.
 * The workspace holds scores: at most 256 MiB, or what one sequence takes, 4 bytes for each row of the window, kv head and block of max_context, where that is more. */
llm42_status llm42_kv_select_workspace_bytes(const llm42_heads* heads, int32_t num_seqs, int32_t window, int32_t max_context,
                                             int32_t budget, size_t* out_bytes);
llm42_status llm42_kv_select(
    const llm42_heads*    heads,
    int32_t               layer,
    const llm42_kv_cache* kv_cache,        /* its block table and num_blocks (kv_base is not read) */
    const void*           kv_bounds,       /* dev, 16-byte aligned                         */
    const void*           q,               /* dev bf16 rows of n_q_heads * head_dim        */
    int64_t               q_stride,
    const int32_t*        seq_lens,
    int32_t               window,
    const int32_t*        n_valid,
    int32_t               num_seqs,
    int32_t               max_context,
    int32_t               budget,          /* 1 .. LLM42_MAX_SELECTED                      */
    int32_t               sink,            /* >= 0                                         */
    int32_t               recent,          /* >= 1, sink + recent <= budget                */
    int32_t*              selected,        /* dev [num_seqs][window][n_kv_heads][budget]   */
    int32_t*              seq_status,
    void*                 workspace,       /* dev, 256-byte aligned                        */
    size_t                workspace_bytes,
    void*                 hip_stream);

/* Attention of row (s, i) over the blocks selected[s][i][kv head][0 .. width - 1], in any order (llm42_kv_select's lists or others): out = softmax(scale * q . k) v over
 * the positions of those blocks up to seq_lens[s] + i, all of which must have been stored; head h uses kv head h / (n_q_heads / n_kv_heads).
 * An entry < 0 or beyond the row's own block counts for nothing, one that is listed twice counts twice; a row that lists nothing gets zeros.
 * Sums are fp32; weights enter the products with V as a sum of two bf16 (off by 2^-16 of a weight).
 * scale 0 stands for 1 / sqrt(head_dim).  Block-table entries are needed for the listed blocks only: where one of a (row, kv head)'s is out of range, the heads of that kv head
 * are left as they were and the sequence's status is LLM42_SEQ_BAD_BLOCK; the other rows are written. */
llm42_status llm42_kv_sparse_attention_workspace_bytes(const llm42_heads* heads, int32_t num_seqs, int32_t window, int32_t width,
                                                       size_t* out_bytes);
llm42_status llm42_kv_sparse_attention(
    const llm42_heads*    heads,
    int32_t               layer,
    const llm42_kv_cache* kv_cache,
    const void*           q,               /* dev bf16 rows of n_q_heads * head_dim        */
    int64_t               q_stride,
    const int32_t*        seq_lens,
    int32_t               window,
    const int32_t*        n_valid,
    int32_t               num_seqs,
    int32_t               max_context,
    const int32_t*        selected,        /* dev [num_seqs][window][n_kv_heads][width]    */
    int32_t               width,           /* 1 .. LLM42_MAX_SELECTED                      */
    float                 scale,           /* 0 .. 2^126                                   */
    void*                 out,             /* dev bf16 rows of n_q_heads * head_dim        */
    int64_t               out_stride,
    int32_t*              seq_status,
    void*                 workspace,       /* dev, 256-byte aligned                        */
    size_t                workspace_bytes,
    void*                 hip_stream);

/* ---- the fast path ---------------------------------------------------------------------------------------- */

/* llm42_decode_step_sampled with attention over selected blocks: the same arguments, effects, errors and status, and for each sequence, layer and kv
 * head llm42_kv_select's choice of `budget` blocks (sequences of no more blocks read all of them) in kv_bounds, the bounds of kv_cache (its model's numbers as llm42_heads).
 * Those of blocks that are whole below seq_lens[s] must have been stored; the step stores those of a block that its token makes whole.
 * The verifier overwrites the window's entries of the cache; llm42_kv_bounds_store behind the commit follows it.
 * workspace: llm42_decode_step_sparse_workspace_bytes for any call of 1 .. max_seqs sequences, contexts up to max_context and this budget;
 * 256-byte aligned. */
llm42_status llm42_decode_step_sparse_workspace_bytes(const llm42_model* model, int32_t max_seqs, int32_t max_context, int32_t budget,
                                                      size_t* out_bytes);
llm42_status llm42_decode_step_sparse(
    const llm42_model*    model,
    const llm42_kv_cache* kv_cache,
    void*                 kv_bounds,       /* dev, 16-byte aligned                         */
    int32_t               budget,          /* as in llm42_kv_select                        */
    int32_t               sink,
    int32_t               recent,
    const int32_t*        seq_lens,        /* dev [num_seqs]                               */
    const int32_t*        tokens,          /* dev [num_seqs]                               */
    int32_t               num_seqs,
    int32_t               max_context,     /* up to 2^30                                   */
    int32_t*              out_tokens,      /* dev [num_seqs]                               */
    int32_t*              seq_status,      /* dev [num_seqs] or NULL                       */
    void* workspace, size_t workspace_bytes, void* hip_stream,
    const llm42_sampling* sampling);       /* or NULL                                      */

#ifdef __cplusplus
}
#endif
#endif /* LLM42_PAGED_H_ */
