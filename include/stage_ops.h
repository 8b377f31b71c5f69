/*
 * stage_ops.h -- operators around a decoder layer's projections, on the caller's own tensors.
 *
 * The stage (include/stage.h) runs whole layers on its own cache and workspaces.  These functions give
 * a program that keeps its own cache, or runs layers of another make, the same kernels one by one: the
 * norm of each query and key head with the position rotation and the append to a paged cache, attention
 * with a sliding window and sinks over that cache, and low-rank adapters beside a shared projection.
 *
 * Conventions, besides those of stage.h (0 or a negative stage_status; nothing throws or aborts):
 *  - Every pointer in the structs is device memory of `device`, unless stated otherwise.  A call checks its
 *    arguments on the host before it enqueues anything; what only the device knows (row starts, lengths,
 *    block ids, positions, adapter ids) is checked by the kernels, which leave out what is out of range
 *    as each function states, so no value of theirs is read or written out of bounds.
 *  - Work is enqueued on `stream` (a hipStream_t of `device`; NULL: its null stream) and the call returns before
 *    it runs; its buffers, workspace among them, must stay until then.  Nothing is allocated and nothing waits, so
 *    calls may be captured into a HIP graph.  Calls may run at once on several streams and host threads if they share
 *    no output and no workspace.
 *  - Row strides (*_ld) are in elements.  Rows start on 16-byte boundaries: pointers and row strides in
 *    bytes are multiples of 16 (EINVAL otherwise).
 *  - EINVAL: a size, type, stride or pointer that the function does not take; ENOMEM: the workspace is
 *    smaller than the function's *_workspace says; EHIP: the launch failed.
 */
#ifndef PAPER_2512_21835_STAGE_OPS_H
#define PAPER_2512_21835_STAGE_OPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define STAGE_F32 0
#define STAGE_BF16 1

/* Most rows of a call, most sequences, and most block-table entries of a sequence. */
#define STAGE_OPS_MAX_ROWS 1048560
#define STAGE_OPS_MAX_SEQS 65536
#define STAGE_OPS_MAX_BLOCKS 1048576
#define STAGE_OPS_MAX_RANK 256

/* The sequences of a call and their rows.  Sequence i owns rows row_start[i] .. row_start[i + 1] - 1 of the
   call's buffers and holds length[i] tokens (0 to 2^30) once they are counted in: its row t sits at position length[i]
   - (row_start[i + 1] - row_start[i]) + t.  A sequence may have no row.  row_start ascends; rows before row_start[0] and
   from row_start[n_seqs] on are padding, which no function writes and no result depends on.  Position p is in block
   block_table[i][p / 16], place p % 16. */
typedef struct {
    int32_t n_seqs;
    int32_t max_rows;   /* no sequence has more rows (rows beyond are left out) */
    int32_t max_len;    /* no sequence holds more tokens (tokens beyond are left out); <= 16 max_blocks */
    int32_t max_blocks; /* entries of a block-table row */
    const int32_t *row_start;   /* [n_seqs + 1] */
    const int32_t *length;      /* [n_seqs] */
    const int32_t *block_table; /* [n_seqs][max_blocks] */
} stage_batch;

/* The paged cache of one layer, laid out as the stage's: [n_blocks][K|V][n_kv_heads][16][head_dim]. */
typedef struct {
    void *pool;
    int32_t n_blocks, n_kv_heads;
    int32_t head_dim; /* 64 or 128 */
    int32_t type;     /* STAGE_F32 or STAGE_BF16 */
} stage_cache;

/* Norm of the query and key heads, rotation, and append to the cache, in one pass.

   For each row: the heads of qkv are n_q_heads query heads, then the cache's n_kv_heads key heads and as
   many value heads, head_dim wide.  A query (key) head x becomes x / sqrt(mean(x^2) + eps) * q_gain (k_gain), or
   stays x where the gain is NULL; then its pairs (i, i + head_dim / 2) turn by the angle of pair i at the
   row's position (rotate-half: y_i = x_i cos - x_i' sin, y_i' = x_i sin + x_i' cos).  Queries go to q_out, keys and
   values (as they are) to the row's position of the cache.  Sums and rotation are in fp32; each result is rounded
   once, to nearest even.

   positions NULL: the angle's position is the row's position in its sequence.  Else positions [n_axes][rows], and
   with n_axes 3 the first section[0] pairs take the first axis (time), the next section[1] the second
   (height), the last section[2] the third (width), for images and video; n_axes 1: section[0] is head_dim / 2.

   A row is left out (q_out and the cache keep what they hold) if its position is negative, not below max_len, or its
   block id is not one of the pool's, or if an angle's position is not in [0, n_angles); positions of an axis without
   pairs do not matter.  Two rows of a call must not name the same place of the cache.  q_out may be qkv itself, with the
   same type and stride. */
typedef struct {
    int32_t device;
    stage_batch batch;
    stage_cache cache;
    int32_t rows;      /* rows that qkv, q_out and positions hold */
    int32_t n_q_heads; /* n_kv_heads times 1, 2, 4 or 8 */
    const void *qkv;   /* [rows, qkv_ld >= (n_q_heads + 2 n_kv_heads) head_dim] */
    void *q_out;       /* [rows, q_ld >= n_q_heads head_dim] */
    int64_t qkv_ld, q_ld;
    int32_t qkv_type, q_type;
    const void *q_gain, *k_gain; /* bf16 [head_dim], or NULL */
    float eps;
    int32_t n_angles;            /* rows of cos and sin */
    const float *cos, *sin;      /* [n_angles][head_dim / 2] */
    const int32_t *positions;    /* [n_axes][rows], or NULL */
    int32_t n_axes;              /* 1 or 3 */
    int32_t section[3];          /* pairs per axis; they sum to head_dim / 2 */
} stage_append_args;
int stage_norm_rope_append(const stage_append_args *a, void *stream);

/* Grouped-query attention over the paged cache with a sliding window and sinks, for prompts and single tokens
   in one call: a row at position p sees the positions j <= p of its sequence with j > p - window or j < sinks
   (window 0: every j <= p).  out = sum_j softmax_j(scale q k_j) v_j; query head h reads KV head h / (n_q_heads /
   n_kv_heads).  Products, softmax statistics and sums are in fp32 or more exact: with fp32 activations the
   operands of the matrix instructions are exact sums of bf16 terms (or fp32, with an fp32 cache); with bf16
   activations the probabilities, and the values of an fp32 cache, may be held to 2^-16 of their sizes.  Nothing of
   a place that a row does not see reaches its result, infinities and NaN among it; those that it sees give what they give
   in the formula.  Tokens in blocks whose id is not one of the pool's are not seen; a row that sees none (its position is
   negative, say), or none of a score above -inf, becomes 0.  out may be q itself, with the same stride; else they share
   no element.  The order in which a row's keys are added up goes by the call's sizes (rows, sequences, longest length): the
   same call gives the same bits, the same row in another call the same to rounding. */
typedef struct {
    int32_t device;
    stage_batch batch;
    stage_cache cache;
    int32_t rows;      /* rows that q and out hold */
    int32_t n_q_heads; /* n_kv_heads times 1, 2, 4 or 8 */
    int32_t window;    /* >= 0; 0: no window */
    int32_t sinks;     /* >= 0 */
    float scale;       /* 0: 1 / sqrt(head_dim); else of a size from 1e-30 to 1e30 */
    const void *q;     /* [rows, q_ld >= n_q_heads head_dim] */
    void *out;         /* [rows, out_ld >= n_q_heads head_dim] */
    int64_t q_ld, out_ld;
    int32_t type;      /* of q and out */
} stage_window_args;
/* Bytes of workspace that the call with these arguments takes (0: none; pointers are not looked at). */
int stage_window_workspace(const stage_window_args *a, int64_t *bytes);
/* workspace: 16-byte aligned; holds nothing between calls and need not be cleared. */
int stage_window_attention(const stage_window_args *a, void *workspace, int64_t workspace_bytes, void *stream);

/* Low-rank adapters of many requests beside a shared projection:
       out[r] = base[r] + scales[i] * B_i (A_i x[r]),  i = ids[r],
   with the first ranks[i] rows of A_i and columns of B_i (NULL: all max_rank); a row whose id is not in [0, n_adapters)
   has no adapter and becomes base[r].  Sums are in fp32 (A_i x[r] too), the operands of the matrix instructions exact
   (fp32 ones as sums of bf16 terms); each result is rounded once.  Infinities and NaN give what they give in the formula.  out may be base itself, with the same stride. */
typedef struct {
    int32_t device;
    int32_t rows;
    int32_t k, n;              /* widths of x and out; multiples of 8 */
    int32_t n_adapters;
    int32_t max_rank;          /* a multiple of 4, at most STAGE_OPS_MAX_RANK */
    int32_t type;              /* of x, base and out */
    const void *x;             /* [rows, x_ld >= k] */
    const void *base;          /* [rows, base_ld >= n]; base_ld up to 2^25 */
    void *out;                 /* [rows, out_ld >= n] */
    int64_t x_ld, base_ld, out_ld;
    const void *a;             /* bf16 [n_adapters][max_rank][k] */
    const void *b;             /* bf16 [n_adapters][n][max_rank] */
    const int32_t *ids;        /* [rows] */
    const int32_t *ranks;      /* [n_adapters], or NULL */
    const float *scales;       /* [n_adapters], or NULL: 1 */
} stage_adapter_args;
int stage_adapter_workspace(const stage_adapter_args *a, int64_t *bytes);
int stage_adapter_add(const stage_adapter_args *a, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PAPER_2512_21835_STAGE_OPS_H */
