/*
 * jdob_edge.h — C ABI of the edge operators for MI355X (gfx950): what the
 * edge GPU computes for the users that a policy offloads.
 *
 * jdob.h decides which users offload after which sub-task of a shared DNN
 * and takes the latency alpha_l + beta_l*b of a batch of b users as given.
 * The calls here compute sub-tasks of a decoder network for such a batch:
 * the users' rows stand packed one after the other in one array (sequences
 * of different lengths, no padding), all users share the network's weights
 * and each may have a low-rank adapter of their own.
 *
 *   jdob_edge_norm     RMS norm of rows with the residual's addition; the
 *                      output in the rows' type, or in 8 bits with a scale
 *                      a row, as the 8-bit projection takes it
 *   jdob_edge_project  the shared projection of all rows beside each row's
 *                      low-rank adapter
 *   jdob_edge_attend   causal attention of packed sequences with grouped
 *                      heads; the new rows stand at the end of the
 *                      sequence's keys (a whole prompt, a chunk after a
 *                      history, a single token)
 *   jdob_edge_cache_write, jdob_edge_cache_read
 *                      new rows' keys and values into the pages of a
 *                      cache, 16-bit or quantised to 8 bits, and back
 *   jdob_edge_attend_paged
 *                      causal attention of sequences' newest rows (a
 *                      single token, a few at once) over such pages
 *
 * The conventions are those of jdob.h: array pointers are DEVICE pointers
 * owned by the caller; calls enqueue work on `hip_stream` and return without
 * synchronizing; the library allocates no device memory, keeps no mutable
 * global state and is thread-safe; the return value is a jdob_status; only
 * host-detectable errors are reported, before anything is launched
 * (JDOB_ERR_INVALID_ARG, JDOB_ERR_UNSUPPORTED), besides a failed launch
 * (JDOB_ERR_HIP).  Calls with no rows launch nothing and return JDOB_OK;
 * their array pointers may be NULL.  Calls can be captured in a HIP graph.
 * Results do not depend on what else runs: equal calls give equal bits.
 * Strides are in elements; the innermost dimension is contiguous.  Arrays
 * need the alignment of their element type only; rows whose starts are
 * multiples of 16 bytes are read faster.  Index arrays on the device are not
 * checked by the host: entries out of range never lead to an access out of
 * bounds (they are clamped, the row counts as one without an adapter, or the
 * key as absent).
 * Outputs must not overlap inputs unless an argument says that they may.
 * The operators are forward passes.
 */
#ifndef JDOB_EDGE_H
#define JDOB_EDGE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { JDOB_EDGE_BF16 = 0, JDOB_EDGE_F16 = 1, JDOB_EDGE_F32 = 2 } jdob_edge_dtype;

#define JDOB_EDGE_MAX_ROWS 1073741824
#define JDOB_EDGE_MAX_NORM_DIM 16384
#define JDOB_EDGE_MAX_PROJECT_DIM 1048576 /* 8 bits: in_dim to 131072      */
#define JDOB_EDGE_MAX_RANK 256
#define JDOB_EDGE_MAX_HEAD_DIM 128
#define JDOB_EDGE_MAX_SEQUENCES 65535

/* h = x + residual;  y_i = h_i * weight_i / sqrt(mean(h^2) + eps).
 * Sums are binary32 and start from the unrounded h; where the squares leave
 * binary32 the row is scaled by a power of two first.  8-bit output:
 * scale = max|y| / 127, q_i = y_i / scale (y before it is rounded to dtype,
 * a binary32 division) rounded to the nearest integer (to even) in
 * [-127, 127], so that q_i * scale stands for y_i (coarser below
 * max|y| = 2^-119, whose scales are subnormal); a row whose y are zeros, or
 * whose scale binary32 has no number for, has scale 0; a row with a NaN or an
 * infinity in y has scale NaN, and so has a row of zeros with eps = 0.  `sum`
 * may be x or residual itself (same stride): each row is read whole before
 * it is written.  out and q may both be asked for; sum needs a residual. */
typedef struct {
  int32_t rows, dim;       /* rows >= 0, dim >= 1, to the limits above       */
  int32_t dtype;           /* of x, residual, weight, sum, out               */
  float eps;               /* >= 0, finite                                   */
  const void *x;           /* [rows][dim]                                    */
  int64_t x_stride;        /* elements from row to row, >= dim               */
  const void *residual;    /* [rows][dim], or NULL                           */
  int64_t residual_stride;
  const void *weight;      /* [dim]                                          */
  void *sum;               /* [rows][dim] h rounded to dtype, or NULL        */
  int64_t sum_stride;
  void *out;               /* [rows][dim] y rounded to dtype, or NULL        */
  int64_t out_stride;
  int8_t *q;               /* [rows][dim] 8-bit y, or NULL                   */
  int64_t q_stride;
  float *scale;            /* [rows], with q                                 */
} jdob_edge_norm_args;

int jdob_edge_norm(const jdob_edge_norm_args *a, void *hip_stream);

/* out = x W^T + gain_a ((x A_a^T) B_a^T), a = row_adapter[row].
 * x and W are of dtype (16 bits), or both 8-bit integers that stand for
 * x * x_scale[row] and W * weight_scale[column]; the adapters are of dtype
 * always.  Sums are binary32 (8-bit products: integers, exact for any codes,
 * in_dim <= 131072); the low-rank rows x A_a^T are kept in binary32 in the
 * workspace or, from 65 rows on, as two 16-bit parts (16 bits of mantissa with
 * bfloat16; 22 with binary16, whatever their size, for ranks that are not more
 * than 2^17 times smaller than the largest of 16).
 * An adapter with a rank below max_rank uses the first `rank` rows of A and
 * columns of B; what lies behind them is not used.                          */
typedef struct {
  int32_t rows, in_dim, out_dim;  /* rows >= 0, the others >= 1              */
  int32_t dtype;                  /* BF16 or F16: out, adapters, 16-bit x, W */
  int32_t bits8;                  /* 1: x and W are int8_t, with scales      */
  const void *x;                  /* [rows][in_dim]                          */
  int64_t x_stride;
  const float *x_scale;           /* [rows], 8 bits only                     */
  const void *weight;             /* [out_dim][in_dim]                       */
  int64_t weight_stride;
  const float *weight_scale;      /* [out_dim], 8 bits only                  */
  int32_t num_adapters, max_rank; /* 0: no adapters, the arrays are not read */
  const void *down;               /* A [num_adapters][max_rank][in_dim]      */
  const void *up;                 /* B [num_adapters][out_dim][max_rank]     */
  const float *gain;              /* [num_adapters]                          */
  const int32_t *rank;            /* [num_adapters], or NULL: max_rank       */
  const int32_t *row_adapter;     /* [rows]; outside [0, num_adapters): none */
  void *out;                      /* [rows][out_dim]                         */
  int64_t out_stride;
  void *workspace;                /* jdob_edge_project_workspace bytes       */
  int64_t workspace_bytes;
} jdob_edge_project_args;

/* Bytes that jdob_edge_project needs (16-byte aligned; 0 without adapters);
 * -1 where the arguments are not valid.  Only the sizes are read.           */
int64_t jdob_edge_project_workspace(const jdob_edge_project_args *a);
int jdob_edge_project(const jdob_edge_project_args *a, void *hip_stream);

/* Causal attention.  Sequence u has rows query_start[u] .. query_start[u+1]-1
 * of q and out (n of them) and rows key_start[u] .. +key_count[u]-1 of k and v
 * (m of them); its row i sees its keys 0 .. m - n + i:
 *   out = sum_j p_j v_j,  p = softmax_j(scale * q . k_j).
 * Head h reads key head h / (num_heads / num_kv_heads).  A row that sees no
 * key (m - n + i < 0) is zero.  Keys and values that a row does not see never
 * change it, infinities and NaN among them; an infinite value that it does
 * see makes its column an infinity or a NaN.  Scores, maxima, sums and the
 * output are binary32; p is rounded to dtype before it is multiplied with v
 * (relative error 2^-8 or 2^-11 of each term, the size of out's own rounding;
 * binary16 has fewer bits of p below 2^-14 of the largest and nothing of it
 * below 2^-25, which the sum that divides has).  Division comes last: sums of
 * values beyond 2^119 / m may pass binary32.
 * max_queries and max_keys are at least the largest n and m (both only size
 * the launch and choose the kernel for all of the call's sequences); rows
 * beyond max_queries may be left unwritten.                                */
typedef struct {
  int32_t num_sequences;          /* 0 .. JDOB_EDGE_MAX_SEQUENCES            */
  int32_t num_heads, num_kv_heads;/* num_heads a multiple of num_kv_heads, to 1024 */
  int32_t head_dim;               /* a multiple of 8, to JDOB_EDGE_MAX_HEAD_DIM */
  int32_t dtype;                  /* BF16 or F16                             */
  int32_t max_queries, max_keys;  /* >= 0                                    */
  float scale;                    /* > 0, finite                             */
  int64_t query_rows, key_rows;   /* rows of q and out, of k and v           */
  const void *q;                  /* [query_rows][num_heads][head_dim]       */
  int64_t q_stride, q_head_stride;
  const void *k;                  /* [key_rows][num_kv_heads][head_dim]      */
  int64_t k_stride, k_head_stride;
  const void *v;
  int64_t v_stride, v_head_stride;
  const int32_t *query_start;     /* [num_sequences + 1], ascending          */
  const int64_t *key_start;       /* [num_sequences]                         */
  const int32_t *key_count;       /* [num_sequences]                         */
  void *out;                      /* [query_rows][num_heads][head_dim]       */
  int64_t out_stride, out_head_stride; /* no two rows or heads share elements  */
  void *workspace;                /* jdob_edge_attend_workspace bytes        */
  int64_t workspace_bytes;
} jdob_edge_attend_args;

/* Bytes that jdob_edge_attend needs (16-byte aligned; 0 where the keys are
 * not split over workgroups); -1 where the arguments are not valid.  Only
 * the sizes are read.                                                       */
int64_t jdob_edge_attend_workspace(const jdob_edge_attend_args *a);
int jdob_edge_attend(const jdob_edge_attend_args *a, void *hip_stream);

/* A paged cache of keys and values.  Key j of a sequence stands on page
 * table[j / page_size] of the sequence's row of a table, in slot
 * j % page_size.  A key is absent where j / page_size is not below the table's
 * width or the entry is outside [0, num_pages): pages that have been given
 * back (keys behind a window) or not been taken yet.  Sequences may share
 * pages that none of them writes.
 * With bits8 = 0 k and v hold rows of dtype.  With bits8 = 1 they hold 8-bit
 * codes that stand for code * scale of their slot and head:
 *   scale = max|x| / 127,  code = x / scale (binary32 divisions) rounded to
 * the nearest integer (to even) in [-127, 127]; zeros have scale 0, a row
 * with a NaN or an infinity has codes 0 and scale NaN (below max|x| = 2^-119
 * scales are subnormal and codes coarser).  dtype is then that of the rows
 * outside the cache.  Slots that no row was written to may hold anything.   */
#define JDOB_EDGE_MAX_PAGE_SIZE 65536

typedef struct {
  int32_t num_pages, page_size;   /* >= 0; 1 .. JDOB_EDGE_MAX_PAGE_SIZE      */
  int32_t num_kv_heads, head_dim; /* 1 .. 1024; as in jdob_edge_attend       */
  int32_t dtype;                  /* BF16 or F16                             */
  int32_t bits8;                  /* 1: k and v are int8_t, with scales      */
  void *k;                        /* [num_pages][num_kv_heads][page_size][head_dim] */
  int64_t k_page_stride, k_head_stride, k_slot_stride; /* any order of the three */
  void *v;
  int64_t v_page_stride, v_head_stride, v_slot_stride;
  float *k_scale;                 /* [num_pages][num_kv_heads][page_size], 8 bits only */
  int64_t k_scale_page_stride, k_scale_head_stride, k_scale_slot_stride;
  float *v_scale;
  int64_t v_scale_page_stride, v_scale_head_stride, v_scale_slot_stride;
} jdob_edge_cache;

/* Sequence u has rows row_start[u] .. row_start[u+1]-1 of k and v (n of
 * them), which are the last of its m = key_count[u] keys: its row i is key
 * m - n + i.  jdob_edge_cache_write puts the rows into the cache; a row whose
 * key is absent or negative, or that belongs to no sequence, is left out, and
 * nothing else of the cache changes.  At most one row may be written to a
 * slot.  jdob_edge_cache_read does the reverse with the same arguments:
 * 8-bit rows become code * scale rounded to dtype, a row whose key is absent
 * or negative becomes zeros, a row of no sequence is left as it was; there no
 * two rows or heads of k or of v may share elements.                        */
typedef struct {
  jdob_edge_cache cache;
  int32_t num_sequences;          /* 0 .. JDOB_EDGE_MAX_SEQUENCES            */
  int32_t table_width;            /* >= 0                                    */
  const int32_t *table;           /* [num_sequences][table_width]            */
  int64_t table_stride;           /* >= table_width                          */
  const int32_t *row_start;       /* [num_sequences + 1], ascending          */
  const int32_t *key_count;       /* [num_sequences]                         */
  int32_t rows;                   /* of k and v                              */
  void *k;                        /* [rows][num_kv_heads][head_dim]          */
  int64_t k_stride, k_head_stride;
  void *v;
  int64_t v_stride, v_head_stride;
} jdob_edge_cache_rows_args;

int jdob_edge_cache_write(const jdob_edge_cache_rows_args *a, void *hip_stream);
int jdob_edge_cache_read(const jdob_edge_cache_rows_args *a, void *hip_stream);

/* jdob_edge_attend with keys and values on pages: sequence u's rows
 * query_start[u] .. query_start[u+1]-1 stand at the end of its key_count[u]
 * keys and see those of them that are there.  Made for few rows a sequence:
 * the keys are read once for every 32 rows times heads of a key head.  All
 * else is as in jdob_edge_attend, but that p (with an 8-bit cache p * scale of
 * the value) goes into its product as 16-bit parts that hold 16 bits of its
 * mantissa from 2^-118 on (with a binary16 cache from 2^-76 on: what less
 * weight adds, such an output cannot show), and that sums of values pass
 * binary32 nowhere: a mean of finite values is finite, and then rounded to
 * dtype.  How the keys are split, and with it the order of sums, follows from
 * the lengths of all sequences.                                             */
typedef struct {
  jdob_edge_cache cache;
  int32_t num_sequences, table_width;
  const int32_t *table;
  int64_t table_stride;
  const int32_t *query_start;     /* [num_sequences + 1], ascending          */
  const int32_t *key_count;       /* [num_sequences]                         */
  int32_t num_heads;              /* a multiple of num_kv_heads, to 1024     */
  int32_t max_queries, max_keys;  /* >= 0, as in jdob_edge_attend            */
  float scale;                    /* > 0, finite                             */
  int64_t query_rows;             /* rows of q and out                       */
  const void *q;                  /* [query_rows][num_heads][head_dim]       */
  int64_t q_stride, q_head_stride;
  void *out;                      /* [query_rows][num_heads][head_dim]       */
  int64_t out_stride, out_head_stride; /* no two rows or heads share elements  */
  void *workspace;                /* jdob_edge_attend_paged_workspace bytes  */
  int64_t workspace_bytes;
} jdob_edge_attend_paged_args;

/* Bytes that jdob_edge_attend_paged needs (16-byte aligned; 0 where the keys
 * are not split over workgroups); -1 where the arguments are not valid.  Only
 * the sizes are read.                                                       */
int64_t jdob_edge_attend_paged_workspace(const jdob_edge_attend_paged_args *a);
int jdob_edge_attend_paged(const jdob_edge_attend_paged_args *a, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* JDOB_EDGE_H */
