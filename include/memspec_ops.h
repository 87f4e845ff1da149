/*
 * memspec_ops.h - op-level entry points of the same library (libmemspec.so).
 *
 * These expose single kernels of the draft-then-verify step so that each can
 * be checked and timed on its own.  Same conventions as memspec.h: device
 * pointers are caller-owned, work is enqueued on the given stream, arguments
 * are validated before anything is enqueued.
 */
#ifndef MEMSPEC_OPS_H_
#define MEMSPEC_OPS_H_

#include "memspec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Scratch bytes that memspec_op_linear needs for (rows, n_out, k): arrival
 * counters and split-K partial sums. */
memspec_status memspec_op_linear_scratch_bytes(int32_t rows, int32_t n_out, int32_t k,
                                               size_t* bytes);

/* y[rows][n_out] (fp32) = x[rows][k] (bf16, row-major) . w[n_out][k]^T (bf16).
 * A weight-streaming GEMM: TMA-staged weight tiles, tcgen05 MMA into TMEM,
 * stream-K over the SMs, deterministic split-K reduction (above 16 rows, split
 * row tiles are finished by a second launch on the same stream, one CTA per
 * row tile and 16-row chunk).  Up to 16 rows and from 161 it runs the kernels
 * of the verify and draft passes' projections (Q/K/V, O, gate/up, down, LM
 * head) with one activation plane for their two; from 17 to 160 one that no
 * pass runs.
 * rows in 1..256, k a multiple of 8, n_out >= 1, and
 * ceil(n_out/128) * ceil(k/64) * (SMs + 1) below 2^32.
 * scratch_dev: memspec_op_linear_scratch_bytes bytes, 256-byte aligned, zeroed
 * once before its first use.  One scratch of the largest call's size serves
 * calls of any sizes that run one after another; calls that may overlap (other
 * streams) need scratches of their own.
 * status_dev: uint32 device word, bits set on in-kernel errors (may be NULL).
 * x, w: 16-byte aligned.  Errors: INVALID_ARG, UNSUPPORTED, CUDA. */
memspec_status memspec_op_linear(const void* x_dev, const void* w_dev, float* y_dev,
                                 int32_t rows, int32_t n_out, int32_t k,
                                 void* scratch_dev, size_t scratch_bytes,
                                 uint32_t* status_dev, void* stream);

/* The same product as memspec_op_linear (y = x . w^T, fp32 out), by the kernel
 * that it runs for 17 to 160 rows, for callers that cannot allocate device
 * memory: plug-ins whose host application owns all device memory, fixed-budget
 * deployments that allocate only at start-up, and latency-critical loops that
 * cannot afford cudaMalloc / cudaFree (which may synchronise the device).  The
 * paper has no counterpart; this is a property of the library's interface.
 * Instead of a scratch argument it uses one file-scope device array of about
 * 2.6 MB that every GPU loading the library keeps until the process exits.
 * Limits: rows in 1..16, n_out in 1..131072, k a positive multiple of 8 up to
 * 2^20; x and w 16-byte aligned.  Larger sizes return MEMSPEC_ERR_INVALID_ARG
 * (message in memspec_op_last_error) and enqueue nothing.  The call allocates
 * nothing; it enqueues a clear of the array's counters and the kernel on
 * `stream`.  Its kernel and split-K grid differ from memspec_op_linear's, so
 * results agree with it within rounding, not bit for bit.
 * All calls share the array: calls that overlap on the GPU (other streams,
 * other host threads) race - serialise them.  The first call on a device looks
 * up the array's address on that device; make it before any stream capture.
 * status_dev: optional uint32 device word for in-kernel error bits (NULL: an
 * internal word that the caller cannot read is used). */
memspec_status memspec_op_linear_noalloc(const void* x_dev, const void* w_dev, float* y_dev,
                                         int32_t rows, int32_t n_out, int32_t k,
                                         uint32_t* status_dev, void* stream);

/* Group-wise INT4 weight-only linear layer (the paper's targets are GPTQ INT4
 * models, Section 4.1).  The weights W[n_out][k] are given GPTQ-style,
 *   W[r][c] = (q[r][c] - zeros[r][c/128]) * scales[r][c/128],
 *   qweight: uint8 [n_out][k/2], byte j of row r = q[r][2j] | q[r][2j+1] << 4
 *   scales:  bf16  [n_out][k/128];   zeros: uint8 [n_out][k/128], values 0..15
 * and are repacked once, by memspec_int4_pack, into the kernel's layout (one
 * 1072-byte record per 16-row tile and 128-column group, codes regrouped
 * within each 32-bit word; rows past n_out are zero-filled).  The layout is private to this library: only
 * memspec_op_linear_int4 reads it.
 *
 * memspec_int4_packed_bytes: bytes of the packed copy, or -1 for bad sizes
 * (n_out >= 1, k a positive multiple of 128). */
int64_t memspec_int4_packed_bytes(int32_t n_out, int32_t k);

/* Repack on `stream` (device pointers; qweight 4-byte, scales 2-byte, packed
 * 16-byte aligned; packed holds memspec_int4_packed_bytes).  The caller owns
 * every buffer; nothing is allocated.  Errors: INVALID_ARG (n_out outside
 * 1..1048576, k not a positive multiple of 128, NULL, misalignment), CUDA. */
memspec_status memspec_int4_pack(const void* qweight_dev, const void* scales_dev, const void* zeros_dev,
                                 int32_t n_out, int32_t k, void* packed_dev, void* stream);

/* y[rows][n_out] (fp32) = x[rows][k] (bf16, row-major) . W^T, enqueued on
 * `stream`.  rows in 1..16; x and packed 16-byte aligned, y 4-byte aligned;
 * the activations (rows (2k + 64) bytes) plus a ring of at least two
 * 1072-byte records per warp (16 warps) must fit in 220 KB of shared memory
 * (else UNSUPPORTED: e.g. rows 9..16 at k = 11008).  Results are
 * deterministic.  status_dev: optional uint32 device word; bit 0 is set if a
 * wait for a bulk copy ran out (about a second; y is then incomplete).
 * Allocates nothing and keeps no state between calls.
 * Errors: INVALID_ARG (sizes, NULL, misalignment), UNSUPPORTED, CUDA. */
memspec_status memspec_op_linear_int4(const void* x_dev, const void* packed_dev, float* y_dev, int32_t rows,
                                      int32_t n_out, int32_t k, uint32_t* status_dev, void* stream);

/* Categorical sampling of each row of logits[rows][vocab] (fp32): with T > 0,
 * out[r] = smallest j with sum_{i<=j} exp(z_i/T - m) > u[r] * sum_i exp(z_i/T - m);
 * with T == 0, out[r] = argmax (lowest id on ties).  u_dev: fp32 [rows] in
 * (0,1) (ignored for T == 0).  This is the draft-token sampler of
 * memspec_draft_step. */
memspec_status memspec_op_sample(const float* logits_dev, int32_t rows, int32_t vocab,
                                 float temperature, const float* u_dev, int32_t* out_dev,
                                 void* stream);

/* ---- sampling rules -------------------------------------------------------
 * What a row of logits is cut down to before it is drawn from.  Weights are
 * w_i = exp((z_i - max z) / T); the row's ids are ordered by descending logit,
 * equal logits by ascending id; each part keeps a prefix of that order, and the
 * shortest one counts:
 *   top_k  the first k ids (0: all)
 *   top_p  of those, the shortest prefix whose weights sum to at least top_p
 *          times the sum over them (1: all)
 *   min_p  the ids with w_i >= min_p (0: all)
 * temperature 0: the first id of the largest logit alone; above 0 and below
 * 1e-30: 1e-30.
 * A NaN logit counts as -inf, +inf as the largest finite float; an id at -inf is
 * never kept.  Sums and their comparisons are exact over weights that are off by
 * at most 2^-29.9 of themselves (and 2^-46 of the largest; below 2^-45 of it they
 * are 0): the same input gives the same result however the work is split.
 * Each part is one number for all rows, or (pointer not NULL) a device array of
 * one value per row, which the call cannot check: there a temperature that is
 * not above 0 (NaN too) is 0, a top_k below 1 and a top_p of 1 or more or NaN
 * are off, a top_p of 0 or less keeps one id, a min_p that is not above 0 is
 * off, one above 1 counts as 1. */
typedef struct memspec_filter {
  float temperature;            /* >= 0 */
  int32_t top_k;                /* >= 0 */
  float top_p;                  /* in (0, 1] */
  float min_p;                  /* in [0, 1] */
  const float* temperature_dev; /* [rows] or NULL */
  const int32_t* top_k_dev;
  const float* top_p_dev;
  const float* min_p_dev;
} memspec_filter;

/* out[r] = the smallest kept id j of row r with sum_{i<=j} w_i > u[r] sum_i w_i
 * over the kept ids; -1 for a row without any finite logit.  With no part of the
 * rule on this is memspec_op_sample's draw (but for roundings at a border
 * between two ids, which here are those of the weights alone).
 * logits_dev: row r (fp32) starts at logits_dev + r * ld, ld >= vocab; u_dev:
 * fp32 [rows] in [0, 1) (below: as 0, 1 and above: the last kept id).  rows in
 * 1..65535, vocab in 1..131072.  Enqueued on `stream`; nothing is allocated.
 * Errors: INVALID_ARG, CUDA. */
memspec_status memspec_op_sample_filtered(const float* logits_dev, int64_t ld, int32_t rows, int32_t vocab,
                                          const memspec_filter* filter, const float* u_dev,
                                          int32_t* out_dev, void* stream);

/* The same cut as a mask: out[r][i] = logits[r][i] where id i is kept (as it
 * counts: +inf as the largest finite float), else -inf.  out_dev may be
 * logits_dev (then out_ld == ld); otherwise the two must not overlap.  Columns
 * past vocab are not written.  Otherwise as memspec_op_sample_filtered. */
memspec_status memspec_op_filter_logits(const float* logits_dev, int64_t ld, int32_t rows, int32_t vocab,
                                        const memspec_filter* filter, float* out_dev, int64_t out_ld,
                                        void* stream);

/* ---- low-rank adapters beside a shared projection --------------------------
 * The adapters of one projection, stacked: adapter a adds scale[a] * B[a] A[a]
 * to the projection's weight.  Adapters of smaller rank occupy the first
 * ranks[a] rows of A[a] and columns of B[a]; the rest is not used. */
typedef struct memspec_lora {
  const void* a_dev;          /* bf16 [n_adapters][rank][k] */
  const void* b_dev;          /* bf16 [n_adapters][n_out][rank] */
  const float* scales_dev;    /* fp32 [n_adapters], or NULL: 1 */
  const int32_t* ranks_dev;   /* [n_adapters], clamped to 0..rank, or NULL: rank */
  int32_t n_adapters;
  int32_t rank;               /* a multiple of 8 in 8..128 */
} memspec_lora;

/* Scratch bytes of memspec_op_lora.  Errors: INVALID_ARG. */
memspec_status memspec_op_lora_scratch_bytes(int32_t rows, int32_t n_out, int32_t k, int32_t rank,
                                             size_t* bytes);

/* y[r] = base[r] + scale[a] * B[a] (A[a] x[r]) with a = ids[r], the adapter of
 * row r (ids_dev: int32 [rows]; an id outside 0..n_adapters-1: no adapter,
 * y[r] = base[r]).  base_dev is typically what memspec_op_linear or
 * memspec_op_linear_int4 gave for the same x, or NULL for 0; it may be y_dev
 * (then ld_base == ldy), otherwise the two must not overlap; y and scratch
 * overlap nothing else.  x bf16, base and y fp32; rows at strides ldx, ld_base,
 * ldy (elements, at least a row and at most 2^40; ldx a multiple of 8; of a
 * single row they are not read).  rows in 1..256, k a positive multiple of 8,
 * n_adapters, n_out and k at most 2^24; x, A, B and scratch 16-byte aligned.
 * Products are of bf16 values, sums fp32; A x enters the second product with
 * all its 24 bits.
 * Deterministic.  A row of x or an adapter with an infinity or a NaN among the
 * values that are used makes its own rows of y unspecified, no others.
 * scratch_dev: memspec_op_lora_scratch_bytes bytes of any content; calls that
 * may overlap need scratches of their own.
 * Errors: INVALID_ARG, CUDA. */
memspec_status memspec_op_lora(const memspec_lora* adapters, const void* x_dev, int64_t ldx,
                               const int32_t* ids_dev, const float* base_dev, int64_t ld_base,
                               float* y_dev, int64_t ldy, int32_t rows, int32_t n_out, int32_t k,
                               void* scratch_dev, size_t scratch_bytes, void* stream);

/* ---- a layer's cache and attention -----------------------------------------
 * What lies between a layer's Q/K/V projection and its O projection, for callers
 * that put layers together from the calls above; the steps' own projections and
 * attention are others.
 *
 * The keys and values of one layer: position `pos` of sequence `seq` in head h
 * starts at k_dev + seq * seq_stride + h * head_stride + pos * pos_stride
 * (elements; a stride of a dimension of size 1 is not read), head_dim values
 * without gaps.  Without scales they are bf16 (a layer of a context's own cache is
 * one of these); with them signed 8-bit codes, value = code * scale, one fp32
 * scale per vector at scale + seq * scale_seq_stride + ...  A scale below 2^-64
 * counts as 2^-64.  k and v 16-byte aligned, their strides multiples of 16 bytes and
 * at most 2^38 elements, positions at least head_dim apart.  Sequences or heads may
 * lie on one another (stride 0) in a cache that is only read. */
typedef struct memspec_kv {
  void* k_dev;
  void* v_dev;
  float* k_scale_dev;       /* NULL, then v_scale_dev too: bf16 */
  float* v_scale_dev;
  int64_t seq_stride, head_stride, pos_stride;
  int64_t scale_seq_stride, scale_head_stride, scale_pos_stride;
  int32_t n_seq, n_heads;   /* heads: 1..1024 */
  int32_t max_pos;          /* positions: 1..2^30 */
  int32_t head_dim;         /* 64 or 128 */
} memspec_kv;

/* Which rows of a call belong to which sequence: rows starts[b] .. starts[b+1]-1
 * to the cache's b-th, whose positions with these rows' own are lens[b]; row j of
 * the n has slot lens[b] - n + j.  A sequence may have no rows.  Both arrays are
 * the device's and cannot be checked: starts have to ascend; what lies outside the
 * call's rows, and slots outside 0..max_pos-1, do not count.  Rows in no sequence
 * are left as they were in every output. */
typedef struct memspec_batch {
  const int32_t* starts_dev;   /* [n_seq + 1] */
  const int32_t* lens_dev;     /* [n_seq] */
  int32_t n_seq;               /* 1..1024, at most the cache's */
  int32_t rows;                /* of the call's tensors: 1..65535 */
} memspec_batch;

typedef enum memspec_value_type { MEMSPEC_F32 = 0, MEMSPEC_BF16 = 1 } memspec_value_type;

/* cos and sin of pos * base^(-2i/head_dim), angles in 64 bits: fp32
 * [2][positions][head_dim/2]. */
memspec_status memspec_op_rope_table(int32_t positions, int32_t head_dim, float base, float* table_dev,
                                     void* stream);

typedef struct memspec_append {
  const void* qkv_dev;        /* rows of [n_heads | kv heads | kv heads][head_dim] */
  int32_t qkv_type;           /* memspec_value_type */
  int32_t n_heads;            /* 1..1024 */
  int64_t ld;                 /* elements from row to row, even (of a single row not read) */
  const float* rope_dev;      /* memspec_op_rope_table's, or NULL: no rotation */
  int32_t rope_positions;
  int32_t prefix_len;         /* positions before the cache's first slot */
  const int32_t* offsets_dev; /* [rows] or NULL: j */
  const void* q_gain_dev;     /* bf16 [head_dim], or NULL with k_gain_dev: no norms */
  const void* k_gain_dev;
  float eps;                  /* >= 0 */
  void* q_dev;                /* out: bf16 [rows][n_heads][head_dim] */
} memspec_append;

/* The rows of a Q/K/V projection (memspec_op_linear's result, say) into queries and
 * into the cache, at the rows' slots.  Each head's q and k become
 * x / sqrt(mean(x^2) + eps) * gain, then the pairs (i, i + head_dim/2) are turned by
 * the angles of position prefix_len + lens[b] - n + offset (a draft tree's row: its
 * depth).  q is rounded to bf16; k and v to bf16, or to codes rint(x / s) with
 * s = max(max|x|, 127 * 2^-64) / 127 over the vector.  Arithmetic is fp32,
 * a norm's squares and their mean too.  A row
 * whose slot or position (where there is a table) is out of range leaves the cache
 * as it was, and its q is 0.  A vector with an infinity or a NaN is not finite when
 * it is read, others are not affected.  The cache's vectors must not overlap, nor
 * q any other argument.  qkv is aligned to two elements, the table to 16 bytes, q
 * and gains to 8.
 * Allocates nothing.  Errors: INVALID_ARG, CUDA. */
memspec_status memspec_op_kv_append(const memspec_batch* batch, const memspec_kv* kv,
                                    const memspec_append* args, void* stream);

/* The rows' keys and values as the cache holds them: bf16 [rows][kv heads][head_dim]
 * each, 8-byte aligned, codes times their scale rounded once; 0 at a slot out of
 * range.  Allocates
 * nothing.  Errors: INVALID_ARG, CUDA. */
memspec_status memspec_op_kv_read(const memspec_batch* batch, const memspec_kv* kv, void* k_out_dev,
                                  void* v_out_dev, void* stream);

typedef struct memspec_attention {
  const void* q_dev;            /* bf16 [rows][n_heads][head_dim], 16-byte aligned */
  int64_t ldq;                  /* elements from row to row, a multiple of 8 */
  void* out_dev;                /* bf16 [rows][n_heads][head_dim], 16-byte aligned */
  int64_t ldo;                  /* as ldq (of a single row neither is read) */
  int32_t n_heads;              /* a multiple of the cache's, up to 64 times it */
  float scale;                  /* of q . k, up to 2e38 either way */
  const int32_t* tree_dev;      /* [rows] or NULL */
  const memspec_kv* prefix;     /* or NULL: its sequence 0 is before every sequence's positions */
  int32_t prefix_len;           /* 0..prefix->max_pos */
  int32_t max_rows;             /* of one sequence: what the call is laid out for (1..rows; rows of many
                                   short sequences take up to twice the time if it is rows) */
} memspec_attention;

/* Scratch bytes of memspec_op_attention.  Errors: INVALID_ARG. */
memspec_status memspec_op_attention_scratch_bytes(const memspec_batch* batch, const memspec_kv* kv,
                                                  const memspec_attention* args, size_t* bytes);

/* out = sum_i w_i v_i / sum_i w_i, w_i = exp(scale q . k_i), for every row and head
 * (head h reads head h / (n_heads / kv heads) of the cache), over the prefix and the
 * sequence's slots up to the row's own; with tree_dev over its slots before the
 * first row's own and those of the rows j < 32 of the sequence whose bit j is set.
 * A row that sees nothing gives 0.  All sequences share the prefix, which is read
 * once for all of them; it has the cache's heads and head_dim, its own strides and
 * type.  q . k and sums are fp32; the weights enter the product with v in 16 bits
 * (of bf16 caches bf16, of codes fp16), off by half a step of it each, of codes
 * also by 2^-31 of the largest weight times scale.  With more than 16 query vectors
 * a head of k and v (max_rows, of a prefix rows, times heads of a group), keys and
 * values of codes count as fp16: off by 2^-10 of themselves, or by 2^-15 of the
 * largest scale among their 128 positions.
 * Slots that a row does not see do not reach it, whatever they hold (but for the
 * scales among those 128 positions); an infinity
 * or a NaN in q, in a key or value that it sees, or among its scores, makes that row
 * and head unspecified.  out overlaps no other argument.
 * A sequence of more than max_rows rows gives the same, at another speed.
 * Deterministic.  scratch_dev: 16-byte aligned, any content; calls that may overlap
 * need scratches of their own.  Every wait on the device is bounded (a second or
 * more; none takes so long): should one run out, the rows it concerns are NaN.
 * Allocates nothing.  Errors: INVALID_ARG, CUDA. */
memspec_status memspec_op_attention(const memspec_batch* batch, const memspec_kv* kv,
                                    const memspec_attention* args, void* scratch_dev, size_t scratch_bytes,
                                    void* stream);

/* Message describing the last failed op-level call (or memspec_init) on this
 * host thread; never NULL. */
const char* memspec_op_last_error(void);

/* Overwrite an internal buffer of ctx (same ids as memspec_read_buffer) from
 * host memory; synchronous.  Lets tests feed the acceptance step synthetic
 * logits and set sequence state.  Writable: TARGET_LOGITS, DRAFT_LOGITS,
 * DRAFT_TOKENS, TOKENS, SEQ_STATE, SEEDS. */
memspec_status memspec_write_buffer(memspec_ctx* ctx, int32_t buffer, const void* src_host,
                                    size_t bytes);

#ifdef __cplusplus
}
#endif
#endif /* MEMSPEC_OPS_H_ */
