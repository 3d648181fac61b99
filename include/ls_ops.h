/*
 * ls_ops.h - C ABI of the decoder-layer operators around the sparse FFN.
 *
 * ls_ffn.h computes the FFN half of a decoder layer.  These calls are the other half, for the
 * same decode loop: the norms around a block with its gated residual update, the 8-bit integer
 * projections, the append of rotated keys and values to a paged cache, and the attention of a
 * batch whose sequences share a prefix.
 *
 * Conventions, beyond those of ls_ffn.h (status codes, nothing aborts or throws, argument
 * validation is synchronous, sticky LS_E_DEVICE, one host thread per context, the same bits on
 * every run):
 *  - A context (ls_ops) owns a device workspace and borrows a stream.  Tensors, weights, page
 *    tables and caches are the caller's device memory; calls enqueue on the context's stream,
 *    so data made on another stream has to be ordered before it by the caller.
 *  - No call allocates, copies to the host or synchronises: every call may be recorded into a
 *    HIP graph, which then reads the device arguments (lengths, page tables, slots) anew at
 *    every replay.
 *  - Strides are in elements and may exceed 32 bits in bytes.  The innermost dimension is
 *    contiguous.  Outputs must not overlap inputs except where a call says so.
 *  - Calls of one context share its workspace: its stream orders them.
 */
#ifndef LS_OPS_H
#define LS_OPS_H

#include <stdint.h>

#include "ls_ffn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ls_ops ls_ops; /* opaque context; owns the workspace */

#define LS_I8 ((ls_dtype)3) /* 8-bit integers: inputs of ls_linear_i8 only */

#define LS_OPS_WORKSPACE_DEFAULT (256ull << 20)

typedef struct {
    uint64_t workspace_bytes; /* 0: LS_OPS_WORKSPACE_DEFAULT; otherwise at least 1 MiB */
    void* stream;             /* hipStream_t borrowed for every call (NULL: the null stream);
                                 must outlive the context */
    uint32_t debug_flags;     /* reserved, 0 */
} ls_ops_desc;

/* Create a context on the current HIP device, which every later call must be made on (LS_E_STATE
 * otherwise).  On success *out receives a context the caller owns and releases with
 * ls_ops_destroy; on failure *out is NULL and ls_ops_last_error(NULL) describes it. */
ls_status ls_ops_create(const ls_ops_desc* desc, ls_ops** out);

/* Wait for the context's stream and release the context.  LS_E_INVAL for a NULL ctx. */
ls_status ls_ops_destroy(ls_ops* ctx);

/* Wait for all work enqueued on the context's stream. */
ls_status ls_ops_sync(ls_ops* ctx);

/* Text of the last failure on ctx (or of the last failed ls_ops_create of this host thread when
 * ctx is NULL); valid until the next call on ctx. */
const char* ls_ops_last_error(const ls_ops* ctx);

/* Norms before and after a block, with its gate and residual scale:
 *   t  = y, or rms(y) * post_weight                       (post_norm)
 *   x' = x_scale x + y_scale gate t     -> x_out
 *   h  = x', or rms(x') * pre_weight                      (pre_norm)  -> h
 *   rms(v) = v / sqrt(mean(v^2) + eps), each token on its own; a NULL weight or gate is ones.
 * y NULL: x' = x_scale x (a norm alone).  x and x_out are fp32 (the residual of ls_ffn.h) and
 * may be the same array; y, gate, the weights and h are of type dtype, rounded once when h is
 * written.  Either output may be NULL, not both.  Sums and norms are fp32.
 * gate_stride 0: one row [d] for every token; otherwise a row per token.
 * Any d in 1 .. 32768; n_tokens 0 does nothing. */
typedef struct {
    int32_t n_tokens, d;
    ls_dtype dtype;
    int32_t post_norm, pre_norm; /* 0 or 1 */
    float x_scale, y_scale, eps; /* eps >= 0 */
    const float* x;
    int64_t x_stride;
    const void* y;
    int64_t y_stride;
    const void* gate;
    int64_t gate_stride;
    const void* post_weight; /* [d] or NULL */
    const void* pre_weight;  /* [d] or NULL */
    float* x_out;
    int64_t x_out_stride;
    void* h;
    int64_t h_stride;
} ls_norm_args;
ls_status ls_norm_residual(ls_ops* ctx, const ls_norm_args* a);

/* Matrix product in 8-bit integers with a scale for each token and output channel:
 *   out[t, n] = s_t w_scale[n] sum_k q_tk w[n, k] + bias[n]
 * x of type LS_I8: q = x and s = x_scale [n_tokens] (fp32).  x of a floating type: quantised on
 * the way, s_t = max_k |x_tk| / 127 and q_tk = round(127 x_tk / max_k |x_tk|), to nearest, ties to
 * even, in fp32 (x_scale must be NULL).  A token of zeros (or whose s_t is below the smallest
 * normal fp32 number) has s_t = 0; one that holds an infinity or NaN gives NaN in its whole row.
 * The sums are exact in 32-bit integers; s_t, then w_scale, then the bias (fp32 [n] or NULL) are
 * applied in fp32 and rounded once to out_type (LS_F32, LS_F16 or LS_BF16): a token's row has the
 * same bits whatever tokens are beside it.
 * w: int8 [n, k] (nn.Linear layout, quantised by row).  k: a multiple of 16, at most 131056;
 * rows of x and w 16-byte aligned.  n >= 1; n_tokens 0 does nothing; n_tokens < 2^23 where x is
 * quantised on the way.
 * LS_E_CAPACITY if the quantised tokens (n_tokens (k + 4) bytes, each part rounded up to 256)
 * exceed the workspace; one to four tokens of up to 16384 elements need none. */
typedef struct {
    int32_t n_tokens, k, n;
    ls_dtype x_type, out_type;
    const void* x;
    int64_t x_stride;
    const float* x_scale;
    const int8_t* w;
    int64_t w_stride;
    const float* w_scale;
    const float* bias;
    void* out;
    int64_t out_stride;
} ls_linear_i8_args;
ls_status ls_linear_i8(ls_ops* ctx, const ls_linear_i8_args* a);

/* A paged cache of one layer's keys and values.  Entry (page, head, i) of k is at
 * k + page * page_stride + head * head_stride + i * token_stride, head_dim contiguous elements;
 * v likewise.  So heads or tokens may be outermost within a page. */
typedef struct {
    void* k;
    void* v;
    ls_dtype dtype;      /* LS_F16 or LS_BF16 (ls_kv_append also takes LS_F32) */
    int32_t n_pages;
    int32_t page_size;   /* tokens per page: a power of two, 1 .. 4096; n_pages * page_size < 2^31 */
    int32_t n_kv_heads, head_dim;
    int64_t page_stride, head_stride, token_stride;
} ls_kv_cache;

/* Which elements of a head turn together: HALF pairs i with i + rot_dim / 2, PAIR pairs 2i with 2i + 1. */
typedef enum { LS_ROPE_HALF = 0, LS_ROPE_PAIR = 1 } ls_rope;

/* Append keys and values to the cache, the keys (and the queries, if given) turned to their
 * positions on the way: for pair i of the first rot_dim elements of a head, with c = cos(i) and
 * s = sin(i) of the token's position,
 *   (a, b) -> (a c - b s, b c + a s),  in fp32, rounded once;
 * the other elements, and values, are copied.
 * cos_sin: fp32 [n_pos, rot_dim], a row holding the rot_dim / 2 cosines, then the sines.
 * positions: dev int32 [n_tokens]; slots: dev int32 [n_tokens], slot = page * page_size + place.
 * A token whose slot is outside the cache writes no key or value (-1 marks padding); one whose
 * position is outside [0, n_pos) writes nothing at all, its query row included.  Slots of one
 * call must differ.  q: [n_tokens, n_heads, head_dim] of the cache's type, written to q_out,
 * which may be q itself; both NULL (n_heads 0): keys and values alone.  Any head_dim in 1 .. 1024,
 * rot_dim even, 0 .. head_dim (0: a plain append; positions and cos_sin may then be NULL). */
typedef struct {
    int32_t n_tokens, n_heads, rot_dim, n_pos;
    ls_rope style;
    const void* k;
    int64_t k_token_stride, k_head_stride;
    const void* v;
    int64_t v_token_stride, v_head_stride;
    const void* q;
    int64_t q_token_stride, q_head_stride;
    void* q_out;
    int64_t q_out_token_stride, q_out_head_stride;
    const int32_t* positions;
    const int32_t* slots;
    const float* cos_sin;
} ls_append_args;
ls_status ls_kv_append(ls_ops* ctx, const ls_kv_cache* cache, const ls_append_args* a);

/* Attention of n_seqs sequences that share a prefix, n_q query tokens each (1: a decode step),
 * over a paged cache.  Query token i of sequence s sees every key of the prefix and the keys
 * j <= lens[s] - n_q + i of the sequence's own pages (its n_q tokens being the last appended):
 *   out = sum_j p_j v_j,  p = softmax over the visible keys of scale * (q . k_j)
 * with query head h reading key/value head h / (n_heads / n_kv_heads).  The prefix's keys are
 * read once for the whole batch.
 * A row that sees no key (no prefix and lens[s] < 1, or every page invalid) is zeros, and so is
 * every row of a sequence with lens[s] < 0, an idle slot.  Nothing else of a masked key reaches
 * the result, whatever it holds.  A page id outside [0, n_pages) masks its keys.
 * prefix_pages: dev int32, ceil(prefix_len / page_size) ids; pages: dev int32
 * [n_seqs, pages_stride]; lens: dev int32 [n_seqs], of which at most max_len counts (the work is
 * shared out by max_len: a bound far above the lengths gives each sequence fewer workgroups);
 * pages_stride * page_size >= max_len unless max_len is 0.
 * q, out: [n_seqs * n_q, n_heads, head_dim] of the cache's type (f16 or bf16; LS_E_UNSUPPORTED
 * for LS_F32).  head_dim: a multiple of 8, at most 256; pointers and strides of q, out, k and v
 * 16-byte aligned.  1 <= n_q <= 16; prefix_len, max_len < 2^22; scale > 0.
 * Scores, the softmax's maxima and sums and the outputs are fp32; probabilities are rounded to
 * the cache's type for the product with the values (to a step of 2^-31 of the row's largest, at
 * the finest, in f16).
 * LS_E_CAPACITY if the workspace cannot hold the parts of one split
 * (n_seqs n_q n_heads 2 (head_dim + 2) floats; of more than 2^20 rows n_seqs n_q n_heads as many
 * whole sequences as 2^20 hold are taken at a time). */
typedef struct {
    int32_t n_seqs, n_q, n_heads;
    int32_t prefix_len, max_len;
    float scale;
    const void* q;
    int64_t q_token_stride, q_head_stride;
    void* out;
    int64_t out_token_stride, out_head_stride;
    const int32_t* prefix_pages;
    const int32_t* pages;
    int64_t pages_stride;
    const int32_t* lens;
} ls_attend_args;
ls_status ls_attend(ls_ops* ctx, const ls_kv_cache* cache, const ls_attend_args* a);

#ifdef __cplusplus
}
#endif
#endif /* LS_OPS_H */
