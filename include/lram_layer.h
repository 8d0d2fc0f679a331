/*
 * lram_layer.h -- C ABI of the operators around the lattice memory in a transformer layer (liblram.so, gfx950):
 * layer norm with the residual add in front of it, attention over packed sequences, and the learned relative
 * position bias inside the attention.  The memory replaces the layer's feed-forward part (Sec. 3.1); these are the
 * rest of the layer of the paper's model (Sec. 3.2).
 *
 * Conventions, beyond those of lram.h (streams, caller-owned memory, status codes, host checks before any launch,
 * nothing kept between calls):
 *   - dtype is that of the activations and their gradients, LRAM_F32 or LRAM_BF16; wdtype that of the learned weights and
 *     theirs: LRAM_F32, or LRAM_BF16 beside bf16 activations.  Sums, statistics, maxima, lse and partial results are fp32; a
 *     result is rounded once, to nearest even.  In bf16 the matrix cores take bf16 operands, so that the softmax's weights
 *     and, backward, ds = p (dO.v - dO.out) are rounded to bf16 too before the products that use them (the weights' own
 *     sum is of the unrounded ones); fp32 rounds nothing in between.
 *   - Every result is the same, bit for bit, on every call with the same inputs: no sum's order depends on timing.
 *   - Tensors are dense row-major unless a stride is given, and 16-byte aligned; fp32 per-row arrays, int32 arrays
 *     and learned weights need the alignment of an element.
 */
#ifndef LRAM_LAYER_H
#define LRAM_LAYER_H

#include "lram.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LRAM_NORM_MAX_WIDTH 16384

/* hipError_t of the most recent LRAM_EHIP of this header's entry points on the calling thread (0 if none). */
int lram_layer_last_hip_error(void);

/*
 * lram_layer_norm_forward -- for each of `rows` rows of `width` elements (1 to LRAM_NORM_MAX_WIDTH)
 *     h = x + residual   (rounded to dtype; h = x without a residual)
 *     y = (h - mean h) / sqrt(mean (h - mean h)^2 + eps) * weight + bias
 *   residual  nullable; `sum` then receives h and must be given (it may be x's or residual's own buffer)
 *   mean, rstd [rows] fp32: nullable (both or none); what the backward needs beside h.
 * y may be x's or residual's own buffer where it is not `sum`'s.
 */
int lram_layer_norm_forward(const void* x, const void* residual, const void* weight, const void* bias, int dtype,
                            int wdtype, int64_t rows, int64_t width, double eps, void* sum, void* y, float* mean,
                            float* rstd, void* stream);

/* Device workspace of an lram_layer_norm_backward that gives the weight gradients (host only); without them it needs none. */
int lram_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width, int dtype, size_t* bytes);

/*
 * lram_layer_norm_backward -- with g = grad_y weight and n = (h - mean) rstd:
 *     grad_x = rstd (g - mean g - n mean(g n)) + grad_sum   (the gradient of x and of residual alike)
 *     grad_weight = sum over rows of grad_y n,  grad_bias = sum over rows of grad_y   (overwritten, in wdtype)
 *   grad_sum  nullable: the gradient that reaches h other than through y
 *   grad_weight, grad_bias  nullable (both or none).
 * grad_x may be grad_y's or grad_sum's own buffer.  With rows = 0 the weight gradients are written as zeros.
 */
int lram_layer_norm_backward(const void* h, const void* weight, const float* mean, const float* rstd,
                             const void* grad_y, const void* grad_sum, int dtype, int wdtype, int64_t rows,
                             int64_t width, void* grad_x, void* grad_weight, void* grad_bias, void* workspace,
                             size_t ws_bytes, void* stream);

/*
 * Attention over packed sequences.  Sequence b has the rows start_q[b] ... start_q[b + 1] - 1 of q (nq of them) and the
 * first nk rows from start_k[b] on of k and v, nk = used_k[b], or all up to start_k[b + 1] without used_k.  With
 * G = heads / kv_heads, query i of head h meets key j of head h / G if j < nk and, causal, j <= i + nk - nq (the ends
 * of queries and keys are aligned: a prompt, a piece of one, or one token over a cache):
 *     s_ij = scale q_i . k_j + rel_weight[h][rel_bucket[clamp(j - i - (nk - nq), -rel_reach, rel_reach) + rel_reach]]
 *     out_i = sum_j softmax_j(s_ij) v_j,   0 where a query meets no key
 * The bias (Sec. 3.2's model learns positions; here by bucketed distance, as T5's does) is nullable.  A weight of -inf
 * hides its keys as `causal` does.  Finite weights of 1.16e7 (2^24 / log2 e) and more in magnitude, a type's lowest value
 * among them, count alike: no score matters beside them, so that a query that meets no other keys has the even average of
 * theirs.  Scores themselves have to stay below that in magnitude: fp32 holds no digit of them behind the point from there
 * on, so that gradients mean nothing, and from 128 times it on results may be NaN.
 *
 * The lengths stay on the device: nothing waits for them, and a captured call may be replayed over others.  max_q and
 * max_k are the longest nq and nk expected, from which the host chooses how to divide the work; lengths beyond them
 * cost time, not results.  Rows of q before the first sequence and past the last one give zeros, and whatever the device
 * arrays hold, no row outside the tensors is addressed.  A value that is not finite can reach
 * every query of its own sequence (a product with weight 0 is formed in a tile), never another sequence's, and keys
 * at and past nk are not read into any result.
 */
typedef struct {
  int32_t dtype;              /* of q, k, v and every result: LRAM_F32, LRAM_BF16 */
  int32_t wdtype;             /* of rel_weight */
  int32_t heads, kv_heads;    /* heads a multiple of kv_heads, at most 64 times it */
  int32_t head_dim;           /* 32, 64 or 128 */
  int32_t batch;              /* sequences, at least 0 */
  int32_t causal;             /* 0 or 1 */
  float scale;                /* finite, > 0 */
  int64_t tq, tk;             /* rows of q, of k and v; tq heads / kv_heads <= 2^30, tk <= 2^30 */
  int64_t max_q, max_k;
  const void *q, *k, *v;      /* [tq][heads][head_dim], [tk][kv_heads][head_dim] with the strides below */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head; /* in elements: multiples of 16 bytes, rows at least head_dim
                                                          and at most 2^22 */
  const int32_t *start_q, *start_k; /* [batch + 1], ascending (device) */
  const int32_t* used_k;      /* [batch] (device), nullable */
  const void* rel_weight;     /* [heads][rel_buckets], nullable */
  const int32_t* rel_bucket;  /* [2 rel_reach + 1] (device), each in [0, rel_buckets) */
  int32_t rel_buckets;        /* 1 ... 256 */
  int32_t rel_reach;          /* >= 0, heads / kv_heads (2 rel_reach + 193) <= 4096; in fp32 with head_dim 128
                                 2 rel_reach + 193 <= 1365 */
} lram_attention;

/*
 * lram_attention_forward -- out [tq][heads][head_dim] in dtype.
 *   lse      [tq][heads] fp32: nullable; log2 sum_j 2^(s_ij log2 e), -inf where a query meets no key (the base that the
 *            kernels work in); +-2^126 (1 + log2(n) / 32) where the n keys that count are those of weights that count alike
 *   residue  as out, nullable, bf16 only: out before its rounding minus out.  With it the backward's
 *            <grad_out, out> is that of the unrounded result.
 *   workspace: lram_attention_forward_workspace_bytes (0 unless the keys are divided because rows are few).
 */
int lram_attention_forward_workspace_bytes(const lram_attention* a, size_t* bytes);
int lram_attention_forward(const lram_attention* a, void* out, float* lse, void* residue, void* workspace,
                           size_t ws_bytes, void* stream);

/*
 * lram_attention_backward -- gradients of <grad_out, out>, from the same arguments and what the forward wrote:
 *   grad_q [tq][heads][head_dim], grad_k, grad_v [tk][kv_heads][head_dim]  dense, in dtype, overwritten (rows that no
 *          query meets, those of a cache past used_k among them: zeros)
 *   grad_rel [heads][rel_buckets] in wdtype, overwritten; given exactly where rel_weight is
 *   residue  nullable (the forward's).
 */
int lram_attention_backward_workspace_bytes(const lram_attention* a, size_t* bytes);
int lram_attention_backward(const lram_attention* a, const void* out, const void* residue, const float* lse,
                            const void* grad_out, void* grad_q, void* grad_k, void* grad_v, void* grad_rel,
                            void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LRAM_LAYER_H */
