/*
 * lram_cache.h -- C ABI of what serves the layer around the lattice memory token by token (liblram.so, gfx950): rotary
 * positions (in training too), a key-value cache in pages, attention of new tokens over it, and eviction from it by
 * accumulated attention weight.
 *
 * The conventions are those of lram.h and lram_layer.h: the caller's memory and stream, status codes, checks on the host
 * before any launch, nothing kept between calls, results that have the same bits on every call.  dtype is LRAM_F32 or
 * LRAM_BF16.  Angles are exact to 2^-32 of a turn, their sines and cosines fp32; a rotated value is rounded once.  Attention's
 * sums, statistics, weights and partial results are fp32.  In bf16 the softmax's weights enter the product with the values
 * with 16 bits (less than 2^-15 of one is lost) where a call expects at most 16 new rows times heads / kv_heads of a sequence
 * (by max_q and by rows / batch), otherwise rounded to bf16; their sums, and the weights that keys gather, are of the
 * unrounded ones.
 */
#ifndef LRAM_CACHE_H
#define LRAM_CACHE_H

#include "lram_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rotary positions (Su et al., arXiv 2104.09864).  Pair i < pairs of a head, (x[2i], x[2i + 1]) interleaved or
 * (x[i], x[i + pairs]) otherwise, turns by a = 2 pi frac(position turns[i] / 2^64):
 *     (magnitude (x1 cos a - x2 sin a), magnitude (x1 sin a + x2 cos a)),
 * and the head's dimensions from 2 pairs on stay as they are.
 */
typedef struct {
  int32_t pairs;         /* 1 ... head_dim / 2 */
  int32_t interleaved;   /* 0 or 1 */
  float magnitude;       /* finite */
  const int64_t* turns;  /* [pairs] (device): turns a token, times 2^64, modulo 2^64 */
} lram_rotary;

#define LRAM_ROTARY_MAX_HEAD_DIM 1024

/*
 * lram_positions -- position[row] = first[b] + row - start[b] of the sequence b with start[b] <= row < start[b + 1]
 * (start ascending, [batch + 1], device); 0 for rows of none.  first [batch]: nullable, zeros.
 */
int lram_positions(const int32_t* start, const int32_t* first, int32_t batch, int64_t rows, int32_t* position, void* stream);

/*
 * lram_rotate -- q [rows][heads][head_dim] and k [rows][kv_heads][head_dim], with their strides in elements (multiples of 16
 * bytes), into dense q_out and k_out, at position [rows] (any int32).  backward != 0 turns the other way round, which takes
 * the results' gradients to the arguments'.  k is nullable (kv_heads = 0).  head_dim: a multiple of 8, at most
 * LRAM_ROTARY_MAX_HEAD_DIM.  Results are not their arguments' own memory.
 */
int lram_rotate(const lram_rotary* r, int dtype, int backward, int64_t rows, int32_t head_dim, const int32_t* position,
                const void* q, int64_t q_row, int64_t q_head, int32_t heads, void* q_out, const void* k, int64_t k_row,
                int64_t k_head, int32_t kv_heads, void* k_out, void* stream);

/*
 * A cache in pages.  A pool holds `pages` pages of `page` keys for each key head.  table[b] names the pages of sequence b in
 * their order (what is not in 0 ... pages - 1 is no page: keys there are not met, and rows that belong there are left out);
 * used[b] counts its keys, seen[b] the tokens it has had.  Every layer has a pool of its own, and all share table and lengths.
 * No page belongs to two sequences of a call that writes (append, attention that weighs, evict).
 *
 * A step's new rows are packed: those of sequence b are start[b] ... start[b + 1] - 1.  lram_paged_extend adds their numbers
 * to used and seen first; from then on they are the last of both: row i of nq has position seen[b] - nq + i and key slot
 * used[b] - nq + i.  Slots from width * page on are left out, in append as in attention.
 *
 * In a page the keys of a head lie in the order in which the matrix cores take them, so that a wave's load is 1 KiB in
 * one piece and no value is moved between lanes.  With E = 16 bytes of elements and F = E / 4, slot t of the page is
 *     k [page][kv_head][t / 16][d / E][t % 16][d % E]
 *     v [page][kv_head][t / (16 F)][d / 16][t % 16 / 4][d % 16][t % (16 F) / 16 * 4 + t % 4]
 * and position, weight [page][kv_head][t]: the key's position in its text, the attention weight that it has gathered.  As long
 * as used[b] = seen[b], which says that no key was evicted, slot t holds the key of position t.
 */
typedef struct {
  int32_t dtype;
  int32_t heads, kv_heads;   /* heads a multiple of kv_heads, at most 64 times it */
  int32_t head_dim;          /* 32, 64 or 128 */
  int32_t batch;             /* sequences, at least 0 */
  int32_t page;              /* 32, 64, 128 or 256 keys */
  int64_t pages;             /* pages * page <= 2^30 */
  int64_t width;             /* of a table's row; width * page <= 2^30 */
  void *k, *v;               /* 16-byte aligned */
  int32_t* position;         /* 16-byte aligned, like weight */
  float* weight;             /* nullable where nothing gathers */
  const int32_t* table;      /* [batch][width] (device) */
  const int32_t *used, *seen; /* [batch] (device) */
  const int32_t* start;      /* [batch + 1], ascending (device) */
  int64_t rows;              /* of q (k, v); rows * heads <= 2^30 */
  int64_t max_q, max_k;      /* longest numbers of new rows and of keys expected: past them calls cost time, not results */
} lram_paged;

/* lram_paged_extend -- used[b] and seen[b] grow by start[b + 1] - start[b]. */
int lram_paged_extend(const int32_t* start, int32_t batch, int32_t* used, int32_t* seen, void* stream);

/*
 * lram_paged_append -- the new rows' keys k [rows][kv_heads][head_dim] (strides in elements: multiples of 16 bytes, as for
 * attention) and values v into their slots, keys rotated where r is given; their positions, and, where the pool has weights,
 * `given` [rows][kv_heads] fp32 or 0.  q [rows][heads][head_dim] is nullable; q_out is q rotated, dense (only with r); rows
 * of no sequence have position 0.  p->weight nullable.
 */
int lram_paged_append(const lram_paged* p, const lram_rotary* r, const void* k, int64_t k_row, int64_t k_head,
                      const void* v, int64_t v_row, int64_t v_head, const float* given, const void* q, int64_t q_row,
                      int64_t q_head, void* q_out, void* stream);

/*
 * lram_paged_attention -- out [rows][heads][head_dim]: query i of sequence b, of position p_i, meets the used keys of position
 * p_j <= p_i, with the score and the bias of lram_attention (rel_bucket by p_j - p_i; at most 256 buckets,
 * heads / kv_heads (2 rel_reach + 193) <= 4096):
 *     s_ij = scale q_i . k_j + rel_weight[h][rel_bucket[clamp(p_j - p_i, -rel_reach, rel_reach) + rel_reach]]
 *     out_i = sum_j softmax_j(s_ij) v_j,   0 where a query meets no key;  rows of no sequence: 0
 * weigh != 0: weight of each key that is met grows by the sum of its softmax_j(s_ij) over the sequence's queries and the
 * heads that share it.  Everything else about values that are not finite, vast weights and scores is as for lram_attention.
 */
typedef struct {
  const void* q;             /* [rows][heads][head_dim] */
  int64_t q_row, q_head;     /* as for lram_attention */
  float scale;               /* finite, > 0 */
  int32_t weigh;             /* 0 or 1 */
  int32_t wdtype;            /* of rel_weight */
  int32_t rel_buckets, rel_reach;
  const void* rel_weight;    /* [heads][rel_buckets], nullable */
  const int32_t* rel_bucket; /* [2 rel_reach + 1] (device) */
} lram_paged_queries;

int lram_paged_attention_workspace_bytes(const lram_paged* p, const lram_paged_queries* a, size_t* bytes);
int lram_paged_attention(const lram_paged* p, const lram_paged_queries* a, void* out, void* workspace, size_t ws_bytes,
                         void* stream);

/*
 * lram_paged_evict -- cuts the sequences that use more than `budget` keys down to it, for each key head by itself.  What stays:
 * the keys of the positions from seen - recent on, and of the others those of the largest weight; of equal weights the lowest
 * position, of equal positions the lowest slot.  A weight that is NaN counts as less than any, and a slot below the budget that
 * lies in no page is taken.  Those that stay past slot `budget` move, in their order, into the slots below that are left, with
 * their positions and weights.  used is left as it is, since every layer's pool is cut by the same lengths: lram_paged_shrink
 * follows the last of them.  1 <= budget, 0 <= recent <= budget.  rows, start, max_q are not read.
 */
int lram_paged_evict_workspace_bytes(const lram_paged* p, int64_t budget, size_t* bytes);
int lram_paged_evict(const lram_paged* p, int64_t budget, int64_t recent, void* workspace, size_t ws_bytes, void* stream);

/* lram_paged_shrink -- used[b] = min(used[b], budget), budget >= 1. */
int lram_paged_shrink(int64_t budget, int32_t batch, int32_t* used, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LRAM_CACHE_H */
