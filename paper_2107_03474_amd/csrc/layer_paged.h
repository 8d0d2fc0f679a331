// layer_paged.h -- part of liblram: the key-value cache in pages.
//
// A page of a key head holds its keys as operands of the matrix cores (lane l: row l % 16, group g = l / 16):
//   k: blocks of 16 keys; the scores' product S^T = K Q^T takes key l % 16 and, per load, E dimensions E (4 c + g) ... + E - 1,
//      E = 16 bytes of elements: 1 KiB in one piece.
//   v: blocks of 16 F keys (F = E / 4 results of S^T); the lane that holds S^T's rows 4 g ... 4 g + 3 of F blocks of 16 holds
//      these F times 4 keys as its k elements of O^T = V^T P^T, so v has them side by side for dimension l % 16: again 1 KiB
//      in one piece, and the softmax's results are an operand as they stand.

#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../../include/lram_cache.h"
#include "layer_common.h"

namespace {

template <typename T>
struct PageTile {
  static constexpr int E = 16 / (int)sizeof(T);  // elements of 16 bytes
  static constexpr int F = E / 4;                // blocks of 16 keys in one of v
  static constexpr int KEYS = 16 * F;            // of a block of v
};
constexpr int PAGE_BLOCK = 32;  // every page size is a multiple: 2 blocks of 16 keys

// A sequence of the cache: nq new rows from q0 on (those that lie in the tensor: from row `skip` of the sequence's own on), nk
// keys that pages can hold, the position of the row q0, and whether every token's key is there.
struct CacheSeq {
  int64_t q0;
  int nq, nk, used, at;
  bool whole;
};

struct Pool {
  void *k, *v;
  int32_t* position;
  float* weight;
  const int32_t *table, *used, *seen, *start;
  int64_t rows, width;
  int pages, page, log_page, batch, heads, kv_heads, group;
};

__device__ __forceinline__ int64_t clamp_row(int64_t x, int64_t rows) { return x < 0 ? 0 : x > rows ? rows : x; }

// Whatever the arrays hold, rows lie in the tensors and slots in the table.
__device__ __forceinline__ CacheSeq cache_seq(const Pool& p, int b) {
  const int64_t s0 = p.start[b], s1 = p.start[b + 1];
  CacheSeq s;
  s.q0 = clamp_row(s0, p.rows);
  const int64_t q1 = clamp_row(s1, p.rows);
  s.nq = q1 > s.q0 ? (int)(q1 - s.q0) : 0;
  const int64_t most = p.width << p.log_page;
  s.used = p.used[b];
  s.nk = s.used < 0 ? 0 : s.used > most ? (int)most : s.used;
  const int seen = p.seen[b];
  s.at = seen - (int)(s1 - s.q0);
  s.whole = s.used == seen;
  return s;
}

// The page of a slot of sequence b, -1 where there is none.
__device__ __forceinline__ int page_of(const Pool& p, int b, int slot) {
  const int page = p.table[(int64_t)b * p.width + (slot >> p.log_page)];
  return page >= 0 && page < p.pages ? page : -1;
}

// The same for a slot that is one for the whole wave.  Through the scalar cache: a vector load here would wait for every load
// that the wave has on its way.
__device__ __forceinline__ int page_of_wave(const Pool& p, int b, int slot) {
  const int at = __builtin_amdgcn_readfirstlane(slot >> p.log_page);
  const auto* const row = (const __attribute__((address_space(4))) int32_t*)(p.table + (int64_t)b * p.width);
  const int page = row[at];
  return page >= 0 && page < p.pages ? page : -1;
}

// First element of a page's keys of a head (k and v alike), and of its positions.
__device__ __forceinline__ int64_t page_rows(const Pool& p, int page, int head) {
  return ((int64_t)page * p.kv_heads + head) << p.log_page;
}

inline int check_pool(const lram_paged& p, bool queries) {
  if (p.dtype != LRAM_F32 && p.dtype != LRAM_BF16) return LRAM_EDTYPE;
  if (p.head_dim != 32 && p.head_dim != 64 && p.head_dim != 128) return LRAM_EDTYPE;
  if (p.kv_heads < 1 || p.kv_heads > 1024) return LRAM_EINVAL;
  if (p.page != 32 && p.page != 64 && p.page != 128 && p.page != 256) return LRAM_EINVAL;
  if (p.batch < 0 || p.batch > 1 << 20 || p.pages < 0 || p.pages > (1 << 30) / p.page || p.width < 0 ||
      p.width > (1 << 30) / p.page || p.max_k < 0)
    return LRAM_EINVAL;
  if (p.pages && (!p.k || !p.v || !p.position)) return LRAM_EINVAL;
  if (off_align(p.k, 16) || off_align(p.v, 16) || off_align(p.position, 16) || off_align(p.weight, 16)) return LRAM_EINVAL;
  if (p.batch && (!p.used || !p.seen || (p.width && !p.table))) return LRAM_EINVAL;
  if (off_align(p.used, 4) || off_align(p.seen, 4) || off_align(p.table, 4)) return LRAM_EINVAL;
  if (!queries) return LRAM_OK;
  if (p.heads < 1 || p.heads % p.kv_heads || p.heads / p.kv_heads > 64 || p.heads > 65536) return LRAM_EINVAL;
  if (p.rows < 0 || p.rows > (1 << 30) / p.heads || p.max_q < 0 || !p.start || off_align(p.start, 4)) return LRAM_EINVAL;
  return LRAM_OK;
}

inline bool bad_strides(int64_t row, int64_t head, int64_t heads, int64_t dim, int dtype) {
  const int64_t per = 16 / (int64_t)elem_size(dtype);
  return row < dim || row > 1 << 22 || row % per || head < 0 || head > INT64_MAX / 2 / heads || head % per;
}

inline Pool pool_of(const lram_paged& p) {
  Pool x{};
  x.k = p.k, x.v = p.v, x.position = p.position, x.weight = p.weight;
  x.table = p.table, x.used = p.used, x.seen = p.seen, x.start = p.start;
  x.rows = p.rows, x.width = p.width, x.pages = (int)p.pages, x.page = p.page, x.log_page = __builtin_ctz(p.page);
  x.batch = p.batch, x.heads = p.heads, x.kv_heads = p.kv_heads, x.group = p.heads / p.kv_heads;  // 0 where no queries are given
  return x;
}

template <typename F>
int by_form(int dtype, int dim, F f) {
  const auto of = [&](auto t) {
    return dim == 128 ? f(t, std::integral_constant<int, 128>())
           : dim == 64 ? f(t, std::integral_constant<int, 64>())
                       : f(t, std::integral_constant<int, 32>());
  };
  return dtype == LRAM_BF16 ? of(bf16()) : of(float());
}

}  // namespace
