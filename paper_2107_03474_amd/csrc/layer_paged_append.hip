// layer_paged_append.hip -- part of liblram: new rows into the pages of the cache.
//
// One launch: workgroups that rotate q's rows, and workgroups that each take 32 key slots of a head, through LDS from
// the rows' order into the pages' (keys are rotated on the way out).  Bound by HBM for prompts, by its launch for
// single tokens.

#include "layer_paged.h"
#include "layer_rotary.h"

namespace {

constexpr int APPEND_THREADS = 256;

struct Append {
  Pool p;
  const void *k, *v, *q;
  void* q_out;
  const float* given;
  const int64_t* turns;  // null: nothing is rotated
  int64_t k_row, k_head, v_row, v_head, q_row, q_head;
  int pairs, interleaved;
  float magnitude;
  int tiles;         // workgroups of a sequence and key head
  unsigned q_groups;  // workgroups of q's rows, the first ones of the grid
};

// x's E elements from e0 on, rotated; row: the head's whole row.
template <typename T, int E>
__device__ __forceinline__ void turned(const Append& a, const T* row, int e0, int position, float (&f)[E]) {
  load_n<T, E>(row + e0, f);
  if (!a.turns || e0 >= 2 * a.pairs) return;
  if (a.interleaved) {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const int pair = (e0 + e) / 2;
      if (pair >= a.pairs) break;
      const Turn t = turn_of(a.turns[pair], position, a.magnitude, 1.0f);
      const float u = f[e], v = f[e + 1];
      f[e] = fmaf(u, t.c, -v * t.s);
      f[e + 1] = fmaf(u, t.s, v * t.c);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e0 + e;
      if (i >= 2 * a.pairs) break;
      const bool second = i >= a.pairs;
      const int pair = second ? i - a.pairs : i;
      const Turn t = turn_of(a.turns[pair], position, a.magnitude, 1.0f);
      const float other = (float)row[second ? i - a.pairs : i + a.pairs];
      f[e] = second ? fmaf(other, t.s, f[e] * t.c) : fmaf(f[e], t.c, -other * t.s);
    }
  }
}

// The position of a row, 0 where it belongs to no sequence.
__device__ __forceinline__ int position_of(const Pool& p, int64_t row) {
  int lo = 0, hi = p.batch + 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (p.start[mid] <= row)
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo == 0 || lo > p.batch ? 0 : p.seen[lo - 1] - (int)(p.start[lo] - row);
}

template <typename T, int D>
__global__ __launch_bounds__(APPEND_THREADS) void k_paged_append(Append a) {
  using Ti = PageTile<T>;
  constexpr int E = Ti::E, F = Ti::F, CH = D / E;
  const Pool& p = a.p;
  if (blockIdx.x < a.q_groups) {
    const int64_t id = (int64_t)blockIdx.x * APPEND_THREADS + threadIdx.x;
    const int64_t at = id / CH, row = at / p.heads;
    if (row >= p.rows) return;
    const int h = (int)(at % p.heads), e0 = (int)(id % CH) * E;
    float f[E];
    turned<T, E>(a, (const T*)a.q + row * a.q_row + h * a.q_head, e0, position_of(p, row), f);
    store_n<T, E>((T*)a.q_out + (row * p.heads + h) * D + e0, f);
    return;
  }
  __shared__ __align__(16) T rows_k[PAGE_BLOCK][D], rows_v[PAGE_BLOCK][D + E];
  const int64_t group = blockIdx.x - a.q_groups;
  const int head = (int)(group % p.kv_heads), tile = (int)(group / p.kv_heads % a.tiles);
  const int b = (int)(group / p.kv_heads / a.tiles);
  const CacheSeq s = cache_seq(p, b);
  const int first = s.used - (int)(p.start[b + 1] - s.q0);  // slot of the row q0
  const int low = max(first, 0), high = min(first + s.nq, s.nk);
  for (int64_t block = (low >> 5) + tile; block * PAGE_BLOCK < high; block += a.tiles) {
    const int slot0 = (int)block * PAGE_BLOCK;
    const int page = page_of(p, b, slot0);
    if (page < 0) continue;  // all threads alike
    const int t0 = slot0 & (p.page - 1);
    const int from = max(low - slot0, 0), to = min(high - slot0, PAGE_BLOCK);
    const int64_t keys = page_rows(p, page, head) + t0;
    for (int i = threadIdx.x; i < PAGE_BLOCK * CH; i += APPEND_THREADS) {
      const int t = i / CH, c = i % CH * E;
      if (t < from || t >= to) continue;
      const int64_t row = s.q0 + (slot0 + t - first);
      *(Packed<T, E>*)&rows_k[t][c] = *(const Packed<T, E>*)((const T*)a.k + row * a.k_row + head * a.k_head + c);
      *(Packed<T, E>*)&rows_v[t][c] = *(const Packed<T, E>*)((const T*)a.v + row * a.v_row + head * a.v_head + c);
    }
    if (threadIdx.x < PAGE_BLOCK && (int)threadIdx.x >= from && (int)threadIdx.x < to) {
      const int row = slot0 + threadIdx.x - first;
      p.position[keys + threadIdx.x] = s.at + row;
      if (p.weight) p.weight[keys + threadIdx.x] = a.given ? a.given[(s.q0 + row) * p.kv_heads + head] : 0.0f;
    }
    __syncthreads();
    T* const k = (T*)p.k + keys * D;
    for (int i = threadIdx.x; i < PAGE_BLOCK * CH; i += APPEND_THREADS) {
      const int half = i / (16 * CH), c = i / 16 % CH, t = half * 16 + i % 16;
      if (t < from || t >= to) continue;
      float f[E];
      turned<T, E>(a, rows_k[t], c * E, s.at + slot0 + t - first, f);
      store_n<T, E>(k + (int64_t)i * E, f);
    }
    T* const v = (T*)p.v + keys * D;
    for (int i = threadIdx.x; i < PAGE_BLOCK * CH; i += APPEND_THREADS) {  // as many times E values
      const int d16 = i % 16, g = i / 16 % 4, d = i / 64 % (D / 16) * 16 + d16, t1 = i / (4 * D) * Ti::KEYS + g * 4;
      Packed<T, E> o;
      bool whole = true;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int t = t1 + e / 4 * 16 + e % 4;
        whole = whole && t >= from && t < to;
        o.v[e] = rows_v[t][d];
      }
      if (whole) {
        *(Packed<T, E>*)(v + (int64_t)i * E) = o;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int t = t1 + e / 4 * 16 + e % 4;
          if (t >= from && t < to) v[(int64_t)i * E + e] = o.v[e];
        }
      }
    }
    __syncthreads();
  }
  (void)F;
}

constexpr int EXTEND_THREADS = 256;
__global__ __launch_bounds__(EXTEND_THREADS) void k_paged_extend(const int32_t* start, int batch, int32_t* used, int32_t* seen) {
  const int b = blockIdx.x * EXTEND_THREADS + threadIdx.x;
  if (b >= batch) return;
  const int n = max(start[b + 1] - start[b], 0);
  used[b] += n;
  seen[b] += n;
}

}  // namespace

extern "C" {

int lram_paged_extend(const int32_t* start, int32_t batch, int32_t* used, int32_t* seen, void* stream) {
  if (batch < 0 || batch > 1 << 20) return LRAM_EINVAL;
  if (batch == 0) return LRAM_OK;
  if (!start || !used || !seen || off_align(start, 4) || off_align(used, 4) || off_align(seen, 4)) return LRAM_EINVAL;
  hipLaunchKernelGGL(k_paged_extend, dim3((unsigned)((batch + EXTEND_THREADS - 1) / EXTEND_THREADS)), dim3(EXTEND_THREADS), 0,
                     (hipStream_t)stream, start, (int)batch, used, seen);
  return layer_launched();
}

int lram_paged_append(const lram_paged* p, const lram_rotary* r, const void* k, int64_t k_row, int64_t k_head,
                      const void* v, int64_t v_row, int64_t v_head, const float* given, const void* q, int64_t q_row,
                      int64_t q_head, void* q_out, void* stream) {
  if (!p) return LRAM_EINVAL;
  if (int rc = check_pool(*p, true)) return rc;
  if (r)
    if (int rc = check_rotary(*r, p->head_dim)) return rc;
  if (bad_strides(k_row, k_head, p->kv_heads, p->head_dim, p->dtype) || bad_strides(v_row, v_head, p->kv_heads, p->head_dim, p->dtype))
    return LRAM_EINVAL;
  if ((q != nullptr) != (q_out != nullptr) || (q && !r) || (given && !p->weight)) return LRAM_EINVAL;
  if (q && (bad_strides(q_row, q_head, p->heads, p->head_dim, p->dtype) || off_align(q, 16) || off_align(q_out, 16)))
    return LRAM_EINVAL;
  if (p->rows == 0) return LRAM_OK;
  if (!k || !v || off_align(k, 16) || off_align(v, 16) || off_align(given, 4)) return LRAM_EINVAL;
  Append a{};
  a.p = pool_of(*p);
  a.k = k, a.v = v, a.q = q, a.q_out = q_out, a.given = given;
  a.k_row = k_row, a.k_head = k_head, a.v_row = v_row, a.v_head = v_head, a.q_row = q_row, a.q_head = q_head;
  if (r) a.turns = r->turns, a.pairs = r->pairs, a.interleaved = r->interleaved, a.magnitude = r->magnitude;
  // n rows touch (n + 30) / 32 + 1 blocks at most; a grid holds fewer than 2^32 threads
  const int64_t each = 16 / (int64_t)elem_size(p->dtype), expected = std::min(p->max_q, p->rows);
  const int64_t groups_q = q ? (p->rows * p->heads * (p->head_dim / each) + APPEND_THREADS - 1) / APPEND_THREADS : 0;
  const int64_t most = ((int64_t)1 << 32) / APPEND_THREADS - 1 - groups_q, lists = (int64_t)p->batch * p->kv_heads;
  if (groups_q + lists >= ((int64_t)1 << 32) / APPEND_THREADS) return LRAM_EINVAL;
  a.q_groups = (unsigned)groups_q;
  if (lists) a.tiles = (int)std::max<int64_t>(1, std::min((expected + 30) / PAGE_BLOCK + 1, most / lists));
  const int64_t grid = groups_q + lists * a.tiles;
  if (grid == 0) return LRAM_OK;
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(APPEND_THREADS), 0, (hipStream_t)stream, a);
    return layer_launched();
  };
  if (p->dtype == LRAM_BF16)
    return p->head_dim == 128 ? go(k_paged_append<bf16, 128>)
           : p->head_dim == 64 ? go(k_paged_append<bf16, 64>)
                               : go(k_paged_append<bf16, 32>);
  return p->head_dim == 128 ? go(k_paged_append<float, 128>)
         : p->head_dim == 64 ? go(k_paged_append<float, 64>)
                             : go(k_paged_append<float, 32>);
}

}  // extern "C"
