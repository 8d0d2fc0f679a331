// layer_rotary.hip -- part of liblram: rotary positions for gfx950.
//
// Bound by HBM: every element is read and written once, and the angle's 30 operations a pair are shared out over heads.  A
// thread owns a chunk of a head: 16 bytes of the first halves and their partners, or 16 bytes of neighbours.  It forms
// the chunk's sines and cosines once and goes over the heads of its row with them.

#include <algorithm>

#include "layer_rotary.h"

namespace {

constexpr int ROTATE_THREADS = 256;

struct Rotate {
  const void *q, *k;
  void *q_out, *k_out;
  int64_t q_row, q_head, k_row, k_head;
  const int64_t* turns;
  const int32_t* position;
  int64_t rows;
  int heads, kv_heads, dim, pairs;
  int chunks;       // of a head
  int pair_chunks;  // of them rotated, the first ones
  int teams;        // threads that share a row's heads for one chunk
  float magnitude, sign;
};

// Up to N elements of a chunk; all of them at once where it is whole.
template <typename T, int N>
__device__ __forceinline__ void load_some(const T* p, int n, float (&f)[N]) {
  if (n == N) {
    load_n<T, N>(p, f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = e < n ? (float)p[e] : 0.0f;
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, int n, const float (&f)[N]) {
  if (n == N) {
    store_n<T, N>(p, f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = (T)f[e];
  }
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(ROTATE_THREADS) void k_rotate(Rotate a) {
  constexpr int E = 16 / (int)sizeof(T);
  const int64_t id = (int64_t)blockIdx.x * ROTATE_THREADS + threadIdx.x;
  const int chunk = (int)(id % a.chunks);
  const int64_t rest = id / a.chunks, row = rest / a.teams;
  if (row >= a.rows) return;
  const int all = a.heads + a.kv_heads;
  // the chunk's first element, and how many it has
  const bool turned = chunk < a.pair_chunks;
  const int first = INTERLEAVED || turned ? chunk * E : 2 * a.pairs + (chunk - a.pair_chunks) * E;
  const int n = min(E, (turned && !INTERLEAVED ? a.pairs : a.dim) - first);
  const int position = a.position[row];
  Turn t[INTERLEAVED ? E / 2 : E];
  if (turned) {
#pragma unroll
    for (int e = 0; e < (INTERLEAVED ? E / 2 : E); ++e) {
      const int pair = INTERLEAVED ? first / 2 + e : first + e;
      t[e] = pair < a.pairs ? turn_of(a.turns[pair], position, a.magnitude, a.sign) : Turn{1.0f, 0.0f};
    }
  }
#pragma unroll 2
  for (int head = (int)(rest % a.teams); head < all; head += a.teams) {
    const bool of_q = head < a.heads;
    const int h = of_q ? head : head - a.heads;
    const T* const x = (of_q ? (const T*)a.q + row * a.q_row + h * a.q_head : (const T*)a.k + row * a.k_row + h * a.k_head);
    T* const y = of_q ? (T*)a.q_out + (row * a.heads + h) * a.dim : (T*)a.k_out + (row * a.kv_heads + h) * a.dim;
    float f[E], g[E];
    load_some<T, E>(x + first, n, f);
    if constexpr (INTERLEAVED) {
      if (turned) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float u = f[2 * e], v = f[2 * e + 1];
          f[2 * e] = fmaf(u, t[e].c, -v * t[e].s);
          f[2 * e + 1] = fmaf(u, t[e].s, v * t[e].c);
        }
      }
    } else if (turned) {
      load_some<T, E>(x + a.pairs + first, n, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float u = f[e], v = g[e];
        f[e] = fmaf(u, t[e].c, -v * t[e].s);
        g[e] = fmaf(u, t[e].s, v * t[e].c);
      }
      store_some<T, E>(y + a.pairs + first, n, g);
    }
    store_some<T, E>(y + first, n, f);
  }
}

__global__ __launch_bounds__(ROTATE_THREADS) void k_positions(const int32_t* start, const int32_t* first, int batch,
                                                             int64_t rows, int32_t* position) {
  const int64_t row = (int64_t)blockIdx.x * ROTATE_THREADS + threadIdx.x;
  if (row >= rows) return;
  int lo = 0, hi = batch + 1;  // start[lo - 1] <= row < start[hi]
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (start[mid] <= row)
      lo = mid + 1;
    else
      hi = mid;
  }
  position[row] = lo == 0 || lo > batch ? 0 : (first ? first[lo - 1] : 0) + (int)(row - start[lo - 1]);
}

// Threads that share a row's heads: one goes over all of them where rows are many, so that an angle is formed once for up to
// HEADS_EACH heads; where rows are few, each takes one.
constexpr int HEADS_EACH = 8;
constexpr int64_t MANY_THREADS = 256 * 1024;
int teams_of(int64_t rows, int chunks, int heads) {
  for (int each = HEADS_EACH; each > 1; each /= 2)
    if (rows * chunks * ((heads + each - 1) / each) >= MANY_THREADS) return (heads + each - 1) / each;
  return heads;
}

bool bad_heads(const void* x, const void* y, int64_t row, int64_t head, int64_t heads, int64_t dim, int64_t per) {
  return !x || !y || off_align(x, 16) || off_align(y, 16) || row < dim || row > 1 << 22 || row % per || head < 0 ||
         head > INT64_MAX / 2 / heads || head % per;
}

}  // namespace

extern "C" {

int lram_positions(const int32_t* start, const int32_t* first, int32_t batch, int64_t rows, int32_t* position, void* stream) {
  if (batch < 0 || batch > 1 << 24 || rows < 0 || rows > 1 << 30) return LRAM_EINVAL;
  if (rows == 0) return LRAM_OK;
  if (!start || !position || off_align(start, 4) || off_align(first, 4) || off_align(position, 4)) return LRAM_EINVAL;
  hipLaunchKernelGGL(k_positions, dim3((unsigned)((rows + ROTATE_THREADS - 1) / ROTATE_THREADS)), dim3(ROTATE_THREADS), 0,
                     (hipStream_t)stream, start, first, (int)batch, rows, position);
  return layer_launched();
}

int lram_rotate(const lram_rotary* r, int dtype, int backward, int64_t rows, int32_t head_dim, const int32_t* position,
                const void* q, int64_t q_row, int64_t q_head, int32_t heads, void* q_out, const void* k, int64_t k_row,
                int64_t k_head, int32_t kv_heads, void* k_out, void* stream) {
  if (dtype != LRAM_F32 && dtype != LRAM_BF16) return LRAM_EDTYPE;
  if (!r || head_dim < 8 || head_dim > LRAM_ROTARY_MAX_HEAD_DIM || head_dim % 8) return LRAM_EINVAL;
  if (int rc = check_rotary(*r, head_dim)) return rc;
  if (rows < 0 || rows > 1 << 30 || heads < 1 || heads > 65536 || kv_heads < 0 || kv_heads > 65536) return LRAM_EINVAL;
  if (rows == 0) return LRAM_OK;
  const int64_t per = 16 / (int64_t)elem_size(dtype);
  if (bad_heads(q, q_out, q_row, q_head, heads, head_dim, per)) return LRAM_EINVAL;
  if (kv_heads && bad_heads(k, k_out, k_row, k_head, kv_heads, head_dim, per)) return LRAM_EINVAL;
  if (!position || off_align(position, 4)) return LRAM_EINVAL;
  Rotate a{q, k, q_out, k_out, q_row, q_head, k_row, k_head, r->turns, position, rows, heads, kv_heads, head_dim, r->pairs};
  const int64_t turned = r->interleaved ? 2 * r->pairs : r->pairs;
  a.pair_chunks = (int)((turned + per - 1) / per);
  a.chunks = r->interleaved ? (int)(head_dim / per) : a.pair_chunks + (int)((head_dim - 2 * r->pairs + per - 1) / per);
  a.teams = teams_of(rows, a.chunks, heads + kv_heads);
  a.magnitude = r->magnitude;
  a.sign = backward ? -1.0f : 1.0f;
  const int64_t each = (int64_t)a.chunks * a.teams;  // threads of a row
  const int64_t most = ((int64_t)1 << 31) / each;    // rows of a launch: fewer than 2^32 threads
  for (int64_t row = 0; row < rows; row += most) {
    Rotate part = a;
    part.rows = std::min(rows - row, most);
    part.position = position + row;
    const int64_t size = (int64_t)elem_size(dtype);
    part.q = (const char*)q + row * q_row * size;
    part.q_out = (char*)q_out + row * heads * head_dim * size;
    if (kv_heads) {
      part.k = (const char*)k + row * k_row * size;
      part.k_out = (char*)k_out + row * kv_heads * head_dim * size;
    }
    const auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((part.rows * each + ROTATE_THREADS - 1) / ROTATE_THREADS)),
                         dim3(ROTATE_THREADS), 0, (hipStream_t)stream, part);
      return layer_launched();
    };
    const int rc = dtype == LRAM_BF16 ? r->interleaved ? go(k_rotate<bf16, true>) : go(k_rotate<bf16, false>)
                   : r->interleaved   ? go(k_rotate<float, true>)
                                      : go(k_rotate<float, false>);
    if (rc) return rc;
  }
  return LRAM_OK;
}

}  // extern "C"
