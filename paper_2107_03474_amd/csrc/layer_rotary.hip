// layer_rotary.hip -- part of liblram: rotary positions for gfx950.
//
// Bound by HBM: every element is read and written once (rotate_chunk).  16,384 rows of 32/8 heads of 128 bf16: 61 us, 5.5 TB/s
// (52 where the same rows are rotated again and again); 8,192 rows of 8/8 heads of 64 7.7 us, 4.4 TB/s; 17 pairs of 64 dimensions
// in fp32, 5,003 rows of 12/4 heads, 10 us, 4.0 TB/s.

#include <algorithm>

#include "layer_rotary.h"

namespace {

template <typename T, Form FORM>
__global__ __launch_bounds__(ROTATE_THREADS) void k_rotate(Rotate a) {
  const auto position_of = [&](int64_t row) { return a.position[row]; };
  if (a.past)
    rotate_chunk<T, FORM, true>(a, blockIdx.x * ROTATE_THREADS + threadIdx.x, position_of);
  else
    rotate_chunk<T, FORM, false>(a, blockIdx.x * ROTATE_THREADS + threadIdx.x, position_of);
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
  Rotate a{q, k, q_out, k_out, q_row, q_head, k_row, k_head, r->turns, position, rows, heads, kv_heads, head_dim};
  const int64_t each = divide(a, *r, dtype);  // threads of a row
  a.sign = backward ? -1.0f : 1.0f;
  const int64_t most = ((int64_t)1 << 31) / each;    // rows of a launch: at most 2^31 threads
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
    const Form form = form_of(*r, dtype);
    const auto of = [&](auto t) {
      using T = decltype(t);
      return form == NEIGHBOURS ? go(k_rotate<T, NEIGHBOURS>) : form == HALVES ? go(k_rotate<T, HALVES>) : go(k_rotate<T, ODD_HALVES>);
    };
    if (int rc = dtype == LRAM_BF16 ? of(bf16()) : of(float())) return rc;
  }
  return LRAM_OK;
}

}  // extern "C"
