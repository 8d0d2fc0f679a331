// layer_norm.hip -- part of liblram: layer norm, forward and backward, for gfx950.
//
//     h = x + r;  y = (h - mu) rs w + b,  mu = mean h,  rs = 1 / sqrt(mean (h - mu)^2 + eps)
//     g = dy w;   dx = rs (g - mean g - n mean(g n)) + dh,  n = (h - mu) rs;  dw = sum dy n,  db = sum dy
//
// Bound by HBM: a row is read once and stays in registers between its statistics and its result (mean first, then
// the squared distances from it: no cancellation).  A row belongs to a wave or a workgroup; a thread owns the same columns of
// every row, so that in the backward pass the weights' gradients add up in its registers over the rows that the group
// takes, and only one partial row per workgroup goes through memory to the second kernel.

#include <algorithm>

#include "layer_common.h"

namespace {

thread_local int g_hip_error = 0;

constexpr int CHUNK_BYTES = 16;
constexpr int NORM_WAVES = 4;  // waves of a workgroup whose waves take rows of their own

// Sums over a row's threads.  G: threads of a row; a workgroup's sums go through LDS, in the waves' order.
template <int G, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float (*lds)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
  if constexpr (G > WAVE) {
    const int w = threadIdx.x / WAVE;
    __syncthreads();  // the last sums have been read
    if (threadIdx.x % WAVE == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[w][i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0;
#pragma unroll
    for (int v = 0; v < G / WAVE; ++v)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += lds[v][i];
  }
}

// The columns of thread t of a row's G threads: chunk i starts at (t + i G) V.  A chunk that the row's end cuts is
// moved element by element.
template <typename T, int V>
__device__ __forceinline__ void load_cols(const T* row, int c, int width, float (&f)[V]) {
  if (c + V <= width) {
    load_n<T, V>(row + c, f);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = c + e < width ? (float)row[c + e] : 0.0f;
  }
}

template <typename T, int V>
__device__ __forceinline__ void store_cols(T* row, int c, int width, const float (&f)[V]) {
  if (c + V <= width) {
    store_n<T, V>(row + c, f);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (c + e < width) row[c + e] = (T)f[e];
  }
}

template <typename T>
constexpr int vec() { return CHUNK_BYTES / (int)sizeof(T); }

constexpr int threads_of(int G) { return G == WAVE ? NORM_WAVES * WAVE : G; }

template <typename T, typename W, int G, int NC, bool RES>
__global__ __launch_bounds__(threads_of(G)) void k_norm_forward(const T* x, const T* r, const W* w,
                                                               const W* b, int64_t rows, int width, float eps, T* sum,
                                                               T* y, float* mean, float* rstd) {
  constexpr int V = vec<T>();
  __shared__ float lds[G > WAVE ? G / WAVE : 1][1];
  const int t = G == WAVE ? threadIdx.x % WAVE : threadIdx.x;
  const int64_t row = G == WAVE ? (int64_t)blockIdx.x * NORM_WAVES + threadIdx.x / WAVE : blockIdx.x;
  if (row >= rows) return;  // whole waves of the wave form only, which meets no barrier
  const int64_t at = row * width;
  float h[NC][V];
  float s[1] = {0};
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = (t + i * G) * V;
    load_cols<T, V>(x + at, c, width, h[i]);
    if constexpr (RES) {
      float f[V];
      load_cols<T, V>(r + at, c, width, f);
#pragma unroll
      for (int e = 0; e < V; ++e) h[i][e] = (float)(T)(h[i][e] + f[e]);  // what the caller gets is what is normed
    }
#pragma unroll
    for (int e = 0; e < V; ++e) s[0] += h[i][e];
  }
  if constexpr (RES) {
#pragma unroll
    for (int i = 0; i < NC; ++i) store_cols<T, V>(sum + at, (t + i * G) * V, width, h[i]);
  }
  row_sum<G>(s, lds);
  const float mu = s[0] / (float)width;
  s[0] = 0;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = (t + i * G) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      h[i][e] -= mu;
      s[0] = c + e < width ? fmaf(h[i][e], h[i][e], s[0]) : s[0];
    }
  }
  row_sum<G>(s, lds);
  const float rs = 1.0f / sqrtf(s[0] / (float)width + eps);
  if (mean && t == 0) {
    mean[row] = mu;
    rstd[row] = rs;
  }
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = (t + i * G) * V;
    float fw[V], fb[V];
    load_cols<W, V>(w, c, width, fw);
    load_cols<W, V>(b, c, width, fb);
#pragma unroll
    for (int e = 0; e < V; ++e) h[i][e] = fmaf(h[i][e] * rs, fw[e], fb[e]);
    store_cols<T, V>(y + at, c, width, h[i]);
  }
}

// part: [workgroups][2][width] sums of dy n and dy over the workgroup's rows; ONE: the only workgroup writes the
// weights' gradients themselves.
template <typename T, typename W, int G, int NC>
__global__ __launch_bounds__(threads_of(G)) void k_norm_backward(const T* __restrict__ h, const W* w, const float* mean,
                                                                const float* rstd, const T* dy, const T* dh,
                                                                int64_t rows, int width, T* dx, float* part, W* dw,
                                                                W* db) {
  constexpr int V = vec<T>();
  constexpr int TEAMS = G == WAVE ? NORM_WAVES : 1;  // rows in flight in a workgroup
  __shared__ float lds[G > WAVE ? G / WAVE : 1][2];
  const int t = G == WAVE ? threadIdx.x % WAVE : threadIdx.x;
  const int team = G == WAVE ? threadIdx.x / WAVE : 0;
  const float inv = 1.0f / (float)width;
  float sw[NC][V] = {}, sb[NC][V] = {}, fw[NC][V];
#pragma unroll
  for (int i = 0; i < NC; ++i) load_cols<W, V>(w, (t + i * G) * V, width, fw[i]);
  for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < rows; row += (int64_t)gridDim.x * TEAMS) {
    const int64_t at = row * width;
    float n[NC][V], g[NC][V];
    float s[2] = {0, 0};
    const float mu = mean[row], rs = rstd[row];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      load_cols<T, V>(h + at, (t + i * G) * V, width, n[i]);
      load_cols<T, V>(dy + at, (t + i * G) * V, width, g[i]);
    }
    float f[NC][V];
    if (dh) {
#pragma unroll
      for (int i = 0; i < NC; ++i) load_cols<T, V>(dh + at, (t + i * G) * V, width, f[i]);
    }
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // past the row's end dy is 0, and with it every term
        n[i][e] = (n[i][e] - mu) * rs;
        sw[i][e] = fmaf(g[i][e], n[i][e], sw[i][e]);
        sb[i][e] += g[i][e];
        g[i][e] *= fw[i][e];
        s[0] += g[i][e];
        s[1] = fmaf(g[i][e], n[i][e], s[1]);
      }
    row_sum<G>(s, lds);
    const float a = s[0] * inv, c = s[1] * inv;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = rs * (g[i][e] - a - n[i][e] * c);
        g[i][e] = dh ? d + f[i][e] : d;
      }
      store_cols<T, V>(dx + at, (t + i * G) * V, width, g[i]);
    }
  }
  if (!part && !dw) return;
  if constexpr (TEAMS > 1) {  // the waves' sums, in their order
    __shared__ float team_sum[TEAMS - 1][V][WAVE];
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float(&v)[V] = k ? sb[i] : sw[i];
        __syncthreads();
        if (team)
#pragma unroll
          for (int e = 0; e < V; ++e) team_sum[team - 1][e][t] = v[e];
        __syncthreads();
        if (!team)
#pragma unroll
          for (int o = 0; o < TEAMS - 1; ++o)
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += team_sum[o][e][t];
      }
    if (team) return;
  }
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = (t + i * G) * V;
    if (c >= width) continue;
    if (dw) {
      store_cols<W, V>(dw, c, width, sw[i]);
      store_cols<W, V>(db, c, width, sb[i]);
    } else {
      float* p = part + (int64_t)blockIdx.x * 2 * width;
      store_cols<float, V>(p, c, width, sw[i]);
      store_cols<float, V>(p + width, c, width, sb[i]);
    }
  }
}

// The workgroups' partial rows [n][2 width] added up: 16 columns to a workgroup, 64 threads to a column, each a fixed
// set of the partial rows.
constexpr int FIN_COLS = 16, FIN_ROWS = 64;
template <typename W>
__global__ __launch_bounds__(FIN_COLS* FIN_ROWS) void k_norm_finish(const float* part, int n, int width, W* dw, W* db) {
  __shared__ float lds[FIN_ROWS][FIN_COLS];
  const int c = threadIdx.x % FIN_COLS, r = threadIdx.x / FIN_COLS;
  const int col = blockIdx.x * FIN_COLS + c;
  float s = 0;
  if (col < 2 * width) {
#pragma unroll 8
    for (int p = r; p < n; p += FIN_ROWS) s += part[(int64_t)p * 2 * width + col];
  }
  lds[r][c] = s;
  __syncthreads();
#pragma unroll
  for (int half = FIN_ROWS / 2; half > 0; half /= 2) {
    if (r < half) lds[r][c] += lds[r + half][c];
    __syncthreads();
  }
  if (r == 0 && col < 2 * width) {
    if (col < width)
      dw[col] = (W)lds[0][c];
    else
      db[col - width] = (W)lds[0][c];
  }
}

// Threads of a row and chunks of a thread: a thread to a chunk, which is the shortest way through a row, but waves take
// rows of up to four chunks a lane where there are many (us of a thread to a chunk / waves: 64 rows x 2,048 bf16 3.2 / 5.4,
// 1,024 x 2,048 4.8 / 6.4, 2,048 x 1,024 6.1 / 5.2, 5,003 x 500 fp32 11.4 / 7.2; of one chunk / four to 256 threads:
// 16,384 x 8,192 bf16 192 / 200, 64 x 8,192 4.2 / 5.8).  With more than two chunks a lane the two are close, and one rule
// serves both types though bf16 leans the other way (with a residual: fp32 8,192 x 520 15.2 / 13.1, 40,000 x 520 77 / 61,
// 8,192 x 1,024 23.8 / 24.2, 2,048 x 800 7.6 / 8.1; bf16 40,000 x 1,040 94 / 84, 8,192 x 2,048 23.8 / 24.1, 8,192 x 1,600
// 19.9 / 23.0, 2,048 x 1,600 8.3 / 10.5).
constexpr int64_t FEW_ROWS = 1024;
struct Shape {
  int G, NC;
};
Shape shape_of(int64_t rows, int64_t width, int dtype) {
  const int64_t chunks = (width + CHUNK_BYTES / (int)elem_size(dtype) - 1) / (CHUNK_BYTES / (int)elem_size(dtype));
  for (int NC : {1, 2, 4})
    if ((NC == 1 || rows > FEW_ROWS) && chunks <= WAVE * NC) return {WAVE, NC};
  for (int G : {4 * WAVE, 8 * WAVE, 16 * WAVE})
    if (chunks <= G) return {G, 1};
  return {16 * WAVE, chunks <= 32 * WAVE ? 2 : 4};
}

// The backward pass holds three rows and the weights' sums, so its rows take more threads with a chunk each (16,384 rows of
// 8,192 bf16 with grad_sum: 256 threads with four chunks each 526 us, 1,024 with one 222 us).
Shape backward_shape_of(int64_t width, int dtype) {
  const int64_t chunks = (width + CHUNK_BYTES / (int)elem_size(dtype) - 1) / (CHUNK_BYTES / (int)elem_size(dtype));
  if (chunks <= 2 * WAVE) return {WAVE, chunks <= WAVE ? 1 : 2};
  for (int G : {4 * WAVE, 8 * WAVE, 16 * WAVE})
    if (chunks <= G) return {G, 1};
  return {16 * WAVE, chunks <= 32 * WAVE ? 2 : 4};
}

// Workgroups of the backward pass: enough to keep HBM busy, and few against the rows, since each leaves a partial row
// of its own for the second kernel (us of both kernels with half, as many and twice as many: 8,192 x 512 bf16 13.9 / 12.8 /
// 17.8, 5,003 x 1,021 fp32 21.7 / 20.4 / 24.0, 16,384 x 8,192 bf16 382 / 230 / 236).
int64_t groups_of(int64_t rows, const Shape& sh) {
  const int64_t teams = sh.G == WAVE ? NORM_WAVES : 1;
  const int64_t all = (rows + teams - 1) / teams;
  const int64_t most = sh.G > 4 * WAVE ? 4096 * WAVE / sh.G : 1024;
  return all < most ? all : most;
}

template <typename F>
int by_shape(const Shape& sh, F f) {
#define LRAM_SHAPE(g, n) \
  if (sh.G == g && sh.NC == n) return f(std::integral_constant<int, g>(), std::integral_constant<int, n>());
  LRAM_SHAPE(64, 1) LRAM_SHAPE(64, 2) LRAM_SHAPE(64, 4)
  LRAM_SHAPE(256, 1) LRAM_SHAPE(512, 1) LRAM_SHAPE(1024, 1) LRAM_SHAPE(1024, 2) LRAM_SHAPE(1024, 4)
#undef LRAM_SHAPE
  return LRAM_EINVAL;
}

template <typename F>
int by_types(int dtype, int wdtype, F f) {
  if (dtype == LRAM_F32 && wdtype == LRAM_F32) return f(float(), float());
  if (dtype == LRAM_BF16 && wdtype == LRAM_F32) return f(bf16(), float());
  if (dtype == LRAM_BF16 && wdtype == LRAM_BF16) return f(bf16(), bf16());
  return LRAM_EDTYPE;
}

int check_norm(int dtype, int wdtype, int64_t rows, int64_t width) {
  if (rows < 0 || width < 1 || width > LRAM_NORM_MAX_WIDTH || rows > INT32_MAX) return LRAM_EINVAL;
  if (dtype != LRAM_F32 && dtype != LRAM_BF16) return LRAM_EDTYPE;
  if (wdtype != LRAM_F32 && !(wdtype == LRAM_BF16 && dtype == LRAM_BF16)) return LRAM_EDTYPE;
  return LRAM_OK;
}

}  // namespace

int layer_failed(hipError_t e) {
  g_hip_error = (int)e;
  return LRAM_EHIP;
}

int layer_launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LRAM_OK : layer_failed(e);
}

extern "C" {

int lram_layer_last_hip_error(void) { return g_hip_error; }

int lram_layer_norm_forward(const void* x, const void* residual, const void* weight, const void* bias, int dtype,
                            int wdtype, int64_t rows, int64_t width, double eps, void* sum, void* y, float* mean,
                            float* rstd, void* stream) {
  if (int rc = check_norm(dtype, wdtype, rows, width)) return rc;
  if (!(eps >= 0) || (residual != nullptr) != (sum != nullptr) || (mean != nullptr) != (rstd != nullptr))
    return LRAM_EINVAL;
  if (rows == 0) return LRAM_OK;
  if (!x || !weight || !bias || !y || y == sum) return LRAM_EINVAL;
  if (off_align(x, 16) || off_align(residual, 16) || off_align(sum, 16) || off_align(y, 16) || off_align(mean, 4) ||
      off_align(rstd, 4) || off_align(weight, elem_size(wdtype)) || off_align(bias, elem_size(wdtype)))
    return LRAM_EINVAL;
  const Shape sh = shape_of(rows, width, dtype);
  return by_types(dtype, wdtype, [&](auto t, auto v) {
    using T = decltype(t);
    using W = decltype(v);
    return by_shape(sh, [&](auto g, auto n) {
      constexpr int G = decltype(g)::value, NC = decltype(n)::value;
      constexpr int64_t EACH = G == WAVE ? NORM_WAVES : 1;  // rows of a workgroup
      constexpr int64_t MOST = ((int64_t(1) << 32) / threads_of(G) - 1) * EACH;  // of a launch: less than 2^32 threads
      const auto go = [&](auto kernel) {
        for (int64_t row = 0; row < rows; row += MOST) {
          const int64_t n = std::min(rows - row, MOST), at = row * width;
          hipLaunchKernelGGL(kernel, dim3((unsigned)((n + EACH - 1) / EACH)), dim3(threads_of(G)), 0, (hipStream_t)stream,
                             (const T*)x + at, residual ? (const T*)residual + at : nullptr, (const W*)weight,
                             (const W*)bias, n, (int)width, (float)eps, sum ? (T*)sum + at : nullptr, (T*)y + at,
                             mean ? mean + row : nullptr, rstd ? rstd + row : nullptr);
          if (int rc = layer_launched()) return rc;
        }
        return (int)LRAM_OK;
      };
      return residual ? go(k_norm_forward<T, W, G, NC, true>) : go(k_norm_forward<T, W, G, NC, false>);
    });
  });
}

int lram_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width, int dtype, size_t* bytes) {
  if (!bytes) return LRAM_EINVAL;
  if (int rc = check_norm(dtype, LRAM_F32, rows, width)) return rc;
  const int64_t n = groups_of(rows, backward_shape_of(width, dtype));
  *bytes = n > 1 ? (size_t)n * 2 * width * 4 : 0;
  return LRAM_OK;
}

int lram_layer_norm_backward(const void* h, const void* weight, const float* mean, const float* rstd,
                             const void* grad_y, const void* grad_sum, int dtype, int wdtype, int64_t rows,
                             int64_t width, void* grad_x, void* grad_weight, void* grad_bias, void* workspace,
                             size_t ws_bytes, void* stream) {
  if (int rc = check_norm(dtype, wdtype, rows, width)) return rc;
  if ((grad_weight != nullptr) != (grad_bias != nullptr)) return LRAM_EINVAL;
  if (rows == 0 && !grad_weight) return LRAM_OK;
  if (rows && (!h || !mean || !rstd || !grad_y || !grad_x)) return LRAM_EINVAL;
  if (!weight) return LRAM_EINVAL;
  if (off_align(h, 16) || off_align(grad_y, 16) || off_align(grad_sum, 16) || off_align(grad_x, 16) ||
      off_align(mean, 4) || off_align(rstd, 4) || off_align(weight, elem_size(wdtype)) ||
      off_align(grad_weight, elem_size(wdtype)) || off_align(grad_bias, elem_size(wdtype)))
    return LRAM_EINVAL;
  const Shape sh = backward_shape_of(width, dtype);
  const int64_t groups = groups_of(rows, sh);
  const bool two = grad_weight && groups > 1;
  if (two && (!workspace || off_align(workspace, 16) || ws_bytes < (size_t)groups * 2 * width * 4))
    return LRAM_EWORKSPACE;
  return by_types(dtype, wdtype, [&](auto t, auto v) {
    using T = decltype(t);
    using W = decltype(v);
    const int rc = by_shape(sh, [&](auto g, auto n) {
      constexpr int G = decltype(g)::value, NC = decltype(n)::value;
      // no rows: one workgroup, whose sums are the zeros that the weights' gradients are
      hipLaunchKernelGGL((k_norm_backward<T, W, G, NC>), dim3((unsigned)(groups ? groups : 1)), dim3(threads_of(G)), 0,
                         (hipStream_t)stream, (const T*)h, (const W*)weight, mean, rstd, (const T*)grad_y,
                         (const T*)grad_sum, rows, (int)width, (T*)grad_x, two ? (float*)workspace : nullptr,
                         two ? nullptr : (W*)grad_weight, two ? nullptr : (W*)grad_bias);
      return layer_launched();
    });
    if (rc || !two) return rc;
    hipLaunchKernelGGL(k_norm_finish<W>, dim3((unsigned)((2 * width + FIN_COLS - 1) / FIN_COLS)),
                       dim3(FIN_COLS * FIN_ROWS), 0, (hipStream_t)stream, (const float*)workspace, (int)groups,
                       (int)width, (W*)grad_weight, (W*)grad_bias);
    return layer_launched();
  });
}

}  // extern "C"
