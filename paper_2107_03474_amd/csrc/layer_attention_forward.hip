// layer_attention_forward.hip -- part of liblram: attention over packed sequences, forward (see layer_attention.h for
// the formulas and the tiles).
//
// k_attention: prompts.  A workgroup holds 128 packed rows, 32 to a wave, whose queries stay in registers; keys and values
// pass through LDS in tiles of 64, the next tile's loads in flight while one is used.  One pass: running maximum m and
// sum l a row, accumulators rescaled only when the maximum grows by more than 2^8 (the weights stay exact in that
// range, and the branch is rarely taken).  A tile's scores are formed while the one before it is weighed.  Weights go into
// the product with the values rounded to the values' type, the matrix cores' own; their sum is of the unrounded ones.
// k_attention_few: a few queries over many keys.  The four waves of a workgroup share the same 32 rows and take key
// tiles in turn, each through LDS of its own without barriers, and join their sums at the end.
// Where rows are few against the chip the keys are divided into pieces (either kernel) that k_attention_join joins.

#include "layer_attention.h"

namespace {

constexpr int MAX_SPLITS = 64;
constexpr float GROWTH = 8;  // log2 of how far weights may pass 1 before the sums are rescaled

struct Out {
  void* out;
  void* residue;
  float* lse;
  float *part, *part_lse;  // [splits][tq heads][D], [splits][tq heads]
};

// A wave's running softmax over its 32 rows (a row to a lane and its twin in the other half).
template <int D>
struct Running {
  f32x16 o[D / 32];
  float m, l;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[b][r] = 0;
    m = -INFINITY;
    l = 0;
  }
};

// Scores of 32 keys (a block of rows of the tile at kt) with the wave's 32 rows.
template <typename T, int D>
__device__ __forceinline__ f32x16 scores(const typename Frag<T>::type (&q)[D / 16], Lds kt, uint32_t ka, int first_key) {
  f32x16 s;
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) s = mma(Tile<T, D>::row_frag(kt, ka, k, first_key), q[k], s);
  return s;
}

// Asks the compiler to spread a step's matrix instructions over its vector instructions and LDS reads: a block's products
// with the keys, each followed by six vector instructions of the weights, then those with the values.  (8,192 causal
// tokens, 16/8 heads of 64, bias: 191 -> 183 us; with heads of 128 the compiler's own order is the faster: 555 us, 585 with
// this one.)
template <typename T, int D>
__device__ __forceinline__ void interleave() {
  if constexpr (sizeof(T) == 2 && D <= 64) {
    constexpr int MFMA = 0x8, VALU = 0x2, DS_READ = 0x100;
    __builtin_amdgcn_sched_group_barrier(DS_READ, 2, 0);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(VALU, 6, 0);
      __builtin_amdgcn_sched_group_barrier(DS_READ, 1, 0);
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      __builtin_amdgcn_sched_group_barrier(DS_READ, 2, 0);
      __builtin_amdgcn_sched_group_barrier(MFMA, 1, 0);
      __builtin_amdgcn_sched_group_barrier(VALU, 1, 0);
    }
  }
}

// What a wave adds to scores of the 32 keys from j on: z = unit s + far after it.  near: the bias differs from pair to pair, and
// `bias` is the lane's row of its table at distance -(i + off); else one value of it, `far`, serves the block.
// masked: some row of the wave does not see every key; lim: the last key that the lane's row sees.
template <bool BIAS>
__device__ __forceinline__ void prepare(f32x16& s, float c, int j, const float* bias, bool near, bool masked, int lim) {
  const int h = threadIdx.x >> 5 & 1;
  if constexpr (BIAS) {
    if (near) {
      const float* at = bias + j + 4 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], c, at[8 * (r >> 2) + (r & 3)]);
    }
  }
  if (masked) {
    const int last = lim - j - 4 * h;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) <= last ? s[r] : -INFINITY;
  }
}

// The running maximum after a block's scores; the sums are rescaled if it grew by more than GROWTH in some row.
template <int D>
__device__ __forceinline__ void grow(Running<D>& st, const f32x16& s, float unit, float far) {
  float top = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
  top = fmaf(max_halves(top), unit, far);
  if (__builtin_amdgcn_ballot_w64(top > st.m + GROWTH)) {
    const float m = fmaxf(st.m, top);
    const float a = __builtin_amdgcn_exp2f(st.m - (m == -INFINITY ? 0.0f : m));
    st.m = m;
    st.l *= a;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[b][r] *= a;
  }
}

// The weights of a block, in place of its scores.
template <int D>
__device__ __forceinline__ void weigh(Running<D>& st, f32x16& s, float unit, float far) {
  const float less = far - (st.m == -INFINITY ? 0.0f : st.m);
  float l = 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], unit, less));
    l += s[r];
  }
  st.l += l;
}

// The block's weights times its values, rows first_key ... of the tile at vt (a multiple of 32).
template <typename T, int D>
__device__ __forceinline__ void collect(Running<D>& st, const f32x16& s, Lds vt, uint32_t va, int first_key) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    f32x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = s[8 * k + e];
    const auto f = to_frag<T>(p);
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
      st.o[b] = mma(Tile<T, D>::col_frag(vt, va, b, first_key / 16 + k), f, st.o[b]);
  }
}

// Results of flat row `at` = (row of q) heads + head: 4 elements from d on.
template <typename T, int D>
__device__ __forceinline__ void put(const Args& a, const Out& o, int split, int64_t at, int d, f32x4 x) {
  if (a.splits > 1) {
    *(f32x4*)(o.part + ((int64_t)split * a.tq * a.heads + at) * D + d) = x;
    return;
  }
  T* p = (T*)o.out + at * D + d;
  store4<T>(p, x);
  if constexpr (sizeof(T) == 2) {
    if (o.residue) {
      f32x4 left;
#pragma unroll
      for (int e = 0; e < 4; ++e) left[e] = x[e] - (float)(T)x[e];
      store4<T>((T*)o.residue + at * D + d, left);
    }
  }
}
__device__ __forceinline__ void put_lse(const Args& a, const Out& o, int split, int64_t at, float lse) {
  if (a.splits > 1)
    o.part_lse[(int64_t)split * a.tq * a.heads + at] = lse;
  else if (o.lse)
    o.lse[at] = lse;
}

// TEAMS: of four waves each, which share the rows and take the tiles of keys in turn; the second joins its sums to the
// first's at the end (plan_of: when).
template <typename T, int D, int TEAMS>
constexpr int prompt_bytes() { return TEAMS * ring_bytes<T, D>(); }
template <typename T, int D, bool BIAS, int TEAMS>
__global__ __launch_bounds__(TEAMS* THREADS, (waves_per_simd<T, D>())) void k_attention(Args a, Out o) {
  using Ti = Tile<T, D>;
  constexpr int M = WAVES * ROWS;
  extern __shared__ __attribute__((aligned(256))) char smem[];
  Work w;
  if (!find_work<M>(a, &w)) return;
  using Ring = KeyAhead<T, D, TEAMS>;
  Ring ring(a, w, (Lds)smem, __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE) % WAVES, l = threadIdx.x % WAVE;
  const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  const int G = a.group, off = w.s.nk - w.s.nq, first = w.row0 + wave * ROWS, rows = w.s.nq * G;
  const Row r = row_of(a, w.s, first + (l & 31));
  const int head = w.head.first + r.g;
  if (a.splits > 1 && w.kbeg >= w.kend) {  // a piece without keys: the join leaves it out
    if (r.valid && l < 32 && !team) put_lse(a, o, w.split, (w.s.q0 + r.i) * a.heads + head, -INFINITY);
    return;
  }
  typename Frag<T>::type q[D / 16];
  load_query<T, D>(a, (const T*)a.q, a.q_row, a.q_head, w.s, head, r, q);
  // last key of the lane's row, and of the wave's first and last rows
  const int lim = a.causal && r.valid ? min(r.i + off, w.s.nk - 1) : w.s.nk - 1;
  const int i_first = first / G, i_last = (min(first + ROWS, rows) - 1) / G;
  const int lim_first = a.causal ? min(i_first + off, w.s.nk - 1) : w.s.nk - 1;
  const int lim_last = first >= rows ? -1 : (a.causal ? min(i_last + off, w.s.nk - 1) : w.s.nk - 1);
  const float* bias = nullptr;
  float near_far[2] = {0, 0}, far_unit[2] = {a.c, a.c};
  if constexpr (BIAS) {
    float* table = (float*)(smem + prompt_bytes<T, D, TEAMS>());
    fill_bias(a, w.head.first, G, table);
    bias = table + r.g * bias_width(a) + a.reach + BIAS_PAD - (r.i + off);
    __syncthreads();
    const float* mine = table + (r.valid ? r.g : 0) * bias_width(a);
    near_far[0] = mine[0];
    near_far[1] = mine[bias_width(a) - 1];
#pragma unroll
    for (int side = 0; side < 2; ++side) far_unit[side] = unit_beside(near_far[side], a.c);
  }
  const uint32_t ka = Ti::row_base(l & 31), va = Ti::col_base();
  Running<D> st;
  st.clear();
  // The scores of a tile are formed one tile ahead, between the weights of this one: the matrix cores and the vector
  // units work at the same time.
  f32x16 s[KEYS / 32], next[KEYS / 32];
  const auto tile = [&](int j0, Lds kt, Lds vt, auto more) {
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b) {
      const int j = j0 + 32 * b;
      bool near = false, above = false;
      float far = 0;
      if constexpr (BIAS) {
        const bool below = j + 31 - (i_first + off) <= -a.reach;
        above = j - (i_last + off) >= a.reach;
        near = !below && !above;
        // a block past the wave's last key meets no distance of its own, and that one's weight may hold anything
        far = near || j > lim_last ? 0.0f : near_far[above];
      }
      const float unit = near ? 1.0f : BIAS ? far_unit[above] : a.c;
      prepare<BIAS>(s[b], a.c, j, bias, near, j + 31 > lim_first, lim);
      grow(st, s[b], unit, far);
      if constexpr (decltype(more)::value) next[b] = scores<T, D>(q, kt, ka, 32 * b);
      weigh(st, s[b], unit, far);
      collect<T, D>(st, s[b], vt, va, 32 * b);
      interleave<T, D>();
    }
    if constexpr (decltype(more)::value)
#pragma unroll
      for (int b = 0; b < KEYS / 32; ++b) s[b] = next[b];
  };
  const int mine = team * KEYS, at_lds = mine * Ti::ROW;  // the team's tile of a step
  if (w.kbeg < w.kend) {
    const Lds kt = ring.first() + at_lds;
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b) s[b] = scores<T, D>(q, kt, ka, 32 * b);
  }
  int j0 = w.kbeg;
  for (; j0 + Ring::STEP < w.kend; j0 += Ring::STEP) {
    ring.next(j0);
    if (j0 + mine <= lim_last) tile(j0 + mine, ring.keys() + at_lds, ring.values() + at_lds, std::true_type());
  }
  if (j0 < w.kend) {
    ring.next(j0);
    if (j0 + mine <= lim_last) tile(j0 + mine, ring.keys() + at_lds, ring.values() + at_lds, std::false_type());
  }
  float sum = add_halves(st.l);
  if constexpr (TEAMS == 2) {  // the second team's sums join the first one's, through the LDS that held the tiles
    constexpr int SUMS = D / 2;  // accumulators of a lane
    static_assert((SUMS + 2) * THREADS * 4 <= prompt_bytes<T, D, TEAMS>(), "they fit");
    float* const to = (float*)smem + threadIdx.x % THREADS;
    __syncthreads();
    if (team) {
      to[0] = st.m;
      to[THREADS] = sum;
#pragma unroll
      for (int e = 0; e < SUMS; ++e) to[(2 + e) * THREADS] = st.o[e / 16][e % 16];
    }
    __syncthreads();
    if (team) return;
    const float other = to[0], m = fmaxf(st.m, other), m0 = m == -INFINITY ? 0.0f : m;
    const float f = __builtin_amdgcn_exp2f(st.m - m0), g = __builtin_amdgcn_exp2f(other - m0);
    sum = sum * f + to[THREADS] * g;
    st.m = m;
#pragma unroll
    for (int e = 0; e < SUMS; ++e)
      st.o[e / 16][e % 16] = fmaf(to[(2 + e) * THREADS], g, st.o[e / 16][e % 16] * f);
  }
  if (!r.valid) return;
  const float inv = sum == 0 ? 0.0f : 1.0f / sum;
  const int64_t at = (w.s.q0 + r.i) * a.heads + head;
  if (l < 32) put_lse(a, o, w.split, at, lse_of(st.m, sum, BIAS));
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = st.o[b][4 * u + e] * inv;
      put<T, D>(a, o, w.split, at, 32 * b + 8 * u + 4 * (l >> 5), x);
    }
}

// Buffers of a wave's key and value tiles in k_attention_few: two where LDS holds them.
template <typename T, int D>
constexpr int few_stages() { return WAVES * 2 * 2 * 32 * Tile<T, D>::ROW <= 128 * 1024 ? 2 : 1; }
template <typename T, int D>
constexpr int few_bytes() { return WAVES * few_stages<T, D>() * 2 * 32 * Tile<T, D>::ROW; }

template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(THREADS, 1) void k_attention_few(Args a, Out o) {
  using Ti = Tile<T, D>;
  constexpr int N = 32, BYTES = N * Ti::ROW, STAGES = few_stages<T, D>();
  constexpr int LOADS = 2 * N * Ti::CH / 64;  // of a tile of keys and values
  extern __shared__ __attribute__((aligned(256))) char smem[];
  Work w;
  if (!find_work<ROWS>(a, &w)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), l = threadIdx.x % WAVE;
  Lds lds = (Lds)smem + wave * STAGES * 2 * BYTES;
  const int G = a.group, off = w.s.nk - w.s.nq, rows = w.s.nq * G;
  const Row r = row_of(a, w.s, w.row0 + (l & 31));
  const int head = w.head.first + r.g;
  if (a.splits > 1 && w.kbeg >= w.kend) {
    if (r.valid && threadIdx.x < 32) put_lse(a, o, w.split, (w.s.q0 + r.i) * a.heads + head, -INFINITY);
    return;
  }
  typename Frag<T>::type q[D / 16];
  load_query<T, D>(a, (const T*)a.q, a.q_row, a.q_head, w.s, head, r, q);
  const int lim = a.causal && r.valid ? min(r.i + off, w.s.nk - 1) : w.s.nk - 1;
  const int i_first = w.row0 / G, i_last = (min(w.row0 + ROWS, rows) - 1) / G;
  const int lim_first = a.causal ? min(i_first + off, w.s.nk - 1) : w.s.nk - 1;
  const float* bias = nullptr;
  float near_far[2] = {0, 0}, far_unit[2] = {a.c, a.c};
  if constexpr (BIAS) {
    float* table = (float*)(smem + few_bytes<T, D>());
    fill_bias(a, w.head.first, G, table);
    bias = table + r.g * bias_width(a) + a.reach + BIAS_PAD - (r.i + off);
    __syncthreads();
    const float* mine = table + (r.valid ? r.g : 0) * bias_width(a);
    near_far[0] = mine[0];
    near_far[1] = mine[bias_width(a) - 1];
#pragma unroll
    for (int side = 0; side < 2; ++side) far_unit[side] = unit_beside(near_far[side], a.c);
  }
  const uint32_t ka = Ti::row_base(l & 31), va = Ti::col_base();
  Running<D> st;
  st.clear();
  const T* kh = (const T*)a.k + w.s.k0 * a.k_row + w.head.kv * a.k_head;
  const T* vh = (const T*)a.v + w.s.k0 * a.v_row + w.head.kv * a.v_head;
  auto load = [&](int j0, int buf) {
    load_rows<T, D, N, 1>(kh, a.k_row, j0, w.s.nk, lds + buf * 2 * BYTES, 0);
    load_rows<T, D, N, 1>(vh, a.v_row, j0, w.s.nk, lds + buf * 2 * BYTES + BYTES, 0);
  };
  const int step = WAVES * N;
  int j0 = w.kbeg + wave * N;
  if (STAGES == 2 && j0 < w.kend) load(j0, 0);
  for (int buf = 0; j0 < w.kend; j0 += step, buf ^= STAGES - 1) {
    reads_done();  // of the buffer that is loaded next
    if (STAGES == 1) load(j0, 0);
    const bool more = STAGES == 2 && j0 + step < w.kend;
    if (more) {
      load(j0 + step, buf ^ 1);
      loads_left<LOADS>();
    } else {
      loads_left<0>();
    }
    bool near = false, above = false;
    float far = 0;
    if constexpr (BIAS) {
      const bool below = j0 + N - 1 - (i_first + off) <= -a.reach;
      above = j0 - (i_last + off) >= a.reach;
      near = !below && !above;
      far = near ? 0.0f : near_far[above];
    }
    const float unit = near ? 1.0f : BIAS ? far_unit[above] : a.c;
    f32x16 s = scores<T, D>(q, lds + buf * 2 * BYTES, ka, 0);
    prepare<BIAS>(s, a.c, j0, bias, near, j0 + N - 1 > lim_first, lim);
    grow(st, s, unit, far);
    weigh(st, s, unit, far);
    collect<T, D>(st, s, lds + buf * 2 * BYTES + BYTES, va, 0);
  }
  // join the waves: maxima and sums, then the scaled accumulators, through LDS
  constexpr int PITCH = D * 4 + 16;
  static_assert(WAVES * ROWS * PITCH + 2 * WAVES * ROWS * 4 <= few_bytes<T, D>() || D == 32, "the join fits");
  float* ml = (float*)(smem + WAVES * ROWS * PITCH);
  const float mine = add_halves(st.l);
  __syncthreads();
  if (l < 32) {
    ml[wave * ROWS + l] = st.m;
    ml[(WAVES + wave) * ROWS + l] = mine;
  }
  __syncthreads();
  float m = -INFINITY, sum = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) m = fmaxf(m, ml[v * ROWS + (l & 31)]);
  const float m0 = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int v = 0; v < WAVES; ++v)
    sum += ml[(WAVES + v) * ROWS + (l & 31)] * __builtin_amdgcn_exp2f(ml[v * ROWS + (l & 31)] - m0);
  const float f = sum == 0 ? 0.0f : __builtin_amdgcn_exp2f(st.m - m0) / sum;
  const int64_t at = (w.s.q0 + r.i) * a.heads + head;
  if (wave == 0 && l < 32 && r.valid) put_lse(a, o, w.split, at, lse_of(m, sum, BIAS));
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = st.o[b][4 * u + e] * f;
      *(f32x4*)(smem + (wave * ROWS + (l & 31)) * PITCH + (32 * b + 8 * u + 4 * (l >> 5)) * 4) = x;
    }
  __syncthreads();
  for (int t = threadIdx.x; t < ROWS * D / 4; t += THREADS) {
    const int row = t / (D / 4), d = t % (D / 4) * 4;
    const Row rr = row_of(a, w.s, w.row0 + row);
    if (!rr.valid) continue;
    f32x4 x = *(const f32x4*)(smem + row * PITCH + d * 4);
#pragma unroll
    for (int v = 1; v < WAVES; ++v) {
      const f32x4 y = *(const f32x4*)(smem + (v * ROWS + row) * PITCH + d * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    put<T, D>(a, o, w.split, (w.s.q0 + rr.i) * a.heads + w.head.first + rr.g, d, x);
  }
}

// The pieces of a flat row joined: a row to D / 4 lanes.
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void k_attention_join(Args a, Out o) {
  constexpr int PER = D / 4;  // lanes of a row
  const int64_t n = a.tq * a.heads;
  const int64_t at = ((int64_t)blockIdx.x * THREADS + threadIdx.x) / PER;
  const int d = threadIdx.x % PER * 4;
  if (at >= n) return;
  float m = -INFINITY;
  for (int s = 0; s < a.splits; ++s) m = fmaxf(m, parts_of(o.part_lse[s * n + at], a.rel_weight).top);
  const float m0 = m == -INFINITY ? 0.0f : m;
  float sum = 0;
  f32x4 x = {0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
    const float lse = o.part_lse[s * n + at];
    if (lse == -INFINITY) continue;  // a piece without keys
    const LseParts part = parts_of(lse, a.rel_weight);
    const float f = __builtin_amdgcn_exp2f(part.top - m0 + part.rest);
    sum += f;
    const f32x4 y = *(const f32x4*)(o.part + (s * n + at) * D + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], f, x[e]);
  }
  const float inv = sum == 0 ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  a.splits = 1;
  put<T, D>(a, o, 0, at, d, x);
  if (d == 0) put_lse(a, o, 0, at, lse_of(m, sum, a.rel_weight));
}

struct Plan {
  bool few;
  bool teams;  // two of them
  int group, slots, splits, piece;
};

// Few rows: a sequence's packed rows fit one wave.  Pieces of the keys, where row tiles are few against the chip: as many
// as make a round of workgroups (two rounds of k_attention where sequences differ in bf16), none shorter than 1,024 keys
// (128 where fp32 products, a sixteenth of the rate, make them long).  us, with the join: 32 tokens over caches of 256 to
// 8,192, 32/8 heads of 128, half a round / one / two / four 122 / 122 / 144 / 139; 4 x 100 queries over 12,345, 300, 8,000
// and 101 keys, one / two / three / four 103 / 84 / 83 / 86; 2 x 2,048 causal tokens, 16/8 heads of 128, one / two 62 /
// 88; five texts of 1 to 1,000 in fp32, 8/4 heads of 64, one / two / four 43 / 50 / 57.
// Two teams where k_attention's tiles leave a compute unit one workgroup, or causal ones of many lengths not much more, and
// the longest walk is what counts; a round is then a workgroup a unit.  us without / with (bf16): causal, 16/8 heads of 64
// and bias, 1,024 tokens 24 / 19, 2,176 45 / 34, 2,560 52 / 39, 3,500 71 / 67, 4,097 84 / 84; 8/8 heads of 64, 4,097 72 / 50,
// 6,000 104 / 71; 16/4 heads of 128, 2,048 44 / 40; both directions, 8/8 heads of 64, 4,096 64 / 55, 4,224 89 / 97; 24 x 256 13 / 18,
// 32 x 64 5.6 / 6.3; pieces of prompts over caches of 101 to 12,345, 32/8 heads of 128, 78 / 83; 8 heads of 64 in fp32, 2,048
// tokens, 63 / 93.
Plan plan_of(const lram_attention& call) {
  const lram_attention a = bounded(call);
  Plan p;
  const int64_t G = a.heads / a.kv_heads;
  p.few = a.max_q * G <= ROWS;
  const int tile = p.few ? ROWS : WAVES * ROWS;
  p.group = a.rel_weight && !p.few ? 1 : (int)G;
  p.slots = slots_of(a.tq, p.group, tile, a.batch);
  const int64_t heads = a.heads / p.group;
  const int64_t real = heads * tiles_of(a, a.max_q * p.group, a.tq * p.group, tile, p.slots);
  const bool even = p.few || a.dtype == LRAM_F32 || alike(a);
  p.teams = !p.few && a.dtype == LRAM_BF16 && even && a.max_k > 256 &&
            real <= (a.causal && a.max_k > 1024 ? 3 * UNITS / 2 : UNITS);
  int64_t splits = real > 0 ? (p.teams ? UNITS : even ? ROUND : 2 * ROUND) / real : 1;
  const int64_t shortest = a.dtype == LRAM_F32 && !p.few ? 128 : 1024;
  splits = std::min<int64_t>({splits, MAX_SPLITS, (a.max_k + shortest - 1) / shortest});
  if (splits < 1 || !few_enough(heads * p.slots)) splits = 1;
  p.piece = (int)std::min<int64_t>(((a.max_k + splits - 1) / splits + 127) / 128 * 128, INT32_MAX / 2);
  if (p.piece < 128) p.piece = 128;
  p.splits = (int)std::min<int64_t>(splits, std::max<int64_t>(1, (a.max_k + p.piece - 1) / p.piece));
  return p;
}

size_t workspace_of(const lram_attention& a, const Plan& p) {
  return p.splits > 1 ? (size_t)p.splits * a.tq * a.heads * (a.head_dim + 1) * 4 : 0;
}

template <typename T, int D, bool BIAS>
int go(Args x, const Out& o, const Plan& p, hipStream_t s) {
  const unsigned grid = (unsigned)(x.heads / x.group) * x.slots * x.splits;
  const size_t table = BIAS ? (size_t)x.group * (2 * (x.reach + BIAS_PAD) + 1) * 4 : 0;
  const auto launch = [&](auto kernel, size_t bytes, int threads) {
    if (int rc = allow_lds((const void*)kernel, bytes)) return rc;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), bytes, s, x, o);
    return layer_launched();
  };
  const auto prompt = [&](auto teams) {
    constexpr int TEAMS = decltype(teams)::value;
    return launch(k_attention<T, D, BIAS, TEAMS>, prompt_bytes<T, D, TEAMS>() + table, TEAMS * THREADS);
  };
  int rc = LRAM_OK;
  if constexpr (sizeof(T) == 2)
    if (p.teams) rc = prompt(std::integral_constant<int, 2>());
  if (p.few)
    rc = launch(k_attention_few<T, D, BIAS>,
                std::max<size_t>(few_bytes<T, D>(), WAVES * ROWS * (D * 4 + 16 + 8)) + table, THREADS);
  else if (!p.teams)
    rc = prompt(std::integral_constant<int, 1>());
  if (rc || x.splits == 1) return rc;
  const int64_t threads = x.tq * x.heads * (D / 4);
  hipLaunchKernelGGL((k_attention_join<T, D>), dim3((unsigned)((threads + THREADS - 1) / THREADS)), dim3(THREADS), 0, s,
                     x, o);
  return layer_launched();
}

}  // namespace

extern "C" {

int lram_attention_forward_workspace_bytes(const lram_attention* a, size_t* bytes) {
  if (!a || !bytes) return LRAM_EINVAL;
  if (int rc = check_attention(*a, false)) return rc;
  *bytes = a->tq ? workspace_of(*a, plan_of(*a)) : 0;
  return LRAM_OK;
}

int lram_attention_forward(const lram_attention* a, void* out, float* lse, void* residue, void* workspace,
                           size_t ws_bytes, void* stream) {
  if (!a) return LRAM_EINVAL;
  if (int rc = check_attention(*a, true)) return rc;
  if (a->tq == 0) return LRAM_OK;
  if (!out || off_align(out, 16) || off_align(residue, 16) || off_align(lse, 4)) return LRAM_EINVAL;
  if (residue && a->dtype != LRAM_BF16) return LRAM_EDTYPE;
  const Plan p = plan_of(*a);
  const size_t need = workspace_of(*a, p);
  if (need && (!workspace || off_align(workspace, 16) || ws_bytes < need)) return LRAM_EWORKSPACE;
  Args x = args_of(*a);
  x.group = p.group;
  x.slots = p.slots;
  x.splits = p.splits;
  x.piece = p.piece;
  Out o{out, residue, lse, (float*)workspace, nullptr};
  o.part_lse = o.part ? o.part + (size_t)p.splits * a->tq * a->heads * a->head_dim : nullptr;
  return by_kind(*a, [&](auto t, auto d, auto bias) {
    return go<decltype(t), decltype(d)::value, decltype(bias)::value>(x, o, p, (hipStream_t)stream);
  });
}

}  // extern "C"
