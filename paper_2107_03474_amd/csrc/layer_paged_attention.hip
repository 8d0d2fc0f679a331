// layer_paged_attention.hip -- part of liblram: attention of new tokens over the cache in pages, for gfx950.
//
// In units of log 2, z_ij = c q_i . k_j + t_h(p_j - p_i), c = scale log2 e; p_ij = 2^(z_ij - m_i) / l_i; out_i = sum_j p_ij v_j;
// weight_j += sum p_ij.  The G = heads / kv_heads query heads of a key head and the sequence's tokens are columns of one
// matrix (column n: token n / G, head n % G of the group), 16 to a product of the matrix cores.
//
// A single token meets every key once: bound by HBM.  A wave takes blocks of 16 F keys straight from HBM into the operands'
// registers (the pages hold them in that order), forms S^T = K Q^T, moves the maximum only when it grows by more than 2^8,
// and has in its results the second operand of O^T += V^T P^T.  No value crosses lanes but the maximum, and LDS is met once,
// when the four waves of a workgroup join what they have.  Long caches are cut into pieces, joined by a second kernel, which
// also adds up the weights that keys gather.  Measured: 32 tokens over caches of 256 to 8,192, 32/8 heads of 128 bf16, 531 MB
// in 88 us, 6.0 TB/s where a plain read reaches 6.9; one token over 131,072 keys 84 us, 6.4 TB/s, and 100 where scores are kept
// for the weights.
//
// Prompts and pieces of them take tiles of 32 columns, so that a load serves two products, and leave out keys that no query of
// the tile may meet.  4,096 causal tokens, 32/8 heads of 128 bf16: 207 to 232 us, 590 to 660 TFLOP/s of what is met, bound by the
// softmax's vector instructions (0.61 of a unit's issue) and by waits for keys; 4 x 100 tokens over 101 to 12,345 keys 126 us and
// a join of 17.  A form with 128 columns a workgroup, whose waves shared keys through LDS, was timed without leaving keys out:
// there it took 272 us for the prompt, this one 398, and for the pieces 174, this one 146.  With it, it was not built.

#include "layer_paged.h"

namespace {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

constexpr int ATTEND_WAVES = 4, ATTEND_THREADS = ATTEND_WAVES * WAVE;
constexpr int BIAS_MOST = 4096;  // group (2 reach + 193): a group's table by distance 0 ... reach is half of it
constexpr float GROW = 8;

template <typename T>
struct Operand;  // 16 bytes of elements
template <>
struct Operand<bf16> {
  using type = bf16x8;
};
template <>
struct Operand<float> {
  using type = f32x4;
};

struct Attend {
  Pool p;
  const void* q;
  void* out;
  int64_t q_row, q_head;
  float c;
  const void* rel_weight;
  const int32_t* rel_bucket;
  int buckets, reach, rel_bf16;
  int tiles, pieces, piece;  // workgroups along a sequence's columns, along its keys, and keys of one of these
  float* part;               // [piece][row][head][dim]
  float2* stat;              // [piece][row][head]: maximum and sum
  float* scores;             // [sequence][kv_head][score_cols][scored]: of few columns, kept for the weights; null: none are
  int score_cols;
  int64_t scored;
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// The maximum and the sum over the four lanes l, l + 16, l + 32, l + 48, the same in all of them.
__device__ __forceinline__ float of_groups(float x, bool sum) {
  const int a = __builtin_bit_cast(int, x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const float u = __builtin_bit_cast(float, (unsigned)r[0]), v = __builtin_bit_cast(float, (unsigned)r[1]);
  const float y = sum ? u + v : fmaxf(u, v);
  const int b = __builtin_bit_cast(int, y);
  const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  const float w = __builtin_bit_cast(float, (unsigned)s[0]), z = __builtin_bit_cast(float, (unsigned)s[1]);
  return sum ? w + z : fmaxf(w, z);
}

// Keys that queries up to the token-th may meet: of a sequence that has lost none (used = seen) those up to its own, since slot t
// then has position t.
__device__ __forceinline__ int64_t keys_met(const CacheSeq& s, int64_t token) {
  return s.whole ? min((int64_t)s.nk, max((int64_t)s.at + min(token, (int64_t)s.nq - 1) + 1, (int64_t)0)) : (int64_t)s.nk;
}

// The columns of a tile that a lane holds: its query's operand, position and place.
template <typename T, int D>
struct Column {
  static constexpr int CH = D / (4 * PageTile<T>::E);
  typename Operand<T>::type q[CH];
  int position, head;  // head: of the group
  int64_t row;         // -1: none

  __device__ __forceinline__ void load(const Attend& a, const CacheSeq& s, int kv_head, int64_t n) {  // n < 2^31
    const uint32_t i = (uint32_t)n / (uint32_t)a.p.group;
    load(a, s, kv_head, (int)i, (int)((uint32_t)n - i * (uint32_t)a.p.group));
  }
  __device__ __forceinline__ void load(const Attend& a, const CacheSeq& s, int kv_head, int i, int of_group) {
    const int lane = threadIdx.x % WAVE;
    head = of_group;
    row = i < s.nq ? s.q0 + i : -1;
    position = i < s.nq ? s.at + i : INT32_MIN;
    const T* const x = (const T*)a.q + (row < 0 ? 0 : row * a.q_row + (kv_head * a.p.group + head) * a.q_head);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      q[c] = {};
      if (row >= 0) q[c] = *(const typename Operand<T>::type*)(x + (4 * c + lane / 16) * PageTile<T>::E);
    }
  }
};

// Whether a sequence's scores are kept for its keys' weights: the host expects few columns, and the sequence has no more.
__device__ __forceinline__ bool keeps_scores(const Attend& a, const CacheSeq& s) {
  return a.scores && s.nk <= a.scored && (int64_t)s.nq * a.p.group <= a.score_cols;
}

// Pieces that hold a part of a sequence's results; 1: the results themselves are there.
__device__ __forceinline__ int pieces_of(const Attend& a, const CacheSeq& s) {
  return (int)max(min(((int64_t)s.nk + a.piece - 1) / a.piece, (int64_t)a.pieces), (int64_t)1);
}

// The bias of a group's heads by distance, in LDS.
__device__ __forceinline__ void load_bias(const Attend& a, int kv_head, float* bias) {
  const int n = a.reach + 1;
  for (int i = threadIdx.x; i < a.p.group * n; i += blockDim.x) {
    const int h = i / n, far = i - h * n, bucket = a.rel_bucket[a.reach - far];
    const int64_t at = (int64_t)(kv_head * a.p.group + h) * a.buckets + min(max(bucket, 0), a.buckets - 1);
    bias[i] = in_log2(a.rel_bf16 ? (float)((const bf16*)a.rel_weight)[at] : ((const float*)a.rel_weight)[at]);
  }
}

// Scores of a block of 16 F keys of which `left` are used: z[h][r] of key 16 h + 4 (lane / 16) + r, -inf where it is not met.
template <typename T, int D, bool BIAS>
__device__ __forceinline__ void scores(const Attend& a, const Column<T, D>& col,
                                       const typename Operand<T>::type (&k)[PageTile<T>::F][Column<T, D>::CH],
                                       const int4 (&at)[PageTile<T>::F], int left, const float* bias,
                                       f32x4 (&z)[PageTile<T>::F]) {
  const int g = threadIdx.x % WAVE / 16;
#pragma unroll
  for (int h = 0; h < PageTile<T>::F; ++h) {
    f32x4 s = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < Column<T, D>::CH; ++c) s = mma(k[h][c], col.q[c], s);
    const int p[4] = {at[h].x, at[h].y, at[h].z, at[h].w};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool met = p[r] <= col.position && h * 16 + 4 * g + r < left;
      float x = s[r] * a.c;
      if constexpr (BIAS) {
        const uint32_t far = (uint32_t)col.position - (uint32_t)p[r];
        x += bias[col.head * (a.reach + 1) + (int)min(met ? far : 0, (uint32_t)a.reach)];
      }
      z[h][r] = met ? x : -INFINITY;
    }
  }
}

// Keys that no other workgroup meets pass the caches by (ONCE): 32 tokens over caches of 256 to 8,192, 32/8 heads of 128, bf16:
// 113 -> 100 us.
template <bool ONCE, typename V>
__device__ __forceinline__ V fetch(const V* x) {
  if constexpr (ONCE)
    return __builtin_nontemporal_load(x);
  else
    return *x;
}

template <typename T, int D, bool ONCE>
__device__ __forceinline__ void load_keys(const Pool& p, int64_t keys,
                                          typename Operand<T>::type (&k)[PageTile<T>::F][Column<T, D>::CH],
                                          int4 (&at)[PageTile<T>::F]) {
  using Ti = PageTile<T>;
  const int lane = threadIdx.x % WAVE;
  const T* const x = (const T*)p.k + keys * D + lane * Ti::E;
#pragma unroll
  for (int h = 0; h < Ti::F; ++h) {
#pragma unroll
    for (int c = 0; c < Column<T, D>::CH; ++c)
      k[h][c] = fetch<ONCE>((const typename Operand<T>::type*)(x + h * 16 * D + c * WAVE * Ti::E));
    at[h] = *(const int4*)(p.position + keys + h * 16 + lane / 16 * 4);
  }
}

// A softmax weight as operands of the product with the values.  fp32: itself.  bf16, 16 columns (FINE): its first 8 bits, and the
// rest rounded to 8 more in a second product, so that 2^-15 of a weight is lost and not 2^-8; HBM hides it (us of 32 tokens over
// caches of 256 to 8,192, 32/8 heads of 128, one product / two: 93.8 / 93.8; of one over 777 keys, 8 heads of 64 with bias, 9.2 /
// 9.7).  A weight that is not 0 leaves a rest that is not 0 (2^-23 of it is added), so that an infinite value stays that
// infinity.  Tiles of 32 columns are bound by their products, and take weights rounded to bf16 as attention over packed
// rows does (4,096 tokens, 32/8 heads of 128: 207 / 245).
template <bool FINE>
__device__ __forceinline__ void split(float e, bf16& first, bf16& rest) {
  if constexpr (FINE) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, e);
    first = __builtin_bit_cast(bf16, (uint16_t)(bits >> 16));
    rest = (bf16)fmaf(e, 1.0f + 0x1p-23f, -__builtin_bit_cast(float, bits & 0xffff0000u));
  } else {
    first = (bf16)e;
  }
}
template <bool FINE>
__device__ __forceinline__ void split(float e, float& first, float&) {
  first = e;
}

// A block's scores of column t and its values into the results: the maximum moves only when it grows by more than 2^GROW.
template <typename T, int D, int CT>
__device__ __forceinline__ void absorb(int t, const f32x4 (&z)[PageTile<T>::F], const typename Operand<T>::type (&v)[D / 16],
                                       f32x4 (&o)[D / 16][CT], float (&m)[CT], float (&l)[CT]) {
  constexpr int F = PageTile<T>::F, DB = D / 16;
  constexpr bool FINE = sizeof(T) == 2 && CT == 1;
  float top = z[0][0];
#pragma unroll
  for (int h = 0; h < F; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) top = fmaxf(top, z[h][r]);
  top = of_groups(top, false);
  if (__builtin_amdgcn_ballot_w64(top > m[t] + GROW)) {
    const float now = fmaxf(m[t], top), f = now == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[t] - now);
    m[t] = now;
    l[t] *= f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d][t] *= f;
  }
  const float used = m[t] == -INFINITY ? 0.0f : m[t];
  typename Operand<T>::type w, rest;
#pragma unroll
  for (int h = 0; h < F; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = __builtin_amdgcn_exp2f(z[h][r] - used);
      l[t] += e;
      T first, second;
      split<FINE>(e, first, second);
      w[h * 4 + r] = first;
      if constexpr (FINE) rest[h * 4 + r] = second;
    }
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d][t] = mma(v[d], w, o[d][t]);
  if constexpr (FINE)
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d][t] = mma(v[d], rest, o[d][t]);
}

// Rows of no sequence get zeros, shared out over the workgroups of a head.
template <typename T, int D>
__device__ __forceinline__ void clear_rows(const Attend& a, int head) {
  const Pool& p = a.p;
  const int64_t before = clamp_row(p.start[0], p.rows), behind = max(clamp_row(p.start[p.batch], p.rows), before);
  const int all = gridDim.x / p.kv_heads;
  for (int64_t i = blockIdx.x / p.kv_heads; i < before + (p.rows - behind); i += all) {
    T* const row = (T*)a.out + ((i < before ? i : behind + (i - before)) * p.heads + head * p.group) * D;
#pragma clang loop unroll(disable) vectorize(disable)
    for (int d = threadIdx.x; d < p.group * D; d += ATTEND_THREADS) row[d] = (T)0.0f;
  }
}

// Four waves take blocks of keys in turn.  Two workgroups a compute unit (three: 112 us for 98, the reads disturb each other), so
// that 256 registers hold everything and the matrix cores take them as they are: with more, the compiler keeps the results in
// the other half of the register file and moves them to and fro (4 x 100 tokens over 101 to 12,345 keys 262 -> 154 us).
template <typename T, int D, int CT, bool BIAS>
__global__ __launch_bounds__(ATTEND_THREADS, 2) void k_paged_attention(Attend a) {
  using Ti = PageTile<T>;
  using Op = typename Operand<T>::type;
  constexpr int E = Ti::E, F = Ti::F, KEYS = Ti::KEYS, DB = D / 16, COLS = 16 * CT, STEP = ATTEND_WAVES * KEYS;
  __shared__ __align__(16) float joined[ATTEND_WAVES][16][D + 4];
  __shared__ float2 stats[ATTEND_WAVES][COLS];
  __shared__ float bias[BIAS ? BIAS_MOST / 2 : 1];
  const Pool& p = a.p;
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), g = lane / 16;
  int64_t id = blockIdx.x;
  const int head = (int)(id % p.kv_heads);
  id /= p.kv_heads;
  const int b = (int)(id % p.batch);
  id /= p.batch;
  const int tile0 = a.tiles - 1 - (int)(id % a.tiles), piece = (int)(id / a.tiles);  // a prompt's longest tiles first
  const CacheSeq s = cache_seq(p, b);
  clear_rows<T, D>(a, head);
  if (piece && (int64_t)piece * a.piece >= s.nk) return;
  const bool keeps = keeps_scores(a, s);
  const bool alone = pieces_of(a, s) == 1;
  if constexpr (BIAS) {
    load_bias(a, head, bias);
    __syncthreads();
  }
  for (int64_t tile = tile0; tile * COLS < (int64_t)s.nq * p.group; tile += a.tiles) {
    Column<T, D> col[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) col[t].load(a, s, head, tile * COLS + t * 16 + lane % 16);
    f32x4 o[DB][CT] = {};
    float m[CT], l[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) m[t] = -INFINITY, l[t] = 0;
    const int64_t met = keys_met(s, (tile * COLS + COLS - 1) / p.group);
    for (int64_t base = (int64_t)piece * a.piece; base < met; base += (int64_t)a.pieces * a.piece) {
      const int end = (int)min(base + a.piece, met);
      // A block's values are on their way while its scores are formed, and the next one's keys (of a page looked up a block
      // before) while it is finished.  Loads are made whatever the table says, of page 0 where it names none: where some were
      // left out, the wait for keys would be one for everything.
      const auto look = [&](int at) { return page_of_wave(p, b, min(at, end - 1)); };
      const auto keys_of = [&](int page, int at) { return page_rows(p, max(page, 0), head) + (at & (p.page - 1)); };
      int slot = (int)base + wave * KEYS;
      if (slot >= end) continue;
      int page = look(slot), next = look(slot + STEP);
      Op k[F][Column<T, D>::CH], v[DB];
      int4 at[F];
      load_keys<T, D, CT == 1>(p, keys_of(page, slot), k, at);
      const auto block = [&](auto more) {
        const int left = page < 0 ? 0 : s.nk - slot;  // 0: no key is met
        const T* const x = (const T*)p.v + keys_of(page, slot) * D + lane * E;
#pragma unroll
        for (int d = 0; d < DB; ++d) v[d] = fetch<CT == 1>((const Op*)(x + d * WAVE * E));
        __builtin_amdgcn_sched_barrier(0);  // first the values, then the next keys: they are waited for in this order
        f32x4 z[CT][F];
#pragma unroll
        for (int t = 0; t < CT; ++t) scores<T, D, BIAS>(a, col[t], k, at, left, bias, z[t]);
        if constexpr (more.value) {
          __builtin_amdgcn_sched_barrier(0);
          load_keys<T, D, CT == 1>(p, keys_of(next, slot + STEP), k, at);
          __builtin_amdgcn_sched_barrier(0);
          page = next;
          next = look(slot + 2 * STEP);
        }
        if (left == 0) return;
        if (left < KEYS) {  // what lies past the last key is never met, NaN or not
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (e / 4 * 16 + 4 * g + e % 4 >= left) v[d][e] = 0;
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          if (CT == 1 && keeps && lane % 16 < s.nq * p.group) {
            float* const to = a.scores + ((int64_t)(b * p.kv_heads + head) * a.score_cols + lane % 16) * a.scored + slot + 4 * g;
#pragma unroll
            for (int h = 0; h < F; ++h) *(f32x4*)(to + 16 * h) = z[t][h];
          }
          absorb<T, D, CT>(t, z[t], v, o, m, l);
        }
      };
      for (; slot + STEP < end; slot += STEP) block(std::true_type());
      block(std::false_type());
    }
    // the waves' parts, in their order
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      l[t] = of_groups(l[t], true);
      if (g == 0) stats[wave][t * 16 + lane] = {m[t], l[t]};
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) top = fmaxf(top, stats[w][t * 16 + lane % 16].x);
        const float f = m[t] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[t] - top);
#pragma unroll
        for (int d = 0; d < DB; ++d) *(f32x4*)&joined[wave][lane % 16][d * 16 + 4 * g] = o[d][t] * f;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * (D / 4); i += ATTEND_THREADS) {
        const int n = i / (D / 4), d = i % (D / 4) * 4;
        const int64_t at = tile * COLS + t * 16 + n, token = at / p.group;
        if (token >= s.nq) continue;
        const int64_t place = (s.q0 + token) * p.heads + head * p.group + (at - token * p.group);
        float top = -INFINITY, sum = 0;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) top = fmaxf(top, stats[w][t * 16 + n].x);
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) {
          const float2 st = stats[w][t * 16 + n];
          sum += st.x == -INFINITY ? st.y : st.y * __builtin_amdgcn_exp2f(st.x - top);  // NaN stays
          x += *(const f32x4*)&joined[w][n][d];
        }
        if (alone) {
          const float inv = sum == 0 ? 0.0f : 1.0f / sum;
          const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
          store_n<T, 4>((T*)a.out + place * D + d, y);
          if (a.stat && d == 0) a.stat[place] = {top, sum};
        } else {
          const int64_t to = (int64_t)piece * p.rows * p.heads + place;
          *(f32x4*)(a.part + to * D + d) = x;
          if (d == 0) a.stat[to] = {top, sum};
        }
      }
      __syncthreads();
    }
  }
}

// The pieces' parts of a query and head joined.
template <typename T, int D>
__device__ __forceinline__ void join_rows(const Attend& a, int64_t id, int rows_each) {
  constexpr int LANES = D / 4, TEAMS = ATTEND_THREADS / LANES;
  __shared__ float tops[ATTEND_WAVES];
  __shared__ __align__(16) float parts[TEAMS][D];
  __shared__ float sums[TEAMS];
  const Pool& p = a.p;
  const int h = (int)(id % p.heads), b = (int)(id / p.heads % p.batch), first = (int)(id / p.heads / p.batch);
  const CacheSeq s = cache_seq(p, b);
  const int pieces = pieces_of(a, s);
  if (pieces == 1) return;
  const int team = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
  const int64_t step = p.rows * p.heads;
  for (int i = first; i < s.nq; i += rows_each) {
    const int64_t place = (s.q0 + i) * p.heads + h;
    const auto stat = [&](int n) { return a.stat[n * step + place]; };
    const auto part = [&](int n) { return *(const f32x4*)(a.part + (n * step + place) * D + d); };
    float top = stat(min((int)threadIdx.x, pieces - 1)).x;
    const int own = min(team, pieces - 1);
    const float2 st0 = stat(own);  // on their way while the maximum is found
    const f32x4 y0 = part(own);
    for (int n = threadIdx.x + ATTEND_THREADS; n < pieces; n += ATTEND_THREADS) top = fmaxf(top, stat(n).x);
#pragma unroll
    for (int o = WAVE / 2; o; o /= 2) top = fmaxf(top, __shfl_xor(top, o));
    if (threadIdx.x % WAVE == 0) tops[threadIdx.x / WAVE] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    float sum = 0;
    f32x4 x = {0, 0, 0, 0};
    const auto add = [&](float2 st, f32x4 y) {
      const float f = st.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st.x - top);
      sum += st.x == -INFINITY ? st.y : st.y * f;
      x += y * f;
    };
    if (team < pieces) add(st0, y0);
#pragma unroll 4
    for (int n = team + TEAMS; n < pieces; n += TEAMS) add(stat(n), part(n));
    *(f32x4*)&parts[team][d] = x;
    if (d == 0) sums[team] = sum;
    __syncthreads();
    if (team == 0) {
      for (int n = 1; n < TEAMS; ++n) {
        x += *(const f32x4*)&parts[n][d];
        sum += sums[n];
      }
      const float inv = sum == 0 ? 0.0f : 1.0f / sum;
      const float y[4] = {x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
      store_n<T, 4>((T*)a.out + place * D + d, y);
    }
    __syncthreads();
  }
}

template <typename T, int D>
__global__ __launch_bounds__(ATTEND_THREADS) void k_paged_join(Attend a, int rows_each) {
  join_rows<T, D>(a, blockIdx.x, rows_each);
}

// The maximum and 1 / sum of a row and head, by the `step` neighbouring lanes that share it (a power of 2; first: this one's).
__device__ __forceinline__ float2 whole_of(const Attend& a, int64_t place, int pieces, int first, int step) {
  const int64_t all = a.p.rows * a.p.heads;
  float top = -INFINITY, sum = 0;
  for (int n = first; n < pieces; n += step) top = fmaxf(top, a.stat[n * all + place].x);
  for (int o = 1; o < step; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  for (int n = first; n < pieces; n += step) {
    const float2 st = a.stat[n * all + place];
    sum += st.x == -INFINITY ? st.y : st.y * __builtin_amdgcn_exp2f(st.x - top);
  }
  for (int o = 1; o < step; o *= 2) sum += __shfl_xor(sum, o);
  return {top, sum == 0 ? 0.0f : 1.0f / sum};
}

// The weight that each key gathers, in a fixed order, beside the join.  Of a single token's few columns the scores were kept (16
// bytes a key for four heads that share it, beside the 256 of its k); a thread then takes four keys of each stretch.  Otherwise a workgroup
// keeps a block of keys and forms their scores again, its waves sharing out the sequence's queries.
constexpr int WEIGH_CHUNK = 4 * ATTEND_THREADS;  // keys of a workgroup
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(ATTEND_THREADS, sizeof(T) * D == 512 ? 3 : 4) void k_paged_weigh(Attend a, int joins, int rows_each, int chunks, int chunk) {
  using Ti = PageTile<T>;
  using Op = typename Operand<T>::type;
  constexpr int F = Ti::F, KEYS = Ti::KEYS;
  __shared__ float bias[BIAS ? BIAS_MOST / 2 : 1];
  __shared__ float2 whole[16];
  if (blockIdx.x < (unsigned)joins) {
    join_rows<T, D>(a, blockIdx.x, rows_each);
    return;
  }
  const Pool& p = a.p;
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const unsigned id = blockIdx.x - joins;
  const int head = (int)(id % p.kv_heads), b = (int)(id / p.kv_heads % p.batch);
  const int64_t first = id / p.kv_heads / p.batch;
  const CacheSeq s = cache_seq(p, b);
  if (s.nq == 0 || first * chunk >= s.nk) return;
  const int pieces = pieces_of(a, s);
  if (keeps_scores(a, s)) {
    const int cols = s.nq * p.group, mine = threadIdx.x / 16;
    const int64_t met = keys_met(s, s.nq - 1);  // scores were kept of these
    f32x4 x[16], had, *w = nullptr;
    const auto load = [&](int64_t slot) {
      w = nullptr;
      const int page = slot < met ? page_of(p, b, (int)slot) : -1;
      if (page < 0) return;
      w = (f32x4*)(p.weight + page_rows(p, page, head) + (slot & (p.page - 1)));
      had = *w;
      const float* const z = a.scores + (int64_t)(b * p.kv_heads + head) * a.score_cols * a.scored + slot;
#pragma unroll
      for (int c = 0; c < 16; ++c)
        if (c < cols) x[c] = *(const f32x4*)(z + c * a.scored);
    };
    int64_t slot = first * chunk + 4 * threadIdx.x;
    load(slot);  // on its way while the sums are formed
    if (mine < cols) {
      const int64_t place = (s.q0 + mine / p.group) * p.heads + head * p.group + mine % p.group;
      const float2 st = whole_of(a, place, pieces, threadIdx.x % 16, 16);
      if (threadIdx.x % 16 == 0) whole[mine] = st;
    }
    __syncthreads();
    while (slot < met) {
      if (w) {
        f32x4 got = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 16; ++c)
          if (c < cols)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              got[r] += x[c][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x[c][r] - whole[c].x) * whole[c].y;
        if (slot + 4 <= met) {
          *w = had + got;
        } else {
          for (int r = 0; slot + r < met; ++r) ((float*)w)[r] = had[r] + got[r];
        }
      }
      slot += (int64_t)chunks * chunk;
      load(slot);
    }
    return;
  }
  if constexpr (BIAS) {
    load_bias(a, head, bias);
    __syncthreads();
  }
  constexpr uint32_t STEP = ATTEND_WAVES * 16;
  __shared__ float sums[ATTEND_WAVES][KEYS];
  const uint32_t group = p.group, all = (uint32_t)s.nq * group;  // columns
  for (int64_t base = first * chunk; base < s.nk; base += (int64_t)chunks * chunk) {
    const int end = (int)min(base + chunk, (int64_t)s.nk);
    for (int slot = (int)base; slot < end; slot += KEYS) {
      const int page = page_of_wave(p, b, slot);
      if (page < 0) continue;  // all waves alike
      const int64_t keys = page_rows(p, page, head) + (slot & (p.page - 1));
      const int left = s.nk - slot;
      Op k[F][Column<T, D>::CH];
      int4 at[F];
      load_keys<T, D, false>(p, keys, k, at);
      // queries before the lowest position meet none of these keys
      int lowest = INT32_MAX;
#pragma unroll
      for (int h = 0; h < F; ++h) {
        const int x[4] = {at[h].x, at[h].y, at[h].z, at[h].w}, key = h * 16 + lane / 16 * 4;
#pragma unroll
        for (int r = 0; r < 4; ++r) lowest = key + r < left ? min(lowest, x[r]) : lowest;
      }
      lowest = min(lowest, __shfl_xor(lowest, 16));
      lowest = min(lowest, __shfl_xor(lowest, 32));
      const int64_t skipped = min(max((int64_t)__builtin_amdgcn_readfirstlane(lowest) - s.at, (int64_t)0), (int64_t)s.nq);
      // this lane's columns: one of each 16, every fourth 16 of them the wave's; the next one's query is on its way
      const uint32_t tile0 = ((uint32_t)skipped * group & ~15u) + wave * 16;
      uint32_t i = (tile0 + lane % 16) / group, h0 = tile0 + lane % 16 - i * group;
      const uint32_t step_i = STEP / group, step_h = STEP - step_i * group;
      const T* query = (const T*)a.q + (s.q0 + i) * a.q_row + (int64_t)(head * group + h0) * a.q_head + lane / 16 * Ti::E;
      const float2* stat = a.stat + (s.q0 + i) * p.heads + head * group + h0;
      const int64_t query_step = step_i * a.q_row + step_h * a.q_head, query_wrap = a.q_row - (int64_t)group * a.q_head;
      f32x4 got[F] = {};
      Column<T, D> col;
      float2 st;
      const auto get = [&] {
        const bool has = i < (uint32_t)s.nq;
        col.head = (int)h0;
        col.position = has ? s.at + (int)i : INT32_MIN;
        st = {0, 0};
#pragma unroll
        for (int c = 0; c < Column<T, D>::CH; ++c) col.q[c] = {};
        if (has) {
#pragma unroll
          for (int c = 0; c < Column<T, D>::CH; ++c) col.q[c] = *(const Op*)(query + c * 4 * Ti::E);
          st = pieces == 1 ? *stat : whole_of(a, stat - a.stat, pieces, 0, 1);
        }
      };
      get();
      for (uint32_t tile = tile0; tile < all; tile += STEP) {
        const Column<T, D> mine = col;
        const float2 mine_st = {st.x, pieces > 1 ? st.y : st.y == 0 ? 0.0f : __builtin_amdgcn_rcpf(st.y)};
        const bool wraps = h0 + step_h >= group;
        i += step_i + wraps;
        h0 += step_h - (wraps ? group : 0);
        query += query_step + (wraps ? query_wrap : 0);
        stat += (int64_t)step_i * p.heads + step_h + (wraps ? p.heads - (int64_t)group : 0);
        if (tile + STEP < all) get();
        f32x4 z[F];
        scores<T, D, BIAS>(a, mine, k, at, left, bias, z);
#pragma unroll
        for (int h = 0; h < F; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            got[h][r] += z[h][r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(z[h][r] - mine_st.x) * mine_st.y;
      }
#pragma unroll
      for (int h = 0; h < F; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int o = 1; o < 16; o *= 2) got[h][r] += __shfl_xor(got[h][r], o);
          if (lane % 16 == 0) sums[wave][h * 16 + lane / 16 * 4 + r] = got[h][r];
        }
      __syncthreads();
      if ((int)threadIdx.x < min(KEYS, left)) {
        float sum = 0;
#pragma unroll
        for (int w = 0; w < ATTEND_WAVES; ++w) sum += sums[w][threadIdx.x];
        p.weight[keys + threadIdx.x] += sum;
      }
      __syncthreads();
    }
  }
}

template <typename T>
__global__ __launch_bounds__(ATTEND_THREADS) void k_paged_clear(T* out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * ATTEND_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * ATTEND_THREADS)
    out[i] = (T)0.0f;
}

struct Plan {
  int cols;  // of a tile: 16 or 32
  int64_t tiles, pieces, piece;
  int64_t score_cols, scored;        // of kept scores; 0: none
  size_t part, scores, stat;  // bytes
  size_t all() const { return part + scores + stat; }
};

// Pieces: a round of two workgroups a unit for a single sequence, and up to four rounds for several, which are rarely of one
// length (us of one round / four: one token over 131,072 keys, 32/8 heads of 128 bf16 with weights, 123 / 130; 32 tokens over
// 256 to 8,192 keys 107 / 97).
// The least piece is 128 keys where workgroups are fewer than units even so, and few parts are joined (us of kernels, 256 / 128:
// one token over 4,000 keys, 32/8 heads of 128 fp32 with weights 15.5 / 13.0, over 1,500 in bf16 10.9 / 10.2; 50 over 1,000, 16/8
// heads of 64 fp32, 16.6 / 14.3; with more of them: four over 1,500, 32/8 heads of 128 bf16, 9.8 / 10.7; one over 20,000 of one
// head of 64 10.1 / 11.0, for its join), otherwise 256.
// Few keys take one piece, which needs no join (us of a call / of its kernels, one piece and pieces of 256: one token over 777
// keys, 8 heads of 64 bf16, 15.9 / 8.3 and 19.9 / 9.0; four over 300, 32/8 heads of 128, 13.9 / 7.4 and 17.8 / 9.7, with
// weights 17.9 / 12.1 and 18.0 / 11.0; over 777 of these 13.9 / 12.0 and 17.8 / 10.3).  Results are the same with weights
// and without.
constexpr int64_t PIECE_STEP = 128, PIECE_LEAST = 256, ROUND = 512, ROUNDS = 4, UNITS = 256, JOINED = 64;
// So do more keys where heads of sequences fill a round by themselves (us, four rounds / one piece, all sequences as long as
// said or of lengths from 16 on: 64 tokens over 1,024 keys, 32/8 heads of 128 bf16, 50.7 / 41.3 and 22.5 / 16.9, over 2,048
// 92.7 / 81.6 and 30.2 / 27.3; over 4,096 174 / 160 and 43.3 / 46.2, which stays in pieces).
constexpr int64_t FEW_BYTES = 256 << 10, ALONE_BYTES = 1 << 20;  // of a sequence's keys and values of a head
constexpr int64_t SCORE_BYTES = 256 << 20;
constexpr int64_t WEIGH_GROUPS = 8192;  // more go over several stretches each: where few keys are met of many expected, they only start
constexpr int64_t MOST_GROUPS = ((int64_t)1 << 32) / ATTEND_THREADS - 1;

int64_t over(int64_t a, int64_t b) { return (a + b - 1) / b; }

Plan plan_of(const lram_paged& p, bool weigh) {
  Plan x{};
  const int64_t G = p.heads / p.kv_heads, lists = std::max<int64_t>(1, (int64_t)p.batch * p.kv_heads);
  // a plan that understates the rows is found out by how many there are
  const int64_t tokens = std::max({std::min(p.max_q, p.rows), over(p.rows, std::max(p.batch, 1)), (int64_t)1});
  const int64_t keys = std::max<int64_t>(1, std::min(p.max_k, p.width * p.page));
  x.cols = tokens * G <= 16 ? 16 : 32;
  x.tiles = std::max<int64_t>(1, std::min(over(tokens * G, x.cols), MOST_GROUPS / lists));
  const int64_t wanted = std::min(over(ROUND * std::min<int64_t>(std::max(p.batch, 1), ROUNDS), lists * x.tiles), MOST_GROUPS / (lists * x.tiles));
  x.piece = over(over(keys, std::max<int64_t>(1, wanted)), PIECE_STEP) * PIECE_STEP;
  const int64_t most_pieces = over(keys, PIECE_STEP);
  x.piece = std::max(x.piece, most_pieces <= JOINED && lists * x.tiles * most_pieces <= UNITS ? PIECE_STEP : PIECE_LEAST);
  if (keys * p.head_dim * 2 * (int64_t)elem_size(p.dtype) <= (lists * x.tiles >= ROUND ? ALONE_BYTES : FEW_BYTES))
    x.piece = over(keys, PIECE_STEP) * PIECE_STEP;
  x.pieces = over(keys, x.piece);
  const size_t places = (size_t)p.rows * p.heads;
  if (x.pieces > 1) x.part = (size_t)x.pieces * places * p.head_dim * sizeof(float);
  if (x.pieces > 1 || weigh) x.stat = (size_t)x.pieces * places * sizeof(float2);
  if (weigh && tokens * G <= 16) {
    x.score_cols = tokens * G;
    // longer sequences' scores, of a plan that expects the whole of a large cache, are formed again
    const int64_t most = SCORE_BYTES / (lists * x.score_cols * (int64_t)sizeof(float)) / PIECE_STEP * PIECE_STEP;
    x.scored = std::min(x.pieces * x.piece, most);
    x.scores = (size_t)lists * x.score_cols * x.scored * sizeof(float);
  }
  return x;
}

int check_queries(const lram_paged& p, const lram_paged_queries& a) {
  if (int rc = check_pool(p, true)) return rc;
  const int64_t G = p.heads / p.kv_heads;
  if (!(a.scale > 0) || !(a.scale < INFINITY) || (a.weigh & ~1) || (a.weigh && p.pages && !p.weight)) return LRAM_EINVAL;
  if (bad_strides(a.q_row, a.q_head, p.heads, p.head_dim, p.dtype)) return LRAM_EINVAL;
  if ((int64_t)p.batch * p.heads > MOST_GROUPS / 2) return LRAM_EINVAL;
  if (a.rel_weight) {
    if (a.wdtype != LRAM_F32 && !(a.wdtype == LRAM_BF16 && p.dtype == LRAM_BF16)) return LRAM_EDTYPE;
    if (!a.rel_bucket || a.rel_buckets < 1 || a.rel_buckets > 256 || a.rel_reach < 0 || a.rel_reach > BIAS_MOST ||
        G * (2 * (int64_t)a.rel_reach + 193) > BIAS_MOST)
      return LRAM_EINVAL;
    if (off_align(a.rel_weight, elem_size(a.wdtype)) || off_align(a.rel_bucket, 4)) return LRAM_EINVAL;
  }
  return LRAM_OK;
}

}  // namespace

extern "C" {

int lram_paged_attention_workspace_bytes(const lram_paged* p, const lram_paged_queries* q, size_t* bytes) {
  if (!p || !q || !bytes) return LRAM_EINVAL;
  if (int rc = check_queries(*p, *q)) return rc;
  const Plan x = plan_of(*p, q->weigh);
  *bytes = x.all();
  return LRAM_OK;
}

int lram_paged_attention(const lram_paged* p, const lram_paged_queries* q, void* out, void* workspace, size_t ws_bytes,
                         void* stream) {
  if (!p || !q) return LRAM_EINVAL;
  if (int rc = check_queries(*p, *q)) return rc;
  if (p->rows == 0) return LRAM_OK;
  if (!q->q || !out || off_align(q->q, 16) || off_align(out, 16)) return LRAM_EINVAL;
  const Plan x = plan_of(*p, q->weigh);
  const size_t need = x.all();
  if (need && (!workspace || off_align(workspace, 16) || ws_bytes < need)) return LRAM_EWORKSPACE;
  Attend a{};
  a.p = pool_of(*p);
  a.q = q->q, a.out = out, a.q_row = q->q_row, a.q_head = q->q_head;
  a.c = q->scale * LOG2E;
  a.rel_weight = q->rel_weight, a.rel_bucket = q->rel_bucket, a.buckets = q->rel_buckets, a.reach = q->rel_reach;
  a.rel_bf16 = q->wdtype == LRAM_BF16;
  a.tiles = (int)x.tiles, a.pieces = (int)x.pieces, a.piece = (int)x.piece;
  char* const ws = (char*)workspace;
  if (x.part) a.part = (float*)ws;
  if (x.scores) a.scores = (float*)(ws + x.part), a.score_cols = (int)x.score_cols, a.scored = x.scored;
  if (x.stat) a.stat = (float2*)(ws + x.part + x.scores);
  if (p->batch == 0 || p->pages == 0) {
    const int64_t n = p->rows * p->heads * p->head_dim;
    const dim3 grid((unsigned)std::min<int64_t>(over(n, ATTEND_THREADS), 4096));
    if (p->dtype == LRAM_BF16)
      hipLaunchKernelGGL(k_paged_clear<bf16>, grid, dim3(ATTEND_THREADS), 0, (hipStream_t)stream, (bf16*)out, n);
    else
      hipLaunchKernelGGL(k_paged_clear<float>, grid, dim3(ATTEND_THREADS), 0, (hipStream_t)stream, (float*)out, n);
    return layer_launched();
  }
  return by_form(p->dtype, p->head_dim, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    const auto go = [&](auto kernel, int64_t groups, auto... more) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(ATTEND_THREADS), 0, (hipStream_t)stream, a, more...);
      return layer_launched();
    };
    const int64_t lists = (int64_t)p->batch * p->kv_heads, groups = lists * x.tiles * x.pieces;
    const auto of = [&](auto bias) {
      constexpr bool BIAS = decltype(bias)::value;
      return x.cols == 16 ? go(k_paged_attention<T, D, 1, BIAS>, groups) : go(k_paged_attention<T, D, 2, BIAS>, groups);
    };
    int rc = q->rel_weight ? of(std::true_type()) : of(std::false_type());
    if (rc != LRAM_OK || (!x.part && !q->weigh)) return rc;
    const int64_t all = (int64_t)p->batch * p->heads;
    const int64_t each = std::max<int64_t>(1, std::min({p->max_q, p->rows, MOST_GROUPS / 2 / all}));
    const int64_t joins = x.part ? all * each : 0;
    if (!q->weigh) return go(k_paged_join<T, D>, joins, (int)each);
    const int64_t keys = std::max<int64_t>(1, std::min(p->max_k, p->width * p->page));
    const int64_t chunk = x.scores ? WEIGH_CHUNK : PageTile<T>::KEYS;
    const int64_t chunks = std::max<int64_t>(1, std::min({over(keys, chunk), over(WEIGH_GROUPS, lists), (MOST_GROUPS - joins) / lists}));
    rc = q->rel_weight ? go(k_paged_weigh<T, D, true>, joins + lists * chunks, (int)joins, (int)each, (int)chunks, (int)chunk)
                       : go(k_paged_weigh<T, D, false>, joins + lists * chunks, (int)joins, (int)each, (int)chunks, (int)chunk);
    return rc;
  });
}

}  // extern "C"
