// layer_attention_backward.hip -- part of liblram: attention over packed sequences, backward (see layer_attention.h for
// the formulas and the tiles).
//
//     p_ij = 2^(z_ij - lse_i),  dv_j = sum_i p_ij do_i,  ds_ij = p_ij (do_i . v_j - delta_i),  delta_i = do_i . o_i
//     dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dW_h(d) = sum over j - i - off = d of ds_ij
//
// Two kernels, each forming p again, so that every sum has one owner and one order: k_attention_dq keeps 128 packed
// rows and walks over the keys (scores transposed, as in the forward pass), k_attention_dkv keeps 128 keys and walks over
// the packed rows, the G heads of its group among them.  Seven products instead of the five of a single kernel, whose dq
// would be added up in memory by atomics, in an order that varies.  p and ds are rounded to the operands' type, the matrix
// cores' own, half a unit of which is what q, k, v and the results carry anyway; sums and delta stay in fp32.
//
// The bias's gradient: k_attention_dq adds up the diagonals of its 32 x 32 blocks of ds.  Rows are lanes and keys registers, so
// a sum that moves on by one lane with every key collects a diagonal in a lane (diagonals); a block's sums then go to the
// wave's own table in LDS (one instruction, no two lanes in an entry: the order is fixed).  Blocks past reach go into a
// register.  A workgroup leaves its sums by bucket, and relative_grad adds up the workgroups'.

#include "layer_attention.h"

namespace {

// The value of the lane before, going round the wave.
__device__ __forceinline__ float next_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x13c, 0xf, 0xf, true));
}

struct Grads {
  const void *out, *residue, *grad_out;
  const float* lse;
  void *gq, *gk, *gv, *grel;
  // workspace: row_lse, delta and (with a bias) share [tq heads], [slots][heads][buckets], [pieces][tk][kv_heads][2][D] or
  // [splits][tq][heads][D] (dq first)
  float *row_lse, *delta, *share, *rel, *part;
  int rel_rows;
};

// A block of 32 keys x 32 rows (a row to a lane) summed along its diagonals: lane p < 63 of the result holds the sum over
// lane c's key k with c + 31 - k = p.
__device__ __forceinline__ float diagonals(const f32x16& s) {
  float sum = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float part[8];  // keys 8 u ..., one each: its rows in the lower half's lanes, zeros beside them
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, (float)s[4 * u + e]), 0, false, false);
      const unsigned lower = r[0], upper = r[1];
      part[e] = __builtin_bit_cast(float, lower);
      part[4 + e] = __builtin_bit_cast(float, upper);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = u + k ? next_lane(sum) + part[k] : part[k];
  }
  return sum;
}

// TEAMS: as in k_attention.
template <typename T, int D, bool BIAS, int TEAMS>
__global__ __launch_bounds__(TEAMS* THREADS, (waves_per_simd<T, D>())) void k_attention_dq(Args a, Grads o) {
  using Ti = Tile<T, D>;
  using F = typename Frag<T>::type;
  constexpr int M = WAVES * ROWS, ALL = TEAMS * THREADS, TABLES = TEAMS * WAVES;
  extern __shared__ __attribute__((aligned(256))) char smem[];
  constexpr int IDS = 2;  // of a thread, asked for while the work is looked up
  int ids[IDS];
  if constexpr (BIAS)
#pragma unroll
    for (int t = 0; t < IDS; ++t) ids[t] = bucket_of(a, (int)(t * ALL + threadIdx.x) - a.reach - BIAS_PAD);
  Work w;
  const bool found = find_work<M>(a, &w);
  float* const rel_row = o.rel + (((int64_t)w.slot * a.splits + w.split) * a.heads + w.head.first) * a.buckets;
  if (!found) {
    if constexpr (BIAS)  // an empty slot's sums are zero
      for (int t = threadIdx.x; t < a.buckets; t += ALL) rel_row[t] = 0;
    return;
  }
  using Ring = KeyRing<T, D, TEAMS>;
  const int place = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), l = threadIdx.x % WAVE, h = l >> 5;
  Ring ring(a, w, (Lds)smem, place);
  const int wave = place % WAVES, team = place / WAVES;
  const int G = a.group, off = w.s.nk - w.s.nq, first = w.row0 + wave * ROWS, rows = w.s.nq * G;
  const Row r = row_of(a, w.s, first + (l & 31));
  const int head = w.head.first + r.g;
  const int64_t at = (w.s.q0 + r.i) * a.heads + head;
  F q[D / 16], g[D / 16];
  load_query<T, D>(a, (const T*)a.q, a.q_row, a.q_head, w.s, head, r, q);
  load_query<T, D>(a, (const T*)o.grad_out, (int64_t)a.heads * D, D, w.s, head, r, g);
  float delta = 0, lse = 0, share = 1;  // share: what p lacks beside 2^(z - lse) (parts_of)
  {
    F x[D / 16];
    load_query<T, D>(a, (const T*)o.out, (int64_t)a.heads * D, D, w.s, head, r, x);
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)g[k][e], (float)x[k][e], delta);
    if (o.residue) {
      load_query<T, D>(a, (const T*)o.residue, (int64_t)a.heads * D, D, w.s, head, r, x);
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf((float)g[k][e], (float)x[k][e], delta);
    }
    delta = add_halves(delta);
    if (r.valid) {
      // a row that meets no key, each of its weights -inf among the reasons: 2^(-inf - inf) = 0 is the p of all its pairs
      lse = o.lse[at];
      lse = lse == -INFINITY ? INFINITY : lse;
      if constexpr (BIAS) {
        const LseParts part = parts_of(lse, BIAS);
        lse = part.top;
        share = __builtin_amdgcn_exp2f(-part.rest);
      }
      if (l < 32 && !team) {
        o.row_lse[at] = lse;
        o.delta[at] = delta;
        if constexpr (BIAS) o.share[at] = share;
      }
      if constexpr (BIAS) delta *= share;
    }
  }
  // last key of the lane's row, and of the wave's first and last rows.  With a bias, rows past the last query see none:
  // their weight is 2^bias, which passes fp32's range from a bias of 89 on, and inf times their zeros would be NaN.
  const bool part = BIAS && first + ROWS > rows;
  const int lim = BIAS && !r.valid ? -1 : a.causal && r.valid ? min(r.i + off, w.s.nk - 1) : w.s.nk - 1;
  const int i_first = first / G, i_last = (min(first + ROWS, rows) - 1) / G;
  const int lim_first = part ? -1 : a.causal ? min(i_first + off, w.s.nk - 1) : w.s.nk - 1;
  const int lim_last = first >= rows ? -1 : (a.causal ? min(i_last + off, w.s.nk - 1) : w.s.nk - 1);
  // with a bias G = 1: the lane's row is query i of one head
  const float* bias = nullptr;
  float far_bias[2] = {0, 0}, far_unit[2] = {a.c, a.c}, far_sum[2] = {0, 0};
  const int width = bias_width(a);
  float* const table = (float*)(smem + TEAMS * ring_bytes<T, D>());
  float* const sums = table + width;              // [TABLES][width]
  float* const mine = sums + place * width;
  int* const of = (int*)(sums + TABLES * width);  // buckets
  if constexpr (BIAS) {
    for (int n = 0, t = threadIdx.x; t < width; ++n, t += ALL) {
      const int id = n == 0 ? ids[0] : n == 1 ? ids[1] : bucket_of(a, t - a.reach - BIAS_PAD);
      of[t] = id;
      table[t] = in_log2(rel_weight(a, w.head.first, id));
    }
    for (int t = threadIdx.x; t < TABLES * width; t += ALL) sums[t] = 0;
    bias = table + a.reach + BIAS_PAD - (r.i + off);
    __syncthreads();
    far_bias[0] = table[0];
    far_bias[1] = table[width - 1];
#pragma unroll
    for (int side = 0; side < 2; ++side) far_unit[side] = unit_beside(far_bias[side], a.c);
  }
  const uint32_t ka = Ti::row_base(l & 31), ca = Ti::col_base();
  f32x16 acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[b][e] = 0;
  for (int j0 = w.kbeg; j0 < w.kend; j0 += Ring::STEP) {
    const Lds kt = ring.next(j0) + team * KEYS * Ti::ROW, vt = kt + Ring::BYTES;
#pragma unroll
    for (int b = 0; b < KEYS / 32; ++b) {
      const int j = j0 + team * KEYS + 32 * b;
      if (j > lim_last) continue;
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) s = mma(Ti::row_frag(kt, ka, k, 32 * b), q[k], s);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) dp = mma(Ti::row_frag(vt, ka, k, 32 * b), g[k], dp);
      bool whole = true, above = false;
      float far = 0;
      if constexpr (BIAS) {
        above = j - (i_last + off) >= a.reach;
        whole = above || j + 31 - (i_first + off) <= -a.reach;
        far = far_bias[above];
      }
      if (whole) {
        const float unit = BIAS ? far_unit[above] : a.c;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], unit, far - lse));
      } else {
        const float* t = bias + j + 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], a.c, t[8 * (e >> 2) + (e & 3)]) - lse);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] *= BIAS ? fmaf(dp[e], share, -delta) : dp[e] - delta;
      if (j + 31 > lim_first) {
        const int last = lim - j - 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + (e & 3) <= last ? s[e] : 0.0f;
      }
      if constexpr (BIAS) {
        if (whole) {
          float sum = 0;
#pragma unroll
          for (int e = 0; e < 16; ++e) sum += s[e];
          far_sum[0] += above ? 0.0f : sum;
          far_sum[1] += above ? sum : 0.0f;
        } else {
          // lane p holds the sum at distance j - (first + off) + 31 - p.  (One such instruction to a block and not one to
          // 8 keys: LDS takes 100 cycles and more for it; dq of 32 x 256 tokens, 8 heads of 64: 32 and 27 us.)
          const float sum = diagonals(s);
          if (l < 63)
            __hip_atomic_fetch_add(mine + a.reach + BIAS_PAD + j - (first + off) + 31 - l, sum, __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_WORKGROUP);
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f32x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = s[8 * k + e];
        const auto f = to_frag<T>(p);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) acc[d] = mma(Ti::col_frag(kt, ca, d, 2 * b + k), f, acc[d]);
      }
    }
  }
  if constexpr (TEAMS == 2) {  // the second team's sums join the first one's, through the LDS that held the tiles
    float* const to = (float*)smem + threadIdx.x % THREADS;
    __syncthreads();
    if (team)
#pragma unroll
      for (int e = 0; e < D / 2; ++e) to[e * THREADS] = acc[e / 16][e % 16];
    __syncthreads();
    if (!team)
#pragma unroll
      for (int e = 0; e < D / 2; ++e) acc[e / 16][e % 16] += to[e * THREADS];
  }
  if (r.valid && !team) {
    T* const p = (T*)o.gq + at * D + 4 * h;
    float* const part = o.part + ((int64_t)w.split * a.tq * a.heads + at) * D + 4 * h;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = acc[b][4 * u + e] * a.scale;
        if (a.splits > 1)
          *(f32x4*)(part + 32 * b + 8 * u) = x;
        else
          store4<T>(p + 32 * b + 8 * u, x);
      }
  }
  if constexpr (BIAS) {
    // the waves' tables added up, then the entries past reach, with the far blocks' sums, into the last one's
    __syncthreads();
    for (int t = threadIdx.x; t < width; t += ALL) {
      float x = 0;
#pragma unroll
      for (int v = 0; v < TABLES; ++v) x += sums[v * width + t];
      sums[t] = x;
    }
    float* const far = (float*)smem;  // [2][TABLES]; the tiles are done with
    const float below = wave_sum(far_sum[0]), above = wave_sum(far_sum[1]);
    if (l == 0) {
      far[place] = below;
      far[TABLES + place] = above;
    }
    __syncthreads();
    if (threadIdx.x < 2) {  // the far blocks' sums into the last entry of their side
      float x = sums[threadIdx.x ? width - 1 : 0];
#pragma unroll
      for (int v = 0; v < TABLES; ++v) x += far[threadIdx.x * TABLES + v];
      sums[threadIdx.x ? width - 1 : 0] = x;
    }
    __syncthreads();
    for (int e0 = 0; e0 < width; e0 += 8 * WAVE) {
      int b[8];
      float y[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int e = e0 + t * WAVE + l;
        b[t] = of[min(e, width - 1)];
        y[t] = e < width ? sums[e] : 0.0f;
      }
      for (int k = place; k < a.buckets; k += TABLES) {
        float x = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) x += b[t] == k ? y[t] : 0.0f;
        x = wave_sum(x);
        if (l == 0) rel_row[k] = e0 ? rel_row[k] + x : x;
      }
    }
  }
}

// The pieces' dq added up, in their order.
template <typename T>
__global__ __launch_bounds__(THREADS) void k_attention_dq_join(const float* part, int64_t n, int splits, T* gq) {
  const int64_t at = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * 4;
  if (at >= n) return;
  f32x4 x = *(const f32x4*)(part + at);
  for (int p = 1; p < splits; ++p) {
    const f32x4 y = *(const f32x4*)(part + p * n + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += y[e];
  }
  store4<T>(gq + at, x);
}

// k_attention_dkv: a wave's 32 keys stay in registers, and so do their values while a row of them takes 128 bytes; longer
// ones stay in LDS, where the tiles are then half as long.  (2 x 8,192 causal tokens, 32/8 heads of 128, bf16: values in
// registers, tiles of 64 rows 4.28 ms with 76 registers spilled; in LDS, tiles of 32 rows 2.47 ms.  32 x 256 tokens, 8
// heads of 64: 39 and 42 us.)
template <typename T, int D>
constexpr bool values_in_lds() { return Tile<T, D>::ROW >= 256; }
template <typename T, int D>
constexpr int tile_rows() { return values_in_lds<T, D>() ? 32 : 64; }  // packed rows
constexpr int DKV_KEYS = WAVES * 32;
template <typename T, int D, int TEAMS>
constexpr int dkv_bytes() {
  return TEAMS * STAGES * 2 * tile_rows<T, D>() * Tile<T, D>::ROW +
         (values_in_lds<T, D>() ? DKV_KEYS * Tile<T, D>::ROW : 0);
}
template <typename T, int D>
constexpr int dkv_waves() { return dkv_bytes<T, D, 1>() > 72 * 1024 ? 1 : 2; }  // a SIMD
// The bias's gradient from k_attention_dq's sums [rel_rows][heads][buckets], by the workgroup of a head at the end of the
// grid of k_attention_dkv (a kernel of its own cost 4 us): 8 threads to a bucket, each a fixed set of the rows.
__device__ __forceinline__ void relative_grad(const Args& a, const Grads& o, int head, float* lds) {
  constexpr int COLS = 32, PARTS = THREADS / COLS;
  const int c = threadIdx.x % COLS, p = threadIdx.x / COLS;
  for (int k0 = 0; k0 < a.buckets; k0 += COLS) {
    float x = 0;
    if (k0 + c < a.buckets)
#pragma unroll 8
      for (int s = p; s < o.rel_rows; s += PARTS) x += o.rel[((int64_t)s * a.heads + head) * a.buckets + k0 + c];
    lds[p * COLS + c] = x;
    __syncthreads();
    if (p == 0 && k0 + c < a.buckets) {
#pragma unroll
      for (int t = 1; t < PARTS; ++t) x += lds[t * COLS + c];
      const int64_t at = (int64_t)head * a.buckets + k0 + c;
      if (a.rel_bf16)
        ((bf16*)o.grel)[at] = (bf16)x;
      else
        ((float*)o.grel)[at] = x;
    }
    __syncthreads();
  }
}

// What it keeps of a tile's queries beside them: lse, delta and, with a bias, share.
enum { LSE, DELTA, SHARE };
template <bool BIAS>
constexpr int stats_of() { return BIAS ? 3 : 2; }

// The key tile of a workgroup and its piece of the queries, lo to hi (lo >= hi: none meets the tile).  It walks from the last
// queries to the first, and over the heads of its group at each: the workgroups of a sequence that run side by side read
// the same rows at the same time, whatever the first query is that sees their keys, and share them in their L2 (2 x 8,192
// causal tokens, 32/8 heads of 128: head by head from the first query on 64 % of the reads missed it, 8.8 GB of them; in
// step 12 %, 1.6 GB).
struct KeyWork {
  Seq s;
  int j0, seen;  // queries from `seen` on see a key of the tile
  int lo, hi;
};
__device__ __forceinline__ bool key_work(const Args& a, int slot, KeyWork* w) {
  const Place at = place_of<true>(a, 1, DKV_KEYS, slot);
  w->s = at.s;
  const int64_t from = at.tile * DKV_KEYS;
  if (from >= w->s.cap) return false;
  w->j0 = (int)from;
  w->seen = w->j0 >= w->s.nk ? w->s.nq : a.causal ? max(w->j0 - (w->s.nk - w->s.nq), 0) : 0;
  return true;
}
__device__ __forceinline__ void take_piece(const Args& a, int piece, KeyWork* w) {
  const int range = piece / a.parts, last = a.splits / a.parts - 1;
  const int64_t lo = (int64_t)range * a.piece;
  w->hi = range < last ? (int)min(lo + a.piece, (int64_t)w->s.nq) : w->s.nq;
  w->lo = (int)min((int64_t)max(w->seen, (int)min(lo, (int64_t)w->s.nq)), (int64_t)w->hi);
}

// TEAMS: of four waves each, which share the keys and take the tiles of queries in turn.
template <typename T, int D, bool BIAS, int TEAMS>
__global__ __launch_bounds__(TEAMS* THREADS, (dkv_waves<T, D>())) void k_attention_dkv(Args a, Grads o) {
  using Ti = Tile<T, D>;
  using F = typename Frag<T>::type;
  constexpr int TROWS = tile_rows<T, D>(), BYTES = TROWS * Ti::ROW;
  constexpr bool VLDS = values_in_lds<T, D>();
  constexpr int STATS = stats_of<BIAS>();
  extern __shared__ __attribute__((aligned(256))) char smem[];
  Lds lds = (Lds)smem;
  if constexpr (BIAS) {
    const int tiles = a.kv_heads * a.slots * a.splits;
    if ((int)blockIdx.x >= tiles) {
      if (threadIdx.x >= THREADS) return;
      relative_grad(a, o, blockIdx.x - tiles, (float*)smem);
      return;
    }
  }
  const int hk = blockIdx.x % a.kv_heads;
  const int tile = in_turn(blockIdx.x / a.kv_heads, a.slots * a.splits, a.kv_heads);
  const int piece = tile % a.splits, slot = tile / a.splits;  // the first keys, which most rows see, first
  KeyWork w;
  if (!key_work(a, slot, &w)) return;
  take_piece(a, piece, &w);
  const Seq& s = w.s;
  const bool any = w.lo < w.hi;
  if (a.splits > 1 && !any) return;  // k_attention_dkv_join leaves it out
  const int at_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), l = threadIdx.x % WAVE, h = l >> 5;
  const int wave = at_wave % WAVES, team = at_wave / WAVES;
  const int off = s.nk - s.nq;
  const int jw = w.j0 + 32 * wave, j = jw + (l & 31);
  const bool valid = j < s.nk;
  // the wave's keys are seen by queries from `some` on, and all of them by those from `all` on
  const int some = a.causal ? jw - off : 0, all = a.causal ? jw + 31 - off : 0;
  F k[D / 16], v[VLDS ? 1 : D / 16];
  const Lds vt = lds + TEAMS * STAGES * 2 * BYTES;
  if (VLDS && any)
    load_rows<T, D, DKV_KEYS, TEAMS * WAVES>((const T*)a.v + s.k0 * a.v_row + hk * a.v_head, a.v_row, w.j0, s.nk, vt,
                                             at_wave);
  {
    const T* kp = (const T*)a.k + (s.k0 + j) * a.k_row + hk * a.k_head + 8 * h;
    const T* vp = (const T*)a.v + (s.k0 + j) * a.v_row + hk * a.v_head + 8 * h;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      F z = {};
      k[e] = valid ? *(const F*)(kp + 16 * e) : z;
      if constexpr (!VLDS) v[e] = valid ? *(const F*)(vp + 16 * e) : z;
    }
  }
  // The tiles of queries and their grad_out pass through LDS; queries i0 ... of head g, the next to load (into place
  // `place`) and the one in use.
  // beside the tiles: [TEAMS][STAGES][STATS][TROWS], then the bias table
  const Lds tiles_at = lds + team * STAGES * 2 * BYTES;
  const Lds stats = lds + dkv_bytes<T, D, TEAMS>() + team * STAGES * STATS * TROWS * 4;
  float* const table = (float*)(smem + dkv_bytes<T, D, TEAMS>()) + TEAMS * STAGES * STATS * TROWS;
  const int width = bias_width(a);
  const int64_t g_row = (int64_t)a.heads * D;
  const int top = (w.hi - 1) / TROWS * TROWS;
  const int g_first = a.ratio / a.parts * (piece % a.parts), g_end = g_first + a.ratio / a.parts;
  int place = 0, next_i = top, next_g = g_first;
  const auto load = [&] {
    const int hq = hk * a.ratio + next_g;
    const Lds to = tiles_at + place * 2 * BYTES;
    load_rows<T, D, TROWS, WAVES>((const T*)a.q + s.q0 * a.q_row + hq * a.q_head, a.q_row, next_i, w.hi, to, wave);
    load_rows<T, D, TROWS, WAVES>((const T*)o.grad_out + s.q0 * g_row + hq * D, g_row, next_i, w.hi, to + BYTES, wave);
    if (wave < STATS && l < TROWS) {  // past the end: zeros, as in the tiles
      const float* const from = (wave == LSE ? o.row_lse : wave == DELTA ? o.delta : o.share) + (s.q0 + next_i) * a.heads + hq;
      const int rows = min(w.hi - next_i, TROWS);
      dma4(resource(from, (uint32_t)((rows - 1) * a.heads + 1) * 4), stats + (place * STATS + wave) * TROWS * 4,
           (uint32_t)(l * a.heads) * 4);
    }
    place ^= 1;
  };
  const auto advance = [&](int steps, int& i, int& g) {
#pragma unroll
    for (int t = 0; t < TEAMS; ++t)
      if (t < steps && ++g == g_end) {
        g = g_first;
        i -= TROWS;
      }
  };
  // tiles of all heads that the piece meets, from the last queries on
  int left = any ? (top / TROWS - w.lo / TROWS + 1) * (g_end - g_first) : 0;
  advance(team, next_i, next_g);
  int i0 = next_i, g = next_g;
  if (team < left) load();
  bool vast = false;  // some weight is: rows have a share
  if constexpr (BIAS) {
    char* const flags = (char*)(table + a.ratio * width);  // a wave's each
    const bool mine = __builtin_amdgcn_ballot_w64(fill_bias(a, hk * a.ratio, a.ratio, table)) != 0;
    if (l == 0) flags[at_wave] = mine;
    __syncthreads();
    vast = __builtin_amdgcn_ballot_w64(l < TEAMS * WAVES && flags[l & (TEAMS * WAVES - 1)]) != 0;
  }
  uint32_t ra = Ti::row_base(l & 31), ca = Ti::col_base();
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[b][e] = dv[b][e] = 0;
  for (; left > 0; left -= TEAMS) {
    loads_done();
    __syncthreads();
    if (team >= left) break;  // the last step of an odd number: nothing to wait for but the end
    const int in_use = place ^ 1;
    advance(TEAMS, next_i, next_g);
    if (team + TEAMS < left)
      load();
    else
      place ^= 1;
    asm volatile("" : "+v"(ra), "+v"(ca));  // the addresses are formed at their use: kept, they would not fit the registers
    const Lds qt = tiles_at + in_use * 2 * BYTES, gt = qt + BYTES;
    const Lds st = stats + (in_use * STATS * TROWS + 4 * h) * 4;
#pragma unroll
    for (int rb = 0; rb < TROWS / 32; ++rb) {
      const int i = i0 + 32 * rb;
      if (jw >= s.nk || i + 31 < some || i >= w.hi) continue;  // none of the queries meets the wave's keys
      bool near = false;  // past reach one value of the bias serves the whole block
      float far = 0;
      if constexpr (BIAS) {
        const bool below = jw + 31 - (i + off) <= -a.reach, above = jw - (i + 31 + off) >= a.reach;
        near = !below && !above;
        far = near ? 0.0f : table[g * width + (above ? width - 1 : 0)];
      }
      f32x16 p, ds;
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = ds[e] = 0;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) p = mma(Ti::row_frag(qt, ra, x, 32 * rb), k[x], p);
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        if constexpr (VLDS)
          ds = mma(Ti::row_frag(gt, ra, x, 32 * rb), Ti::row_frag(vt, ra, x, 32 * wave), ds);
        else
          ds = mma(Ti::row_frag(gt, ra, x, 32 * rb), v[x], ds);
      }
      float unit = BIAS && vast ? unit_beside(far, a.c) : a.c;
      if constexpr (BIAS) {
        if (near) {  // entry of distance j - (i + 31) - off, the block's queries from there downwards
          const float* from = table + g * width + a.reach + BIAS_PAD + j - (i + 31 + off) - 4 * h;
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = fmaf(p[e], a.c, from[31 - 8 * (e >> 2) - (e & 3)]);
          unit = 1;
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 lse =
            *(const __attribute__((address_space(3))) f32x4*)(st + (LSE * TROWS + 32 * rb + 8 * u) * 4);
        const f32x4 delta =
            *(const __attribute__((address_space(3))) f32x4*)(st + (DELTA * TROWS + 32 * rb + 8 * u) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[4 * u + e] = __builtin_amdgcn_exp2f(fmaf(p[4 * u + e], unit, BIAS ? far - lse[e] : -lse[e]));
          ds[4 * u + e] = p[4 * u + e] * (ds[4 * u + e] - delta[e]);
        }
      }
      // Rows past the last query: p = 1 and with zeros beside it p dO = ds = 0, but p = 2^bias with one, and no number from a
      // bias of 89 on.
      const bool part = BIAS && i + 32 > w.hi;
      if (i < all || part || vast) {
        const int need = i < all ? j - off - i - 4 * h : -4 * h, end = w.hi - i - 4 * h;
        const unsigned many = max(end - need, 0);  // rows from `need` on, up to the last
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = 8 * (e >> 2) + (e & 3);
          const bool sees = BIAS ? (unsigned)(row - need) < many : row >= need;
          p[e] = sees ? p[e] : 0.0f;
          ds[e] = sees ? ds[e] : 0.0f;
        }
        if (BIAS && vast) {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const f32x4 share =
                *(const __attribute__((address_space(3))) f32x4*)(st + (SHARE * TROWS + 32 * rb + 8 * u) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[4 * u + e] *= share[e];
              ds[4 * u + e] *= share[e];
            }
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        f32x8 x, y;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = p[8 * c + e];
          y[e] = ds[8 * c + e];
        }
        const auto fx = to_frag<T>(x), fy = to_frag<T>(y);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) dv[b] = mma(Ti::col_frag(gt, ca, b, 2 * rb + c), fx, dv[b]);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) dk[b] = mma(Ti::col_frag(qt, ca, b, 2 * rb + c), fy, dk[b]);
      }
    }
    advance(TEAMS, i0, g);
  }
  if constexpr (TEAMS == 2) {  // the second team's sums join the first one's, through the LDS that held the tiles
    static_assert(D / 2 * THREADS * 4 <= dkv_bytes<T, D, TEAMS>(), "they fit");
    float* const to = (float*)smem + threadIdx.x % THREADS;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f32x16(&sum)[D / 32] = k ? dv : dk;
      __syncthreads();
      if (team)
#pragma unroll
        for (int e = 0; e < D / 2; ++e) to[e * THREADS] = sum[e / 16][e % 16];
      __syncthreads();
      if (!team)
#pragma unroll
        for (int e = 0; e < D / 2; ++e) sum[e / 16][e % 16] += to[e * THREADS];
    }
    if (team) return;
  }
  if (a.splits > 1) {
    if (j >= s.nk) return;
    float* const to = o.part + (((int64_t)piece * a.tk + s.k0 + j) * a.kv_heads + hk) * 2 * D + 4 * h;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f32x4 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = dk[b][4 * u + e] * a.scale;
          y[e] = dv[b][4 * u + e];
        }
        *(f32x4*)(to + 32 * b + 8 * u) = x;
        *(f32x4*)(to + D + 32 * b + 8 * u) = y;
      }
    return;
  }
  if (j >= s.cap) return;
  const int64_t at = ((s.k0 + j) * a.kv_heads + hk) * D + 4 * h;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f32x4 x, y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // rows of a cache past the sequence's keys: zeros
        x[e] = valid ? dk[b][4 * u + e] * a.scale : 0.0f;
        y[e] = valid ? dv[b][4 * u + e] : 0.0f;
      }
      store4<T>((T*)o.gk + at + 32 * b + 8 * u, x);
      store4<T>((T*)o.gv + at + 32 * b + 8 * u, y);
    }
}

// The pieces of a key tile's gradients added up, in their order; JOIN_PARTS workgroups to a tile and key head.
constexpr int JOIN_PARTS = 8;
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void k_attention_dkv_join(Args a, Grads o) {
  const int hk = blockIdx.x % a.kv_heads, part = blockIdx.x / a.kv_heads % JOIN_PARTS;
  KeyWork w;
  if (!key_work(a, blockIdx.x / a.kv_heads / JOIN_PARTS, &w)) return;
  unsigned used = 0;  // pieces with rows that meet the tile
  for (int p = 0; p < a.splits; ++p) {
    take_piece(a, p, &w);
    used |= (unsigned)(w.lo < w.hi) << p;
  }
  constexpr int KEYS_EACH = DKV_KEYS / JOIN_PARTS, VECS = 2 * D / 4;
  for (int t = threadIdx.x; t < KEYS_EACH * VECS; t += THREADS) {
    const int j = w.j0 + part * KEYS_EACH + t / VECS, d = t % VECS * 4;
    if (j >= w.s.cap) return;
    const int64_t at = (w.s.k0 + j) * a.kv_heads + hk;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (int p = 0; p < a.splits; ++p) {
      f32x4 y = {0, 0, 0, 0};
      if (j < w.s.nk && (used >> p & 1))
        y = *(const f32x4*)(o.part + ((int64_t)p * a.tk * a.kv_heads + at) * 2 * D + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += y[e];
    }
    store4<T>((d < D ? (T*)o.gk + d : (T*)o.gv + d - D) + at * D, x);
  }
}

// How the two kernels divide the work: keys (dq) and queries (dk, dv) come in pieces where the tiles are few against the
// chip, none shorter than 1,024 rows (128 in fp32, whose products take sixteen times as long).  dq: a round of workgroups,
// two where sequences differ in bf16.  dk and dv: causal tiles meet half of the pieces, so n of them make (n + 1) / 2
// workgroups a tile.  us with the join, 2 x 2,048 causal tokens, 16/8 heads of 128: dq of one round / two 76 / 108, dk and
// dv in 2 / 3 (a round) / 4 pieces 120 / 115 / 153; 8 packed texts of 1 to 4,321, 16/4 heads of 128, dk and dv for 768 /
// 1,024 / 1,536 / 2,048 workgroups 407 / 343 / 319 / 325.
// In fp32, dk and dv for 512 / 1,024 / 2,048 workgroups: 2,048 causal tokens, 8 heads of 64, 108 / 146 / 139; 2,000, 8 heads of 128,
// 322 / 265 / 265; texts of 1 to 500, 64/8 heads of 128, 599 / 470 / 401; of 1 to 1,000, 8/4 heads of 64, 85 / 83 / 81.
// k_attention_dq with two teams, as in the forward pass, us without / with: causal, 16/8 heads of 64 and bias, 300 tokens 17.4 /
// 16.1, 1,024 33 / 26, 2,304 60 / 45, 4,097 107 / 110; 8/8 heads of 64, 512 13.5 / 14.2, 6,000 107 / 85; 16/4 heads of 128, 2,600
// 80 / 68, 4,096 140 / 146; both directions, 8/8 heads of 64, 4,096 71 / 66, 4,224 108 / 118.
// k_attention_dkv with two teams, where its workgroups leave each a compute unit of its own (UNITS) and the rows are no shorter
// than 256, us without / with, the join included: causal, 16/8 heads of 64 and bias, 256 tokens 20.7 / 17.0, 1,024 40 / 32, 2,048 (320
// workgroups) 50 / 60; 16/4 heads of 128, 512 52 / 41, 2,048 (288) 74 / 89; 8/8 heads of 64, 2,048 35 / 30; 32 x 256 (512) 22.6 / 29.6.
// They also take the place of two pieces where sequences differ: six texts of 20 to 3,000, 32/8 heads of 128, 433 / 353, 8 heads of
// 64 with bias 133 / 109; three of 200 to 6,000, 24/8 heads of 128, 707 / 603; eight of 1 to 3,321, 8 heads of 64, 75 / 78.
constexpr int MAX_PIECES = 16;
struct Pieces {
  int n, size, parts;
};
// rows: units of work that one of `length` stands for, heads that pieces can share out (parts); tiles: of the grid.
Pieces pieces_of(int64_t wanted, int64_t length, int rows, int dtype, int64_t tiles) {
  const int64_t shortest = dtype == LRAM_F32 ? 128 : 1024;
  const int64_t step = dtype == LRAM_F32 ? KEYS : 2 * KEYS;  // whole steps of two teams
  const auto at_least = [&](int64_t work) {
    return few_enough(tiles) ? std::min<int64_t>({wanted, (length * rows + work - 1) / work, MAX_PIECES}) : 1;
  };
  int64_t n = std::max<int64_t>(1, std::min(at_least(shortest), (length + step - 1) / step));
  const int64_t size = std::max<int64_t>(step, ((length + n - 1) / n + step - 1) / step * step);
  n = std::max<int64_t>(1, std::min(n, (length + size - 1) / size));
  // queries that cannot be divided any further are, by their heads (in fp32 down to 64 rows; 8/1 heads of 128 and 200 queries:
  // dk and dv 156 -> 58 us)
  const int64_t most = at_least(dtype == LRAM_F32 ? KEYS : shortest);
  int parts = 1;
  for (int p = 2; p <= rows; ++p)
    if (rows % p == 0 && n * p <= most) parts = p;
  return {(int)n * parts, (int)std::min<int64_t>(size, 1 << 30), parts};
}
struct Plan {
  int group, row_slots, key_slots;
  bool teams, key_teams;  // two of them in k_attention_dq, in k_attention_dkv
  Pieces keys, rows;
  size_t stats, rel, part;  // floats of workspace; stats: of row_lse, of delta and of share each
  int kinds;                // how many of those there are
};
Plan plan_of(const lram_attention& call) {
  const lram_attention a = bounded(call);
  Plan p;
  const int64_t G = a.heads / a.kv_heads;
  p.group = a.rel_weight ? 1 : (int)G;
  p.row_slots = slots_of(a.tq, p.group, WAVES * ROWS, a.batch);
  p.key_slots = slots_of(a.tk, 1, DKV_KEYS, a.batch);
  const bool even = a.dtype == LRAM_F32 || alike(a);
  const auto tiles = [&](int64_t longest, int64_t rows, int64_t slots, int64_t heads) {
    return std::max<int64_t>(1, tiles_of(a, longest, rows, 128, slots) * heads);
  };
  const int64_t row_tiles = tiles(a.max_q * p.group, a.tq * p.group, p.row_slots, a.heads / p.group);
  // of a cache, what its sequences have in use
  const int64_t key_tiles = tiles(a.max_k, a.used_k ? 0 : a.tk, p.key_slots, a.kv_heads);
  p.teams = a.dtype == LRAM_BF16 && even && a.max_k > (a.rel_weight ? 256 : 512) && dq_lds(a, 2) <= LDS_BYTES &&
            row_tiles <= (a.causal && a.max_k > 1024 ? 3 * UNITS / 2 : UNITS);
  p.keys = pieces_of((p.teams ? UNITS : even ? ROUND : 2 * ROUND) / row_tiles, a.max_k, 1, a.dtype,
                     (int64_t)p.row_slots * (a.heads / p.group));
  const int64_t wanted = a.dtype == LRAM_F32 ? (!alike(a) ? 4 : a.head_dim == 128 ? 2 : 1) * ROUND / key_tiles
                         : !even             ? 3 * ROUND / key_tiles
                         : a.causal          ? 2 * ROUND / key_tiles - 1
                                             : ROUND / key_tiles;
  const auto rows_of = [&](int64_t n) {
    return pieces_of(n, a.max_q, (int)G, a.dtype, (int64_t)p.key_slots * a.kv_heads);
  };
  p.rows = rows_of(wanted);
  const int64_t busy = a.causal ? key_tiles * (p.rows.n + 1) / 2 : key_tiles * p.rows.n;
  const bool halves = !even && p.rows.n == 2;
  if (halves) p.rows = rows_of(1);
  p.key_teams = a.dtype == LRAM_BF16 && a.max_q * G >= 256 && (halves || busy <= UNITS);
  p.stats = ((size_t)a.tq * a.heads + 3) / 4 * 4;
  p.kinds = a.rel_weight ? 3 : 2;
  p.rel = a.rel_weight ? ((size_t)p.row_slots * p.keys.n * a.heads * a.rel_buckets + 3) / 4 * 4 : 0;
  // dq's pieces are joined before those of dk and dv are written
  const size_t dq = p.keys.n > 1 ? (size_t)p.keys.n * a.tq * a.heads * a.head_dim : 0;
  const size_t dkv = p.rows.n > 1 ? (size_t)p.rows.n * a.tk * a.kv_heads * 2 * a.head_dim : 0;
  p.part = std::max(dq, dkv);
  return p;
}

template <typename T, int D, bool BIAS>
int go(Args x, const Grads& g, const Plan& p, hipStream_t s) {
  const size_t width = BIAS ? (size_t)(2 * (x.reach + BIAS_PAD) + 1) * 4 : 0;
  const auto launch = [&](auto kernel, int64_t grid, size_t bytes, int threads = THREADS) {
    if (int rc = allow_lds((const void*)kernel, bytes)) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), bytes, s, x, g);
    return layer_launched();
  };
  if (x.tq) {
    x.group = p.group;
    x.slots = p.row_slots;
    x.splits = p.keys.n;
    x.piece = p.keys.size;
    const auto dq = [&](auto teams) {
      constexpr int TEAMS = decltype(teams)::value;
      return launch(k_attention_dq<T, D, BIAS, TEAMS>, (int64_t)(x.heads / x.group) * x.slots * x.splits,
                    TEAMS * ring_bytes<T, D>() + width * (2 + TEAMS * WAVES), TEAMS * THREADS);
    };
    int rc = LRAM_OK;
    if constexpr (sizeof(T) == 2)
      if (p.teams) rc = dq(std::integral_constant<int, 2>());
    if (!p.teams) rc = dq(std::integral_constant<int, 1>());
    if (rc) return rc;
    if (x.splits > 1) {
      const int64_t n = x.tq * x.heads * D;
      hipLaunchKernelGGL(k_attention_dq_join<T>, dim3((unsigned)((n / 4 + THREADS - 1) / THREADS)), dim3(THREADS), 0, s,
                         (const float*)g.part, n, x.splits, (T*)g.gq);
      if (int rc = layer_launched()) return rc;
    }
  }
  if (x.tk || BIAS) {
    x.slots = x.tk ? p.key_slots : 0;
    x.splits = p.rows.n;
    x.piece = p.rows.size;
    x.parts = p.rows.parts;
    const auto dkv = [&](auto teams) {
      constexpr int TEAMS = decltype(teams)::value;
      return launch(k_attention_dkv<T, D, BIAS, TEAMS>,
                    (int64_t)x.kv_heads * x.slots * x.splits + (BIAS ? x.heads : 0),
                    dkv_bytes<T, D, TEAMS>() + TEAMS * STAGES * stats_of<BIAS>() * tile_rows<T, D>() * 4 +
                        (BIAS ? width * x.ratio + TEAMS * WAVES : 0),
                    TEAMS * THREADS);
    };
    int rc = LRAM_OK;
    if constexpr (sizeof(T) == 2)
      if (p.key_teams) rc = dkv(std::integral_constant<int, 2>());
    if (!p.key_teams) rc = dkv(std::integral_constant<int, 1>());
    if (rc) return rc;
    if (x.tk && x.splits > 1)
      return launch(k_attention_dkv_join<T, D>, (int64_t)x.kv_heads * x.slots * JOIN_PARTS, 0);
  }
  return LRAM_OK;
}

}  // namespace

extern "C" {

int lram_attention_backward_workspace_bytes(const lram_attention* a, size_t* bytes) {
  if (!a || !bytes) return LRAM_EINVAL;
  if (int rc = check_attention(*a, false)) return rc;
  const Plan p = plan_of(*a);
  *bytes = (p.kinds * p.stats + p.rel + p.part) * 4;
  return LRAM_OK;
}

int lram_attention_backward(const lram_attention* a, const void* out, const void* residue, const float* lse,
                            const void* grad_out, void* grad_q, void* grad_k, void* grad_v, void* grad_rel,
                            void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return LRAM_EINVAL;
  if (int rc = check_attention(*a, true)) return rc;
  if (a->tq && (!out || !lse || !grad_out || !grad_q)) return LRAM_EINVAL;
  if (a->tk && (!grad_k || !grad_v)) return LRAM_EINVAL;
  if ((a->rel_weight != nullptr) != (grad_rel != nullptr)) return LRAM_EINVAL;
  if (off_align(out, 16) || off_align(residue, 16) || off_align(grad_out, 16) || off_align(grad_q, 16) ||
      off_align(grad_k, 16) || off_align(grad_v, 16) || off_align(lse, 4) ||
      off_align(grad_rel, elem_size(a->wdtype)))
    return LRAM_EINVAL;
  if (residue && a->dtype != LRAM_BF16) return LRAM_EDTYPE;
  const Plan p = plan_of(*a);
  const size_t need = (p.kinds * p.stats + p.rel + p.part) * 4;
  if (need && (!workspace || off_align(workspace, 16) || ws_bytes < need)) return LRAM_EWORKSPACE;
  Args x = args_of(*a);
  x.splits = 1;
  float* const ws = (float*)workspace;
  const Grads g{out, residue, grad_out, lse, grad_q, grad_k, grad_v, grad_rel, ws, ws + p.stats,
                ws + 2 * p.stats, ws + p.kinds * p.stats, ws + p.kinds * p.stats + p.rel, a->tq ? p.row_slots * p.keys.n : 0};
  return by_kind(*a, [&](auto t, auto d, auto bias) {
    return go<decltype(t), decltype(d)::value, decltype(bias)::value>(x, g, p, (hipStream_t)stream);
  });
}

}  // extern "C"
