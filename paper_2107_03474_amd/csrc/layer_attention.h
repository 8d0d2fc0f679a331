// layer_attention.h -- part of liblram: what the attention kernels share.
//
// For a sequence of nq queries and nk keys, off = nk - nq; query i of head h sees key j if j < nk and, causal,
// j <= i + off.  In units of log 2:
//     z_ij = c q_i . k_j + t_h(j - i - off),  c = scale log2 e,  t_h the bias by distance, times log2 e
//     p_ij = 2^(z_ij - m_i) / l_i,  o_i = sum_j p_ij v_j,  lse_i = m_i + log2 l_i
//
// The heads / kv_heads query heads that share a key head are rows of one matrix: with G = heads / kv_heads, packed row r of a
// sequence is query r / G of head r % G of the group, so a few queries fill a tile, and a tile meets a key once for all
// G heads.  Row tiles of prompts with a bias keep to one head (G = 1): its rows' distances to a key are consecutive.
//
// Tiles.  Products run on the matrix cores as 32 x 32 blocks with K = 16 (fp32: eight steps of K = 2).  A lane's operand is
// 8 elements: A row (lane & 31), k = 8 (lane >> 5) .. + 7, B column the same; a result's lane holds column lane & 31,
// rows 8 (r >> 2) + 4 (lane >> 5) + (r & 3) for r < 16.  Scores are formed transposed (keys x rows), so a lane owns one row of
// the softmax, and its 8 results r = 8 c .. 8 c + 7 are the B operand of the next product for keys 16 c .. 16 c + 15 as
// they stand, with the k order (4 h + 0..3, 8 + 4 h + 0..3) that the other operand's loads follow (col_frag).

#pragma once

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layer_common.h"

namespace {

using f32x16 = float __attribute__((ext_vector_type(16)));
using f32x8 = float __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using bf16x4 = __bf16 __attribute__((ext_vector_type(4)));
using s16x4 = short __attribute__((ext_vector_type(4)));
using Lds = __attribute__((address_space(3))) char*;

constexpr float LOG2E = 1.4426950408889634f;
constexpr int ROWS = 32;     // packed rows (or keys) of a wave
constexpr int KEYS = 64;     // keys of a tile in LDS
constexpr int WAVES = 4, THREADS = WAVES * WAVE;
constexpr int BIAS_PAD = 96;  // distances that a tile reaches past the last one with a bias of its own

// Device-side view of a call.
struct Args {
  const void *q, *k, *v;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head;  // strides in elements
  const int32_t *start_q, *start_k, *used_k;
  const void* rel_weight;
  const int32_t* rel_bucket;
  int64_t tq, tk;
  int32_t heads, kv_heads, batch;
  int32_t ratio;  // heads of a key head
  int32_t group;  // of them, those packed in a tile: ratio or 1
  int32_t causal, buckets, reach;
  int32_t rel_bf16;
  int32_t slots;   // row (or key) tiles of all stretches (sequence), some of them empty
  int32_t splits;  // pieces of the keys (dk, dv: of the rows)
  int32_t piece;   // keys (queries) of a piece
  int32_t parts;   // dk, dv: so many pieces share a piece's queries, by their heads
  float c;         // scale log2 e
  float scale;
};

// A sequence's place.  The starts live in device memory, where no host check sees them: whatever they hold, no row
// outside the tensors is addressed.
struct Seq {
  int64_t q0, k0;
  int32_t nq, nk, cap;  // queries, keys, rows that the sequence has in k and v
};

__device__ __forceinline__ int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : (x > hi ? hi : x); }

// The tensors' rows come in batch + 2 stretches: those before the first sequence (0), the sequences (1 ... batch) and those
// past the last one (batch + 1).  The first and the last see nothing.
__device__ __forceinline__ Seq sequence(const Args& a, int e) {
  const int from = e ? e - 1 : 0, to = e <= a.batch ? e : a.batch;  // starts
  const bool real = from < to;
  const int64_t q0 = a.start_q[from], q1 = a.start_q[to], k0 = a.start_k[from], k1 = a.start_k[to];
  const int64_t used = a.used_k && real ? a.used_k[from] : INT32_MAX;
  Seq s;
  s.q0 = e ? clamp64(q0, 0, a.tq) : 0;
  s.k0 = e ? clamp64(k0, 0, a.tk) : 0;
  s.nq = (int32_t)((e <= a.batch ? clamp64(q1, s.q0, a.tq) : a.tq) - s.q0);
  s.cap = (int32_t)((e <= a.batch ? clamp64(k1, s.k0, a.tk) : a.tk) - s.k0);
  s.nk = real ? (int32_t)clamp64(used, 0, s.cap) : 0;
  return s;
}

// Which stretch and which of its tiles a slot of the grid is, without knowing the lengths on the host.  Tiles hold `tile`
// packed rows, `scale` to a query (BY_KEYS: rows of k and v, 1 to a row).  The grid has slots_of slots, at least as many as
// there are tiles; those left over are empty.
//
// Up to 62 sequences, a lane for each stretch, all of whose places are read at once: the longest come first, ties in their
// order, so that the workgroups that start last are short.  More sequences: stretch e, which begins at row r, takes the
// slots from r scale / tile + e on, which leaves each as many as it needs, and is found by a wave that looks at 64 places
// at once.
inline int slots_of(int64_t rows, int64_t scale, int tile, int batch) { return (int)(rows * scale / tile + batch + 2); }
struct Place {
  Seq s;
  int64_t tile;  // past the stretch's last one: an empty slot
};
__device__ __forceinline__ int64_t first_slot(const int32_t* start, int64_t rows, int e, int scale, int tile) {
  return (e ? clamp64(start[e - 1], 0, rows) : 0) * scale / tile + e;
}
__device__ __forceinline__ int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
template <bool BY_KEYS>
__device__ __forceinline__ Place place_of(const Args& a, int scale, int tile, int slot) {
  const int lane = threadIdx.x % WAVE, last = a.batch + 1;
  if (last < WAVE) {
    const Seq s = sequence(a, lane <= last ? lane : last);
    const int mine = lane > last ? 0 : (int)(((int64_t)(BY_KEYS ? s.cap : s.nq) * scale + tile - 1) / tile);
    const int one = of_lane(mine, 1);
    int first;  // slot of the stretch's first tile
    if (__builtin_amdgcn_ballot_w64(lane && lane < last && mine != one) == 0 && of_lane(mine, 0) == 0 &&
        of_lane(mine, last) <= one) {
      first = (lane - 1) * one;  // like sequences from row 0 on
    } else {
      first = 0;
      for (int e = 0; e <= last; ++e) {
        const int other = of_lane(mine, e);
        first += other > mine || (other == mine && e < lane) ? other : 0;
      }
    }
    const uint64_t at = __builtin_amdgcn_ballot_w64(lane <= last && first <= slot && slot - first < mine);
    Place p{};
    p.tile = INT32_MAX;
    if (!at) return p;
    const int e = __ffsll((unsigned long long)at) - 1;
    p.s.q0 = of_lane((int)s.q0, e);  // the starts are 32-bit
    p.s.k0 = of_lane((int)s.k0, e);
    p.s.nq = of_lane(s.nq, e);
    p.s.nk = of_lane(s.nk, e);
    p.s.cap = of_lane(s.cap, e);
    p.tile = slot - of_lane(first, e);
    return p;
  }
  const int32_t* const start = BY_KEYS ? a.start_k : a.start_q;
  const int64_t rows = BY_KEYS ? a.tk : a.tq;
  int lo = 0, n = last + 1;  // the last e of lo ... lo + n - 1 with first_slot(e) <= slot
  while (n > 1) {
    const int step = (n + WAVE - 1) / WAVE, e = lo + lane * step;
    const bool at = e < lo + n && first_slot(start, rows, e, scale, tile) <= slot;
    // the first place holds; where the starts do not rise, none may, and the search stays inside them all the same
    const int past = max(__popcll(__builtin_amdgcn_ballot_w64(at)) - 1, 0) * step;
    lo += past;
    n = min(step, n - past);
  }
  const int64_t past = slot - first_slot(start, rows, lo, scale, tile);
  return {sequence(a, lo), past < 0 ? INT32_MAX : past};
}

// The grid's order: tiles of falling length (causal), but every second stretch of as many workgroups as there are compute
// units turned round, so that workgroups that share one, a grid's length apart, are a long and a short one.  idx of n
// tiles, each with `heads` workgroups.  (It is long products that need it: fp32, five texts of 1 to 1,000, 8/4 heads of 64,
// forward 51 -> 37 us; bf16, 2 x 2,048 tokens, the same time both ways.)
constexpr int UNITS = 256, TURN_MOST = 3;
__device__ __forceinline__ int in_turn(int idx, int n, int heads) {
  if ((int64_t)n * heads > TURN_MOST * UNITS) return idx;  // units that run dry take the next one by themselves
  const int stretch = max(1, UNITS / heads), first = idx / stretch * stretch;
  return idx / stretch % 2 ? first + min(stretch, n - first) - 1 - (idx - first) : idx;
}

// Workgroups go round the 8 dies in turn, and neighbours in the grid are different heads: with 8 key heads, or a divisor or
// multiple of 8, the tiles that read the same keys run on the same die and share its L2, and every die gets long and
// short tiles alike.  Packed head n (of heads / group) of the grid's order:
struct Heads {
  int kv, first;  // key head, first query head
};
__device__ __forceinline__ Heads heads_of(const Args& a, int n) {
  Heads h;
  h.kv = n % a.kv_heads;
  h.first = h.kv * a.ratio + n / a.kv_heads * a.group;
  return h;
}

template <typename T>
struct Frag;
template <>
struct Frag<bf16> {
  using type = bf16x8;
};
template <>
struct Frag<float> {
  using type = f32x8;
};

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// Eight fp32 values as an operand (rounded to nearest even).
template <typename T>
__device__ __forceinline__ typename Frag<T>::type to_frag(f32x8 x) {
  if constexpr (sizeof(T) == 4)
    return x;
  else
    return __builtin_convertvector(x, bf16x8);
}

// The values of the lane and of its twin in the other half of the wave.
struct Pair {
  float lower, upper;
};
__device__ __forceinline__ Pair halves(float x) {
  const int a = __builtin_bit_cast(int, x);
  const auto r = __builtin_amdgcn_permlane32_swap(a, a, false, false);
  const unsigned lower = r[0], upper = r[1];
  return {__builtin_bit_cast(float, lower), __builtin_bit_cast(float, upper)};
}
__device__ __forceinline__ float max_halves(float x) {
  const Pair p = halves(x);
  return fmaxf(p.lower, p.upper);
}
__device__ __forceinline__ float add_halves(float x) {
  const Pair p = halves(x);
  return p.lower + p.upper;
}

// A tile of rows x D elements in LDS, row-major, each row's 16-byte chunks permuted by an XOR of the row's low bits so
// that neither a column of chunks (row_frag) nor four rows of 64 bytes (col_frag) meet in one bank.
template <typename T, int D>
struct Tile {
  using F = typename Frag<T>::type;
  static constexpr int ROW = D * (int)sizeof(T);  // bytes
  static constexpr int CH = ROW / 16;
  static constexpr int PER = 16 / (int)sizeof(T);  // elements of a chunk
  static constexpr int STEPS = D / 16, BLOCKS = D / 32;

  static __device__ __forceinline__ int swizzle(int row) {
    const int b0 = row & 1, b1 = row >> 1 & 1, b2 = row >> 2 & 1, b3 = row >> 3 & 1;
    if constexpr (sizeof(T) == 2 && CH == 16) return b1 << 3 | b0 << 2 | b3 << 1 | b2;
    if constexpr (CH == 8) return b1 << 2 | b2 << 1 | b3;
    if constexpr (CH == 4) return b2 << 1 | b3;
    return b2 << 3 | b0 << 2 | b1 << 1 | b3;
  }

  // A lane's operand addresses are a base and, since the swizzle is linear in the row's bits, an XOR with a constant.
  // Row operand: 8 elements of the lane's row, k = 16 s + 8 h ..., of the block that starts at first_row (a multiple of 16).
  static __device__ __forceinline__ uint32_t row_base(int row) {
    const int h = threadIdx.x >> 5 & 1;
    return row * ROW + (8 * h / PER ^ swizzle(row)) * 16;
  }
  static __device__ __forceinline__ F row_frag(Lds tile, uint32_t base, int s, int first_row) {
    if constexpr (sizeof(T) == 2) {
      return *(const __attribute__((address_space(3))) bf16x8*)(tile + (base ^ s * 32) + first_row * ROW);
    } else {
      const f32x4 x = *(const __attribute__((address_space(3))) f32x4*)(tile + (base ^ s * 64) + first_row * ROW);
      const f32x4 y = *(const __attribute__((address_space(3))) f32x4*)(tile + (base ^ (s * 64 + 16)) + first_row * ROW);
      return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }

  // Column operand: column d = 32 block + (lane & 31) of the transposed tile, rows 16 c + (4 h + 0..3, 8 + 4 h + 0..3).
  static __device__ __forceinline__ uint32_t col_base() {
    const int l = threadIdx.x & 63, h = l >> 5;
    if constexpr (sizeof(T) == 2) {  // the transposing read: 16 lanes take 4 rows of 16 columns
      const int row = 4 * h + (l >> 2 & 3), d = (l & 16) + 4 * (l & 3);
      return row * ROW + (d / PER ^ swizzle(row)) * 16 + d % PER * 2;
    } else {
      const int row = 4 * h, d = l & 31;
      return row * ROW + (d / PER ^ swizzle(row)) * 16 + d % PER * 4;
    }
  }
  static __device__ __forceinline__ F col_frag(Lds tile, uint32_t base, int block, int c) {
    if constexpr (sizeof(T) == 2) {
      union {
        s16x4 s[2];
        bf16x8 f;
      } u;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        u.s[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
            tile + (base ^ (32 * block / PER ^ swizzle(8 * i)) * 16) + (16 * c + 8 * i) * ROW));
      return u.f;
    } else {
      f32x8 f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          f[4 * i + e] = *(const __attribute__((address_space(3))) float*)(
              tile + (base ^ (32 * block / PER ^ swizzle(8 * i + e)) * 16) + (16 * c + 8 * i + e) * ROW);
      return f;
    }
  }
};

// 16 bytes a lane from memory straight into LDS at dst + 16 lane; a lane whose offset lies past the resource's end
// gets zeros.  Written out so that the compiler does not wait for it at the next read of any tile: the kernels wait
// themselves (loads_left), before the barrier or the reads that need it.  m0, the destination's register, is named as
// written: the compiler keeps no values there (it says so, in a warning), but may share one setting of it among its own
// instructions.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t src, Lds dst, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"((uint32_t)(uintptr_t)dst), "v"(offset), "s"(src)
               : "memory", "m0");
}
// The same of 4 bytes a lane, to dst + 4 lane.
__device__ __forceinline__ void dma4(__amdgpu_buffer_rsrc_t src, Lds dst, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"((uint32_t)(uintptr_t)dst), "v"(offset), "s"(src)
               : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
}
// Rows [row, row + N) of a head of k or v into a tile, by `waves` waves of which this is number `wave`; rows from `rows` on
// become zeros.
template <typename T, int D, int N, int WAVES>
__device__ __forceinline__ void load_rows(const T* head, int64_t stride, int row, int rows, Lds tile, int wave) {
  using Ti = Tile<T, D>;
  const int left = rows - row;
  const uint32_t bytes = left > 0 ? (uint32_t)(((left < N ? left : N) - 1) * stride + D) * (uint32_t)sizeof(T) : 0;
  const auto src = resource(head + row * stride, bytes);
  constexpr int LOADS = N * Ti::CH / 64 / WAVES;
  static_assert(LOADS * 64 * WAVES == N * Ti::CH, "whole loads");
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int first = (wave * LOADS + i) * 64;  // chunk of lane 0
    const int p = first + (threadIdx.x & 63);
    const int r = p / Ti::CH, ch = (p % Ti::CH) ^ Ti::swizzle(r);
    dma16(src, tile + first * 16, (uint32_t)(r * (int)stride + ch * Ti::PER) * (uint32_t)sizeof(T));
  }
}

// Weights far past any score.  From 2^24 on (a weight of 1.2e7, times log2 e) fp32 holds no digit behind the point, so that
// scores beside such a weight say nothing, and times log2 e the type's lowest value, a common mask, would be -inf, which
// hides a key altogether.  Finite weights from there on all count as +-2^126: a score added to it leaves it as it is, and
// a row that meets no other keys (or one that meets keys of +2^126) has the even average of those.  Its maximum is then
// +-2^126 and its sum a count, which m + log2 l would lose: the row's lse is m (1 + log2 l / 32) instead, l <= 2^30.
constexpr float FAR_WEIGHT = 0x1p24f, VAST = 0x1p126f, BARELY = 0x1p-100f;
__device__ __forceinline__ float in_log2(float weight) {
  const float t = weight * LOG2E;
  return fabsf(t) >= FAR_WEIGHT && fabsf(weight) < INFINITY ? copysignf(VAST, weight) : t;
}
__device__ __forceinline__ bool is_vast(float x) { return fabsf(x) >= VAST && fabsf(x) < 2 * VAST; }
// The scores' factor beside a bias that serves a whole block: next to nothing where the bias is vast, so that subtracting
// the maximum does not bring them back (not 0, which would make the -inf of a key that is not seen NaN).
__device__ __forceinline__ float unit_beside(float far, float c) { return is_vast(far) ? BARELY : c; }
__device__ __forceinline__ float lse_of(float m, float sum, bool bias) {
  const float l = __builtin_amdgcn_logf(sum);
  return sum == 0 ? -INFINITY : bias && fabsf(m) == VAST ? fmaf(m, l * 0x1p-5f, m) : m + l;
}
// An lse as the two parts of log2 of a sum: the maximum where it is vast, and what is left beside it.
struct LseParts {
  float top, rest;
};
__device__ __forceinline__ LseParts parts_of(float lse, bool bias) {
  if (!bias || !is_vast(lse)) return {lse, 0.0f};
  return {copysignf(VAST, lse), fmaf(fabsf(lse), 32 / VAST, -32.0f)};
}

// The bias by distance of the group's heads, times log2 e, in LDS: [G][2 (reach + BIAS_PAD) + 1], constant past reach.
__device__ __forceinline__ int bias_width(const Args& a) { return 2 * (a.reach + BIAS_PAD) + 1; }
__device__ __forceinline__ float rel_weight(const Args& a, int head, int bucket) {
  const int64_t at = (int64_t)head * a.buckets + bucket;
  return a.rel_bf16 ? (float)((const bf16*)a.rel_weight)[at] : ((const float*)a.rel_weight)[at];
}
__device__ __forceinline__ int bucket_of(const Args& a, int d) {
  d = d < -a.reach ? -a.reach : (d > a.reach ? a.reach : d);
  const int b = a.rel_bucket[d + a.reach];
  return b < 0 ? 0 : (b < a.buckets ? b : a.buckets - 1);  // device data: nothing outside the weights is addressed
}
// Whether the thread met a vast one.
__device__ __forceinline__ bool fill_bias(const Args& a, int first_head, int heads, float* table) {
  const int n = bias_width(a);
  bool vast = false;
  for (int i = threadIdx.x; i < heads * n; i += blockDim.x) {
    table[i] = in_log2(rel_weight(a, first_head + i / n, bucket_of(a, i % n - a.reach - BIAS_PAD)));
    vast |= is_vast(table[i]);
  }
  return vast;
}

// Waits of a wave: every load into LDS that it issued has arrived, all but the last N have, every read of LDS has.
template <int N>
__device__ __forceinline__ void loads_left() {
  static_assert(N < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void loads_done() { loads_left<0>(); }
__device__ __forceinline__ void reads_done() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// What a lane knows of its row.
struct Row {
  bool valid;
  int i, g;  // query, head of the group
};
__device__ __forceinline__ Row row_of(const Args& a, const Seq& s, int row) {
  Row r;
  r.valid = row < s.nq * a.group;
  r.i = row / a.group;
  r.g = row - r.i * a.group;
  return r;
}
template <typename T, int D>
__device__ __forceinline__ void load_query(const Args& a, const T* base, int64_t row_stride, int64_t head_stride,
                                           const Seq& s, int head, const Row& r, typename Frag<T>::type (&f)[D / 16]) {
  using F = typename Frag<T>::type;
  const T* p = base + (s.q0 + r.i) * row_stride + head * head_stride + 8 * (threadIdx.x >> 5 & 1);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    F z = {};
    f[k] = r.valid ? *(const F*)(p + 16 * k) : z;
  }
}

// The tile of a workgroup: sequence, first packed row, key range (find_work: false for an empty slot).  The grid
// is slots x splits x packed heads, the last fastest.
struct Work {
  Seq s;
  Heads head;
  int slot, row0, split, kbeg, kend;
};
template <int M>
__device__ __forceinline__ bool find_work(const Args& a, Work* w) {
  const unsigned n = a.heads / a.group;
  w->head = heads_of(a, blockIdx.x % n);
  const int tile = in_turn(blockIdx.x / n, a.slots * a.splits, n);
  w->split = tile % a.splits;
  w->slot = tile / a.splits;
  const Place at = place_of<false>(a, a.group, M, w->slot);
  w->s = at.s;
  // a sequence's last rows, which see most keys (causal), first
  const int64_t tiles = ((int64_t)w->s.nq * a.group + M - 1) / M;
  if (at.tile >= tiles) return false;
  const int64_t row0 = (tiles - 1 - at.tile) * M;
  w->row0 = (int)row0;
  const int rows = w->s.nq * a.group;
  const int last = (w->row0 + M < rows ? w->row0 + M : rows) - 1;
  int end = w->s.nk;
  if (a.causal) {
    const int seen = last / a.group + w->s.nk - w->s.nq + 1;
    end = seen < end ? (seen > 0 ? seen : 0) : end;
  }
  const int64_t from = (int64_t)w->split * a.piece;
  w->kbeg = from < end ? (int)from : end;
  w->kend = w->split == a.splits - 1 || from + a.piece > end ? end : (int)(from + a.piece);
  return true;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 x) {
  using V = T __attribute__((ext_vector_type(4)));
  *(V*)p = __builtin_convertvector(x, V);
}

// Tiles in LDS at once: the one in use and the one on its way.  (Three or four of the smaller ones cost workgroups a CU:
// 32 x 256 tokens, 8 heads of 64, bf16, bias, us with 2 / 3 / 4: forward 20.5 / 22.4 / 25.9, dq 36 / 55 / 56, dk and dv
// 24 / 24 / 33.)
constexpr int STAGES = 2;
template <typename T, int D>
constexpr int ring_bytes() { return STAGES * 2 * KEYS * Tile<T, D>::ROW; }
// Waves per SIMD: two; one where LDS holds one workgroup a CU.
template <typename T, int D>
constexpr int waves_per_simd() { return ring_bytes<T, D>() > 80 * 1024 ? 1 : 2; }

// The tiles of KEYS keys and values of a work item, one to each of the workgroup's teams, passing through LDS; all waves go
// along together.
template <typename T, int D, int TEAMS>
struct KeyRing {
  static constexpr int STEP = TEAMS * KEYS, BYTES = STEP * Tile<T, D>::ROW;
  const T *k, *v;
  int64_t k_row, v_row;
  Lds lds;
  int wave, nk, end, place;

  __device__ __forceinline__ KeyRing(const Args& a, const Work& w, Lds lds_, int wave_)
      : k((const T*)a.k + w.s.k0 * a.k_row + w.head.kv * a.k_head),
        v((const T*)a.v + w.s.k0 * a.v_row + w.head.kv * a.v_head),
        k_row(a.k_row), v_row(a.v_row), lds(lds_), wave(wave_), nk(w.s.nk), end(w.kend), place(0) {
    load(w.kbeg, 0);
  }
  __device__ __forceinline__ void load(int j0, int to) {
    if (j0 >= end) return;
    load_rows<T, D, STEP, TEAMS * WAVES>(k, k_row, j0, nk, lds + to * 2 * BYTES, wave);
    load_rows<T, D, STEP, TEAMS * WAVES>(v, v_row, j0, nk, lds + to * 2 * BYTES + BYTES, wave);
  }
  // The tiles from key j0 on, the next in line: keys here, values BYTES on.
  __device__ __forceinline__ Lds next(int j0) {
    loads_done();
    __syncthreads();  // the tiles are whole, and every wave has left the other place
    const Lds tile = lds + place * 2 * BYTES;
    place ^= 1;
    load(j0 + STEP, place);
    return tile;
  }
};

// The same with the keys a step ahead of the values.
template <typename T, int D, int TEAMS>
struct KeyAhead {
  static constexpr int STEP = TEAMS * KEYS, BYTES = STEP * Tile<T, D>::ROW;
  const T *k, *v;
  int64_t k_row, v_row;
  Lds lds;
  int wave, nk, end, place;  // of the values in use, and of the next keys to be loaded

  __device__ __forceinline__ KeyAhead(const Args& a, const Work& w, Lds lds_, int wave_)
      : k((const T*)a.k + w.s.k0 * a.k_row + w.head.kv * a.k_head),
        v((const T*)a.v + w.s.k0 * a.v_row + w.head.kv * a.v_head),
        k_row(a.k_row), v_row(a.v_row), lds(lds_), wave(wave_), nk(w.s.nk), end(w.kend), place(1) {
    load_k(w.kbeg, 0);
    load_v(w.kbeg, 0);
    load_k(w.kbeg + STEP, 1);
  }
  __device__ __forceinline__ void load_k(int j0, int to) {
    if (j0 < end) load_rows<T, D, STEP, TEAMS * WAVES>(k, k_row, j0, nk, lds + to * BYTES, wave);
  }
  __device__ __forceinline__ void load_v(int j0, int to) {
    if (j0 < end) load_rows<T, D, STEP, TEAMS * WAVES>(v, v_row, j0, nk, lds + (2 + to) * BYTES, wave);
  }
  __device__ __forceinline__ Lds first() {
    loads_done();
    __syncthreads();
    return lds;
  }
  // The tiles from key j0 on become those in use.
  __device__ __forceinline__ void next(int j0) {
    loads_done();
    __syncthreads();  // its values and the next one's keys are whole; every wave has left the other places
    place ^= 1;
    load_k(j0 + 2 * STEP, place);
    load_v(j0 + STEP, place ^ 1);
  }
  __device__ __forceinline__ Lds keys() const { return lds + (place ^ 1) * BYTES; }  // of the tile after it
  __device__ __forceinline__ Lds values() const { return lds + (2 + place) * BYTES; }
};

// ---------------------------------------------------------------------------
// Host side.

constexpr int64_t MOST_GROUPS = int64_t(1) << 24;
// Whether a grid of so many tiles may have 64 pieces of each; the joins, 256 threads to 8 or more rows, then fit too.
bool few_enough(int64_t tiles) { return tiles < MOST_GROUPS / 64; }

// LDS of a workgroup of k_attention_dq: tiles, the bias, sums of it for every wave, buckets.
constexpr int64_t LDS_BYTES = 160 * 1024;
int64_t dq_lds(const lram_attention& a, int teams) {
  const int64_t tiles = (int64_t)STAGES * 2 * KEYS * a.head_dim * (int64_t)elem_size(a.dtype);
  return teams * tiles + (a.rel_weight ? (2 + teams * WAVES) * (2 * ((int64_t)a.rel_reach + BIAS_PAD) + 1) * 4 : 0);
}

int check_attention(const lram_attention& a, bool pointers) {
  if (a.dtype != LRAM_F32 && a.dtype != LRAM_BF16) return LRAM_EDTYPE;
  if (a.head_dim != 32 && a.head_dim != 64 && a.head_dim != 128) return LRAM_EDTYPE;
  if (a.kv_heads < 1 || a.heads < 1 || a.heads % a.kv_heads || a.heads / a.kv_heads > 64 || a.heads > 65536)
    return LRAM_EINVAL;
  const int64_t G = a.heads / a.kv_heads;
  if (a.batch < 0 || a.batch > 1 << 24 || (a.causal & ~1) || !(a.scale > 0) || !(a.scale < INFINITY))
    return LRAM_EINVAL;
  if (a.tq < 0 || a.tk < 0 || a.tk > 1 << 30 || a.tq > (1 << 30) / G || a.max_q < 0 || a.max_k < 0)
    return LRAM_EINVAL;
  // a grid holds less than 2^32 threads: tiles of 32 rows with a workgroup of 256 each, of 128 rows with one of 512 at most;
  // pieces are made where they fit (few_enough, tiles_of)
  if (a.heads * (std::max(a.tq * G, a.tk) / 32 + a.batch + 3) >= MOST_GROUPS) return LRAM_EINVAL;
  if (a.rel_weight) {
    if (a.wdtype != LRAM_F32 && !(a.wdtype == LRAM_BF16 && a.dtype == LRAM_BF16)) return LRAM_EDTYPE;
    if (!a.rel_bucket || a.rel_buckets < 1 || a.rel_buckets > 256 || a.rel_reach < 0 || a.rel_reach > 4096 ||
        G * (2 * (a.rel_reach + BIAS_PAD) + 1) > 4096 || dq_lds(a, 1) > LDS_BYTES)
      return LRAM_EINVAL;
    if (off_align(a.rel_weight, elem_size(a.wdtype)) || off_align(a.rel_bucket, 4)) return LRAM_EINVAL;
  }
  const int64_t per = 16 / (int64_t)elem_size(a.dtype);
  for (int64_t row : {a.q_row, a.k_row, a.v_row})
    if (row < a.head_dim || row > 1 << 22 || row % per) return LRAM_EINVAL;
  for (int64_t head : {a.q_head, a.k_head, a.v_head})
    if (head < 0 || head > INT64_MAX / 2 / a.heads || head % per) return LRAM_EINVAL;
  if (!pointers) return LRAM_OK;
  if (a.tq && (!a.q || off_align(a.q, 16))) return LRAM_EINVAL;
  if (a.tk && (!a.k || !a.v || off_align(a.k, 16) || off_align(a.v, 16))) return LRAM_EINVAL;
  if (!a.start_q || !a.start_k) return LRAM_EINVAL;
  if (off_align(a.start_q, 4) || off_align(a.start_k, 4) || off_align(a.used_k, 4)) return LRAM_EINVAL;
  return LRAM_OK;
}

Args args_of(const lram_attention& a) {
  Args x{};
  x.q = a.q, x.k = a.k, x.v = a.v;
  x.q_row = a.q_row, x.q_head = a.q_head, x.k_row = a.k_row, x.k_head = a.k_head, x.v_row = a.v_row, x.v_head = a.v_head;
  x.start_q = a.start_q, x.start_k = a.start_k, x.used_k = a.used_k;
  x.rel_weight = a.rel_weight, x.rel_bucket = a.rel_bucket;
  x.tq = a.tq, x.tk = a.tk;
  x.heads = a.heads, x.kv_heads = a.kv_heads, x.ratio = x.group = a.heads / a.kv_heads, x.batch = a.batch;
  x.causal = a.causal, x.buckets = a.rel_buckets, x.reach = a.rel_reach, x.rel_bf16 = a.wdtype == LRAM_BF16;
  x.parts = 1;
  x.scale = a.scale;
  x.c = a.scale * LOG2E;
  return x;
}

// Tiles that a call of expected length `longest` has, of `slots` at most: `rows` in all (packed rows, keys) fill as many as
// they do whatever the sequences' lengths, so that an expectation below them does not lead to pieces of many tiles.
int64_t tiles_of(const lram_attention& a, int64_t longest, int64_t rows, int tile, int64_t slots) {
  return std::min(std::max(a.batch * std::max<int64_t>(1, (longest + tile - 1) / tile), rows / tile), slots);
}

// The call with the expected lengths no longer than the tensors, so that no product of them overflows.
lram_attention bounded(lram_attention a) {
  a.max_q = std::min(a.max_q, a.tq);
  a.max_k = std::min(a.max_k, a.tk);
  return a;
}

// Whether the expected lengths make a batch of like sequences, whose tiles run in rounds over the chip: then as many pieces
// as fill one round (two workgroups a CU) are best, where the pieces of ragged ones, which even out, may be twice as
// many.
constexpr int64_t ROUND = 512;
bool alike(const lram_attention& a) {
  return a.batch * (double)a.max_q <= 1.25 * (double)a.tq && a.max_k <= 2 * a.max_q;
}

// More than 64 KB of a workgroup's LDS has to be asked for, once for a kernel and a device.
int allow_lds(const void* kernel, size_t bytes) {
  if (bytes <= 64 * 1024) return LRAM_OK;
  const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  return e == hipSuccess ? LRAM_OK : layer_failed(e);
}

template <typename F>
int by_kind(const lram_attention& a, F f) {
  const auto width = [&](auto t, auto bias) {
    switch (a.head_dim) {
      case 32: return f(t, std::integral_constant<int, 32>(), bias);
      case 64: return f(t, std::integral_constant<int, 64>(), bias);
      default: return f(t, std::integral_constant<int, 128>(), bias);
    }
  };
  const auto type = [&](auto bias) { return a.dtype == LRAM_F32 ? width(float(), bias) : width(bf16(), bias); };
  return a.rel_weight ? type(std::true_type()) : type(std::false_type());
}

}  // namespace
