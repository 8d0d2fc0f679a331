// layer_rotary.h -- part of liblram: the angle of a rotary position.
//
// a = 2 pi frac(p u), u turns a token.  A far position loses its angle in fp32 (p = 10^6: 0.06 of a radian), so u is a 64-bit
// fraction and p u is formed modulo 1 in whole numbers: exact to 2^-64 p of a turn, of which the upper 32 bits are used.
// They are cut into the nearest quarter turn and the rest, |r| <= 1/8 turn, whose sine and cosine are their Taylor sums
// (the first terms left out are below 2 10^-9).

#pragma once

#include <type_traits>

#include "../../include/lram_cache.h"
#include "layer_common.h"

namespace {

struct Turn {
  float c, s;  // cosine and sine, times the magnitude
};

// sign: +1, or -1 to turn the other way round.
__device__ __forceinline__ Turn turn_of(int64_t turns, int position, float magnitude, float sign) {
  const uint32_t u = (uint32_t)(((uint64_t)turns * (uint64_t)(int64_t)position) >> 32);
  const uint32_t quarter = (u + (1u << 29)) >> 30;
  const float x = (float)(int32_t)(u - (quarter << 30)) * (float)(6.283185307179586 * 0x1p-32), x2 = x * x;
  const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
  const float c =
      fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
  float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  a = (quarter + 1) & 2 ? -a : a;  // cosine: negative in quarters 1 and 2
  b = quarter & 2 ? -b : b;
  return {a * magnitude, b * magnitude * sign};
}

// How pairs lie in a head: side by side, in halves that are whole 16-byte chunks, in other halves; PLAIN: nothing turns.
enum Form { PLAIN, NEIGHBOURS, HALVES, ODD_HALVES };
inline Form form_of(const lram_rotary& r, int dtype) {
  return r.interleaved ? NEIGHBOURS : r.pairs % (16 / (int)elem_size(dtype)) == 0 ? HALVES : ODD_HALVES;
}

inline int check_rotary(const lram_rotary& r, int64_t head_dim) {
  if (r.pairs < 1 || 2 * (int64_t)r.pairs > head_dim || (r.interleaved & ~1) || !(r.magnitude - r.magnitude == 0))
    return LRAM_EINVAL;
  if (!r.turns || off_align(r.turns, 8)) return LRAM_EINVAL;
  return LRAM_OK;
}

// Rows rotated as they lie.  A thread owns a chunk of a head: 16 bytes of the first halves and their partners, or 16 bytes of
// neighbours.  It forms the chunk's sines and cosines once and goes over heads of its row with them; the threads of a
// wave lie side by side in the row, so that they meet every channel of the L2 (16 rows at a time, 8 KiB apart: 105 -> 132 us
// for 28,654 rows of 32 heads of 128 bf16).
constexpr int ROTATE_THREADS = 256;
constexpr int AT_ONCE = 4;  // heads whose chunks a thread has on their way at once

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
  bool past;        // results go past the caches
};

// A region of a head that is not whole chunks ends in one that overlaps the one before (both write the same values); one
// shorter than a chunk goes element by element.
template <typename T, Form FORM, bool PAST, typename F>
__device__ __forceinline__ void rotate_chunk(const Rotate& a, uint32_t id, F position_of) {
  using C = Chunk<T>;
  constexpr int E = C::E;
  const uint32_t rest = id / (uint32_t)a.chunks;
  const int chunk = (int)(id - rest * (uint32_t)a.chunks);
  const int64_t row = rest / (uint32_t)a.teams;
  if (row >= a.rows) return;
  const int head0 = (int)(rest - (uint32_t)row * (uint32_t)a.teams), all = a.heads + a.kv_heads;
  const int position = position_of(row);
  const auto from = [&](int head) {
    return head < a.heads ? (const T*)a.q + row * a.q_row + head * a.q_head
                          : (const T*)a.k + row * a.k_row + (head - a.heads) * a.k_head;
  };
  const auto to = [&](int head) {
    return head < a.heads ? (T*)a.q_out + (row * a.heads + head) * a.dim
                          : (T*)a.k_out + (row * a.kv_heads + (head - a.heads)) * a.dim;
  };
  bool turned = chunk < a.pair_chunks;
  int first = chunk * E;
  if constexpr (FORM != NEIGHBOURS) {
    const int base = turned ? 0 : 2 * a.pairs, size = turned ? a.pairs : a.dim - 2 * a.pairs;
    first = base + (turned ? chunk : chunk - a.pair_chunks) * E;
    if (FORM == ODD_HALVES && size < E) {
      for (int head = head0; head < all; head += a.teams)
        for (int i = base; i < base + size; ++i) {
          const T* const x = from(head) + i;
          T* const y = to(head) + i;
          if (turned) {
            const Turn t = turn_of(a.turns[i], position, a.magnitude, a.sign);
            const float u = (float)x[0], v = (float)x[a.pairs];
            y[0] = (T)fmaf(u, t.c, -v * t.s);
            y[a.pairs] = (T)fmaf(u, t.s, v * t.c);
          } else {
            y[0] = x[0];
          }
        }
      return;
    }
    if (FORM == ODD_HALVES) first = min(first, base + size - E);
  }
  using V = std::conditional_t<FORM == ODD_HALVES, typename C::loose, typename C::type>;
  constexpr int TURNS = FORM == NEIGHBOURS ? E / 2 : E;
  Turn t[TURNS];
  if (turned) {
#pragma unroll
    for (int e = 0; e < TURNS; ++e) {
      const int pair = FORM == NEIGHBOURS ? first / 2 + e : first + e;
      t[e] = turn_of(a.turns[FORM == NEIGHBOURS ? min(pair, a.pairs - 1) : pair], position, a.magnitude, a.sign);
    }
  }
  const auto put = [](V* at, typename C::type value) {
    if constexpr (PAST)
      __builtin_nontemporal_store((V)value, at);
    else
      *at = value;
  };
  for (int head1 = head0; head1 < all; head1 += AT_ONCE * a.teams) {
    typename C::type x[AT_ONCE], z[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {  // all of them on their way before the first is stored
      const int head = min(head1 + j * a.teams, all - 1);
      x[j] = *(const V*)(from(head) + first);
      if (FORM != NEIGHBOURS && turned) z[j] = *(const V*)(from(head) + a.pairs + first);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int head = head1 + j * a.teams;
      if (head >= all) break;
      if (turned) {
        typename C::wide f = C::up(x[j]), g;
        if constexpr (FORM == NEIGHBOURS) {
#pragma unroll
          for (int e = 0; e < E / 2; ++e) {
            const float u = f[2 * e], v = f[2 * e + 1];
            const bool turns = first / 2 + e < a.pairs;
            f[2 * e] = turns ? fmaf(u, t[e].c, -v * t[e].s) : u;
            f[2 * e + 1] = turns ? fmaf(u, t[e].s, v * t[e].c) : v;
          }
        } else {
          g = C::up(z[j]);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float u = f[e], v = g[e];
            f[e] = fmaf(u, t[e].c, -v * t[e].s);
            g[e] = fmaf(u, t[e].s, v * t[e].c);
          }
          put((V*)(to(head) + a.pairs + first), C::down(g));
        }
        x[j] = C::down(f);
      }
      put((V*)(to(head) + first), x[j]);
    }
  }
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

// Results that the L2s cannot hold go past them (16,384 rows of 32/8 heads of 128 bf16, two sets of data in turn: 66 -> 62 us).
constexpr int64_t CACHED_BYTES = 32 << 20;

// What a thread does where rows are rotated as they lie; the threads of a row.
inline int64_t divide(Rotate& a, const lram_rotary& r, int dtype) {
  const int per = 16 / (int)elem_size(dtype), turned = r.interleaved ? 2 * r.pairs : r.pairs;
  a.turns = r.turns, a.pairs = r.pairs, a.magnitude = r.magnitude, a.sign = 1.0f;
  a.pair_chunks = (turned + per - 1) / per;
  a.chunks = r.interleaved ? a.dim / per : a.pair_chunks + (a.dim - 2 * r.pairs + per - 1) / per;
  a.past = a.rows * (a.heads + a.kv_heads) * a.dim * (int64_t)elem_size(dtype) > CACHED_BYTES;
  a.teams = teams_of(a.rows, a.chunks, a.heads + a.kv_heads);
  return (int64_t)a.chunks * a.teams;
}

}  // namespace
