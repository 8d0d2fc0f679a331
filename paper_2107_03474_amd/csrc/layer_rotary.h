// layer_rotary.h -- part of liblram: the angle of a rotary position.
//
// a = 2 pi frac(p u), u turns a token.  A far position loses its angle in fp32 (p = 10^6: 0.06 of a radian), so u is a 64-bit
// fraction and p u is formed modulo 1 in whole numbers: exact to 2^-64 p of a turn, of which the upper 32 bits are used.
// They are cut into the nearest quarter turn and the rest, |r| <= 1/8 turn, whose sine and cosine are their Taylor sums
// (the first terms left out are below 2 10^-9).

#pragma once

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

inline int check_rotary(const lram_rotary& r, int64_t head_dim) {
  if (r.pairs < 1 || 2 * (int64_t)r.pairs > head_dim || (r.interleaved & ~1) || !(r.magnitude - r.magnitude == 0))
    return LRAM_EINVAL;
  if (!r.turns || off_align(r.turns, 8)) return LRAM_EINVAL;
  return LRAM_OK;
}

}  // namespace
