// layer_common.h -- part of liblram: what the operators of the layer around the memory share.

#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lram_layer.h"

// Records an error for lram_layer_last_hip_error: a call's, or that of the launch before.
int layer_failed(hipError_t e);
int layer_launched();

namespace {

constexpr int WAVE = 64;

using bf16 = __bf16;

// N consecutive elements, loaded and stored whole.  Rows of odd sizes start on any element: the type promises no
// alignment beyond an element's (the memory system takes such vectors).
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Packed {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, float (&f)[N]) {
  const auto a = *reinterpret_cast<const Packed<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = (float)a.v[i];
}

template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&f)[N]) {
  Packed<T, N> a;
#pragma unroll
  for (int i = 0; i < N; ++i) a.v[i] = (T)f[i];
  *reinterpret_cast<Packed<T, N>*>(p) = a;
}

// 16 bytes of elements as one value, so that they are moved by one instruction; `loose` where they start on any element.
template <typename T>
struct Chunk {
  static constexpr int E = 16 / (int)sizeof(T);
  typedef T type __attribute__((ext_vector_type(E)));
  typedef T loose __attribute__((ext_vector_type(E), aligned(sizeof(T))));
  typedef float wide __attribute__((ext_vector_type(E)));
  static __device__ __forceinline__ wide up(type x) { return __builtin_convertvector(x, wide); }
  static __device__ __forceinline__ type down(wide x) { return __builtin_convertvector(x, type); }
};

// The sum of x over the wave, the same in every lane (a tree of fixed shape).
__device__ __forceinline__ float wave_sum(float x) {
#define LRAM_DPP_ADD(ctrl, rows) \
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), ctrl, rows, 0xf, true))
  LRAM_DPP_ADD(0x111, 0xf);  // shift right by 1, 2, 4, 8 inside each row of 16 lanes
  LRAM_DPP_ADD(0x112, 0xf);
  LRAM_DPP_ADD(0x114, 0xf);
  LRAM_DPP_ADD(0x118, 0xf);
  LRAM_DPP_ADD(0x142, 0xa);  // lane 15 of a row into the next row
  LRAM_DPP_ADD(0x143, 0xc);  // lane 31 into rows 2 and 3
#undef LRAM_DPP_ADD
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Orders LDS traffic between the lanes of one wave: its LDS operations execute in the order of their issue, so that the compiler
// is all there is to hold back.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr float LOG2E = 1.4426950408889634f;

// A bias's weights far past any score.  From 2^24 on (a weight of 1.2e7, times log2 e) fp32 holds no digit behind the point,
// so that scores beside such a weight say nothing, and times log2 e the type's lowest value, a common mask, would be -inf,
// which hides a key altogether.  Finite weights from there on all count as +-2^126: a score added to it leaves it as it is,
// and a row that meets no other keys (or one that meets keys of +2^126) has the even average of those.
constexpr float FAR_WEIGHT = 0x1p24f, VAST = 0x1p126f;
__device__ __forceinline__ float in_log2(float weight) {
  const float t = weight * LOG2E;
  return fabsf(t) >= FAR_WEIGHT && fabsf(weight) < INFINITY ? copysignf(VAST, weight) : t;
}

inline bool off_align(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline uintptr_t elem_size(int dtype) { return dtype == LRAM_BF16 ? 2 : 4; }

}  // namespace
