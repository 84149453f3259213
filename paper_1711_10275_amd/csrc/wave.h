// Reductions over the 64 lanes of a wavefront whose result every lane of the
// group holds, without LDS: exchanges within rows of 16 lanes are data-
// parallel-primitive moves, those across rows are the lane swaps of gfx950.
// The order is fixed, so sums are reproducible.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace sscn {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kQuadXor1 = 0xb1, kQuadXor2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;

struct OpAdd {
  __device__ static float of(float a, float b) { return a + b; }
};
struct OpMax {  // NaN if either is
  __device__ static float of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
};
struct OpMin {
  __device__ static float of(float a, float b) { return fminf(a, b); }
};

// Over groups of 2 * FROM .. TO lanes, v uniform in groups of FROM lanes before.
template <class Op, int FROM = 1, int TO = 64>
__device__ __forceinline__ float wave_reduce(float v) {
  const auto f = [](uint32_t b) { return __uint_as_float(b); };
  if constexpr (FROM < 2 && TO >= 2) v = Op::of(v, f(dpp<kQuadXor1>(__float_as_uint(v))));
  if constexpr (FROM < 4 && TO >= 4) v = Op::of(v, f(dpp<kQuadXor2>(__float_as_uint(v))));
  if constexpr (FROM < 8 && TO >= 8) v = Op::of(v, f(dpp<kMirror8>(__float_as_uint(v))));
  if constexpr (FROM < 16 && TO >= 16) v = Op::of(v, f(dpp<kMirror16>(__float_as_uint(v))));
  if constexpr (FROM < 32 && TO >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = Op::of(f(r[0]), f(r[1]));
  }
  if constexpr (FROM < 64 && TO >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = Op::of(f(r[0]), f(r[1]));
  }
  return v;
}

// How many of the other 15 lanes of this lane's row hold an `of` above v.
template <int N = 1>
__device__ __forceinline__ int above_in_row(float of, float v) {
  if constexpr (N == 16) {
    return 0;
  } else {
    constexpr int kRotate = 0x120 + N;  // the value N lanes away
    return (__uint_as_float(dpp<kRotate>(__float_as_uint(of))) > v ? 1 : 0) + above_in_row<N + 1>(of, v);
  }
}

// Of the other 15 lanes of this lane's row that hold this lane's key: the sum
// of their v, and whether one of them is a lower lane.
struct Same {
  float sum;
  bool before;
};
template <int N = 1>
__device__ __forceinline__ Same same_in_row(int key, float v) {
  if constexpr (N == 16) {
    return {0.f, false};
  } else {
    constexpr int kRotate = 0x120 + N;
    const int lane = (int)threadIdx.x & 15;
    const float other = __uint_as_float(dpp<kRotate>(__float_as_uint(v)));
    const bool same = (int)dpp<kRotate>((uint32_t)key) == key;
    const bool lower = (int)dpp<kRotate>((uint32_t)lane) < lane;
    const Same rest = same_in_row<N + 1>(key, v);
    return {(same ? other : 0.f) + rest.sum, (same && lower) || rest.before};
  }
}

// The largest of the 64-bit keys of L lanes (16 or 64).
__device__ __forceinline__ uint64_t key_max(uint64_t a, uint32_t lo, uint32_t hi) {
  const uint64_t b = (uint64_t)hi << 32 | lo;
  return a > b ? a : b;
}
template <int L = 64>
__device__ __forceinline__ uint64_t wave_max_key(uint64_t v) {
#define SSCN_KEY_STEP(C) v = key_max(v, dpp<C>((uint32_t)v), dpp<C>((uint32_t)(v >> 32)))
  SSCN_KEY_STEP(kQuadXor1);
  SSCN_KEY_STEP(kQuadXor2);
  SSCN_KEY_STEP(kMirror8);
  SSCN_KEY_STEP(kMirror16);
#undef SSCN_KEY_STEP
  if constexpr (L > 16) {
    const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    v = key_max((uint64_t)hi[0] << 32 | lo[0], lo[1], hi[1]);
  }
  if constexpr (L > 32) {
    const auto lo = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap((uint32_t)(v >> 32), (uint32_t)(v >> 32), false, false);
    v = key_max((uint64_t)hi[0] << 32 | lo[0], lo[1], hi[1]);
  }
  return v;
}

}  // namespace sscn
