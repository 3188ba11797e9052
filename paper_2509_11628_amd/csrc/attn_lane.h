// What the attention kernels share at the level of a lane: packed conversions, exponentials, and the reductions over the lanes that hold
// one query of a transposed 16x16 tile (l % 16, in the four groups l / 16).
#pragma once

#include "common.h"

namespace speca {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

// two floats -> packed bf16 pair, round to nearest even, NaN stays NaN (one v_cvt_pk_bf16_f32)
__device__ inline uint32_t cvt_pk_bf16(float a, float b) {
  const floatx2 f = {a, b};
  const bf16x2 r = __builtin_convertvector(f, bf16x2);
  return *reinterpret_cast<const uint32_t*>(&r);
}

// 2^x by the hardware instruction alone (inputs are <= 0 here; results below the normal range flush
// to 0, -inf gives 0): exp2f() wraps it in range checks and a rescale, ~5 vector instructions per value.
__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// maximum and sum over the lanes l % 16 + {0, 16, 32, 48}, which hold one query
__device__ __forceinline__ float max_of_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_of_groups(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// four bf16 values at a time: which are infinite or NaN (0x8000 and 0x80000000 of each word), and the words without them
__device__ inline uint32_t odd_halves(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ inline uint32_t without_odd(uint32_t w) { return w & ~((odd_halves(w) >> 15) * 0xFFFFu); }

}  // namespace speca
