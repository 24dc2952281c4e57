// What the attention kernels share: vector types, matrix products of one wave, the
// order of key rows in LDS, barriers, stores.
#pragma once

#include "decoder.h"

namespace d2moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline f4 mma(u4 a, u4 b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));  // the result gets registers of its own
  return d;
}
__device__ inline f4 mma(float a, float b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));
  return d;
}

// Key rows of CPR 16-byte chunks in LDS: chunk c of row r lies at r CPR + (c ^
// swizzle(r)), so that 16 lanes meet 16 different bank groups both writing (one row) and
// reading (16 rows, one c).
template <int CPR>
__device__ inline int swizzle(int row) {
  return CPR >= 16 ? row & 15 : (row >> 1) & 7;
}

// A barrier for LDS alone: a full one would also wait for the loads under way.
__device__ inline void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// LDS between the lanes of a wave.
__device__ inline void wave_handoff() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four values of a result row.
template <typename T>
__device__ inline void store4(T* p, f4 v) {
  if constexpr (sizeof(T) == 2)
    *(uint2*)p = make_uint2(f2bf(v[0]) | (uint32_t)f2bf(v[1]) << 16,
                            f2bf(v[2]) | (uint32_t)f2bf(v[3]) << 16);
  else
    *(f4*)p = v;
}

}  // namespace
}  // namespace d2moe
