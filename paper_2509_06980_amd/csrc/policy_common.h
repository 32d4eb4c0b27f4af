// What the policy-update operators share: element access by type, checks of their C entry points.
#pragma once
#include "../../include/rl_rollout.h"
#include "kernels.h"

// N consecutive elements as one aligned access where N > 1 (16 bytes: 8 bf16 or 4 floats), widened to 32 bits.
template <int N>
__device__ __forceinline__ void ldv(const float* p, float (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = *p;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) ld4(p + i, v[i], v[i + 1], v[i + 2], v[i + 3]);
  }
}
template <int N>
__device__ __forceinline__ void ldv(const bf16_t* p, float (&v)[N]) {
  if constexpr (N == 1) {
    v[0] = bf2f(*p);
  } else {
    static_assert(N == 8, "16 bytes");
    const u32x4 q = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = bf2f((bf16_t)(q[i] & 0xffffu));
      v[2 * i + 1] = bf2f((bf16_t)(q[i] >> 16));
    }
  }
}
// bf16 of a float, to nearest even; NaN stays NaN (f2bf's rounding carry could turn one into infinity or zero).
__device__ __forceinline__ bf16_t to_bf16(float f) { return __builtin_bit_cast(bf16_t, (__bf16)f); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(bf16_t* p, float v) { *p = to_bf16(v); }
template <int N>
__device__ __forceinline__ void stv(float* p, const float (&v)[N]) {
  if constexpr (N == 1) {
    *p = v[0];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) *(float4*)(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  }
}
template <int N>
__device__ __forceinline__ void stv(bf16_t* p, const float (&v)[N]) {
  if constexpr (N == 1) {
    *p = to_bf16(v[0]);
  } else {
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; i++) q[i] = (uint32_t)to_bf16(v[2 * i]) | ((uint32_t)to_bf16(v[2 * i + 1]) << 16);
    *(u32x4*)p = q;
  }
}

static inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
static inline int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
// Workgroups that one launch takes along a grid's first dimension: its threads are counted in 32 bits, and a launch of more runs some
// of them and reports no error.
constexpr int64_t most_workgroups(int threads) { return ((1ll << 32) - 1) / threads; }
// What a C entry point returns after its launches.
static inline int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? RL_OK : rl_fail(RL_E_HIP, hipGetErrorString(e));
}
