// Numbers on their way into 8-bit pools: E4M3 and int8 codes, and quotients by a page's scale, for the kernels that write them.
// Codes are integers decided by float arithmetic, so everything here is one IEEE float32 operation after another, in an order
// that the interface states.
#pragma once

#include "rollattn_internal.h"

namespace rollattn {

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));

constexpr float kE4m3Max = 448.f;
constexpr float kInt8Max = 127.f;
constexpr float kLeastHeadScale = 0x1p-64f;   // of a page and KV head

// (one instruction, the median, where a minimum of a maximum is two; both make -448 of an undefined value)
__device__ __forceinline__ float clamp448(float x) { return __builtin_amdgcn_fmed3f(x, -kE4m3Max, kE4m3Max); }

// four floats -> four E4M3 codes
__device__ __forceinline__ unsigned int encode4_e4m3(const float* x) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x[0]), clamp448(x[1]), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x[2]), clamp448(x[3]), w, true);
  return (unsigned int)w;
}
// eight floats -> eight E4M3 codes
__device__ __forceinline__ uintx2 encode8(const float* x) { return uintx2{encode4_e4m3(x), encode4_e4m3(x + 4)}; }

// Four floats -> four 8-bit integers, nearest even: 1.5 * 2^23 more has units of one in its last place, and whole numbers of
// either sign there in two's complement.
__device__ __forceinline__ unsigned int encode4_int8(const float* x) {
  unsigned int w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(__builtin_amdgcn_fmed3f(x[i], -kInt8Max, kInt8Max) + 0x1.8p23f);
  const unsigned int lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
  return lo | hi;
}

// x / s for many x of one s: ten instructions apiece as the compiler expands an IEEE division.
// All of them share the divisor, so its refined reciprocal is worked out once and each quotient takes
// the remaining steps of that same expansion (product, two residual corrections, a last fused step) and
// the sign of the dividend, which a quotient that rounds to zero would otherwise lose: six
// instructions, and the same correctly rounded result wherever the expansion's operand scaling would
// have done nothing, i.e. for a divisor of moderate magnitude and every quotient large enough to
// matter (one below 2^-10 encodes to zero whatever its last bits).  Divisors outside that range take
// the plain division; MODERATE: there are none, as with scales from kLeastHeadScale up to the largest float over 127.
template <bool MODERATE = false>
struct Quotients {
  float s, r;
  bool fast;
  __device__ __forceinline__ explicit Quotients(float divisor) : s(divisor), fast(MODERATE || (divisor >= 0x1p-100f && divisor <= 0x1p+100f)) {
    const float r0 = __builtin_amdgcn_rcpf(s);
    r = __builtin_fmaf(__builtin_fmaf(-s, r0, 1.f), r0, r0);
  }
  template <int N>
  __device__ __forceinline__ void divide(float (&x)[N]) const {
    if (fast) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float q0 = x[i] * r;
        const float q1 = __builtin_fmaf(__builtin_fmaf(-s, q0, x[i]), r, q0);
        x[i] = __builtin_copysignf(__builtin_fmaf(__builtin_fmaf(-s, q1, x[i]), r, q1), x[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = x[i] / s;
    }
  }
};

// Four codes -> four floats, exactly.
template <bool INT8>
__device__ __forceinline__ void decode4(unsigned int w, float* x) {
  if constexpr (INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(w >> (8 * e));
  } else {
    const floatx2 f0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), f1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = f0[0]; x[1] = f0[1]; x[2] = f1[0]; x[3] = f1[1];
  }
}

// Sixteen codes: the largest magnitude (undefined ones count for nothing), and the codes of the same values under another scale,
// enc(dec(code) * before / now).
template <bool INT8>
__device__ __forceinline__ float largest16(uintx4 w) {
  float m = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float x[4];
    decode4<INT8>(w[k], x);
#pragma unroll
    for (int e = 0; e < 4; ++e) m = fmaxf(m, __builtin_fabsf(x[e]));
  }
  return m;
}
template <bool INT8>
__device__ __forceinline__ uintx4 again16(uintx4 w, float before, float now) {
  const Quotients<false> by(now);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float x[4];
    decode4<INT8>(w[k], x);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= before;
    by.divide(x);
    w[k] = INT8 ? encode4_int8(x) : encode4_e4m3(x);
  }
  return w;
}

}  // namespace rollattn
