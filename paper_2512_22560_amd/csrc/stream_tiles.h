// What the kernels that stream K and V rows through tiles in LDS share: a tile's layout, codes to operands, small steps across lanes.
#pragma once

#include <type_traits>

#include "plan_device.h"

namespace rollattn {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef int intx2 __attribute__((ext_vector_type(2)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));

typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));

constexpr float kMostBits = 15.f;     // f16 weights: log2 of the most that rounding may make of the largest
constexpr int kQueryBits = 15;        // f16 queries: the largest is below two to this

template <int D, bool FP8>
struct Geo {
  static constexpr int kRowBytes = D * (FP8 ? 1 : 2);
  static constexpr int kChunks = kRowBytes / 16;          // 16-byte chunks per token row
  static constexpr int kRowsPerLoad = 64 / kChunks;        // token rows one wave-wide load covers
  static constexpr int kLoads = kBlockTokens / kRowsPerLoad;  // loads per block, per pool
  static constexpr int kTileBytes = kBlockTokens * kRowBytes; // LDS bytes per block, per pool
  static_assert(kRowsPerLoad <= 16 && 16 % kRowsPerLoad == 0, "a load must stay inside one page");
};

__device__ __forceinline__ float xor32_max(float x) {
  uintx2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor32_add(float x) {
  uintx2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Eight E4M3 codes to bf16, exactly: the scaled conversion with a scale of one, two codes per instruction.
__device__ __forceinline__ bf16x8 fp8x8_to_bf16(uint32_t lo, uint32_t hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  bf16x8 r;
  r[0] = a[0]; r[1] = a[1]; r[2] = b[0]; r[3] = b[1];
  r[4] = c[0]; r[5] = c[1]; r[6] = d[0]; r[7] = d[1];
  return r;
}

__device__ __forceinline__ halfx8 fp8x8_to_f16(uint32_t lo, uint32_t hi) {
  const halfx2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
  const halfx2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const halfx2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
  const halfx2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return halfx8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight 8-bit integers to f16, exactly: with the sign turned round a byte counts from -128 up, as the low bits of 1024.0 it adds
// itself to that, and 1152 less is the value.  (Left out for keys and taken off the scores instead: 73.0 -> 72.6 us, not worth it.)
__device__ __forceinline__ halfx8 int8x8_to_f16(uint32_t lo, uint32_t hi) {
  lo ^= 0x80808080u;
  hi ^= 0x80808080u;
  const halfx2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
  const halfx2 a = __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) + off;
  const halfx2 b = __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) + off;
  const halfx2 c = __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) + off;
  const halfx2 d = __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) + off;
  return halfx8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight codes as an operand of the first or second product.
template <int KV>
__device__ __forceinline__ auto widen_k8(uint32_t lo, uint32_t hi) {
  if constexpr (KV == kKvInt8Head) return int8x8_to_f16(lo, hi);
  else return fp8x8_to_bf16(lo, hi);
}
template <int KV>
__device__ __forceinline__ auto widen_v8(uint32_t lo, uint32_t hi) {
  if constexpr (KV == kKvFp8Head) return fp8x8_to_f16(lo, hi);
  else if constexpr (KV == kKvInt8Head) return int8x8_to_f16(lo, hi);
  else return fp8x8_to_bf16(lo, hi);
}

// (worked out where it is used: the thread's index would take a register over the whole of a worker's rows)
__device__ __forceinline__ int lane_id() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)); }

}  // namespace

}  // namespace rollattn
