// Shared between the translation units of the operators around attention (not part of the public ABI).
#ifndef SPARSE_BLOCK_INTERNAL_H
#define SPARSE_BLOCK_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sparse_attn_internal.h"

namespace sa_block {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
// the same at any multiple of an element's size: the memory instructions take such addresses
typedef bf16x8 __attribute__((aligned(2))) any_bf16x8;
typedef f32x4 __attribute__((aligned(4))) any_f32x4;

// Eight consecutive values as they lie in memory, and as numbers.
template <class T>
struct Pack8;
template <>
struct Pack8<__bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const __bf16* p) { v = *(const bf16x8*)p; }
  __device__ __forceinline__ void load_any(const __bf16* p) { v = *(const any_bf16x8*)p; }
  __device__ __forceinline__ void store_any(__bf16* p) const { *(any_bf16x8*)p = v; }
  __device__ __forceinline__ void load_once(const __bf16* p) { v = __builtin_nontemporal_load((const bf16x8*)p); }
  __device__ __forceinline__ void store_once(__bf16* p) const { __builtin_nontemporal_store(v, (bf16x8*)p); }
  __device__ __forceinline__ void store(__bf16* p) const { *(bf16x8*)p = v; }
  __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
  __device__ __forceinline__ void set(int e, float f) { v[e] = (__bf16)f; }
};
template <>
struct Pack8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ void load_any(const float* p) { a = *(const any_f32x4*)p; b = *(const any_f32x4*)(p + 4); }
  __device__ __forceinline__ void store_any(float* p) const { *(any_f32x4*)p = a; *(any_f32x4*)(p + 4) = b; }
  __device__ __forceinline__ void load_once(const float* p) {
    a = __builtin_nontemporal_load((const f32x4*)p);
    b = __builtin_nontemporal_load((const f32x4*)(p + 4));
  }
  __device__ __forceinline__ void store_once(float* p) const {
    __builtin_nontemporal_store(a, (f32x4*)p);
    __builtin_nontemporal_store(b, (f32x4*)(p + 4));
  }
  __device__ __forceinline__ void store(float* p) const { *(f32x4*)p = a; *(f32x4*)(p + 4) = b; }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e] : b[e - 4]; }
  __device__ __forceinline__ void set(int e, float f) {
    if (e < 4)
      a[e] = f;
    else
      b[e - 4] = f;
  }
};

// Sum / largest over aligned groups of N lanes (N = 4, 8, 16, 32), in every lane of the group.  Data-parallel moves inside a
// row of 16 lanes, which make no trip through LDS; the last step of 32 lanes is a shuffle, which does.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  static_assert(N == 4 || N == 8 || N == 16 || N == 32, "lanes of a group");
  v += moved<0xB1>(v);                        // quad_perm [1,0,3,2]
  v += moved<0x4E>(v);                        // quad_perm [2,3,0,1]
  if (N >= 8) v += moved<0x141>(v);           // row_half_mirror
  if (N >= 16) v += moved<0x140>(v);          // row_mirror
  if (N == 32) v += __shfl_xor(v, 16);
  return v;
}
__device__ __forceinline__ float group16_max(float v) {
  v = fmaxf(v, moved<0xB1>(v));
  v = fmaxf(v, moved<0x4E>(v));
  v = fmaxf(v, moved<0x141>(v));
  return fmaxf(v, moved<0x140>(v));
}
// Sum over the 64 lanes of a wave, wave-uniform.  All lanes have to take part.
__device__ __forceinline__ float wave_sum(float v) {
  v = group_sum<16>(v);
  const int i = __float_as_int(v);
  return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
         (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}

// e4m3 form of a group of 128 values: the exponent e is the least integer >= -126 with amax <= 448 * 2^e (448 = 1.75 * 2^8 is
// the largest e4m3 value), 0 for a group of zeros; stored as the byte e + 127, the scale operand of the matrix instructions.
// amax is over the finite values: an infinity or NaN becomes the e4m3 NaN and leaves its neighbours as they are.
__device__ __forceinline__ int e4m3_exponent(float amax) {
  const unsigned bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return bits == 0 ? 0 : max(e, -126);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.f;
}
// what the conversion below is given for v: an infinity counts as NaN (finite values are at most 448 here)
__device__ __forceinline__ float e4m3_input(float v) { return fabsf(v) < __builtin_inff() ? v : __builtin_nanf(""); }
// four values, already divided by the scale, as four e4m3 bytes (round to nearest, ties to even)
__device__ __forceinline__ int e4m3x4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// A launch has fewer than 2^32 threads along an axis: workgroups beyond kMostBlocks (of up to 1024 threads) go along y.
constexpr long long kMostBlocks = 1 << 21;
inline dim3 grid_of(long long blocks) {
  const long long x = blocks < kMostBlocks ? blocks : kMostBlocks;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ long long block_of() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }     // may be past the last one

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + nb && y < x + na;
}
inline bool finite_nonnegative(float v) { return v >= 0.f && v - v == 0.f; }

}  // namespace sa_block

#endif
