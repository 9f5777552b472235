// Device helpers of the latent-sequence operators: element types, vector
// access at any alignment, wave reductions, 8-bit codes and their scales.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dtst.h"

namespace dtst {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// N elements of T at the alignment of T.  gfx950 takes 16-byte accesses at any
// alignment of global memory, so odd strides and column ranges keep the wide
// form.
template <class T, int N>
struct pack_of {
  typedef T raw __attribute__((ext_vector_type(N)));
  typedef raw type __attribute__((aligned(alignof(T))));
};
template <class T, int N>
using pack_t = typename pack_of<T, N>::type;

// p[0..N) as floats; entries from n on are zero and not read.
template <int N, class T>
__device__ __forceinline__ void load_n(const T* p, int64_t n, float (&out)[N]) {
  if (n >= N) {
    const pack_t<T, N> v = *reinterpret_cast<const pack_t<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = i < n ? float(p[i]) : 0.f;
  }
}

template <int N, class T>
__device__ __forceinline__ void store_n(T* p, int64_t n, const float (&v)[N]) {
  if (n >= N) {
    typename pack_of<T, N>::raw r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = T(v[i]);
    *reinterpret_cast<pack_t<T, N>*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = T(v[i]);
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
  return v;
}

// Orders a wave's LDS accesses before this point with those of its other lanes
// after it (no instruction: a wave's LDS accesses stay in order).
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The value of lane ^ partner within 16 lanes, rotated by R (1, 2, 4 or 8).
template <int R>
__device__ __forceinline__ float row_rotate(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + R, 0xf, 0xf, false));
}

// Largest of the 16 lanes of a row of lanes.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, row_rotate<1>(v));
  v = fmaxf(v, row_rotate<2>(v));
  v = fmaxf(v, row_rotate<4>(v));
  return fmaxf(v, row_rotate<8>(v));
}

// Largest magnitude of a lane's values; no numbers do not count, infinities do.
template <int N>
__device__ __forceinline__ float max_abs(const float (&v)[N]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}
// The same of the finite values alone.
template <int N>
__device__ float max_finite_abs(const float (&v)[N]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(v[i]) <= 3.402823466e38f ? fabsf(v[i]) : 0.f);
  return m;
}
__device__ __forceinline__ bool is_infinite(float m) { return m > 3.402823466e38f; }

// The scale byte of a block whose largest magnitude is amax >= 0: the smallest
// power of two 2^e, e >= -126, with amax <= 448 * 2^e; 448 = 1.75 * 2^8, so e is
// amax's exponent less 8, one more when its significand is above 1.75.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = int(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return amax == 0.f ? 127u : uint32_t(e < 1 ? 1 : e);
}

// 2^(s - 127), s = 1 .. 254.
__device__ __forceinline__ float scale_float(uint32_t s) { return __uint_as_float(s << 23); }

// Values over a scale that leaves them at most 448, infinities or no numbers, to
// codes, nearest even, one rounding; the last two become the code of no number.
// (The conversion divides by the scale's power of two; what it gives is what a
// division in 32 bits and a conversion give, measured for all 16-bit values.)
typedef short code_pairs __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d, float scale) {
  code_pairs r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// The same of two words of two 16-bit values.
template <class T>
__device__ __forceinline__ uint32_t to_codes(uint32_t ab, uint32_t cd, float scale) {
  typedef T pair __attribute__((ext_vector_type(2)));
  const pair p = __builtin_bit_cast(pair, ab), q = __builtin_bit_cast(pair, cd);
  code_pairs r = {0, 0};
  if constexpr (std::is_same_v<T, bf16_t>) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, p, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, q, scale, true);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, p, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, q, scale, true);
  }
  return __builtin_bit_cast(uint32_t, r);
}

// A block of 128 values, eight a lane in 16 lanes: the lane's codes, and the
// block's scale byte.  (All lanes of the wave take part.)
__device__ __forceinline__ uint32_t code_block(const float (&v)[8], uint2& q) {
  float m = row_max(max_abs(v));
  if (__any(is_infinite(m))) m = row_max(max_finite_abs(v));
  const uint32_t s = scale_byte(m);
  const float scale = scale_float(s);
  q.x = to_codes(v[0], v[1], v[2], v[3], scale);
  q.y = to_codes(v[4], v[5], v[6], v[7], scale);
  return s;
}

}  // namespace dtst
