// Rows (and columns) of an array in 8 bits with a power-of-two scale for each
// 128 values (dtst_quantise).  Bound by HBM: x is read once, codes are written
// once.
//
// In both forms 16 lanes hold a row's block of 128 columns, eight neighbouring
// columns each; the row's scale is a maximum within a row of lanes.  For the
// transposed form a workgroup takes 128 x 128 values, a lane 8 x 8 of them: the
// columns' scales are maxima over a lane's rows, lanes and waves, and a lane's
// codes of 8 rows of a column go to LDS as one word, from which each column's 128
// codes are written as one line.  bf16: 4096 x 2048 by rows 5.7 us (4.4 TB/s);
// 4096 x 4608 by rows 10.7, by columns 11.4, both from one reading 21.3 us (3.6
// TB/s: all workgroups are there at once, so that the card first reads, then
// writes; 8192 x 8192: 59 us, 4.5 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

// Scale byte `block` of a row of scales, and after the last one the bytes up to
// a multiple of four.
__device__ __forceinline__ void put_scale(uint8_t* row, int64_t block, int64_t blocks, uint32_t s) {
  row[block] = uint8_t(s);
  if (block == blocks - 1)
    for (int64_t b = blocks; b < (blocks + 3) / 4 * 4; ++b) row[b] = 127;
}

// Rows alone: a block of 128 for every 16 lanes.
template <class T>
__global__ void __launch_bounds__(256)
quantise_rows_kernel(dtst_quantise_desc d, const T* __restrict__ x, uint8_t* q, uint8_t* scale, uint32_t col_blocks) {
  const uint32_t id = blockIdx.x * 16 + (threadIdx.x >> 4), part = threadIdx.x & 15;
  const uint32_t block = id % col_blocks;
  const int64_t row = id / col_blocks, c = int64_t(block) * 128 + part * 8;
  float v[8];
  load_n<8>(x + row * d.ld_x + c, row < d.rows ? d.cols - c : 0, v);
  uint2 codes;
  const uint32_t s = code_block(v, codes);
  if (row >= d.rows) return;
  *reinterpret_cast<uint2*>(q + row * d.ld_q + c) = codes;
  if (part == 0) put_scale(scale + row * d.ld_scale, block, col_blocks, s);
}

// The maxima of a tile's blocks and the codes of a lane's 8 x 8 values.
// 16-bit types: magnitudes compare as integers, two at a time, and the conversion
// takes pairs as they are.
template <class T>
struct Values {
  static constexpr uint32_t kInfinity = std::is_same_v<T, bf16_t> ? 0x7f80 : 0x7c00;
  typedef uint16_t halves __attribute__((ext_vector_type(2)));
  uint32_t w[8][4];  // rows of four words
  bool finite;       // all of the wave's (else infinities and no numbers count for nothing)

  __device__ static uint32_t larger(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(halves, a), __builtin_bit_cast(halves, b)));
  }
  __device__ static float value(uint32_t half) {
    if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(half << 16);
    else return float(__builtin_bit_cast(_Float16, uint16_t(half)));
  }
  __device__ uint32_t magnitude(int i, int k) const {
    const uint32_t a = w[i][k] & 0x7fff7fffu;
    if (finite) return a;
    return ((a & 0xffffu) < kInfinity ? a & 0xffffu : 0) | ((a >> 16) < kInfinity ? a & 0xffff0000u : 0);
  }

  __device__ void set(int i, typename pack_of<T, 8>::raw v) { __builtin_memcpy(w[i], &v, 16); }
  __device__ void largest(uint32_t (&m)[4]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = magnitude(0, k);
#pragma unroll
      for (int i = 1; i < 8; ++i) m[k] = larger(m[k], magnitude(i, k));
    }
  }
  // The largest magnitudes of the columns, to `top` of the wave.
  __device__ void columns(uint32_t* top, int part) {
    uint32_t m[4];
    finite = true;
    largest(m);
    const uint32_t all = larger(larger(m[0], m[1]), larger(m[2], m[3]));
    finite = !__any(max(all & 0xffffu, all >> 16) >= kInfinity);
    if (!finite) largest(m);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = larger(m[k], __shfl_xor(m[k], 16, 64));
      m[k] = larger(m[k], __shfl_xor(m[k], 32, 64));
      if ((threadIdx.x & 48) == 0) top[part * 4 + k] = m[k];
    }
  }
  static constexpr int kTop = 64;  // words of a wave
  __device__ uint32_t column_scale(const uint32_t (*top)[kTop], int part, int j) const {
    const int k = part * 4 + j / 2;
    const uint32_t m = larger(larger(top[0][k], top[1][k]), larger(top[2][k], top[3][k]));
    return scale_byte(value(j % 2 ? m >> 16 : m & 0xffffu));
  }
  __device__ uint2 column_codes(int j, float scale) const {
    const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;  // the same half of two rows
    const int k = j / 2;
    const auto two = [&](int i) { return __builtin_amdgcn_perm(w[i + 1][k], w[i][k], pick); };
    return uint2{to_codes<T>(two(0), two(2), scale), to_codes<T>(two(4), two(6), scale)};
  }
  __device__ uint32_t row(int i, uint2& codes) const {
    const uint32_t m = larger(larger(magnitude(i, 0), magnitude(i, 1)), larger(magnitude(i, 2), magnitude(i, 3)));
    const uint32_t s = scale_byte(row_max(value(max(m & 0xffffu, m >> 16))));
    const float scale = scale_float(s);
    codes = uint2{to_codes<T>(w[i][0], w[i][1], scale), to_codes<T>(w[i][2], w[i][3], scale)};
    return s;
  }
};

template <>
struct Values<float> {
  typename pack_of<float, 8>::raw v[8];

  __device__ void column(int j, float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v[i][j];
  }
  __device__ void set(int i, typename pack_of<float, 8>::raw r) { v[i] = r; }
  __device__ void columns(uint32_t* top, int part) {
    float m[8], all = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float f[8];
      column(j, f);
      m[j] = max_abs(f);
      all = fmaxf(all, m[j]);
    }
    if (__any(is_infinite(all))) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float f[8];
        column(j, f);
        m[j] = max_finite_abs(f);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = fmaxf(m[j], __shfl_xor(m[j], 16, 64));
      m[j] = fmaxf(m[j], __shfl_xor(m[j], 32, 64));
      if ((threadIdx.x & 48) == 0) top[part * 8 + j] = __float_as_uint(m[j]);
    }
  }
  static constexpr int kTop = 128;
  __device__ uint32_t column_scale(const uint32_t (*top)[kTop], int part, int j) const {
    const int k = part * 8 + j;
    return scale_byte(__uint_as_float(max(max(top[0][k], top[1][k]), max(top[2][k], top[3][k]))));  // (none is negative)
  }
  __device__ uint2 column_codes(int j, float scale) const {
    float f[8];
    column(j, f);
    return uint2{to_codes(f[0], f[1], f[2], f[3], scale), to_codes(f[4], f[5], f[6], f[7], scale)};
  }
  __device__ uint32_t row(int i, uint2& codes) const {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = v[i][j];
    return code_block(f, codes);
  }
};

template <class T, bool ROWS>
__global__ void __launch_bounds__(256)
quantise_cols_kernel(dtst_quantise_desc d, const T* __restrict__ x, uint8_t* q, uint8_t* scale, uint8_t* qt,
                     uint8_t* scale_t, int col_tiles) {
  __shared__ uint2 codes[128][16];   // 8 codes of a column each, word w of column c at w ^ (c / 8)
  __shared__ uint32_t top[4][Values<T>::kTop];
  const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
  const int sub = threadIdx.x >> 4, part = threadIdx.x & 15, wave = threadIdx.x >> 6;  // rows 8 sub .., columns 8 part ..
  const int64_t c = ct * 128 + part * 8;
  const int64_t col_blocks = (d.cols + 127) / 128, row_blocks = (d.rows + 127) / 128;
  Values<T> v;
  if (rt * 128 + 128 <= d.rows && ct * 128 + 128 <= d.cols) {
    const T* at = x + (rt * 128 + sub * 8) * d.ld_x + c;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const typename pack_of<T, 8>::raw r = *reinterpret_cast<const pack_t<T, 8>*>(at + i * d.ld_x);
      v.set(i, r);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = rt * 128 + sub * 8 + i;
      float f[8];
      load_n<8>(x + row * d.ld_x + c, row < d.rows ? d.cols - c : 0, f);
      typename pack_of<T, 8>::raw r;
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] = T(f[j]);
      v.set(i, r);
    }
  }
  v.columns(top[wave], part);
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = rt * 128 + sub * 8 + i;
      uint2 r;
      const uint32_t s = v.row(i, r);
      if (row < d.rows) {
        *reinterpret_cast<uint2*>(q + row * d.ld_q + c) = r;
        if (part == 0) put_scale(scale + row * d.ld_scale, ct, col_blocks, s);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t s = v.column_scale(top, part, j);
    codes[part * 8 + j][sub ^ part] = v.column_codes(j, scale_float(s));
    if (sub == 0 && c + j < d.cols) put_scale(scale_t + (c + j) * d.ld_scale_t, rt, row_blocks, s);
  }
  __syncthreads();
  // 8 lanes a column, two words each
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int lc = i * 32 + (threadIdx.x >> 3), pair = threadIdx.x & 7, p = lc >> 3;
    const uint4 two = *reinterpret_cast<const uint4*>(&codes[lc][(pair ^ (p >> 1)) * 2]);
    const int64_t col = ct * 128 + lc;
    if (col < d.cols)
      *reinterpret_cast<uint4*>(qt + col * d.ld_qt + rt * 128 + pair * 16) =
          (p & 1) ? uint4{two.z, two.w, two.x, two.y} : two;
  }
}

template <class T>
int launch(const dtst_quantise_desc& d, const void* x, void* q, void* scale, void* qt, void* scale_t, hipStream_t s) {
  const int64_t ct = (d.cols + 127) / 128, rt = (d.rows + 127) / 128;
  const T* xt = static_cast<const T*>(x);
  uint8_t *q8 = static_cast<uint8_t*>(q), *s8 = static_cast<uint8_t*>(scale);
  if (qt == nullptr) {
    hipLaunchKernelGGL(quantise_rows_kernel<T>, dim3(unsigned((d.rows * ct + 15) / 16)), dim3(256), 0, s, d, xt, q8, s8,
                       uint32_t(ct));
  } else {
    auto* fn = q == nullptr ? quantise_cols_kernel<T, false> : quantise_cols_kernel<T, true>;
    hipLaunchKernelGGL(fn, dim3(unsigned(ct * rt)), dim3(256), 0, s, d, xt, q8, s8, static_cast<uint8_t*>(qt),
                       static_cast<uint8_t*>(scale_t), int(ct));
  }
  return hipGetLastError();
}

}  // namespace

int launch_quantise(const dtst_quantise_desc& d, const void* x, void* q, void* scale, void* qt, void* scale_t,
                    void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.type == DTST_F32) return launch<float>(d, x, q, scale, qt, scale_t, s);
  if (d.type == DTST_BF16) return launch<bf16_t>(d, x, q, scale, qt, scale_t, s);
  return launch<f16_t>(d, x, q, scale, qt, scale_t, s);
}

}  // namespace dtst
