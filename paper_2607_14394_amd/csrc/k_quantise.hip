// Rows (and columns) of an array in 8 bits with a power-of-two scale for each
// 128 values (dtst_quantise).  Bound by HBM: x is read once, codes are written
// once.
//
// In both forms 16 lanes hold a row's block of 128 columns, eight neighbouring
// columns each; the row's scale is a maximum within a row of lanes.  For the
// transposed form a workgroup takes 128 x 128 values, a lane 8 x 8 of them: the
// columns' scales are maxima over a lane's rows, lanes and waves, and a lane's
// codes of 8 rows of a column go to LDS as one word, from which each column's 128
// codes are written as one line.  4096 x 2048 bf16 by rows 6.3 us (4.0 TB/s); 4096
// x 4608 bf16 both ways from one reading 22 us (3.4 TB/s), where its vector
// instructions, some 20 a value, take half.
#include <hip/hip_runtime.h>

#include <algorithm>

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

template <class T, bool ROWS>
__global__ void __launch_bounds__(256)
quantise_cols_kernel(dtst_quantise_desc d, const T* __restrict__ x, uint8_t* q, uint8_t* scale, uint8_t* qt,
                     uint8_t* scale_t, int col_tiles) {
  __shared__ uint2 codes[128][16];   // 8 codes of a column each, word w of column c at w ^ (c / 8)
  __shared__ float top[4][128];
  const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
  const int sub = threadIdx.x >> 4, part = threadIdx.x & 15, wave = threadIdx.x >> 6;  // rows 8 sub .., columns 8 part ..
  const int64_t c = ct * 128 + part * 8;
  const int64_t col_blocks = (d.cols + 127) / 128, row_blocks = (d.rows + 127) / 128;
  // (kept as loaded: as 64 floats they would cost a third of the waves)
  typename pack_of<T, 8>::raw v[8];
  if (rt * 128 + 128 <= d.rows && ct * 128 + 128 <= d.cols) {
    const T* at = x + (rt * 128 + sub * 8) * d.ld_x + c;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const pack_t<T, 8>*>(at + i * d.ld_x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = rt * 128 + sub * 8 + i;
      float f[8];
      load_n<8>(x + row * d.ld_x + c, row < d.rows ? d.cols - c : 0, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = T(f[j]);
    }
  }
  const auto column = [&](int j, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = float(v[i][j]);
  };
  float m[8];
  bool infinite = false;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float f[8];
    column(j, f);
    m[j] = max_abs(f);
    infinite = infinite || is_infinite(m[j]);
  }
  if (__any(infinite)) {
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
    if ((threadIdx.x & 48) == 0) top[wave][part * 8 + j] = m[j];
  }
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = rt * 128 + sub * 8 + i;
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = float(v[i][j]);
      uint2 r;
      const uint32_t s = code_block(f, r);
      if (row < d.rows) {
        *reinterpret_cast<uint2*>(q + row * d.ld_q + c) = r;
        if (part == 0) put_scale(scale + row * d.ld_scale, ct, col_blocks, s);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int lc = part * 8 + j;
    const uint32_t s = scale_byte(fmaxf(fmaxf(top[0][lc], top[1][lc]), fmaxf(top[2][lc], top[3][lc])));
    const float inv = scale_inverse(s);
    float f[8];
    column(j, f);
    uint2 r;
    r.x = to_codes(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
    r.y = to_codes(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
    codes[lc][sub ^ part] = r;
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
