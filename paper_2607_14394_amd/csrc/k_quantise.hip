// Rows (and columns) of an array in 8 bits with a power-of-two scale for each
// 128 values (dtst_quantise).  Bound by HBM: x is read once, codes are written
// once.
//
// A workgroup takes 128 x 128 values.  For the rows' form, 16 lanes hold a
// row's block of 128, eight neighbouring columns each, and its scale is a
// maximum within a row of lanes.  For the transposed form the tile goes through
// LDS: a lane then holds 8 rows of a column, and 16 lanes its 128.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

// LDS pitch of a tile row in floats: the transposed read takes 8 rows of one
// column per lane, 16 lanes a column and 4 columns a wave.
constexpr int PITCH = 129;

__device__ __forceinline__ uint32_t code_block(const float (&v)[8], uint2& q) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fmaxf(m, finite_abs(v[j]));
  const uint32_t s = scale_byte(row_max(m));
  const float inv = scale_inverse(s);
  q.x = to_codes(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  q.y = to_codes(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
  return s;
}

// Scale byte `block` of a row of scales, and after the last one the bytes up to
// a multiple of four.
__device__ __forceinline__ void put_scale(uint8_t* row, int64_t block, int64_t blocks, uint32_t s) {
  row[block] = uint8_t(s);
  if (block == blocks - 1)
    for (int64_t b = blocks; b < (blocks + 3) / 4 * 4; ++b) row[b] = 127;
}

template <class T, bool ROWS, bool COLS>
__global__ void __launch_bounds__(256)
quantise_kernel(dtst_quantise_desc d, const T* __restrict__ x, uint8_t* q, uint8_t* scale, uint8_t* qt,
                uint8_t* scale_t, int col_tiles) {
  __shared__ float tile[COLS ? 128 * PITCH : 1];
  const int64_t rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
  const int sub = threadIdx.x >> 4, part = threadIdx.x & 15;  // 16 rows at a time, 16 lanes a row
  const int64_t c = ct * 128 + part * 8;
  const int64_t col_blocks = (d.cols + 127) / 128, row_blocks = (d.rows + 127) / 128;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int lr = i * 16 + sub;
    const int64_t row = rt * 128 + lr;
    float v[8];
    load_n<8>(x + row * d.ld_x + c, row < d.rows ? d.cols - c : 0, v);
    if constexpr (ROWS) {
      uint2 codes;
      const uint32_t s = code_block(v, codes);
      if (row < d.rows) {
        *reinterpret_cast<uint2*>(q + row * d.ld_q + c) = codes;
        if (part == 0) put_scale(scale + row * d.ld_scale, ct, col_blocks, s);
      }
    }
    if constexpr (COLS) {
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[lr * PITCH + part * 8 + j] = v[j];
    }
  }
  if constexpr (COLS) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int lc = i * 16 + sub;
      const int64_t col = ct * 128 + lc;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = tile[(part * 8 + j) * PITCH + lc];
      uint2 codes;
      const uint32_t s = code_block(v, codes);
      if (col < d.cols) {
        *reinterpret_cast<uint2*>(qt + col * d.ld_qt + rt * 128 + part * 8) = codes;
        if (part == 0) put_scale(scale_t + col * d.ld_scale_t, rt, row_blocks, s);
      }
    }
  }
}

template <class T>
int launch(const dtst_quantise_desc& d, const void* x, void* q, void* scale, void* qt, void* scale_t, hipStream_t s) {
  const int64_t ct = (d.cols + 127) / 128, rt = (d.rows + 127) / 128;
  auto* fn = q == nullptr ? quantise_kernel<T, false, true>
             : qt == nullptr ? quantise_kernel<T, true, false>
                             : quantise_kernel<T, true, true>;
  hipLaunchKernelGGL(fn, dim3(unsigned(ct * rt)), dim3(256), 0, s, d, static_cast<const T*>(x),
                     static_cast<uint8_t*>(q), static_cast<uint8_t*>(scale), static_cast<uint8_t*>(qt),
                     static_cast<uint8_t*>(scale_t), int(ct));
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
