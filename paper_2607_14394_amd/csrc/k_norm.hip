// RMS norm with the residual's addition, and its backward (dtst_rms_norm,
// dtst_rms_norm_adj).
//
//   u = x + res,  r = 1 / sqrt(mean u^2 + eps),  y = u r w
//   g_u = r (t - h mean(t h)) + g_sum,  t = g_y w,  h = u r;   g_w = sum_rows g_y h
//
// A few operations per value: bound by HBM.  A row stays in the registers of
// its RW waves between the sum and the result, so each array is read or written
// once, eight neighbouring columns (16 bytes of a 16-bit type) per access; 16
// lanes then hold a block of 128 columns, whose 8-bit scale is a maximum within
// a row of lanes.  Up to 1024 columns a wave holds a row (no barrier), then four,
// then sixteen.  16384 x 4096 in bf16 with the residual, to 8 bits: 86 us, 5.5
// TB/s, what a large copy reaches; 6001 x 1537 in 32 bits 33 us forward (4.5
// TB/s) and 27 + 5 us backward.
//
// The sum is rounded to the residual's type first and the norm is of what was
// stored, so that the backward differentiates what the forward computed.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

constexpr int VEC = 8;

// Sum over the RW waves of a row (all lanes get it).  part: one slot per wave.
template <int RW>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (RW > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < RW; ++i) v += part[i];
  }
  return v;
}

// The same in 64 bits from 16 lanes' sums on: there the last additions, whose
// roundings weigh most, cost a few instructions a row.
template <int RW>
__device__ __forceinline__ double row_sum64(float v, double* part) {
#pragma unroll
  for (int d = 1; d <= 8; d <<= 1) v += __shfl_xor(v, d, 64);
  double s = v;
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if constexpr (RW > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < RW; ++i) s += part[i];
  }
  return s;
}

// 1 / sqrt(m), rounded once: the 32-bit root, off by a unit in its last place, and
// a step of Newton's (no root of 0, infinity and no number).
__device__ __forceinline__ float rsqrt_of(double m) {
  const float r = rsqrtf(float(m));
  const double x = r;
  return r > 0.f && r <= 3.402823466e38f ? float(x * (1.5 - 0.5 * m * x * x)) : r;
}

// RW waves a row, V vectors of 8 columns a lane: up to 512 RW V columns.  A
// workgroup holds max(RW, 4) waves, so four rows with RW = 1.
template <class TX, class TR, bool Q8, int RW, int V>
__global__ void __launch_bounds__(RW > 4 ? RW * 64 : 256)
rms_norm_kernel(dtst_norm_desc d, double inv_cols, const TX* x, const TR* res, const float* __restrict__ w, TR* sum_out,
                void* y, uint8_t* scale, float* rstd) {
  constexpr int ROWS = RW > 4 ? 1 : 4 / RW;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  __shared__ double part[RW];
  const int64_t row = int64_t(blockIdx.x) * ROWS + wave / RW;
  if (ROWS > 1 && row >= d.rows) return;  // (one wave a row: no barrier follows)
  const int first = ((wave % RW) * 64 + lane) * VEC;
  const int64_t cols = d.cols;
  float u[V][VEC];
  const TX* xr = x + row * d.ld_x;
  const TR* rr = res ? res + row * d.ld_res : nullptr;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    load_n<VEC>(xr + c, cols - c, u[i]);
  }
  if (rr != nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      float r[VEC];
      load_n<VEC>(rr + c, cols - c, r);
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[i][j] = float(TR(u[i][j] + r[j]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[i][j] = float(TR(u[i][j]));
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) ss += u[i][j] * u[i][j];
  const float r = rsqrt_of(row_sum64<RW>(ss, part) * inv_cols + double(d.eps));
  if (rstd != nullptr && first == 0) rstd[row] = r;
  if (sum_out != nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      store_n<VEC>(sum_out + row * d.ld_sum + c, cols - c, u[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    float wv[VEC];
    load_n<VEC>(w + c, cols - c, wv);
#pragma unroll
    for (int j = 0; j < VEC; ++j) u[i][j] = u[i][j] * r * wv[j];
    if constexpr (Q8) {
      if (c + VEC > cols) {  // (not by the product: 1 / rms may be no number)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (c + j >= cols) u[i][j] = 0.f;
      }
      uint2 q;
      const uint32_t s = code_block(u[i], q);
      const int64_t padded = (cols + 127) / 128 * 128, blocks = padded / 128;
      if (c < padded) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(y) + row * d.ld_y + c) = q;
      // a byte for each block, and for the rest of the row's last four
      if ((lane & 15) == 0 && c / 128 < (blocks + 3) / 4 * 4)
        scale[row * d.ld_scale + c / 128] = c < padded ? uint8_t(s) : uint8_t(127);
    } else {
      store_n<VEC>(static_cast<TX*>(y) + row * d.ld_y + c, cols - c, u[i]);
    }
  }
}

template <class TX, class TR, bool Q8, int RW, int V>
int launch_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* w, void* sum_out, void* y,
                void* scale, float* rstd, hipStream_t s) {
  const NormGrid g = rms_norm_grid(d.rows, d.cols);
  hipLaunchKernelGGL((rms_norm_kernel<TX, TR, Q8, RW, V>), dim3(unsigned(g.groups)), dim3(g.threads), 0, s, d,
                     1.0 / double(d.cols),
                     static_cast<const TX*>(x), static_cast<const TR*>(res), w, static_cast<TR*>(sum_out), y,
                     static_cast<uint8_t*>(scale), rstd);
  return hipGetLastError();
}

template <class TX, class TR, bool Q8>
int launch_norm_cols(const dtst_norm_desc& d, const void* x, const void* res, const float* w, void* sum_out, void* y,
                     void* scale, float* rstd, hipStream_t s) {
  const int64_t c = d.cols;
  if (c <= 512) return launch_norm<TX, TR, Q8, 1, 1>(d, x, res, w, sum_out, y, scale, rstd, s);
  if (c <= 1024) return launch_norm<TX, TR, Q8, 1, 2>(d, x, res, w, sum_out, y, scale, rstd, s);
  if (c <= 2048) return launch_norm<TX, TR, Q8, 4, 1>(d, x, res, w, sum_out, y, scale, rstd, s);
  if (c <= 4096) return launch_norm<TX, TR, Q8, 4, 2>(d, x, res, w, sum_out, y, scale, rstd, s);
  if (c <= 8192) return launch_norm<TX, TR, Q8, 4, 4>(d, x, res, w, sum_out, y, scale, rstd, s);
  if (c <= 16384) return launch_norm<TX, TR, Q8, 16, 2>(d, x, res, w, sum_out, y, scale, rstd, s);
  return launch_norm<TX, TR, Q8, 16, 4>(d, x, res, w, sum_out, y, scale, rstd, s);
}

// Backward.  RW waves hold a row, ROWS rows a workgroup at once (one where
// several waves share a row); it takes every gridDim-th of them and keeps its
// columns' sums of g_y h in registers; they go to part (gridDim, cols), which
// sum_parts_kernel adds up.
template <class TX, class TR, int RW, int V, int ROWS>
__global__ void __launch_bounds__(RW * ROWS * 64, V == 2 ? 4 : 1)  // (4: two registers fewer hold one more wave)
rms_norm_adj_kernel(dtst_norm_adj_desc d, const TX* g_y, const TR* u, const float* __restrict__ w,
                    const float* __restrict__ rstd, const TR* g_sum, TR* g_u, TX* g_x, float* part) {
  static_assert(ROWS == 1 || (RW == 1 && V == 1), "a wave a row, in one access");
  __shared__ float red[2][RW];
  const int first = int(threadIdx.x % (RW * 64)) * VEC, sub = threadIdx.x / (RW * 64);
  const int64_t cols = d.cols;
  float wv[V][VEC], gw[V][VEC];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    load_n<VEC>(w + c, cols - c, wv[i]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) gw[i][j] = 0.f;
  }
  int odd = 0;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + sub; row < d.rows; row += int64_t(gridDim.x) * ROWS, odd ^= 1) {
    const float r = rstd[row];
    float g[V][VEC], h[V][VEC];
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      load_n<VEC>(g_y + row * d.ld_g_y + c, cols - c, g[i]);
      load_n<VEC>(u + row * d.ld_u + c, cols - c, h[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        h[i][j] *= r;
        gw[i][j] += g[i][j] * h[i][j];
        g[i][j] *= wv[i][j];
        dot += g[i][j] * h[i][j];
      }
    const float mean = row_sum<RW>(dot, red[odd]) / float(cols);  // (two sets of slots: one barrier a row)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      float e[VEC];
      if (g_sum != nullptr) {
        load_n<VEC>(g_sum + row * d.ld_g_sum + c, cols - c, e);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) e[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) e[j] += r * (g[i][j] - h[i][j] * mean);
      store_n<VEC>(g_u + row * d.ld_g_u + c, cols - c, e);
      if (g_x != nullptr) store_n<VEC>(g_x + row * d.ld_g_x + c, cols - c, e);
    }
  }
  if constexpr (ROWS > 1) {  // (in order)
    __shared__ float sums[ROWS][64 * VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sums[sub][first + j] = gw[0][j];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += ROWS * 64) {
      float t = 0.f;
#pragma unroll
      for (int k = 0; k < ROWS; ++k) t += sums[k][c];
      part[blockIdx.x * cols + c] = t;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    store_n<VEC>(part + blockIdx.x * cols + c, cols - c, gw[i]);
  }
}

// g_w[c] (+)= sum_p part[p][c]: 32 columns a workgroup, 32 lanes a column, each
// taking every 32nd part (64 columns by 16 waves left the loads one after the
// other: 15 us for 751 parts of 1537 columns).
__global__ void __launch_bounds__(1024)
sum_parts_kernel(const float* __restrict__ part, int parts, int64_t cols, int accumulate, float* g_w) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int p = group; p < parts; p += 32) s += part[p * cols + c];
  }
  red[group][lane] = s;
  __syncthreads();
  if (group == 0 && c < cols) {
    float t = accumulate ? g_w[c] : 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += red[i][lane];
    g_w[c] = t;
  }
}

// Workgroups of the backward: two rows a wave or group of waves, until the card
// is full (two groups of 16 waves a CU, four of 4, two of 8 single ones).  Eight
// rows each left CUs idle (backward of 495 x 7931: 33 against 21 us).
constexpr int SINGLE = 512, SINGLE_ROWS = 8;  // up to so many columns a wave holds a row, so many rows a workgroup
int64_t norm_adj_parts(int64_t rows, int64_t cols) {
  const int64_t each = cols <= SINGLE ? 2 * SINGLE_ROWS : 2, most = cols <= SINGLE || cols > 4096 ? 512 : 1024;
  return std::max<int64_t>(1, std::min<int64_t>(most, (rows + each - 1) / each));
}

template <class TX, class TR, int RW, int V, int ROWS = 1>
int launch_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* w, const float* rstd,
                    const void* g_sum, void* g_u, void* g_x, float* part, hipStream_t s) {
  hipLaunchKernelGGL((rms_norm_adj_kernel<TX, TR, RW, V, ROWS>), dim3(unsigned(norm_adj_parts(d.rows, d.cols))),
                     dim3(RW * ROWS * 64), 0, s, d, static_cast<const TX*>(g_y), static_cast<const TR*>(u), w, rstd,
                     static_cast<const TR*>(g_sum), static_cast<TR*>(g_u), static_cast<TX*>(g_x), part);
  return hipGetLastError();
}

template <class TX, class TR>
int launch_norm_adj_cols(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* w,
                         const float* rstd, const void* g_sum, void* g_u, void* g_x, float* part, hipStream_t s) {
  const int64_t c = d.cols;
  if (c <= SINGLE) return launch_norm_adj<TX, TR, 1, 1, SINGLE_ROWS>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
  if (c <= 2048) return launch_norm_adj<TX, TR, 4, 1>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
  if (c <= 4096) return launch_norm_adj<TX, TR, 4, 2>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
  if (c <= 8192) return launch_norm_adj<TX, TR, 16, 1>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
  if (c <= 16384) return launch_norm_adj<TX, TR, 16, 2>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
  return launch_norm_adj<TX, TR, 16, 4>(d, g_y, u, w, rstd, g_sum, g_u, g_x, part, s);
}

// Calls f with values of the types x_type and res_type stand for (checked:
// res_type is x_type or DTST_F32).
template <class F>
int by_types(int x_type, int res_type, F&& f) {
  if (x_type == DTST_F32) return f(float(), float());
  if (x_type == DTST_BF16) return res_type == DTST_F32 ? f(bf16_t(), float()) : f(bf16_t(), bf16_t());
  return res_type == DTST_F32 ? f(f16_t(), float()) : f(f16_t(), f16_t());
}

}  // namespace

int launch_rms_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, void* sum_out,
                    void* y, void* scale, float* rstd, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_types(d.x_type, d.res_type, [&](auto tx, auto tr) {
    using TX = decltype(tx);
    using TR = decltype(tr);
    return d.y_type == DTST_E4M3
               ? launch_norm_cols<TX, TR, true>(d, x, res, weight, sum_out, y, scale, rstd, s)
               : launch_norm_cols<TX, TR, false>(d, x, res, weight, sum_out, y, scale, rstd, s);
  });
}

// (one wave a row up to 1024 columns, four up to 8192, else sixteen)
NormGrid rms_norm_grid(int64_t rows, int64_t cols) {
  if (cols <= 1024) return {(rows + 3) / 4, 256};
  return {rows, cols <= 8192 ? 256 : 1024};
}

size_t rms_norm_adj_workspace(int64_t rows, int64_t cols) { return size_t(norm_adj_parts(rows, cols)) * cols * 4; }

int launch_rms_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                        const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight, void* workspace,
                        void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  float* part = static_cast<float*>(workspace);
  if (d.rows > 0) {  // (the kernel reads the weight before its rows; of none there is nothing to add up)
    const int e = by_types(d.x_type, d.res_type, [&](auto tx, auto tr) {
      return launch_norm_adj_cols<decltype(tx), decltype(tr)>(d, g_y, u, weight, rstd, g_sum, g_u, g_x, part, s);
    });
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(sum_parts_kernel, dim3(unsigned((d.cols + 31) / 32)), dim3(1024), 0, s, part,
                     d.rows > 0 ? int(norm_adj_parts(d.rows, d.cols)) : 0, d.cols, d.accumulate, g_weight);
  return hipGetLastError();
}

}  // namespace dtst
