// RMS norm and layer norm with the residual's addition, and their backward
// (dtst_rms_norm, dtst_rms_norm_adj; MEAN: dtst_layer_norm, dtst_layer_norm_adj).
//
//   u = x + res,  r = 1 / sqrt(mean u^2 + eps),  y = u r w
//   g_u = r (t - h mean(t h)) + g_sum,  t = g_y w,  h = u r;   g_w = sum_rows g_y h
// MEAN: v = u - mean u in the place of u, y = v r w + b,
//   g_u = r (t - mean t - h mean(t h)) + g_sum,   g_b = sum_rows g_y
//
// A few operations per value: bound by HBM.  A row stays in the registers of
// its RW waves between the sum and the result, so each array is read or written
// once, eight neighbouring columns (16 bytes of a 16-bit type) per access; 16
// lanes then hold a block of 128 columns, whose 8-bit scale is a maximum within
// a row of lanes.  Up to 1024 columns a wave holds a row (no barrier), then four,
// then sixteen.  16384 x 4096 in bf16 with the residual, to 8 bits: 86 us, 5.5
// TB/s, what a large copy reaches; 6001 x 1537 in 32 bits 33 us forward (4.5
// TB/s) and 27 + 5 us backward.  MEAN, with two rounds of sums a row: 95
// us, and 29 and 27 + 5.
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
// (A second call on the same slots needs a barrier before it where RW > 1.)
template <int RW>
__device__ __forceinline__ double row_sum64(float v, double* part) {
  double s = row16_sum(v);
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

// Sum over a wave, in all lanes: 16 lanes without LDS, then their four rows.
__device__ __forceinline__ float wave_sum16(float v) {
  v = row16_sum(v);
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Sum of the RW waves' slots, in all lanes, each of which reads one.
template <int RW>
__device__ __forceinline__ float slots_sum(const float* slots) {
  static_assert(RW == 4 || RW == 16, "quads or rows of lanes");
  float v = slots[threadIdx.x & (RW - 1)];
  if constexpr (RW == 16) return row16_sum(v);
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xb1, 0xf, 0xf, false));
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4e, 0xf, 0xf, false));
}

// 1 / sqrt(m), rounded once: the 32-bit root, off by a unit in its last place, and
// a step of Newton's (no root of 0, infinity and no number).
__device__ __forceinline__ float rsqrt_of(double m) {
  const float r = rsqrtf(float(m));
  const double x = r;
  return r > 0.f && r <= 3.402823466e38f ? float(x * (1.5 - 0.5 * m * x * x)) : r;
}

// RW waves a row, V vectors of 8 columns a lane: up to 512 RW V columns.  A
// workgroup holds max(RW, 4) waves, so four rows with RW = 1.  (8: four registers fewer,
// where they do not spill, hold one more wave a SIMD: 96.1 -> 94.8 us for the case above; the
// other forms were not timed with it.)
template <class TX, class TR, bool Q8, int RW, int V, bool MEAN>
__global__ void __launch_bounds__(RW > 4 ? RW * 64 : 256, MEAN && Q8 && RW == 4 && V == 2 && sizeof(TR) == 2 ? 8 : 1)
norm_kernel(dtst_norm_desc d, double inv_cols, const TX* x, const TR* res, const float* __restrict__ w,
            const float* __restrict__ b, TR* sum_out, void* y, uint8_t* scale, float* mean_out, float* rstd) {
  constexpr int ROWS = RW > 4 ? 1 : 4 / RW;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  __shared__ double part[RW], part2[RW], part3[RW];
  double mean = 0.0;
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
  const auto store_sum = [&] {
    if (sum_out == nullptr) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      store_n<VEC>(sum_out + row * d.ld_sum + c, cols - c, u[i]);
    }
  };
  float s = 0.f;
  if constexpr (MEAN) {
    // Deviations from a mean in 32 bits, which a mean far above them shifts all
    // alike by the roundings of its sum: what they have in common, `low`, is taken
    // off them below.
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) s += u[i][j];
    const float high = float(row_sum64<RW>(s, part2) * inv_cols);
    store_sum();
    s = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      if (c + VEC <= cols) {  // (a select for each value would cost as much as its sums)
#pragma unroll
        for (int j = 0; j < VEC; ++j) u[i][j] -= high;
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) u[i][j] = c + j < cols ? u[i][j] - high : 0.f;
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) s += u[i][j];
    }
    mean = high;
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) ss += u[i][j] * u[i][j];
  double low = 0.0, square;
  if constexpr (MEAN) {
    low = row_sum64<RW>(s, part3) * inv_cols;
    mean += low;
    square = row_sum64<RW>(ss, part) * inv_cols - low * low;
    if (square < 0.0) square = 0.0;  // (no number stays)
  } else {
    square = row_sum64<RW>(ss, part) * inv_cols;
  }
  const float r = rsqrt_of(square + double(d.eps)), shift = float(low);
  if (MEAN && mean_out != nullptr && first == 0) mean_out[row] = float(mean);
  if (rstd != nullptr && first == 0) rstd[row] = r;
  if constexpr (!MEAN) store_sum();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    float wv[VEC];
    load_n<VEC>(w + c, cols - c, wv);
#pragma unroll
    for (int j = 0; j < VEC; ++j) u[i][j] = (MEAN ? u[i][j] - shift : u[i][j]) * r * wv[j];
    if (MEAN && b != nullptr) {
      float bv[VEC];
      load_n<VEC>(b + c, cols - c, bv);
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[i][j] += bv[j];
    }
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

struct NormArgs {
  const void *x, *res;
  const float *w, *b;
  void *sum_out, *y, *scale;
  float *mean, *rstd;
};

template <class TX, class TR, bool Q8, int RW, int V, bool MEAN>
int launch_norm(const dtst_norm_desc& d, const NormArgs& a, hipStream_t s) {
  const NormGrid g = norm_grid(d.rows, d.cols);
  hipLaunchKernelGGL((norm_kernel<TX, TR, Q8, RW, V, MEAN>), dim3(unsigned(g.groups)), dim3(g.threads), 0, s, d,
                     1.0 / double(d.cols), static_cast<const TX*>(a.x), static_cast<const TR*>(a.res), a.w, a.b,
                     static_cast<TR*>(a.sum_out), a.y, static_cast<uint8_t*>(a.scale), a.mean, a.rstd);
  return hipGetLastError();
}

template <class TX, class TR, bool Q8, bool MEAN>
int launch_norm_cols(const dtst_norm_desc& d, const NormArgs& a, hipStream_t s) {
  const int64_t c = d.cols;
  if (c <= 512) return launch_norm<TX, TR, Q8, 1, 1, MEAN>(d, a, s);
  if (c <= 1024) return launch_norm<TX, TR, Q8, 1, 2, MEAN>(d, a, s);
  if (c <= 2048) return launch_norm<TX, TR, Q8, 4, 1, MEAN>(d, a, s);
  if (c <= 4096) return launch_norm<TX, TR, Q8, 4, 2, MEAN>(d, a, s);
  if (c <= 8192) return launch_norm<TX, TR, Q8, 4, 4, MEAN>(d, a, s);
  if (c <= 16384) return launch_norm<TX, TR, Q8, 16, 2, MEAN>(d, a, s);
  return launch_norm<TX, TR, Q8, 16, 4, MEAN>(d, a, s);
}

// Backward.  RW waves hold a row, ROWS rows a workgroup at once (one where
// several waves share a row); it takes every gridDim-th of them and keeps its
// columns' sums of g_y h (MEAN: and of g_y) in registers; they go to part
// (gridDim, cols; MEAN: cols twice), which sum_parts_kernel adds up.
//
// MEAN: three sums a row.  Of h from the mean in 32 bits as it is, two would do, and g_u
// would be off by 4e-3 of itself where the mean is 1e5 deviations; 2^25 values a call in 32
// bits, 1537 columns 87 us either way, 8000: 95 and 93, 16000: 149 and 109; with g_y in bf16
// 1537: 74 and 74, 8000: 83 and 86.  (With the single sums' shuffles and every lane adding up
// all slots it took registers that there are not: 16000 columns 232.)
template <class TX, class TR, int RW, int V, int ROWS, bool MEAN>
__global__ void __launch_bounds__(RW * ROWS * 64, V == 2 && !MEAN ? 4 : 1)  // (4: two registers fewer hold one more wave)
norm_adj_kernel(dtst_norm_adj_desc d, const TX* g_y, const TR* u, const float* __restrict__ w,
                const float* __restrict__ mean_of, const float* __restrict__ rstd, const TR* g_sum, TR* g_u, TX* g_x,
                float* part) {
  static_assert(ROWS == 1 || (RW == 1 && V == 1), "a wave a row, in one access");
  __shared__ float red[2][RW], red2[2][RW], red3[2][RW];
  const int first = int(threadIdx.x % (RW * 64)) * VEC, sub = threadIdx.x / (RW * 64);
  const int64_t cols = d.cols;
  float wv[V][VEC], gw[V][VEC], gb[V][VEC];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    load_n<VEC>(w + c, cols - c, wv[i]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) gw[i][j] = gb[i][j] = 0.f;
  }
  int odd = 0;
  for (int64_t row = int64_t(blockIdx.x) * ROWS + sub; row < d.rows; row += int64_t(gridDim.x) * ROWS, odd ^= 1) {
    const float r = rstd[row];
    float g[V][VEC], h[V][VEC];
    float dot = 0.f, sum = 0.f, shift = 0.f, m = 0.f;
    if constexpr (MEAN) m = mean_of[row];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int64_t c = first + i * RW * 64 * VEC;
      load_n<VEC>(g_y + row * d.ld_g_y + c, cols - c, g[i]);
      load_n<VEC>(u + row * d.ld_u + c, cols - c, h[i]);
    }
    if constexpr (MEAN) {
      // Deviations from the mean in 32 bits over the standard deviation, k, have its
      // rounding in common: `low`, their own mean, is taken off as in the forward, in the
      // sums' one round,  h = k - low,  mean(t h) = mean(t k) - low mean t.
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int64_t c = first + i * RW * 64 * VEC;
        if (c + VEC <= cols) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) h[i][j] = (h[i][j] - m) * r;
        } else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) h[i][j] = c + j < cols ? (h[i][j] - m) * r : 0.f;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float t = g[i][j] * wv[i][j];
          gb[i][j] += g[i][j];
          shift += h[i][j];
          sum += t;
          dot += t * h[i][j];
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          h[i][j] *= r;  // (past the row g and w are zero)
          gw[i][j] += g[i][j] * h[i][j];
          g[i][j] *= wv[i][j];
          dot += g[i][j] * h[i][j];
        }
    }
    // (two sets of slots: one barrier a row)
    float mean, mean_t = 0.f;
    if constexpr (!MEAN) {
      mean = row_sum<RW>(dot, red[odd]) / float(cols);
    } else {
      dot = wave_sum16(dot), sum = wave_sum16(sum), shift = wave_sum16(shift);
      if constexpr (RW > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[odd][wave] = dot, red2[odd][wave] = sum, red3[odd][wave] = shift;
        __syncthreads();
        dot = slots_sum<RW>(red[odd]), sum = slots_sum<RW>(red2[odd]), shift = slots_sum<RW>(red3[odd]);
      }
      mean_t = sum / float(cols);
      const float low = shift / float(cols);
      mean = dot / float(cols) - low * mean_t;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          h[i][j] -= low;
          gw[i][j] += g[i][j] * h[i][j];
          g[i][j] *= wv[i][j];
        }
    }
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
      for (int j = 0; j < VEC; ++j) e[j] += r * ((MEAN ? g[i][j] - mean_t : g[i][j]) - h[i][j] * mean);
      store_n<VEC>(g_u + row * d.ld_g_u + c, cols - c, e);
      if (g_x != nullptr) store_n<VEC>(g_x + row * d.ld_g_x + c, cols - c, e);
    }
  }
  part += blockIdx.x * cols * (MEAN ? 2 : 1);
  if constexpr (ROWS > 1) {  // (in order)
    __shared__ float sums[ROWS][64 * VEC];
    const auto add_up = [&](const float (&v)[VEC], float* out) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) sums[sub][first + j] = v[j];
      __syncthreads();
      for (int c = threadIdx.x; c < cols; c += ROWS * 64) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) t += sums[k][c];
        out[c] = t;
      }
    };
    add_up(gw[0], part);
    if constexpr (MEAN) {
      __syncthreads();
      add_up(gb[0], part + cols);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int64_t c = first + i * RW * 64 * VEC;
    store_n<VEC>(part + c, cols - c, gw[i]);
    if constexpr (MEAN) store_n<VEC>(part + cols + c, cols - c, gb[i]);
  }
}

// g_w[c] (+)= sum_p part[p][c] of rows `pitch` apart, and g_b from the columns
// past g_w's, up to `width`: 32 columns a workgroup, 32 lanes a column, each taking every 32nd part
// (64 columns by 16 waves left the loads one after the other: 15 us for 751 parts
// of 1537 columns).
__global__ void __launch_bounds__(1024)
sum_parts_kernel(const float* __restrict__ part, int64_t parts, int64_t pitch, int64_t cols, int64_t width,
                 int accumulate, float* g_w, float* g_b) {
  __shared__ float red[32][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int64_t p = group; p < parts; p += 32) s += part[p * pitch + c];
  }
  red[group][lane] = s;
  __syncthreads();
  if (group == 0 && c < width) {
    float* out = c < cols ? g_w + c : g_b + (c - cols);
    float t = accumulate ? *out : 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += red[i][lane];
    *out = t;
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

struct NormAdjArgs {
  const void *g_y, *u;
  const float *w, *mean, *rstd;
  const void* g_sum;
  void *g_u, *g_x;
  float* part;
};

template <class TX, class TR, bool MEAN, int RW, int V, int ROWS = 1>
int launch_norm_adj(const dtst_norm_adj_desc& d, const NormAdjArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((norm_adj_kernel<TX, TR, RW, V, ROWS, MEAN>), dim3(unsigned(norm_adj_parts(d.rows, d.cols))),
                     dim3(RW * ROWS * 64), 0, s, d, static_cast<const TX*>(a.g_y), static_cast<const TR*>(a.u), a.w,
                     a.mean, a.rstd, static_cast<const TR*>(a.g_sum), static_cast<TR*>(a.g_u), static_cast<TX*>(a.g_x),
                     a.part);
  return hipGetLastError();
}

template <class TX, class TR, bool MEAN>
int launch_norm_adj_cols(const dtst_norm_adj_desc& d, const NormAdjArgs& a, hipStream_t s) {
  const int64_t c = d.cols;
  if (c <= SINGLE) return launch_norm_adj<TX, TR, MEAN, 1, 1, SINGLE_ROWS>(d, a, s);
  if (c <= 2048) return launch_norm_adj<TX, TR, MEAN, 4, 1>(d, a, s);
  if (c <= 4096) return launch_norm_adj<TX, TR, MEAN, 4, 2>(d, a, s);
  if (c <= 8192) return launch_norm_adj<TX, TR, MEAN, 16, 1>(d, a, s);
  if (c <= 16384) return launch_norm_adj<TX, TR, MEAN, 16, 2>(d, a, s);
  return launch_norm_adj<TX, TR, MEAN, 16, 4>(d, a, s);
}

// Calls f with values of the types x_type and res_type stand for (checked:
// res_type is x_type or DTST_F32).
template <class F>
int by_types(int x_type, int res_type, F&& f) {
  if (x_type == DTST_F32) return f(float(), float());
  if (x_type == DTST_BF16) return res_type == DTST_F32 ? f(bf16_t(), float()) : f(bf16_t(), bf16_t());
  return res_type == DTST_F32 ? f(f16_t(), float()) : f(f16_t(), f16_t());
}

template <bool MEAN>
int norm_forward(const dtst_norm_desc& d, const NormArgs& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_types(d.x_type, d.res_type, [&](auto tx, auto tr) {
    using TX = decltype(tx);
    using TR = decltype(tr);
    return d.y_type == DTST_E4M3 ? launch_norm_cols<TX, TR, true, MEAN>(d, a, s)
                                 : launch_norm_cols<TX, TR, false, MEAN>(d, a, s);
  });
}

template <bool MEAN>
int norm_backward(const dtst_norm_adj_desc& d, const NormAdjArgs& a, float* g_weight, float* g_bias, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.rows > 0) {  // (the kernel reads the weight before its rows; of none there is nothing to add up)
    const int e = by_types(d.x_type, d.res_type, [&](auto tx, auto tr) {
      return launch_norm_adj_cols<decltype(tx), decltype(tr), MEAN>(d, a, s);
    });
    if (e != hipSuccess) return e;
  }
  const int64_t width = d.cols * (MEAN ? 2 : 1);
  return launch_sum_parts(a.part, d.rows > 0 ? norm_adj_parts(d.rows, d.cols) : 0, width, d.cols, width, d.accumulate,
                          g_weight, g_bias, stream);
}

}  // namespace

int launch_sum_parts(const float* part, int64_t parts, int64_t pitch, int64_t cols, int64_t width, int accumulate,
                     float* first, float* second, void* stream) {
  hipLaunchKernelGGL(sum_parts_kernel, dim3(unsigned((width + 31) / 32)), dim3(1024), 0,
                     static_cast<hipStream_t>(stream), part, parts, pitch, cols, width, accumulate, first, second);
  return hipGetLastError();
}

int launch_rms_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, void* sum_out,
                    void* y, void* scale, float* rstd, void* stream) {
  return norm_forward<false>(d, NormArgs{x, res, weight, nullptr, sum_out, y, scale, nullptr, rstd}, stream);
}

int launch_layer_norm(const dtst_norm_desc& d, const void* x, const void* res, const float* weight, const float* bias,
                      void* sum_out, void* y, void* scale, float* mean, float* rstd, void* stream) {
  return norm_forward<true>(d, NormArgs{x, res, weight, bias, sum_out, y, scale, mean, rstd}, stream);
}

// (one wave a row up to 1024 columns, four up to 8192, else sixteen)
NormGrid norm_grid(int64_t rows, int64_t cols) {
  if (cols <= 1024) return {(rows + 3) / 4, 256};
  return {rows, cols <= 8192 ? 256 : 1024};
}

size_t rms_norm_adj_workspace(int64_t rows, int64_t cols) { return size_t(norm_adj_parts(rows, cols)) * cols * 4; }
size_t layer_norm_adj_workspace(int64_t rows, int64_t cols) { return 2 * rms_norm_adj_workspace(rows, cols); }

int launch_rms_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                        const float* rstd, const void* g_sum, void* g_u, void* g_x, float* g_weight, void* workspace,
                        void* stream) {
  return norm_backward<false>(
      d, NormAdjArgs{g_y, u, weight, nullptr, rstd, g_sum, g_u, g_x, static_cast<float*>(workspace)}, g_weight, nullptr,
      stream);
}

int launch_layer_norm_adj(const dtst_norm_adj_desc& d, const void* g_y, const void* u, const float* weight,
                          const float* mean, const float* rstd, const void* g_sum, void* g_u, void* g_x,
                          float* g_weight, float* g_bias, void* workspace, void* stream) {
  return norm_backward<true>(
      d, NormAdjArgs{g_y, u, weight, mean, rstd, g_sum, g_u, g_x, static_cast<float*>(workspace)}, g_weight, g_bias,
      stream);
}

}  // namespace dtst
