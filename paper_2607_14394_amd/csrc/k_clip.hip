// The norm of many tensors together, and the tensors scaled down to a largest
// norm (dtst_global_norm, dtst_clip):
//   norm = sqrt(sum of g^2 over all),   out = g min(1, most / norm).
//
// Bound by HBM: the norm reads each value once, the scaling reads and writes it
// once (16-byte accesses, four in flight a lane).  Gradients are hundreds of
// tensors from a few values to many millions, so a launch takes up to so many
// tensors as its arguments hold (4 KB), cut into chunks of 8192 values; each of
// at most 2048 workgroups takes every 2048th, finds its first chunk's tensor and goes
// on from there.  The sums of two squares are added up in 64 bits; each workgroup leaves
// its sum, and one adds those up in a fixed order.  470 MB in bf16: 116 + 5 us (4.1 TB/s)
// and 161 us (5.8 TB/s, half of what it reads from the last-level cache); 264 tensors of
// 32 MB in 32 bits 15 and 23 us, where a call takes 95 us on the host.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

constexpr int VEC = 8, THREADS = 256, CHUNK = 4 * VEC * THREADS, GROUPS = 2048;
constexpr int NORM_TENSORS = 184, CLIP_TENSORS = 128;  // of a launch

// Tensors of one launch.  size: 4 times the count, and the type; first[i]: chunks
// of the tensors before i.
template <int N, int SIDES>
struct Table {
  void* p[SIDES][N];
  int64_t size[N];
  uint32_t first[N + 1];
  int32_t n;
};
using NormTable = Table<NORM_TENSORS, 1>;
using ClipTable = Table<CLIP_TENSORS, 2>;
static_assert(sizeof(NormTable) <= 4000 && sizeof(ClipTable) <= 4000, "what a launch's arguments hold");

// Calls f(tensor, first value, values) for the chunks of this workgroup.
template <class T, class F>
__device__ __forceinline__ void each_chunk(const T& t, F&& f) {
  uint32_t c = blockIdx.x;
  const uint32_t end = t.first[t.n];
  int lo = 0, hi = t.n;  // the last tensor with first <= c (those without chunks lie before it)
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.first[mid] <= c)
      lo = mid;
    else
      hi = mid;
  }
  for (; c < end; c += gridDim.x) {  // (a run each: 87 against 82, and 201 against 178 us for 470 MB in bf16)
    while (c >= t.first[lo + 1]) ++lo;
    const int64_t at = int64_t(c - t.first[lo]) * CHUNK, left = (t.size[lo] >> 2) - at;
    f(lo, at, left < CHUNK ? left : CHUNK);
  }
}

template <class F>
__device__ __forceinline__ void by_type(int type, F&& f) {
  if (type == DTST_F32)
    f(float());
  else if (type == DTST_BF16)
    f(bf16_t());
  else
    f(f16_t());
}

// Sum over a workgroup, in a fixed order; the first thread's result.
template <int WAVES>
__device__ __forceinline__ double group_sum(double s) {
  __shared__ double part[WAVES];
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) s += part[i];
  return s;
}

// The sum of eight squares: those of two neighbours in 32 bits, as conversions to 64 take
// long (470 MB in bf16, with the scaling: 284 us; 283 with all eight in 32 bits, 308 with
// each in 64, or with the roundings of 32 made good).  That is two roundings of 2^-24 of a
// sum at most, one where 32 bits hold a square (16-bit types), of which the root takes half.
// All in 64 where 32 pass them or lose what matters (a square below 2^-126 beside a sum of
// 2^-66).
__device__ __forceinline__ double squares(const float (&v)[VEC]) {
  float p[VEC / 2];
#pragma unroll
  for (int j = 0; j < VEC / 2; ++j) p[j] = fmaf(v[2 * j + 1], v[2 * j + 1], v[2 * j] * v[2 * j]);
  const float s = (p[0] + p[1]) + (p[2] + p[3]);
  if (s >= 1e-20f && s <= 1e30f) return (double(p[0]) + double(p[1])) + (double(p[2]) + double(p[3]));
  double d = 0.0;
#pragma unroll
  for (int j = 0; j < VEC; ++j) d = fma(double(v[j]), double(v[j]), d);
  return d;
}

__global__ void __launch_bounds__(THREADS) square_sums_kernel(const NormTable t, double* sums) {
  double sum[4] = {};  // (of each load's, so that the additions do not wait for one another)
  each_chunk(t, [&](int i, int64_t at, int64_t n) {
    by_type(int(t.size[i] & 3), [&](auto type) {
      using T = decltype(type);
      const T* p = static_cast<const T*>(t.p[0][i]) + at;
      float v[4][VEC];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = (k * THREADS + int(threadIdx.x)) * VEC;
        load_n<VEC>(p + c, n - c, v[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] += squares(v[k]);
    });
  });
  const double s = group_sum<THREADS / 64>((sum[0] + sum[1]) + (sum[2] + sum[3]));
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__global__ void __launch_bounds__(1024) root_kernel(const double* sums, int64_t n, float* norm) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += sums[i];
  s = group_sum<16>(s);
  if (threadIdx.x == 0) *norm = float(sqrt(s));
}

template <bool IN_PLACE>
__global__ void __launch_bounds__(THREADS) clip_kernel(const ClipTable t, const float* norm, float most) {
  const float n = *norm;
  const float f = n <= most ? 1.f : most / n;  // (no number where the norm is none)
  if (IN_PLACE && f == 1.f) return;
  each_chunk(t, [&](int i, int64_t at, int64_t left) {
    by_type(int(t.size[i] & 3), [&](auto type) {
      using T = decltype(type);
      const T* p = static_cast<const T*>(t.p[0][i]) + at;
      T* out = static_cast<T*>(t.p[1][i]) + at;
      float v[4][VEC];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = (k * THREADS + int(threadIdx.x)) * VEC;
        load_n<VEC>(p + c, left - c, v[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = (k * THREADS + int(threadIdx.x)) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[k][j] *= f;
        store_n<VEC>(out + c, left - c, v[k]);
      }
    });
  });
}

// Fills tables with tensors of at least one value and launches each:
// f(table, workgroups) returns a HIP error code.
template <class T, class F>
int each_table(const TensorList& l, int capacity, F&& f) {
  T t;
  t.n = 0, t.first[0] = 0;
  const auto flush = [&] {
    if (t.n == 0) return int(hipSuccess);
    const int e = f(t, int(std::min<uint32_t>(t.first[t.n], GROUPS)));
    t.n = 0;
    return e;
  };
  for (int64_t i = 0; i < l.n; ++i) {
    if (l.counts[i] == 0) continue;
    t.p[0][t.n] = l.p[i];
    if constexpr (sizeof(t.p) > sizeof(t.p[0])) t.p[1][t.n] = l.out != nullptr ? l.out[i] : l.p[i];
    t.size[t.n] = l.counts[i] * 4 + l.types[i];
    t.first[t.n + 1] = t.first[t.n] + uint32_t((l.counts[i] + CHUNK - 1) / CHUNK);
    if (++t.n == capacity) {
      const int e = flush();
      if (e != hipSuccess) return e;
    }
  }
  return flush();
}

}  // namespace

size_t global_norm_workspace(const TensorList& l) {
  // (a sum for each workgroup of each launch)
  int64_t chunks = 0, some = 0;
  for (int64_t i = 0; i < l.n; ++i) chunks += (l.counts[i] + CHUNK - 1) / CHUNK, some += l.counts[i] > 0;
  const int64_t launches = (some + NORM_TENSORS - 1) / NORM_TENSORS;
  return size_t(std::min<int64_t>(chunks, launches * GROUPS)) * 8;
}

int64_t clip_chunks(int64_t count) { return (count + CHUNK - 1) / CHUNK; }

int launch_global_norm(const TensorList& l, float* norm, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  double* sums = static_cast<double*>(workspace);
  int64_t n = 0;
  const int e = each_table<NormTable>(l, NORM_TENSORS, [&](const NormTable& t, int groups) {
    hipLaunchKernelGGL(square_sums_kernel, dim3(groups), dim3(THREADS), 0, s, t, sums + n);
    n += groups;
    return int(hipGetLastError());
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(root_kernel, dim3(1), dim3(1024), 0, s, sums, n, norm);
  return hipGetLastError();
}

int launch_clip(const TensorList& l, const float* norm, float most, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return each_table<ClipTable>(l, CLIP_TENSORS, [&](const ClipTable& t, int groups) {
    if (l.out == nullptr)
      hipLaunchKernelGGL((clip_kernel<true>), dim3(groups), dim3(THREADS), 0, s, t, norm, most);
    else
      hipLaunchKernelGGL((clip_kernel<false>), dim3(groups), dim3(THREADS), 0, s, t, norm, most);
    return int(hipGetLastError());
  });
}

}  // namespace dtst
