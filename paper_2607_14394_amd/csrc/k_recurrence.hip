// Gated linear recurrence along the steps and its backward (dtst_recurrence,
// dtst_recurrence_adj):
//   h_t = s(z_t) h_{t-1} + s(-z_t) v_t,   y_t = h_t o_t s(o_t).
// A few operations per value: bound by HBM (z, v, o read, y written).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

constexpr int SPAN = DTST_RECURRENCE_SPAN;

// s(x) and s(-x), both to full relative precision (1 - s(x) would lose it).
// Infinities give 0 and 1, no number gives no number.
__device__ __forceinline__ void logistic(float x, float& s, float& sn) {
  const float e = __expf(-fabsf(x)), r = 1.f / (1.f + e);
  s = x >= 0.f ? r : e * r;
  sn = x >= 0.f ? e * r : r;
}

struct Strides {
  int64_t b, t;
};
__device__ __forceinline__ int64_t at(Strides s, int64_t b, int64_t t) { return b * s.b + t * s.t; }

struct Args {
  int64_t batch, steps, features;
  Strides z, v, o, y, gz, gv, go;
  const int32_t* lengths;
};

__device__ __forceinline__ int64_t length_of(const Args& p, int64_t b) {
  if (p.lengths == nullptr) return p.steps;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.steps ? p.steps : n;
}

// One lane a feature of a sequence, step by step.
template <class T>
__global__ void __launch_bounds__(64)
recurrence_serial_kernel(Args p, const T* z, const T* v, const T* o, const float* h_zero, T* y, float* h_out,
                         float* states) {
  const int64_t i = int64_t(blockIdx.x) * 64 + threadIdx.x;
  if (i >= p.batch * p.features) return;
  const int64_t b = i / p.features, c = i % p.features, n = length_of(p, b);
  const int64_t spans = (p.steps + SPAN - 1) / SPAN;
  float h = h_zero ? h_zero[i] : 0.f;
  for (int64_t t = 0; t < p.steps; ++t) {
    if (states != nullptr && t % SPAN == 0) states[(b * spans + t / SPAN) * p.features + c] = h;
    float r = 0.f;
    if (t < n) {
      float s, sn, so, son;
      logistic(float(z[at(p.z, b, t) + c]), s, sn);
      h = s * h + sn * float(v[at(p.v, b, t) + c]);
      r = h;
      if (o != nullptr) {
        const float ot = float(o[at(p.o, b, t) + c]);
        logistic(ot, so, son);
        r = h * ot * so;
      }
    }
    y[at(p.y, b, t) + c] = T(r);
  }
  if (h_out != nullptr) h_out[i] = h;
}

// Backward: the spans from the last to the first, the states inside a span
// again from its first.
template <class T>
__global__ void __launch_bounds__(64)
recurrence_adj_serial_kernel(Args p, const T* z, const T* v, const T* o, const float* states, const T* g_y,
                             const float* g_h, T* g_z, T* g_v, T* g_o, float* g_hzero) {
  const int64_t i = int64_t(blockIdx.x) * 64 + threadIdx.x;
  if (i >= p.batch * p.features) return;
  const int64_t b = i / p.features, c = i % p.features, n = length_of(p, b);
  const int64_t spans = (p.steps + SPAN - 1) / SPAN;
  float d = g_h ? g_h[i] : 0.f;
  for (int64_t k = spans - 1; k >= 0; --k) {
    float h[SPAN + 1];
    h[0] = states[(b * spans + k) * p.features + c];
    const int64_t t0 = k * SPAN, len = p.steps - t0 < SPAN ? p.steps - t0 : SPAN;
    for (int j = 0; j < len; ++j) {
      h[j + 1] = h[j];
      if (t0 + j >= n) continue;
      float s, sn;
      logistic(float(z[at(p.z, b, t0 + j) + c]), s, sn);
      h[j + 1] = s * h[j] + sn * float(v[at(p.v, b, t0 + j) + c]);
    }
    for (int j = int(len) - 1; j >= 0; --j) {
      const int64_t t = t0 + j;
      float gz = 0.f, gv = 0.f, go = 0.f;
      if (t < n) {
        float s, sn;
        logistic(float(z[at(p.z, b, t) + c]), s, sn);
        float gy = float(g_y[at(p.y, b, t) + c]);
        if (o != nullptr) {
          const float ot = float(o[at(p.o, b, t) + c]);
          float so, son;
          logistic(ot, so, son);
          go = gy * h[j + 1] * so * (1.f + ot * son);
          gy *= ot * so;
        }
        d += gy;
        gv = d * sn;
        gz = d * (h[j] - float(v[at(p.v, b, t) + c])) * s * sn;
        d *= s;
      }
      g_z[at(p.gz, b, t) + c] = T(gz);
      g_v[at(p.gv, b, t) + c] = T(gv);
      if (g_o != nullptr) g_o[at(p.go, b, t) + c] = T(go);
    }
  }
  if (g_hzero != nullptr) g_hzero[i] = d;
}

Args args_of(const dtst_recurrence_desc& d, const int32_t* lengths) {
  auto st = [](const int64_t (&s)[2]) { return Strides{s[0], s[1]}; };
  return Args{d.batch, d.steps, d.features, st(d.z_stride), st(d.v_stride), st(d.o_stride), st(d.y_stride),
              st(d.g_z_stride), st(d.g_v_stride), st(d.g_o_stride), lengths};
}

template <class F>
int by_type(int type, F&& f) {
  if (type == DTST_F32) return f(float());
  if (type == DTST_BF16) return f(bf16_t());
  return f(f16_t());
}

}  // namespace

size_t recurrence_workspace(int64_t, int64_t, int64_t, int) { return 0; }

int launch_recurrence(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o, const float* h_zero,
                      const int32_t* lengths, void* y, float* h_out, float* states, void*, void* stream) {
  return by_type(d.type, [&](auto t) {
    using T = decltype(t);
    const unsigned blocks = unsigned((d.batch * d.features + 63) / 64);
    hipLaunchKernelGGL(recurrence_serial_kernel<T>, dim3(blocks), dim3(64), 0, static_cast<hipStream_t>(stream),
                       args_of(d, lengths), static_cast<const T*>(z), static_cast<const T*>(v),
                       static_cast<const T*>(o), h_zero, static_cast<T*>(y), h_out, states);
    return int(hipGetLastError());
  });
}

int launch_recurrence_adj(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o,
                          const int32_t* lengths, const float* states, const void* g_y, const float* g_h, void* g_z,
                          void* g_v, void* g_o, float* g_hzero, void*, void* stream) {
  return by_type(d.type, [&](auto t) {
    using T = decltype(t);
    const unsigned blocks = unsigned((d.batch * d.features + 63) / 64);
    hipLaunchKernelGGL(recurrence_adj_serial_kernel<T>, dim3(blocks), dim3(64), 0, static_cast<hipStream_t>(stream),
                       args_of(d, lengths), static_cast<const T*>(z), static_cast<const T*>(v),
                       static_cast<const T*>(o), states, static_cast<const T*>(g_y), g_h, static_cast<T*>(g_z),
                       static_cast<T*>(g_v), static_cast<T*>(g_o), g_hzero);
    return int(hipGetLastError());
  });
}

}  // namespace dtst
