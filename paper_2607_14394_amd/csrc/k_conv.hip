// Short causal convolution along the steps and its backward (dtst_conv,
// dtst_conv_adj), feature by feature:
//   v_t = bias + sum_k w_k x_{t-K+1+k},   y_t = v_t s(v_t)  (or v_t),
//   p_t = g_y_t s(v_t) (1 + v_t s(-v_t)),   g_x_t = sum_k w_k p_{t+K-1-k},
//   g_w_k = sum_t p_t x_{t-K+1+k},   g_bias = sum_t p_t,
// where the rows before step 0 are the state.
//
// K + 10 operations a value: bound by HBM, with the vector unit near in the backward.
// A lane takes 16 bytes of neighbouring features and a run of steps, whose last K - 1
// inputs stay in its registers, so that a run reads only K - 1 rows more than it
// writes; the backward goes the same way, K - 1 steps behind its p.  4 x 4096 x 2048 in
// bf16, four taps: 31 us forward (134 MB, 4.3 TB/s), 53 + 5 us backward (201 MB, 3.8
// TB/s, the vector unit busy 75% of the time); 24 sequences of 731 steps at most, half of them
// live, and 1001 features in 32 bits 39 us, 28 from the last-level cache (104 MB).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 8;  // rows whose loads are in flight together, and the least of a run

struct ConvArgs {
  int64_t batch, steps, features;
  Strides x, y, gx;
  const int32_t* lengths;
  int64_t vectors, runs, run;  // of a row; of a sequence; steps of a run
  int lanes;                   // of a workgroup's threads along the features (backward)
};

__device__ __forceinline__ int64_t conv_length(const ConvArgs& p, int64_t b) {
  if (p.lengths == nullptr) return p.steps;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.steps ? p.steps : n;
}

// Row t of a sequence, of the state before step 0, zeros without one; t < the
// sequence's length.
template <int V, int K, class T>
__device__ __forceinline__ void input_row(const ConvArgs& p, const T* x, const T* state, int64_t b, int64_t t, int64_t f,
                                          float (&out)[V]) {
  if (t >= 0) {
    load_n<V>(x + at(p.x, b, t) + f, p.features - f, out);
  } else if (state != nullptr) {
    load_n<V>(state + (b * (K - 1) + t + K - 1) * p.features + f, p.features - f, out);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = 0.f;
  }
}

template <class T, int K, int V, bool SILU>
__global__ void __launch_bounds__(THREADS)
conv_kernel(const ConvArgs p, const T* x, const float* __restrict__ w, const float* __restrict__ bias, const T* state, T* y,
            T* state_out) {
  const int64_t id = int64_t(blockIdx.x) * THREADS + threadIdx.x;
  const int64_t f = id % p.vectors * V, run = id / p.vectors % p.runs, b = id / p.vectors / p.runs;
  if (b >= p.batch) return;
  const int64_t F = p.features, n = conv_length(p, b), t0 = run * p.run, end = min(t0 + p.run, p.steps);
  const int64_t live = min(end, n);
  float z[K - 1 + BATCH][V], wv[K][V], bv[V];
#pragma unroll
  for (int k = 0; k < K; ++k) load_n<V>(w + k * F + f, F - f, wv[k]);
#pragma unroll
  for (int j = 0; j < V; ++j) bv[j] = 0.f;
  if (bias != nullptr) load_n<V>(bias + f, F - f, bv);
  // the state at the end: rows n - K + 1 .. n - 1; read before it is written, as it may be the first's place, which
  // no other lane reads (a run is longer than the state)
  if (run == 0 && state_out != nullptr) {
    float last[K][V];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) input_row<V, K>(p, x, state, b, n - K + 1 + k, f, last[k]);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) input_row<V, K>(p, x, state, b, k - K + 1, f, z[k]);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) store_n<V>(state_out + (b * (K - 1) + k) * F + f, F - f, last[k]);
  } else if (t0 < live) {
#pragma unroll
    for (int k = 0; k < K - 1; ++k) input_row<V, K>(p, x, state, b, t0 + k - K + 1, f, z[k]);
  }
  // BATCH steps; full: all of them live, and the lane's features all there
  const T* xr = x + at(p.x, b, t0) + f;
  T* yr = y + at(p.y, b, t0) + f;
  const auto steps = [&](auto full_, int64_t rows) {
    constexpr bool FULL = decltype(full_)::value;
    const int64_t left = FULL ? V : F - f;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {  // (past the end the last row again)
      load_n<V>(xr, left, z[K - 1 + i]);
      if (FULL || i + 1 < rows) xr += p.x.t;
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        v[j] = bv[j];
#pragma unroll
        for (int k = 0; k < K; ++k) v[j] = fmaf(z[i + k][j], wv[k][j], v[j]);
        if constexpr (SILU) v[j] *= logistic<T>(v[j]);
      }
      if (FULL || i < rows) store_n<V>(yr, left, v);
      yr += p.y.t;
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) z[k][j] = z[k + BATCH][j];
  };
  for (int64_t t = t0; t < live; t += BATCH) {
    if (__all(t + BATCH <= live && f + V <= F))  // (of the whole wave, which else would take both ways)
      steps(std::true_type(), BATCH);
    else
      steps(std::false_type(), live - t);
  }
  const float zero[V] = {};
  for (int64_t t = max(t0, live); t < end; ++t) store_n<V>(y + at(p.y, b, t) + f, F - f, zero);
}

// part: (workgroups along the runs, K + 1, features), each workgroup's g_w and g_bias.
template <class T, int K, int V, bool SILU>
__global__ void __launch_bounds__(THREADS)
conv_adj_kernel(const ConvArgs p, const T* x, const float* __restrict__ w, const float* __restrict__ bias, const T* state,
                const T* g_y, const T* g_state_out, T* g_x, T* g_state, float* part) {
  constexpr int STEP = 4;  // rows whose loads are in flight together
  __shared__ float sums[(K + 1) * V][THREADS];
  const int lanes = p.lanes, slots = THREADS / lanes, lane = threadIdx.x % lanes, slot = threadIdx.x / lanes;
  const int64_t blocks = (p.vectors + lanes - 1) / lanes;
  const int64_t f = (blockIdx.x % blocks * lanes + lane) * V, unit = blockIdx.x / blocks * slots + slot;
  const int64_t run = unit % p.runs, b = unit / p.runs, F = p.features;
  float gw[K][V], gb[V];
#pragma unroll
  for (int j = 0; j < V; ++j) gb[j] = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) gw[k][j] = 0.f;
  if (f < F && b < p.batch) {
    const int64_t n = conv_length(p, b), t0 = run * p.run, end = min(t0 + p.run, p.steps), live = min(end, n);
    float wv[K][V], bv[V], z[K - 1 + STEP][V], q[K - 1 + STEP][V];  // q: p, the last K - 1 rows of it first
#pragma unroll
    for (int k = 0; k < K; ++k) load_n<V>(w + k * F + f, F - f, wv[k]);
#pragma unroll
    for (int j = 0; j < V; ++j) bv[j] = 0.f;
    if (bias != nullptr) load_n<V>(bias + f, F - f, bv);
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) z[k][j] = q[k][j] = 0.f;
    if (t0 < live) {
#pragma unroll
      for (int k = 0; k < K - 1; ++k) input_row<V, K>(p, x, state, b, t0 + k - K + 1, f, z[k]);
    }
    // The rows of this run, the state's too in the first: written K - 1 steps behind p.
    const int64_t first = run == 0 ? 1 - K : t0;
    const T *xr = x + at(p.x, b, t0) + f, *gr = g_y + at(p.y, b, t0) + f;
    T* to = g_x + (at(p.gx, b, t0) - (K - 1) * p.gx.t) + f;  // (row t - K + 1's place)
    // STEP steps; full: all live, of this run, as are the rows that they finish, and
    // the lane's features all there
    const auto steps = [&](auto full_, int64_t t) {
      constexpr bool FULL = decltype(full_)::value;
      const int64_t left = FULL ? V : F - f;
      float g[STEP][V];
#pragma unroll
      for (int i = 0; i < STEP; ++i) {
        if (FULL || t + i < n) {
          load_n<V>(xr + i * p.x.t, left, z[K - 1 + i]);
          load_n<V>(gr + i * p.y.t, left, g[i]);
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) z[K - 1 + i][j] = g[i][j] = 0.f;
        }
      }
      xr += STEP * p.x.t, gr += STEP * p.y.t;
#pragma unroll
      for (int i = 0; i < STEP; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float v = bv[j], d = g[i][j];
#pragma unroll
          for (int k = 0; k < K; ++k) v = fmaf(z[i + k][j], wv[k][j], v);
          if constexpr (SILU) {
            float s, sn;
            logistic<T>(v, s, sn);
            d *= s * fmaf(v, sn, 1.f);
          }
          if (!FULL && t + i >= n) d = 0.f;  // (v may be no number there)
          q[K - 1 + i][j] = d;
          if (FULL || t + i < live) {
            gb[j] += d;
#pragma unroll
            for (int k = 0; k < K; ++k) gw[k][j] = fmaf(d, z[i + k][j], gw[k][j]);
          }
        }
        const int64_t row = t + i - K + 1;
        if (FULL || (row >= first && row < end)) {
          float r[V] = {};
          if (FULL || row < n) {
#pragma unroll
            for (int k = 0; k < K; ++k)  // (the row's p_{row + K - 1 - k})
#pragma unroll
              for (int j = 0; j < V; ++j) r[j] = fmaf(q[i + K - 1 - k][j], wv[k][j], r[j]);
            if (g_state_out != nullptr && row > n - K) {
              float s[V];
              load_n<V>(g_state_out + (b * (K - 1) + row - (n - K + 1)) * F + f, F - f, s);
#pragma unroll
              for (int j = 0; j < V; ++j) r[j] += s[j];
            }
          }
          if (FULL || row >= 0)
            store_n<V>(to + i * p.gx.t, left, r);
          else if (g_state != nullptr)
            store_n<V>(g_state + (b * (K - 1) + row + K - 1) * F + f, F - f, r);
        }
      }
      to += STEP * p.gx.t;
#pragma unroll
      for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) z[k][j] = z[k + STEP][j], q[k][j] = q[k + STEP][j];
    };
    for (int64_t t = t0; t < end + K - 1; t += STEP) {
      if (__all(t + STEP <= live && t - K + 1 >= max<int64_t>(first, 0) && f + V <= F))
        steps(std::true_type(), t);
      else
        steps(std::false_type(), t);
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) sums[k * V + j][threadIdx.x] = gw[k][j];
#pragma unroll
  for (int j = 0; j < V; ++j) sums[K * V + j][threadIdx.x] = gb[j];
  __syncthreads();
  // (in the order of the runs)
  for (int i = threadIdx.x; i < (K + 1) * V * lanes; i += THREADS) {
    const int c = i % (V * lanes), k = i / (V * lanes), from = c / V;
    const int64_t column = blockIdx.x % blocks * lanes * V + c;
    if (column >= F) continue;
    float s = 0.f;
    for (int u = 0; u < slots; ++u) s += sums[k * V + c % V][u * lanes + from];
    part[(blockIdx.x / blocks * (K + 1) + k) * F + column] = s;
  }
}

// state_out = state, or g_state = g_state_out, where there are no steps.
template <class T>
__global__ void __launch_bounds__(256) copy_rows_kernel(const T* in, T* out, int64_t n) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) out[i] = in != nullptr ? in[i] : T(0.f);
}

template <class T>
int copy_rows(const void* in, void* out, int64_t n, hipStream_t s) {
  if (out == nullptr || out == in || n == 0) return hipSuccess;
  hipLaunchKernelGGL((copy_rows_kernel<T>), dim3(unsigned((n + 255) / 256)), dim3(256), 0, s, static_cast<const T*>(in),
                     static_cast<T*>(out), n);
  return hipGetLastError();
}

// Features of a lane: 16 bytes forward; four in the backward, whose sums and
// windows take more registers.
template <class T>
constexpr int forward_lane() { return 16 / sizeof(T); }
constexpr int BACKWARD_LANE = 4;

// Runs of as many steps as leave 2^17 lanes (two waves a SIMD), of at least BATCH: a run
// reads K - 1 rows again.  (The cases above: 46, 33 and 57 us; with 2^16 lanes 58, 32
// and 72, with 2^18 43, 34 and 68: ragged, forward, backward, in one run of calls.)
ConvArgs conv_args(const dtst_conv_desc& d, const int32_t* lengths, int lane) {
  ConvArgs p{d.batch, d.steps, d.features, {d.x_stride[0], d.x_stride[1]}, {d.y_stride[0], d.y_stride[1]},
             {d.g_x_stride[0], d.g_x_stride[1]}, lengths, 0, 0, 0, 64};
  p.vectors = (d.features + lane - 1) / lane;
  const int64_t rows = std::max<int64_t>(1, (int64_t(1) << 17) / std::max<int64_t>(1, p.vectors));  // runs of all entries
  p.run = std::max<int64_t>(1, d.batch * d.steps / rows);
  p.run = std::min<int64_t>((p.run + BATCH - 1) / BATCH * BATCH, int64_t(1) << 20);
  p.runs = std::max<int64_t>(1, (d.steps + p.run - 1) / p.run);
  while (p.lanes > 1 && p.lanes / 2 >= p.vectors) p.lanes /= 2;
  return p;
}

int64_t adj_parts(const ConvArgs& p) {
  const int64_t slots = THREADS / p.lanes;
  return (p.batch * p.runs + slots - 1) / slots;
}

template <class F>
int by_taps(int64_t taps, int silu, F&& f) {
  using std::integral_constant;
  const auto go = [&](auto k) { return silu ? f(k, std::true_type()) : f(k, std::false_type()); };
  switch (taps) {
    case 1: return go(integral_constant<int, 1>());
    case 2: return go(integral_constant<int, 2>());
    case 3: return go(integral_constant<int, 3>());
    case 4: return go(integral_constant<int, 4>());
    case 5: return go(integral_constant<int, 5>());
    case 6: return go(integral_constant<int, 6>());
    case 7: return go(integral_constant<int, 7>());
    default: return go(integral_constant<int, 8>());
  }
}

template <class F>
int by_type(int type, F&& f) {
  if (type == DTST_F32) return f(float());
  if (type == DTST_BF16) return f(bf16_t());
  return f(f16_t());
}

}  // namespace

// Workgroups of either direction.
int64_t conv_groups(const dtst_conv_desc& d, bool adj) {
  if (adj) {
    const ConvArgs p = conv_args(d, nullptr, BACKWARD_LANE);
    return adj_parts(p) * ((p.vectors + p.lanes - 1) / p.lanes);
  }
  const ConvArgs p = conv_args(d, nullptr, d.type == DTST_F32 ? 4 : 8);
  return (p.batch * p.runs * p.vectors + THREADS - 1) / THREADS;
}

int launch_conv(const dtst_conv_desc& d, const void* x, const float* w, const float* bias, const void* state,
                const int32_t* lengths, void* y, void* state_out, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_type(d.type, [&](auto t) {
    using T = decltype(t);
    if (d.steps == 0) return copy_rows<T>(state, state_out, d.batch * (d.taps - 1) * d.features, s);
    constexpr int V = forward_lane<T>();
    const ConvArgs p = conv_args(d, lengths, V);
    return by_taps(d.taps, d.silu, [&](auto k, auto silu) {
      hipLaunchKernelGGL((conv_kernel<T, decltype(k)::value, V, decltype(silu)::value>), dim3(unsigned(conv_groups(d, false))), dim3(THREADS), 0, s,
                         p, static_cast<const T*>(x), w, bias, static_cast<const T*>(state), static_cast<T*>(y),
                         static_cast<T*>(state_out));
      return int(hipGetLastError());
    });
  });
}

size_t conv_adj_workspace(const dtst_conv_desc& d) {
  if (d.batch == 0 || d.steps == 0 || d.features == 0) return 0;
  return size_t(adj_parts(conv_args(d, nullptr, BACKWARD_LANE))) * (d.taps + 1) * d.features * 4;
}

int launch_conv_adj(const dtst_conv_desc& d, const void* x, const float* w, const float* bias, const void* state,
                    const int32_t* lengths, const void* g_y, const void* g_state_out, void* g_x, float* g_weight,
                    float* g_bias, void* g_state, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  float* part = static_cast<float*>(workspace);
  const ConvArgs p = conv_args(d, lengths, BACKWARD_LANE);
  const bool steps = d.batch > 0 && d.steps > 0;
  const int e = by_type(d.type, [&](auto t) {
    using T = decltype(t);
    if (!steps) return copy_rows<T>(g_state_out, g_state, d.batch * (d.taps - 1) * d.features, s);
    return by_taps(d.taps, d.silu, [&](auto k, auto silu) {
      hipLaunchKernelGGL((conv_adj_kernel<T, decltype(k)::value, BACKWARD_LANE, decltype(silu)::value>),
                         dim3(unsigned(conv_groups(d, true))),
                         dim3(THREADS), 0, s, p, static_cast<const T*>(x), w, bias, static_cast<const T*>(state),
                         static_cast<const T*>(g_y), static_cast<const T*>(g_state_out), static_cast<T*>(g_x),
                         static_cast<T*>(g_state), part);
      return int(hipGetLastError());
    });
  });
  if (e != hipSuccess) return e;
  const int64_t cols = d.taps * d.features;
  return launch_sum_parts(part, steps ? adj_parts(p) : 0, cols + d.features, cols, cols + (g_bias != nullptr ? d.features : 0),
                          d.accumulate, g_weight, g_bias, s);
}

}  // namespace dtst
