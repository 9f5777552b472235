// Selective state-space scan (dtst_scan):
//   D_t = log(1 + exp(delta_t)),  h_t[n] = exp(D_t a[n]) h_{t-1}[n] + D_t x_t b_t[n],
//   y_t = (sum_n c_t[n] h_t[n] + d x_t) o_t s(o_t),
// feature by feature, with N states h[n] each and b_t, c_t common to all features.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "scan_ops.h"

namespace dtst {
namespace {

constexpr int ROWS = 4;     // steps whose loads are in flight together
constexpr int CHUNK = 32;   // steps whose b and c are in LDS together
constexpr int WAVES = 4;    // of a workgroup, 64 features each

// ENDS: the state at each segment's end from a zero state, with the sum and the
// largest of its D, into `carry` (batch, segments, N + 2, features).  Else the
// outputs, from the state that enters each segment: carry's, or h_zero's where
// there is one segment.  EXACT: N = NS.
template <class T, int NS, bool EXACT, bool ENDS>
__global__ void __launch_bounds__(64 * WAVES, NS <= 16 ? 3 : 1)
scan_kernel(const ScanArgs p, const T* x, const T* delta, const float* __restrict__ a, const T* b, const T* c,
            const float* __restrict__ skip, const T* o, const float* h_zero, T* y, float* h_out, float* states,
            float* carry) {
  constexpr int KINDS = ENDS ? 1 : 2;
  __shared__ float bc[2][KINDS][CHUNK][NS];
  constexpr int LOADS = (KINDS * CHUNK * NS + 64 * WAVES - 1) / (64 * WAVES);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int N = EXACT ? NS : p.states;
  const int64_t groups = (p.tiles + WAVES - 1) / WAVES;
  const int64_t tile = blockIdx.x % groups * WAVES + wave, place = blockIdx.x / groups;
  const int segments = ENDS ? p.segments - 1 : p.segments;  // (nothing comes after the last's end)
  const int seg = int(place % segments);
  const int64_t e = place / segments, F = p.features;
  const bool active = tile < p.tiles;
  const int64_t length = scan_length(p, e), t0 = seg * p.segment, end = min(t0 + p.segment, p.steps);
  const int64_t live = min(end, length);
  // (lanes past the end take the last feature too: the same results to the same places)
  const uint32_t f = uint32_t(min<int64_t>((active ? tile : 0) * 64 + lane, F - 1)), ft = lane_offset(f * sizeof(T));
  const uint32_t f4 = lane_offset(f * 4);
  float* mine = carry + (e * p.segments + seg) * (N + 2) * F;

  float h[NS], a2[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    h[n] = a2[n] = 0.f;
    if (EXACT || n < N) {
      a2[n] = get(a + n * F, f4) * LOG2E;
      if constexpr (!ENDS) {
        if (p.segments > 1)
          h[n] = get(mine + n * F, f4);
        else if (h_zero != nullptr)
          h[n] = get(h_zero + (e * N + n) * F, f4);
      }
    }
  }
  const float dv = !ENDS && skip != nullptr ? skip[f] : 0.f;
  float sum = 0.f, most = 0.f;

  // b and c of CHUNK steps from t on
  float staged[LOADS];
  const auto fetch = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 64 * WAVES + int(threadIdx.x), n = at % NS, r = at / NS % CHUNK;
      const bool second = at >= CHUNK * NS;
      staged[i] = 0.f;
      if (n < N && t + r < live && at < KINDS * CHUNK * NS)
        staged[i] = second ? float((c + dtst::at(p.c, e, t + r))[n]) : float((b + dtst::at(p.b, e, t + r))[n]);
    }
  };
  const auto put_staged = [&](int buffer) {
    float* to = &bc[buffer][0][0][0];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 64 * WAVES + int(threadIdx.x);
      if (at < KINDS * CHUNK * NS) to[at] = staged[i];
    }
  };

  // ROWS rows of the sequences, from t on
  T rx[ROWS], rd[ROWS], ro[ROWS] = {};
  const auto rows = [&](int64_t t) {
    const auto all = [&](auto full_) {
      constexpr bool FULL = decltype(full_)::value;
      const int there = int(min<int64_t>(live - t, ROWS));
      get_rows<FULL>(x, p.x, e, t, there, ft, rx);
      get_rows<FULL>(delta, p.delta, e, t, there, ft, rd);
      if (!ENDS && o != nullptr) get_rows<FULL>(o, p.o, e, t, there, ft, ro);
    };
    if (t + ROWS <= live)
      all(std::true_type());
    else
      all(std::false_type());
  };
  const auto keep = [&](int64_t span) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (EXACT || n < N) put(states + ((e * p.spans + span) * N + n) * F, f4, h[n]);
  };

  if (t0 < live) {
    fetch(t0);
    if (active) rows(t0);
    put_staged(0);
  }
  int buffer = 0;
  for (int64_t t = t0; t < live; t += CHUNK, buffer ^= 1) {
    __syncthreads();
    const bool more = t + CHUNK < live;
    if (more) fetch(t + CHUNK);
    if (active) {
      const int last = int(min<int64_t>(CHUNK, live - t));
      for (int r0 = 0; r0 < last; r0 += ROWS) {
        float D[ROWS], Dx[ROWS], direct[ROWS], gate[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          D[i] = softplus<T>(float(rd[i]));
          Dx[i] = D[i] * float(rx[i]);
          if constexpr (!ENDS) {  // (selected, as branches would divide the steps)
            const float v = float(ro[i]);
            direct[i] = skip != nullptr ? dv * float(rx[i]) : 0.f;
            gate[i] = o != nullptr ? v * logistic<T>(v) : 1.f;
          }
        }
        if (t + r0 + ROWS < live) rows(t + r0 + ROWS);
        if (!ENDS && states != nullptr && (t + r0) % SCAN_SPAN == 0) keep((t + r0) / SCAN_SPAN);
        const auto steps = [&](auto full_) {  // full: all rows are live
          constexpr bool FULL = decltype(full_)::value;
          T* to = ENDS ? nullptr : y + dtst::at(p.y, e, t + r0);
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            if (!FULL && r0 + i >= last) continue;
            if constexpr (ENDS) sum += D[i], most = fmaxf(most, D[i]);
            float v = ENDS ? 0.f : direct[i];
#pragma unroll
            for (int n = 0; n < NS; ++n)
              if (EXACT || n < N) {
                h[n] = __builtin_amdgcn_exp2f(D[i] * a2[n]) * h[n] + Dx[i] * bc[buffer][0][r0 + i][n];
                if constexpr (!ENDS) v = fmaf(h[n], bc[buffer][KINDS - 1][r0 + i][n], v);
              }
            if constexpr (!ENDS) {
              put(to, ft, v * gate[i]);
              to += p.y.t;
            }
          }
        };
        if (r0 + ROWS <= last)
          steps(std::true_type());
        else
          steps(std::false_type());
      }
    }
    if (more) put_staged(buffer ^ 1);
  }
  if (!active) return;
  if constexpr (ENDS) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (EXACT || n < N) put(mine + n * F, f4, h[n]);
    put(mine + N * F, f4, sum);
    put(mine + (N + 1) * F, f4, most);
  } else {
    for (int64_t t = max(t0, live); t < end; ++t) put(y + dtst::at(p.y, e, t), ft, 0.f);
    if (states != nullptr)  // (past the end the state stands still)
      for (int64_t t = max(t0, (live + SCAN_SPAN - 1) / SCAN_SPAN * SCAN_SPAN); t < end; t += SCAN_SPAN) keep(t / SCAN_SPAN);
    if (h_out != nullptr && (length > t0 ? length <= end : length == 0 && seg == 0)) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
        if (EXACT || n < N) put(h_out + (e * N + n) * F, f4, h[n]);
    }
  }
}

// What enters each segment, in the place of the end in `carry`; in their order, or
// (a gradient's) from the last to the first.  Segments are many where features are
// few: eight waves compose a run of them each, meet in LDS, and go over their runs.
constexpr int RUNS = 8;
__global__ void __launch_bounds__(64 * RUNS)
scan_carry_kernel(const ScanArgs p, const float* __restrict__ a, const float* first, float* carry, int reverse) {
  constexpr int AHEAD = 8;  // segments whose loads are in flight together
  __shared__ float mapA[RUNS][64], mapH[RUNS][64];
  const int run = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t F = p.features, N = p.states, all = p.batch * N * F;
  const int64_t i = min<int64_t>(int64_t(blockIdx.x) * 64 + lane, all - 1);  // (lanes past the end: the last again)
  const int64_t e = i / (N * F), f = i % F, n = i / F % N;
  const float a2 = a[n * F + f] * LOG2E;
  const int each = (p.segments + RUNS - 1) / RUNS, s0 = min(run * each, p.segments), s1 = min(s0 + each, p.segments);
  const int64_t step = (reverse ? -1 : 1) * (N + 2) * F;
  float* const at = carry + (e * p.segments + (reverse ? p.segments - 1 : 0)) * (N + 2) * F + f;
  // f(segment, its end, its sum of D, its largest D); the last segment has none
  const auto segments = [&](auto&& f) {
    for (int s = s0; s < s1; s += AHEAD) {
      float H[AHEAD], sum[AHEAD], most[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float* from = at + min(s + k, p.segments - 2) * step;
        H[k] = from[n * F], sum[k] = from[N * F], most[k] = from[(N + 1) * F];
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (s + k < s1) f(s + k, H[k], sum[k], most[k]);
    }
  };
  float H = 0.f, total = 0.f, top = 0.f;
  segments([&](int, float end, float sum, float most) {
    H = run_decay(a2, sum, most) * H + end;
    total += sum, top = fmaxf(top, most);
  });
  mapA[run][lane] = run_decay(a2, total, top), mapH[run][lane] = H;
  float h = first != nullptr ? first[i] : 0.f;
  __syncthreads();  // (all ends are read; what follows writes only a wave's own)
  for (int k = 0; k < run; ++k) h = mapA[k][lane] * h + mapH[k][lane];
  segments([&](int s, float end, float sum, float most) {
    at[s * step + n * F] = h;
    h = run_decay(a2, sum, most) * h + end;
  });
}

// h_out = h_zero (g_hzero = g_h) where there are no steps.
__global__ void __launch_bounds__(256) copy_states_kernel(const float* in, float* out, int64_t n) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) out[i] = in != nullptr ? in[i] : 0.f;
}

template <class T, int NS, bool EXACT>
int launch_forms(const ScanArgs& p, const void* x, const void* delta, const float* a, const void* b, const void* c,
                 const float* skip, const void* o, const float* h_zero, void* y, float* h_out, float* states,
                 float* carry, hipStream_t s) {
  const int64_t groups = (p.tiles + WAVES - 1) / WAVES * p.batch;
  const auto go = [&](auto kernel, int segments) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(groups * segments)), dim3(64 * WAVES), 0, s, p, static_cast<const T*>(x),
                       static_cast<const T*>(delta), a, static_cast<const T*>(b), static_cast<const T*>(c), skip,
                       static_cast<const T*>(o), h_zero, static_cast<T*>(y), h_out, states, carry);
    return int(hipGetLastError());
  };
  if (p.segments > 1) {
    int e = go(scan_kernel<T, NS, EXACT, true>, p.segments - 1);
    if (e != hipSuccess) return e;
    e = launch_scan_carry(p, a, h_zero, carry, false, s);
    if (e != hipSuccess) return e;
  }
  return go(scan_kernel<T, NS, EXACT, false>, p.segments);
}

}  // namespace

int launch_scan_carry(const ScanArgs& p, const float* a, const float* first, float* carry, bool reverse, void* stream) {
  const int64_t n = p.batch * p.states * p.features;
  hipLaunchKernelGGL(scan_carry_kernel, dim3(unsigned((n + 63) / 64)), dim3(64 * RUNS), 0,
                     static_cast<hipStream_t>(stream), p, a, first, carry, int(reverse));
  return hipGetLastError();
}

int launch_copy_states(const float* in, float* out, int64_t n, void* stream) {
  if (out == nullptr || out == in || n == 0) return hipSuccess;
  hipLaunchKernelGGL(copy_states_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), in, out, n);
  return hipGetLastError();
}

// Segments of a sequence: as many as give the card 4096 waves, not one more.
int scan_segments(int64_t batch, int64_t steps, int64_t features) {
  const int64_t waves = batch * ((features + 63) / 64), spans = (steps + SCAN_SPAN - 1) / SCAN_SPAN;
  if (waves <= 0 || spans <= 1 || waves >= 2048) return 1;
  const int64_t most = 4096 / waves, each = (spans + most - 1) / most;  // (spans)
  return int((spans + each - 1) / each);
}

ScanArgs scan_args(const dtst_scan_desc& d, const int32_t* lengths) {
  auto st = [](const int64_t (&s)[2]) { return Strides{s[0], s[1]}; };
  ScanArgs p{d.batch, d.steps, d.features, int(d.states), st(d.x_stride), st(d.delta_stride), st(d.b_stride),
             st(d.c_stride), st(d.o_stride), st(d.y_stride), st(d.g_x_stride), st(d.g_delta_stride), st(d.g_b_stride),
             st(d.g_c_stride), st(d.g_o_stride), lengths, 0, 0, 0, 0};
  p.spans = (d.steps + SCAN_SPAN - 1) / SCAN_SPAN;
  p.tiles = (d.features + 63) / 64;
  p.segments = scan_segments(d.batch, d.steps, d.features);
  p.segment = (p.spans + p.segments - 1) / p.segments * SCAN_SPAN;
  return p;
}

size_t scan_carry_bytes(const dtst_scan_desc& d) {
  const int s = scan_segments(d.batch, d.steps, d.features);
  return s > 1 ? size_t(d.batch) * s * (d.states + 2) * d.features * 4 : 0;
}

int launch_scan(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b, const void* c,
                const float* skip, const void* o, const float* h_zero, const int32_t* lengths, void* y, float* h_out,
                float* states, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.steps == 0) return launch_copy_states(h_zero, h_out, d.batch * d.states * d.features, s);
  const ScanArgs p = scan_args(d, lengths);
  const auto by_states = [&](auto t) {
    using T = decltype(t);
    const auto go = [&](auto ns, auto exact) {
      return launch_forms<T, decltype(ns)::value, decltype(exact)::value>(
          p, x, delta, a, b, c, skip, o, h_zero, y, h_out, states, static_cast<float*>(workspace), s);
    };
    using std::integral_constant;
    const auto sized = [&](auto ns) {
      return p.states == decltype(ns)::value ? go(ns, std::true_type()) : go(ns, std::false_type());
    };
    if (p.states <= 8) return sized(integral_constant<int, 8>());
    if (p.states <= 16) return sized(integral_constant<int, 16>());
    if (p.states <= 32) return sized(integral_constant<int, 32>());
    return sized(integral_constant<int, 64>());
  };
  if (d.type == DTST_F32) return by_states(float());
  if (d.type == DTST_BF16) return by_states(bf16_t());
  return by_states(f16_t());
}

}  // namespace dtst
