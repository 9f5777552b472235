// Selective state-space scan (dtst_scan):
//   D_t = log(1 + exp(delta_t)),  h_t[n] = exp(D_t a[n]) h_{t-1}[n] + D_t x_t b_t[n],
//   y_t = (sum_n c_t[n] h_t[n] + d x_t) o_t s(o_t),
// feature by feature, with N states h[n] each and b_t, c_t common to all features.
//
// N values of work a value of the sequences, five to seven instructions each (the
// exponential's two slots among them): bound by the vector unit, not by HBM.  A lane takes
// a feature with all its states in registers, and goes through the steps; where features
// and entries are too few to fill the card, the steps are cut into segments: each one's
// end from a zero state first, what enters each by composing these, then the outputs,
// where each state's exponentials are computed a second time.  (The tables that a first
// pass would have to keep for it are N times the sequences.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "scan_ops.h"

namespace dtst {
namespace {

// What enters each segment, in the place of the end in `carry`; in their order, or
// (a gradient's) from the last to the first.  RUNS waves compose a run of them each,
// meet in LDS, and go over their runs: eight where features are few and segments many
// (195 of 1280 features' 16 states: 17 against 43 us), one where there are a thousand
// waves of them (31 of 4 x 2048 features' 16 states: 11 against 20 us).
template <int RUNS>
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
  float h = first != nullptr ? first[i] : 0.f;
  if constexpr (RUNS > 1) {
    float H = 0.f, total = 0.f, top = 0.f;
    segments([&](int, float end, float sum, float most) {
      H = run_decay(a2, sum, most) * H + end;
      total += sum, top = fmaxf(top, most);
    });
    mapA[run][lane] = run_decay(a2, total, top), mapH[run][lane] = H;
    __syncthreads();
    for (int k = 0; k < run; ++k) h = mapA[k][lane] * h + mapH[k][lane];
  }
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

}  // namespace

int launch_scan_carry(const ScanArgs& p, const float* a, const float* first, float* carry, bool reverse, void* stream) {
  const int64_t n = p.batch * p.states * p.features;
  const auto go = [&](auto kernel, int runs) {
    hipLaunchKernelGGL(kernel, dim3(unsigned((n + 63) / 64)), dim3(64 * runs), 0, static_cast<hipStream_t>(stream), p, a,
                       first, carry, int(reverse));
  };
  if (n < 65536)
    go(scan_carry_kernel<8>, 8);
  else
    go(scan_carry_kernel<1>, 1);
  return hipGetLastError();
}

int launch_copy_states(const float* in, float* out, int64_t n, void* stream) {
  if (out == nullptr || out == in || n == 0) return hipSuccess;
  hipLaunchKernelGGL(copy_states_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), in, out, n);
  return hipGetLastError();
}

// Segments of a sequence: as many as give the card so many waves, not one more: those that
// the forward's kernel has registers for in one go (4 x 4096 x 1024 of 4 or 8 states: 75 and
// 93 us with four a SIMD, 82 and 104 with three; 65536 x 1280 of 16: 589 us with three, 607
// with four; 8 x 2048 x 1024 of 40: 375 with two, 460 with three), two a SIMD twice over, the
// backward's (4 x 4096 x 2048 of 16, both directions: 891 us with 4096 waves; 1315, 912, 937
// and 901 with 1024, 2048, 6144 and 8192).  Whole sequences from 1024 waves on, as at 2048 the
// second pass over the steps costs more than waves side by side save (32 x 1024 x 4096 of 16:
// 571 us whole, 908 in two).  Between, neither wins: 512 steps x 4096 features, 1024, 1280,
// 1536 and 1920 waves, whole and in segments, forward 143 184 185 187 and 137 158 185 213 us
// with 4 states, 211 285 286 287 and 223 318 321 287 with 16, 671 908 911 912 and 756 909 911
// 915 with 64; both directions 488 572 590 608 and 421 524 676 730, 937 1057 1085 1114 and 775
// 1044 1287 1313, 3011 5478 5511 5570 and 3732 4858 5029 6250.  Lengths have no say in it.
int scan_segments(int64_t batch, int64_t steps, int64_t features, int64_t states, bool adj) {
  const int64_t waves = batch * ((features + 63) / 64), spans = (steps + SCAN_SPAN - 1) / SCAN_SPAN;
  if (waves <= 0 || spans <= 1 || waves >= 1024) return 1;
  const int64_t most = (adj ? 4096 : 1024 * scan_waves(int(states))) / waves, each = (spans + most - 1) / most;  // (spans)
  return int((spans + each - 1) / each);
}

ScanArgs scan_args(const dtst_scan_desc& d, const int32_t* lengths, bool adj) {
  auto st = [](const int64_t (&s)[2]) { return Strides{s[0], s[1]}; };
  ScanArgs p{d.batch, d.steps, d.features, int(d.states), st(d.x_stride), st(d.delta_stride), st(d.b_stride),
             st(d.c_stride), st(d.o_stride), st(d.y_stride), st(d.g_x_stride), st(d.g_delta_stride), st(d.g_b_stride),
             st(d.g_c_stride), st(d.g_o_stride), lengths, 0, 0, 0, 0};
  p.spans = (d.steps + SCAN_SPAN - 1) / SCAN_SPAN;
  p.tiles = (d.features + 63) / 64;
  p.segments = scan_segments(d.batch, d.steps, d.features, d.states, adj);
  p.segment = (p.spans + p.segments - 1) / p.segments * SCAN_SPAN;
  return p;
}

size_t scan_carry_bytes(const dtst_scan_desc& d, bool adj) {
  const int s = scan_segments(d.batch, d.steps, d.features, d.states, adj);
  return s > 1 ? size_t(d.batch) * s * (d.states + 2) * d.features * 4 : 0;
}

int launch_scan(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b, const void* c,
                const float* skip, const void* o, const float* h_zero, const int32_t* lengths, void* y, float* h_out,
                float* states, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.steps == 0) return launch_copy_states(h_zero, h_out, d.batch * d.states * d.features, s);
  const ScanArgs p = scan_args(d, lengths, false);
  const ScanPointers q{x, delta, b, c, o, a, skip, h_zero, y, h_out, states, static_cast<float*>(workspace)};
  if (d.type == DTST_F32) return launch_scan_type<float>(p, q, s);
  if (d.type == DTST_BF16) return launch_scan_type<bf16_t>(p, q, s);
  return launch_scan_type<f16_t>(p, q, s);
}

}  // namespace dtst
