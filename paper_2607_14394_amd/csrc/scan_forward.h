// The forward state-space scan's kernel, by type (k_scan_f32.hip, k_scan_bf16.hip,
// k_scan_f16.hip).
//
// Of 16 states, 7.3 vector instructions a state and step for the outputs, 5.7 for the
// segments' ends, with the step size, the gate and the loads shared among the states; the
// exponential takes two slots.  4 x 4096 x 2048 in bf16: 105 us the ends, 145 the outputs
// with the states that the backward needs, the vector unit busy 91% and 89% of the time;
// 65536 x 1280: 249 and 325 us (93%).  b and c come from LDS, the same word for all lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "scan_ops.h"

namespace dtst {
namespace {

// Steps whose loads are in flight together.  (16 states, three waves a SIMD, 4 x 4096 x
// 2048, ends and outputs: 248 us with four; eight and two waves 252, one or two and four
// waves 277 to 292.  With more states, four steps' b and c leave registers for one wave a
// SIMD: 544 against 261 us for 32 sequences of 1333 steps, 168 features and 55 states, 384
// against 240 for 4 x 4096 x 512 of 64.)
constexpr int rows_of_states(int NS) { return NS <= 16 ? 4 : 1; }
constexpr int EACH = 8;  // steps, for each wave of a workgroup, whose b and c are in LDS together

// ENDS: the state at each segment's end from a zero state, with the sum and the
// largest of its D, into `carry` (batch, segments, N + 2, features).  Else the
// outputs, from the state that enters each segment: carry's, or h_zero's where
// there is one segment.  N is NS or (N >= LEAST) below; the states past N are left
// out by branches, as zeros in their place would meet infinities.
template <class T, int NS, int LEAST, int WAVES, bool ENDS>
__global__ void __launch_bounds__(64 * WAVES, scan_waves(NS))
scan_kernel(const ScanArgs p, const T* x, const T* delta, const float* __restrict__ a, const T* b, const T* c,
            const float* __restrict__ skip, const T* o, const float* h_zero, T* y, float* h_out, float* states,
            float* carry) {
  constexpr int KINDS = ENDS ? 1 : 2;
  constexpr int ROWS = rows_of_states(NS);
  constexpr int CHUNK = EACH * WAVES;
  __shared__ float bc[2][KINDS][CHUNK][NS];
  constexpr int LOADS = (KINDS * CHUNK * NS + 64 * WAVES - 1) / (64 * WAVES);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int N = LEAST == NS ? NS : p.states;
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
    if (n < LEAST || n < N) {
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

  // b and c of a chunk of steps from t on
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
      if (n < LEAST || n < N) put(states + ((e * p.spans + span) * N + n) * F, f4, h[n]);
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
            const float *bt = bc[buffer][0][r0 + i], *ct = bc[buffer][KINDS - 1][r0 + i];
            float bv[NS], cv[NS];  // (ahead of the branches, where there are any)
#pragma unroll
            for (int n = LEAST; n < NS; ++n) bv[n] = bt[n], cv[n] = ct[n];
#pragma unroll
            for (int n = 0; n < NS; ++n) {
              if (n < LEAST || n < N) {
                h[n] = __builtin_amdgcn_exp2f(D[i] * a2[n]) * h[n] + Dx[i] * (n < LEAST ? bt[n] : bv[n]);
                if constexpr (!ENDS) v = fmaf(h[n], n < LEAST ? ct[n] : cv[n], v);
              }
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
      if (n < LEAST || n < N) put(mine + n * F, f4, h[n]);
    put(mine + N * F, f4, sum);
    put(mine + (N + 1) * F, f4, most);
  } else {
    for (int64_t t = max(t0, live); t < end; ++t) put(y + dtst::at(p.y, e, t), ft, 0.f);
    if (states != nullptr)  // (past the end the state stands still)
      for (int64_t t = max(t0, (live + SCAN_SPAN - 1) / SCAN_SPAN * SCAN_SPAN); t < end; t += SCAN_SPAN) keep(t / SCAN_SPAN);
    if (h_out != nullptr && (length > t0 ? length <= end : length == 0 && seg == 0)) {
#pragma unroll
      for (int n = 0; n < NS; ++n)
        if (n < LEAST || n < N) put(h_out + (e * N + n) * F, f4, h[n]);
    }
  }
}

template <class T, int NS, int LEAST, int WAVES>
int launch_forms(const ScanArgs& p, const ScanPointers& q, hipStream_t s) {
  const int64_t groups = (p.tiles + WAVES - 1) / WAVES * p.batch;
  const auto go = [&](auto kernel, int segments) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(groups * segments)), dim3(64 * WAVES), 0, s, p, static_cast<const T*>(q.x),
                       static_cast<const T*>(q.delta), q.a, static_cast<const T*>(q.b), static_cast<const T*>(q.c), q.skip,
                       static_cast<const T*>(q.o), q.h_zero, static_cast<T*>(q.y), q.h_out, q.states, q.carry);
    return int(hipGetLastError());
  };
  if (p.segments > 1) {
    int e = go(scan_kernel<T, NS, LEAST, WAVES, true>, p.segments - 1);
    if (e != hipSuccess) return e;
    e = launch_scan_carry(p, q.a, q.h_zero, q.carry, false, s);
    if (e != hipSuccess) return e;
  }
  return go(scan_kernel<T, NS, LEAST, WAVES, false>, p.segments);
}

// Calls f for the number of states that holds N, and the least of its branch-free ones.
// (24 ragged sequences of 731 steps, 1001 features and 12 states: 118 us by twelve, 164 by
// sixteen of which four are branched around.  A form of its own for every N would be 64
// kernels a type.)
template <class F>
int by_states(int N, F&& f) {
  using std::integral_constant;
  const auto sized = [&](auto ns, auto below) {
    return N == decltype(ns)::value ? f(ns, ns) : f(ns, integral_constant<int, decltype(below)::value + 1>());
  };
  if (N <= 4) return sized(integral_constant<int, 4>(), integral_constant<int, 0>());
  if (N <= 8) return sized(integral_constant<int, 8>(), integral_constant<int, 4>());
  if (N <= 12) return sized(integral_constant<int, 12>(), integral_constant<int, 8>());
  if (N <= 16) return sized(integral_constant<int, 16>(), integral_constant<int, 12>());
  if (N <= 24) return sized(integral_constant<int, 24>(), integral_constant<int, 16>());
  if (N <= 32) return sized(integral_constant<int, 32>(), integral_constant<int, 24>());
  if (N <= 40) return sized(integral_constant<int, 40>(), integral_constant<int, 32>());
  if (N <= 48) return sized(integral_constant<int, 48>(), integral_constant<int, 40>());
  if (N <= 56) return sized(integral_constant<int, 56>(), integral_constant<int, 48>());
  return sized(integral_constant<int, 64>(), integral_constant<int, 56>());
}

}  // namespace

template <class T>
int launch_scan_type(const ScanArgs& p, const ScanPointers& q, hipStream_t s) {
  // Four waves share b and c (32 x 1024 x 4096: 568 us, and 727 with one), but those past the
  // features' end only take others' places (8 x 4000 x 320, five of eight: 240 us, and 200
  // with one).
  const bool four = (p.tiles + 3) / 4 * 4 * 100 <= p.tiles * 115;
  return by_states(p.states, [&](auto ns, auto least) {
    constexpr int NS = decltype(ns)::value, LEAST = decltype(least)::value;
    return four ? launch_forms<T, NS, LEAST, 4>(p, q, s) : launch_forms<T, NS, LEAST, 1>(p, q, s);
  });
}

}  // namespace dtst
