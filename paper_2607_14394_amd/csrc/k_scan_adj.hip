// Backward of the state-space scan (dtst_scan_adj).  With E_t = exp(D_t a), the
// gradient g_t = g_y_t o_t s(o_t) of the sum before the gate, and q_t[n] the one
// that reaches h_t[n]:
//   q_t = g_t c_t + e_t,   e_{t-1} = E_t q_t   (the last e_t is g_h)
//   g_c_t = sum_f g_t h_t,   g_b_t = sum_f q_t D_t x_t,   w_t = sum_n q_t b_t
//   g_x_t = D_t w_t + g_t d,   g_a = sum_t D_t e_{t-1} h_{t-1},   g_d = sum_t g_t x_t
//   g_delta_t = (x_t w_t + sum_n a e_{t-1} h_{t-1}) s(delta_t)
//   g_o_t = g_y_t (sum_n c_t h_t + d x_t) s(o_t) (1 + o_t s(-o_t)).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "scan_ops.h"

namespace dtst {
namespace {

constexpr int WAVES = 4;
constexpr int R = SCAN_SPAN / WAVES;  // steps of a wave
static_assert(R == 16, "row_of's order");

// The sums over 64 lanes of 16 values, value row_of(lane) in each lane: a level of
// the tree halves the values as it doubles the lanes of a sum.
__device__ __forceinline__ int row_of(int lane) {
  return (lane >> 5 & 1) | (lane >> 4 & 1) << 1 | (lane >> 3 & 1) << 2 | (lane >> 2 & 1) << 3;
}
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
// b in the lanes of the banks of MASK, a in the others.
template <int MASK>
__device__ __forceinline__ float by_bank(float a, float b) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(a), __float_as_int(b), 0xe4, 0xf, MASK, false));
}
__device__ __forceinline__ float lane_sums(const float (&v)[16]) {
  float s[8], r[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), false, false);
    s[i] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(s[2 * i]), __float_as_uint(s[2 * i + 1]), false, false);
    r[i] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  const float a = by_bank<0xc>(r[0], r[1]) + dpp<0x128>(by_bank<0x3>(r[0], r[1]));  // (rotated by 8)
  const float b = by_bank<0xc>(r[2], r[3]) + dpp<0x128>(by_bank<0x3>(r[2], r[3]));
  float u = by_bank<0xa>(a, b) + dpp<0x141>(by_bank<0x5>(a, b));  // (half rows mirrored)
  u += dpp<0xb1>(u);
  return u + dpp<0x4e>(u);
}

struct AdjArrays {
  float* carry;  // (batch, segments, N + 2, features): the ends, then what enters
  float* parts;  // (batch, segments, N + 1, features): g_a and g_d of a segment
  float* sums;   // (tiles, batch, N, 2, spans SCAN_SPAN): g_b and g_c of a tile of features
};

// One workgroup: 64 features of a segment, its spans from the last to the first; a
// wave takes 16 steps of a span and a lane a feature.  State by state, the waves
// form their steps' maps, meet in LDS, and run them from the states that enter.
// ENDS: only e before the segment's first step, from zero after its last.
template <class T, bool GATED, bool ENDS>
__global__ void __launch_bounds__(64 * WAVES, ENDS ? 4 : 2)
scan_adj_kernel(const ScanArgs p, const AdjArrays w, const T* x, const T* delta, const float* __restrict__ a, const T* b,
                const T* c, const float* __restrict__ skip, const T* o, const float* __restrict__ states, const T* g_y,
                const float* g_h, T* g_x, T* g_delta, T* g_o, float* g_hzero) {
  extern __shared__ float lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, N = p.states;
  // carry[2][N][64], of a span and the next | gA[N][64] | b and c[N][2][SCAN_SPAN] | maps[2][WAVES][3][64] | ga[2][WAVES][64]
  float* const ecarry = lds;
  float* const gA = ecarry + 2 * N * 64;
  float* const bc = gA + N * 64;
  float* const maps = bc + 2 * N * SCAN_SPAN;
  float* const ga_of = maps + 2 * WAVES * 3 * 64;
  const int64_t F = p.features, tile = blockIdx.x % p.tiles, place = blockIdx.x / p.tiles;
  const int64_t seg = place % p.segments, e = place / p.segments;
  const bool own = tile * 64 + lane < F;  // (lanes past the end have no gradient and store nothing)
  const uint32_t f = uint32_t(min<int64_t>(tile * 64 + lane, F - 1));
  const int64_t length = scan_length(p, e), s0 = seg * p.segment, end = min(s0 + p.segment, p.steps);
  const int64_t live_end = min(end, length);
  float* const mine = w.carry + (e * p.segments + seg) * (N + 2) * F;

  for (int n = wave; n < N; n += WAVES) {
    float q = 0.f;
    if (!ENDS && own) {
      if (p.segments > 1)
        q = mine[n * F + f];
      else if (g_h != nullptr)
        q = g_h[(e * N + n) * F + f];
    }
    ecarry[n * 64 + lane] = q;
    gA[n * 64 + lane] = 0.f;
  }
  const float dv = skip != nullptr ? skip[f] : 0.f;
  float gd = 0.f, total = 0.f, most = 0.f;
  int side = 0, turn = 0;  // of ecarry (a span's), of maps and ga (a state's)
  const auto add_ga = [&](int n, int from) {
    float s = gA[n * 64 + lane];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) s += ga_of[(from * WAVES + i) * 64 + lane];
    gA[n * 64 + lane] = s;
  };
  int pending = -1;  // the state whose ga is still to be added

  const int64_t first_span = s0 / SCAN_SPAN, last_span = (end + SCAN_SPAN - 1) / SCAN_SPAN - 1;
  for (int64_t span = last_span; span >= first_span; --span) {
    const int64_t start = span * SCAN_SPAN, t0 = start + wave * R;
    const int rows_all = int(max<int64_t>(0, min<int64_t>(p.steps - t0, R)));    // of the arrays
    const int rows = int(max<int64_t>(0, min<int64_t>(live_end - t0, R)));       // live ones
    if (start >= live_end) {
      if constexpr (!ENDS) {
        for (int i = 0; i < rows_all; ++i)
          if (own) {
            (g_x + at(p.gx, e, t0 + i))[f] = T(0.f);
            (g_delta + at(p.gdelta, e, t0 + i))[f] = T(0.f);
            if constexpr (GATED) (g_o + at(p.go, e, t0 + i))[f] = T(0.f);
          }
      }
      continue;
    }
    // the span's b and c, states first
    __syncthreads();  // (the span before is done with them)
    for (int i = threadIdx.x; i < SCAN_SPAN * N; i += 64 * WAVES) {
      const int t = i / N, n = i % N;
      const bool there = start + t < live_end;
      if constexpr (!ENDS) bc[(2 * n) * SCAN_SPAN + t] = there ? float((b + at(p.b, e, start + t))[n]) : 0.f;
      bc[(2 * n + 1) * SCAN_SPAN + t] = there ? float((c + at(p.c, e, start + t))[n]) : 0.f;
    }
    float D[R], Dx[R], g[R];
    float sum = 0.f, top = 0.f;
    {
      T rx[R], rd[R], rg[R], ro[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int64_t t = min(t0 + i, live_end - 1);
        rx[i] = (x + at(p.x, e, t))[f];
        rd[i] = (delta + at(p.delta, e, t))[f];
        rg[i] = (g_y + at(p.y, e, t))[f];
        if constexpr (GATED) ro[i] = (o + at(p.o, e, t))[f];
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        D[i] = softplus(float(rd[i]));
        g[i] = float(rg[i]);
        if constexpr (GATED) {
          const float v = float(ro[i]);
          g[i] *= v * logistic<float>(v);
        }
        Dx[i] = D[i] * float(rx[i]);
        if (i >= rows) D[i] = g[i] = Dx[i] = 0.f;  // (past the end the states and their gradients stand still)
        if (!own) g[i] = Dx[i] = 0.f;
        sum += D[i], top = fmaxf(top, D[i]);
      }
    }
    total += sum, most = fmaxf(most, top);
    float wb[R], gD[R], yv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) wb[i] = gD[i] = yv[i] = 0.f;
    __syncthreads();

    float a_next = a[f], h_next = 0.f;
    if constexpr (!ENDS) h_next = states[(e * p.spans + span) * N * F + f];
    for (int n = 0; n < N; ++n, turn ^= 1) {
      const float an = a_next, a2 = an * LOG2E;
      float h = own ? h_next : 0.f;
      if (n + 1 < N) {
        a_next = a[(n + 1) * F + f];
        if constexpr (!ENDS) h_next = states[((e * p.spans + span) * N + n + 1) * F + f];
      }
      const float* bn = bc + 2 * n * SCAN_SPAN + wave * R;
      const float* cn = bn + SCAN_SPAN;
      float E[R], H = 0.f, G = 0.f;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        E[i] = __builtin_amdgcn_exp2f(a2 * D[i]);
        if constexpr (!ENDS) H = E[i] * H + Dx[i] * bn[i];
      }
#pragma unroll
      for (int i = R - 1; i >= 0; --i) G = E[i] * fmaf(g[i], cn[i], G);
      float* m = maps + turn * WAVES * 3 * 64;
      m[(wave * 3 + 0) * 64 + lane] = run_decay(a2, sum, top);
      if constexpr (!ENDS) m[(wave * 3 + 1) * 64 + lane] = H;
      m[(wave * 3 + 2) * 64 + lane] = G;
      __syncthreads();
      if constexpr (ENDS) {
        if (wave == n % WAVES) {
          float q = ecarry[n * 64 + lane];
#pragma unroll
          for (int i = WAVES - 1; i >= 0; --i) q = m[i * 3 * 64 + lane] * q + m[(i * 3 + 2) * 64 + lane];
          ecarry[n * 64 + lane] = q;
        }
      } else {
        if (pending >= 0 && wave == pending % WAVES) add_ga(pending, turn ^ 1);
        for (int i = 0; i < wave; ++i) h = m[i * 3 * 64 + lane] * h + m[(i * 3 + 1) * 64 + lane];
        float q = ecarry[(side * N + n) * 64 + lane];
        for (int i = WAVES - 1; i > wave; --i) q = m[i * 3 * 64 + lane] * q + m[(i * 3 + 2) * 64 + lane];
        float hp[R], v[R];  // hp: the states before the steps
#pragma unroll
        for (int i = 0; i < R; ++i) {
          hp[i] = h;
          h = E[i] * h + Dx[i] * bn[i];
          if constexpr (GATED) yv[i] = fmaf(cn[i], h, yv[i]);
          v[i] = g[i] * h;
        }
        const float gc = lane_sums(v);
        float ga = 0.f;
#pragma unroll
        for (int i = R - 1; i >= 0; --i) {
          const float qi = fmaf(g[i], cn[i], q);
          wb[i] = fmaf(qi, bn[i], wb[i]);
          v[i] = qi * Dx[i];
          q = E[i] * qi;
          const float s = q * hp[i];
          gD[i] = fmaf(an, s, gD[i]);
          ga = fmaf(D[i], s, ga);
        }
        const float gb = lane_sums(v);
        if (wave == 0) ecarry[((side ^ 1) * N + n) * 64 + lane] = q;
        ga_of[(turn * WAVES + wave) * 64 + lane] = ga;
        pending = n;
        // two lanes of each four hold a step's sums
        if ((lane & 2) == 0)
          w.sums[((((tile * p.batch + e) * N + n) * 2 + (lane & 1)) * p.spans * SCAN_SPAN) + t0 + row_of(lane)] = lane & 1 ? gc : gb;
      }
    }
    side ^= 1;
    if constexpr (!ENDS) {
      T rx[R], rd[R], rg[R], ro[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const int64_t t = min(t0 + i, live_end - 1);
        rx[i] = (x + at(p.x, e, t))[f];
        rd[i] = (delta + at(p.delta, e, t))[f];
        rg[i] = (g_y + at(p.y, e, t))[f];
        if constexpr (GATED) ro[i] = (o + at(p.o, e, t))[f];
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool there = i < rows;
        const float xv = float(rx[i]);
        gd += there ? g[i] * xv : 0.f;
        if (i >= rows_all || !own) continue;  // (no `break`: the loop stays unrolled)
        (g_x + at(p.gx, e, t0 + i))[f] = T(there ? D[i] * wb[i] + g[i] * dv : 0.f);
        (g_delta + at(p.gdelta, e, t0 + i))[f] = T(there ? (gD[i] + xv * wb[i]) * logistic<float>(float(rd[i])) : 0.f);
        if constexpr (GATED) {
          const float v = float(ro[i]), s = logistic<float>(v);
          (g_o + at(p.go, e, t0 + i))[f] = T(there ? float(rg[i]) * (yv[i] + dv * xv) * (s + v * s * (1.f - s)) : 0.f);
        }
      }
    }
  }
  __syncthreads();
  if constexpr (ENDS) {
    // (total and most are the wave's)
    maps[(wave * 2) * 64 + lane] = total, maps[(wave * 2 + 1) * 64 + lane] = most;
    __syncthreads();
    if (!own) return;
    for (int n = wave; n < N; n += WAVES) mine[n * F + f] = ecarry[n * 64 + lane];
    if (wave == 0) {
#pragma unroll
      for (int i = 1; i < WAVES; ++i)
        total += maps[(i * 2) * 64 + lane], most = fmaxf(most, maps[(i * 2 + 1) * 64 + lane]);
      mine[N * F + f] = total, mine[(N + 1) * F + f] = most;
    }
  } else {
    if (pending >= 0 && wave == pending % WAVES) add_ga(pending, turn ^ 1);
    maps[wave * 64 + lane] = gd;
    __syncthreads();
    if (!own) return;
    float* part = w.parts + (e * p.segments + seg) * (N + 1) * F;
    for (int n = wave; n < N; n += WAVES) {
      part[n * F + f] = gA[n * 64 + lane];
      if (p.segments == 1 && g_hzero != nullptr) g_hzero[(e * N + n) * F + f] = ecarry[(side * N + n) * 64 + lane];
    }
    if (wave == 0) {
#pragma unroll
      for (int i = 1; i < WAVES; ++i) gd += maps[i * 64 + lane];
      part[N * F + f] = gd;
    }
  }
}

// g_b and g_c from the tiles' sums: a wave 64 steps of one of them and one state.
template <class T>
__global__ void __launch_bounds__(256) scan_adj_sums_kernel(const ScanArgs p, const float* __restrict__ sums, T* g_b, T* g_c) {
  const int64_t N2 = 2 * p.states, unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t which = unit % N2, span = unit / N2 % p.spans, e = unit / N2 / p.spans, t = span * SCAN_SPAN + lane;
  if (e >= p.batch || t >= p.steps) return;
  float s = 0.f;
  if (t < scan_length(p, e)) {
    const int64_t pitch = p.batch * N2 * p.spans * SCAN_SPAN;
    const float* from = sums + (e * N2 + which) * p.spans * SCAN_SPAN + t;
#pragma unroll 8
    for (int64_t i = 0; i < p.tiles; ++i) s += from[i * pitch];
  }
  const int64_t n = which / 2;
  if (which & 1)
    (g_c + at(p.gc, e, t))[n] = T(s);
  else
    (g_b + at(p.gb, e, t))[n] = T(s);
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

}  // namespace

size_t scan_adj_workspace(const dtst_scan_desc& d) {
  const ScanArgs p = scan_args(d, nullptr);
  if (d.batch == 0 || d.features == 0) return 0;
  const size_t parts = size_t(p.batch) * p.segments * (p.states + 1) * p.features * 4;
  const size_t sums = size_t(p.tiles) * p.batch * p.states * 2 * p.spans * SCAN_SPAN * 4;
  return round16(scan_carry_bytes(d)) + round16(parts) + sums;
}

int launch_scan_adj(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b,
                    const void* c, const float* skip, const void* o, const int32_t* lengths, const float* states,
                    const void* g_y, const float* g_h, void* g_x, void* g_delta, float* g_a, void* g_b, void* g_c,
                    float* g_skip, void* g_o, float* g_hzero, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const ScanArgs p = scan_args(d, lengths);
  const int N = p.states;
  char* ws = static_cast<char*>(workspace);
  AdjArrays w;
  w.carry = reinterpret_cast<float*>(ws);
  w.parts = reinterpret_cast<float*>(ws + round16(scan_carry_bytes(d)));
  w.sums = w.parts + round16(size_t(p.batch) * p.segments * (N + 1) * p.features * 4) / 4;
  const auto typed = [&](auto t) {
    using T = decltype(t);
    const auto go = [&](auto kernel) {
      const size_t lds = size_t(3 * N * 64 + 2 * N * SCAN_SPAN + 2 * WAVES * 4 * 64) * 4;
      if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return int(e);
      }
      hipLaunchKernelGGL(kernel, dim3(unsigned(p.tiles * p.segments * p.batch)), dim3(64 * WAVES), lds, s, p, w,
                         static_cast<const T*>(x), static_cast<const T*>(delta), a, static_cast<const T*>(b),
                         static_cast<const T*>(c), skip, static_cast<const T*>(o), states, static_cast<const T*>(g_y), g_h,
                         static_cast<T*>(g_x), static_cast<T*>(g_delta), static_cast<T*>(g_o), g_hzero);
      return int(hipGetLastError());
    };
    int r = hipSuccess;
    if (p.segments > 1) {
      r = o != nullptr ? go(scan_adj_kernel<T, true, true>) : go(scan_adj_kernel<T, false, true>);
      if (r == hipSuccess) r = launch_scan_carry(p, a, g_h, w.carry, g_hzero, true, s);
      if (r != hipSuccess) return r;
    }
    r = o != nullptr ? go(scan_adj_kernel<T, true, false>) : go(scan_adj_kernel<T, false, false>);
    if (r != hipSuccess) return r;
    const int64_t units = p.batch * p.spans * 2 * N;
    hipLaunchKernelGGL((scan_adj_sums_kernel<T>), dim3(unsigned((units + 3) / 4)), dim3(256), 0, s, p, w.sums,
                       static_cast<T*>(g_b), static_cast<T*>(g_c));
    return int(hipGetLastError());
  };
  if (d.steps > 0 && d.batch > 0 && d.features > 0) {
    const int r = d.type == DTST_F32 ? typed(float()) : d.type == DTST_BF16 ? typed(bf16_t()) : typed(f16_t());
    if (r != hipSuccess) return r;
  } else {
    const int r = launch_copy_states(g_h, g_hzero, d.batch * N * d.features, s);
    if (r != hipSuccess) return r;
  }
  if (d.features == 0) return hipSuccess;
  const int64_t cols = N * d.features, parts = d.steps > 0 ? d.batch * p.segments : 0;
  return launch_sum_parts(w.parts, parts, cols + d.features, cols, cols + (g_skip != nullptr ? d.features : 0),
                          d.accumulate, g_a, g_skip, s);
}

}  // namespace dtst
