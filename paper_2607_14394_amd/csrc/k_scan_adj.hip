// Backward of the state-space scan (dtst_scan_adj).  With E_t = exp(D_t a), the
// gradient g_t = g_y_t o_t s(o_t) of the sum before the gate, and q_t[n] the one
// that reaches h_t[n]:
//   q_t = g_t c_t + e_t,   e_{t-1} = E_t q_t   (the last e_t is g_h)
//   g_c_t = sum_f g_t h_t,   g_b_t = sum_f q_t D_t x_t,   w_t = sum_n q_t b_t
//   g_x_t = D_t w_t + g_t d,   g_a = sum_t D_t e_{t-1} h_{t-1},   g_d = sum_t g_t x_t
//   g_delta_t = (x_t w_t + sum_n a e_{t-1} h_{t-1}) s(delta_t)
//   g_o_t = g_y_t (sum_n c_t h_t + d x_t) s(o_t) (1 + o_t s(-o_t)).
//
// Bound by the vector unit: 16 instructions a state and step, 13 of them the formulas', two
// the sums over the features, and 5 more of the step itself among 16 states.  The forward's
// states at every 16th step are read; h goes on from there, and all that a state's way back
// needs is in registers (two waves a SIMD).  4 x 4096 x 2048 of 16 states in bf16: 420 us,
// the vector unit busy 79% of the time, after 130 us for the segments' ends (81%), and 19
// for g_b's and g_c's sums.  At 455 us, spans of 8 steps and three waves a SIMD took 454 with
// twice the states kept, b and c from LDS 500, the lanes' sums by exchanges between them 525.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "scan_ops.h"

namespace dtst {
namespace {

constexpr int R = SCAN_SPAN;    // steps of a span, all in a lane's registers
constexpr int WAVES = 4;  // of a workgroup at most
constexpr int PITCH = 64 + 4;  // of a row of lanes' values in LDS: four banks on, so that a read by rows meets none twice
static_assert(R == 16, "lane_sums");

// The sums over 64 lanes of 16 values; that of value i in lanes 4 i .. 4 i + 3.
// Through LDS: a lane writes its values and reads a quarter of one's lanes (17
// additions; by exchanges between lanes, each halving the values, it would take 44
// cycles' worth of instructions more).  Apart, so that other work hides the reading.
__device__ __forceinline__ void read_row(const float* buffer, int lane, float4 (&r)[4]) {
  wave_sync();
  const float4* row = reinterpret_cast<const float4*>(buffer + (lane >> 2) * PITCH + (lane & 3) * 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = row[i];
  wave_sync();
}
__device__ __forceinline__ float row_sum(const float4 (&r)[4]) {
  float4 s = r[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) s.x += r[i].x, s.y += r[i].y, s.z += r[i].z, s.w += r[i].w;
  float t = (s.x + s.y) + (s.z + s.w);
  t += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(t), 0xb1, 0xf, 0xf, false));  // (its neighbour's)
  return t + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(t), 0x4e, 0xf, 0xf, false));
}
struct AdjArrays {
  float* carry;  // (batch, segments, N + 2, features): the ends, then what enters
  float* parts;  // (batch, segments, N + 1, features): g_a and g_d of a segment
  float* sums;   // (tiles, batch, spans, N, 2, SCAN_SPAN): g_b and g_c of a tile of features
  float* bc;     // (batch, N, 2, spans SCAN_SPAN): b and c
};

// b and c in 32 bits, steps next to each other, zeros past a length: so a wave takes
// 16 steps' of a state by a scalar load.  (From LDS, where every lane would read the
// same, they took as long as the arithmetic.)  A thread: LIFT states of a step.  (All
// states of it are a chain of loads: 11 us for 26 rows of 56 states, where four are 4.)
constexpr int LIFT = 4;
template <class T>
__global__ void __launch_bounds__(256) scan_adj_lift_kernel(const ScanArgs p, const T* b, const T* c, float* bc) {
  const int64_t N = p.states, pitch = p.spans * R, t = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t e = t / pitch, step = t % pitch;
  if (e >= p.batch) return;
  const bool live = step < scan_length(p, e);
  const T *from_b = b + at(p.b, e, live ? step : 0), *from_c = c + at(p.c, e, live ? step : 0);
  const int64_t first = int64_t(blockIdx.y) * LIFT, end = min(first + LIFT, N);
  float* to = bc + (e * N + first) * 2 * pitch + step;
  for (int64_t n = first; n < end; ++n, to += 2 * pitch) {
    to[0] = live ? float(from_b[n]) : 0.f;
    to[pitch] = live ? float(from_c[n]) : 0.f;
  }
}

// Floats of LDS: e[N][64] | gA[N][64] | the sums' buffer | a span's sums of some states.
// (Of all 64 states, they leave room for three waves a CU instead of four: 4 x 4096 x 512,
// both directions, 1387 against 1114 us.)
constexpr int TOGETHER = 16;
__host__ __device__ constexpr int adj_lds(int N, bool ends) {
  return N * 64 + (ends ? 0 : N * 64 + R * PITCH + (N < TOGETHER ? N : TOGETHER) * 2 * R);
}

// A wave's turn at its SIMD over others': first what ends in loads, stores or LDS, so that
// the others' arithmetic covers the wait (4 x 4096 x 2048 of 16 states, both directions: 852
// -> 835 us).
template <bool ENDS, int P>
__device__ __forceinline__ void turn() {
  if constexpr (!ENDS) __builtin_amdgcn_s_setprio(P);
}

// A wave: 64 features of a segment, a lane a feature, its spans from the last to
// the first.  A span's steps are in registers; state by state, h goes forward over
// them from the state that the forward kept, then e backward.  ENDS: only e before
// the segment's first step, from zero after its last.
template <class T, bool GATED, bool ENDS>
__global__ void __launch_bounds__(64 * WAVES, ENDS ? 4 : 2)
scan_adj_kernel(const ScanArgs p, const AdjArrays w, const T* x, const T* delta, const float* __restrict__ a,
                const float* __restrict__ bc, const float* __restrict__ skip, const T* o, const float* __restrict__ states, const T* g_y,
                const float* g_h, T* g_x, T* g_delta, T* g_o, float* g_hzero) {
  extern __shared__ __align__(16) float lds[];
  const int lane = threadIdx.x & 63, N = p.states, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = blockDim.x >> 6;
  float* const ecarry = lds + wave * adj_lds(N, ENDS);
  float* const gA = ecarry + N * 64;
  float* const buffer = gA + N * 64;
  float* const bc_sums = buffer + R * PITCH;
  const int64_t groups = (p.tiles + waves - 1) / waves, F = p.features;
  const int64_t tile = blockIdx.x % groups * waves + wave, place = blockIdx.x / groups;
  if (tile >= p.tiles) return;  // (the waves do not meet)
  const int segments = ENDS ? p.segments - 1 : p.segments;  // (nothing comes before the first's end)
  const int64_t seg = place % segments + (ENDS ? 1 : 0), e = place / segments;
  const bool own = tile * 64 + lane < F;  // (lanes past the end have no gradient and store nothing)
  const uint32_t f = uint32_t(min<int64_t>(tile * 64 + lane, F - 1)), ft = lane_offset(f * sizeof(T));
  const uint32_t f4 = lane_offset(f * 4);
  const int64_t length = scan_length(p, e), s0 = seg * p.segment, end = min(s0 + p.segment, p.steps);
  const int64_t live_end = min(end, length);
  float* const mine = w.carry + (e * p.segments + seg) * (N + 2) * F;

  for (int n = 0; n < N; ++n) {
    float q = 0.f;
    if (!ENDS && own) {
      if (p.segments > 1)
        q = get(mine + n * F, f4);
      else if (g_h != nullptr)
        q = get(g_h + (e * N + n) * F, f4);
    }
    ecarry[n * 64 + lane] = q;
    if constexpr (!ENDS) gA[n * 64 + lane] = 0.f;
  }
  const float dv = skip != nullptr ? skip[f] : 0.f;
  float gd = 0.f, total = 0.f, most = 0.f;
  const int64_t pitch = p.spans * R;
  // Of neighbouring lanes one has g_b's sum, one g_c's; two lanes each write the same,
  // as a branch in the loop below would cost more.  (To memory they go together: a
  // store in the loop would be waited for with the next state's loads.)
  float* const sums = bc_sums + (lane & 1) * R + (lane >> 2);

  for (int64_t t0 = (end - 1) / R * R; t0 >= s0; t0 -= R) {
    const int rows_all = int(min<int64_t>(end - t0, R));
    const int rows = int(max<int64_t>(0, min<int64_t>(live_end - t0, R)));  // live ones
    if (rows == 0) {
      if (!ENDS && own) {
        for (int i = 0; i < rows_all; ++i) {
          put(g_x + at(p.gx, e, t0 + i), ft, 0.f);
          put(g_delta + at(p.gdelta, e, t0 + i), ft, 0.f);
          if constexpr (GATED) put(g_o + at(p.go, e, t0 + i), ft, 0.f);
        }
      }
      continue;
    }
    turn<ENDS, 3>();
    float D[R], Dx[R], g[R];
    const auto load = [&](auto full_) {  // full: all rows are live
      constexpr bool FULL = decltype(full_)::value;
      T rx[R], rd[R], rg[R], ro[R];
      if constexpr (!ENDS) get_rows<FULL>(x, p.x, e, t0, rows, ft, rx);
      get_rows<FULL>(delta, p.delta, e, t0, rows, ft, rd);
      get_rows<FULL>(g_y, p.y, e, t0, rows, ft, rg);
      if constexpr (GATED) get_rows<FULL>(o, p.o, e, t0, rows, ft, ro);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        D[i] = softplus<T>(float(rd[i]));
        g[i] = float(rg[i]);
        if constexpr (GATED) {
          const float v = float(ro[i]);
          g[i] *= v * logistic<T>(v);
        }
        if constexpr (!ENDS) Dx[i] = D[i] * float(rx[i]);
        // (past the end the states and their gradients stand still)
        if (!FULL && i >= rows) D[i] = g[i] = Dx[i] = 0.f;
        if (!own) g[i] = Dx[i] = 0.f;
        if constexpr (ENDS) total += D[i], most = fmaxf(most, D[i]);
      }
    };
    if (rows == R)
      load(std::true_type());
    else
      load(std::false_type());
    turn<ENDS, 0>();
    float wb[R], gD[R], yv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) wb[i] = gD[i] = yv[i] = 0.f;

    const float* kept = ENDS ? nullptr : states + (e * p.spans + t0 / R) * N * F;
    // b and c of a state, and of the next
    const float* from = bc + e * N * 2 * pitch + t0;
    float bn[R], cn[R], b_next[R], c_next[R];
    const auto fetch = [&] {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if constexpr (!ENDS) b_next[i] = from[i];
        c_next[i] = from[pitch + i];
      }
    };
    fetch();
    float a_next = get(a, f4), h_next = ENDS ? 0.f : get(kept, f4);
    float4 last[4];  // g_b's terms of the state before, and its sum of g_c
    float last_c = 0.f;
    for (int first = 0; first < N; first += ENDS ? N : TOGETHER) {
      const int past = ENDS ? N : min(first + TOGETHER, N);
      for (int n = first; n < past; ++n) {
        const float an = a_next, a2 = an * LOG2E;
        float h = own ? h_next : 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) bn[i] = b_next[i], cn[i] = c_next[i];
        if (n + 1 < N) {
          from += 2 * pitch;
          if constexpr (ENDS) fetch();
          a_next = get(a + (n + 1) * F, f4);
          if constexpr (!ENDS) h_next = get(kept + (n + 1) * F, f4);
        }
        turn<ENDS, 2>();
        float E[R], q = ecarry[n * 64 + lane];
#pragma unroll
        for (int i = 0; i < R; ++i) E[i] = __builtin_amdgcn_exp2f(a2 * D[i]);
        if constexpr (ENDS) {
#pragma unroll
          for (int i = R - 1; i >= 0; --i) q = E[i] * fmaf(g[i], cn[i], q);
        } else {
          float hp[R], ga = gA[n * 64 + lane];  // hp: the states before the steps
          if (n > first) {
            const float gb = row_sum(last);
            sums[2 * (n - 1 - first) * R] = lane & 1 ? last_c : gb;
          }
#pragma unroll
          for (int i = 0; i < R; ++i) {
            hp[i] = h;
            h = E[i] * h + Dx[i] * bn[i];
            if constexpr (GATED) yv[i] = fmaf(cn[i], h, yv[i]);
            buffer[i * PITCH + lane] = g[i] * h;
          }
          turn<ENDS, 0>();
          float4 terms[4];
          read_row(buffer, lane, terms);
#pragma unroll
          for (int i = R - 1; i >= 0; --i) {
            q = fmaf(g[i], cn[i], q);
            wb[i] = fmaf(q, bn[i], wb[i]);
            buffer[i * PITCH + lane] = q * Dx[i];
            q *= E[i];
            const float s = q * hp[i];
            gD[i] = fmaf(an, s, gD[i]);
            ga = fmaf(D[i], s, ga);
            if (i == R / 2) {
              // The next state's b and c from here on: scalar loads in flight would be
              // waited for with the terms.
              last_c = row_sum(terms);
              __builtin_amdgcn_sched_barrier(0);
              fetch();
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          gA[n * 64 + lane] = ga;
          read_row(buffer, lane, last);
        }
        ecarry[n * 64 + lane] = q;
      }
      if constexpr (!ENDS) {
        const float gb = row_sum(last);
        sums[2 * (past - 1 - first) * R] = lane & 1 ? last_c : gb;
        wave_sync();
        float4* to = reinterpret_cast<float4*>(w.sums + (((tile * p.batch + e) * p.spans + t0 / R) * N + first) * 2 * R);
        for (int i = lane; i < (past - first) * 2 * R / 4; i += 64) to[i] = reinterpret_cast<const float4*>(bc_sums)[i];
        wave_sync();
      }
    }
    turn<ENDS, 3>();
    const auto store = [&](auto full_) {
      constexpr bool FULL = decltype(full_)::value;
      if (!own) return;
      // The rows are read again: kept, they or their addresses would take registers
      // that there are not.
      uint32_t again = ft;
      asm volatile("" : "+v"(again)::"memory");
      T *to_x = g_x + at(p.gx, e, t0), *to_delta = g_delta + at(p.gdelta, e, t0);
      T* to_o = GATED ? g_o + at(p.go, e, t0) : nullptr;
      T rx[R], rd[R], rg[R], ro[R];
      get_rows<FULL>(x, p.x, e, t0, rows, again, rx);
      get_rows<FULL>(delta, p.delta, e, t0, rows, again, rd);
      if constexpr (GATED) get_rows<FULL>(g_y, p.y, e, t0, rows, again, rg);
      if constexpr (GATED) get_rows<FULL>(o, p.o, e, t0, rows, again, ro);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool there = FULL || i < rows;
        const float xv = float(rx[i]);
        const float gx = there ? D[i] * wb[i] + g[i] * dv : 0.f;
        const float gs = there ? (gD[i] + xv * wb[i]) * logistic<T>(float(rd[i])) : 0.f;
        gd += there ? g[i] * xv : 0.f;
        float go = 0.f;
        if constexpr (GATED) {
          const float v = float(ro[i]), u = logistic<T>(v);
          go = there ? float(rg[i]) * (yv[i] + dv * xv) * (u + v * u * (1.f - u)) : 0.f;
        }
        if (FULL || i < rows_all) {  // (no `break`: the loop stays unrolled)
          put(to_x, again, gx);
          put(to_delta, again, gs);
          if constexpr (GATED) put(to_o, again, go);
        }
        to_x += p.gx.t, to_delta += p.gdelta.t;
        if constexpr (GATED) to_o += p.go.t;
      }
    };
    if constexpr (!ENDS) {
      if (rows == R)
        store(std::true_type());
      else
        store(std::false_type());
    }
  }
  if (!own) return;
  if constexpr (ENDS) {
    for (int n = 0; n < N; ++n) put(mine + n * F, f4, ecarry[n * 64 + lane]);
    put(mine + N * F, f4, total);
    put(mine + (N + 1) * F, f4, most);
  } else {
    float* part = w.parts + (e * p.segments + seg) * (N + 1) * F;
    for (int n = 0; n < N; ++n) {
      put(part + n * F, f4, gA[n * 64 + lane]);
      if (seg == 0 && g_hzero != nullptr) put(g_hzero + (e * N + n) * F, f4, ecarry[n * 64 + lane]);
    }
    put(part + N * F, f4, gd);
  }
}

// g_b and g_c from the tiles' sums: a wave 64 neighbours of a span's (two states), so
// that a tile's are a run of 256 bytes (64 steps of one state instead: 23 against 18.6 us
// for 67 MB of sums).
int64_t sums_units(const ScanArgs& p) { return p.batch * p.spans * ((p.states * 2 * R + 63) / 64); }
template <class T>
__global__ void __launch_bounds__(256) scan_adj_sums_kernel(const ScanArgs p, const float* __restrict__ sums, T* g_b, T* g_c) {
  const int64_t unit = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6), block = p.states * 2 * R, units = (block + 63) / 64;
  const int64_t span = unit / units, i = unit % units * 64 + (threadIdx.x & 63);  // (span: of all entries)
  const int64_t e = span / p.spans, t = span % p.spans * R + i % R, n = i / R / 2;
  if (e >= p.batch || i >= block || t >= p.steps) return;
  float s = 0.f;
  if (t < scan_length(p, e)) {
    const int64_t pitch = p.batch * p.spans * block;
    const float* from = sums + span * block + i;
#pragma unroll 8
    for (int64_t k = 0; k < p.tiles; ++k) s += from[k * pitch];
  }
  if (i / R & 1)
    (g_c + at(p.gc, e, t))[n] = T(s);
  else
    (g_b + at(p.gb, e, t))[n] = T(s);
}

size_t round64(size_t n) { return (n + 63) / 64 * 64; }

}  // namespace

size_t scan_adj_workspace(const dtst_scan_desc& d) {
  const ScanArgs p = scan_args(d, nullptr, true);
  if (d.batch == 0 || d.features == 0) return 0;
  const size_t parts = size_t(p.batch) * p.segments * (p.states + 1) * p.features * 4;
  const size_t sums = size_t(p.tiles) * p.batch * p.states * 2 * p.spans * SCAN_SPAN * 4;
  return round64(scan_carry_bytes(d, true)) + round64(parts) + round64(sums) + sums / p.tiles;
}

int launch_scan_adj(const dtst_scan_desc& d, const void* x, const void* delta, const float* a, const void* b,
                    const void* c, const float* skip, const void* o, const int32_t* lengths, const float* states,
                    const void* g_y, const float* g_h, void* g_x, void* g_delta, float* g_a, void* g_b, void* g_c,
                    float* g_skip, void* g_o, float* g_hzero, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const ScanArgs p = scan_args(d, lengths, true);
  const int N = p.states;
  char* ws = static_cast<char*>(workspace);
  AdjArrays w;
  w.carry = reinterpret_cast<float*>(ws);
  w.parts = reinterpret_cast<float*>(ws + round64(scan_carry_bytes(d, true)));
  w.sums = w.parts + round64(size_t(p.batch) * p.segments * (N + 1) * p.features * 4) / 4;
  const int64_t steps = p.batch * p.spans * R;  // (of all entries, whole spans)
  w.bc = w.sums + round64(size_t(p.tiles) * steps * N * 2 * 4) / 4;
  const auto typed = [&](auto t) {
    using T = decltype(t);
    const auto go = [&](auto kernel, bool ends) {
      const int64_t segments = ends ? p.segments - 1 : p.segments;
      // Several waves a workgroup meet in the scalar cache, whose b and c are the same
      // for all, but as many a CU as its LDS holds (eight, by their registers) come first
      // (4 x 4096 x 1024 of 32 states, both directions: 939 us with as many a workgroup as
      // half the LDS holds, 917 so).
      const auto held = [&](int w) { return std::min(8, 160 * 1024 / (w * adj_lds(N, ends) * 4) * w); };
      int waves = WAVES;
      for (int w = WAVES / 2; w >= 1; w /= 2)
        if (held(w) > held(waves) || w >= p.tiles) waves = w;
      const size_t lds = size_t(waves) * adj_lds(N, ends) * 4;
      if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return int(e);
      }
      hipLaunchKernelGGL(kernel, dim3(unsigned((p.tiles + waves - 1) / waves * segments * p.batch)),
                         dim3(64 * waves), lds, s, p, w,
                         static_cast<const T*>(x), static_cast<const T*>(delta), a, w.bc, skip, static_cast<const T*>(o), states, static_cast<const T*>(g_y), g_h,
                         static_cast<T*>(g_x), static_cast<T*>(g_delta), static_cast<T*>(g_o), g_hzero);
      return int(hipGetLastError());
    };
    hipLaunchKernelGGL((scan_adj_lift_kernel<T>), dim3(unsigned((steps + 255) / 256), unsigned((N + LIFT - 1) / LIFT)),
                       dim3(256), 0, s, p, static_cast<const T*>(b), static_cast<const T*>(c), w.bc);
    int r = hipGetLastError();
    if (r != hipSuccess) return r;
    if (p.segments > 1) {
      r = o != nullptr ? go(scan_adj_kernel<T, true, true>, true) : go(scan_adj_kernel<T, false, true>, true);
      if (r == hipSuccess) r = launch_scan_carry(p, a, g_h, w.carry, true, s);
      if (r != hipSuccess) return r;
    }
    r = o != nullptr ? go(scan_adj_kernel<T, true, false>, false) : go(scan_adj_kernel<T, false, false>, false);
    if (r != hipSuccess) return r;
    hipLaunchKernelGGL((scan_adj_sums_kernel<T>), dim3(unsigned((sums_units(p) + 3) / 4)), dim3(256), 0, s, p, w.sums,
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
