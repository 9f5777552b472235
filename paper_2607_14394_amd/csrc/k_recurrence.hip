// Gated linear recurrence along the steps and its backward (dtst_recurrence,
// dtst_recurrence_adj):
//   h_t = s(z_t) h_{t-1} + s(-z_t) v_t,   y_t = h_t o_t s(o_t).
//
// A few operations per value: bound by HBM (z, v, o read and y written once;
// backward: z, v, o, g_y read and g_z, g_v, g_o written once).  Long sequences
// of few features have to be divided along the steps to keep the card's loads in
// flight.  A run of steps maps the state that enters it to the one that leaves
// it as h -> A h + H (A the product of its gates, H its end from a zero state),
// and two neighbouring runs compose to such a map.  So a workgroup takes SPAN
// steps of 128 features: its waves hold 16 steps each in registers (a lane two
// neighbouring features), form their maps, and meet in LDS; the workgroup
// publishes its span's map, composes those of the spans before it until it meets
// one whose leaving state is known already, publishes its own, and runs its
// steps from the state that enters.  Every value is read once.  The backward runs
// the same scheme from the last span to the first on d_t's carry,
// e_{t-1} = s(z_t) (g_t + e_t), g_t = g_y_t o_t s(o_t), and takes the states from
// the one that the forward kept for each span.
//
// 1 x 65536 x 1280 in bf16: 141 us and 5 us for clearing the chain's words, 4.8
// TB/s (two launches, maps then states, would read z and v twice); 4 x 4096 x
// 2048 60 us forward and 107 us backward (4.5 and 4.4 TB/s), where 25 and 47
// vector instructions a value, 4 and 6 of them at a quarter of the rate, come
// close to the time of the loads.
//
// Waiting ends: spans are taken by ticket, spans earlier in the chain have
// earlier tickets, so a workgroup waits only for workgroups that already run,
// and the earliest of those waits for none.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

constexpr int SPAN = DTST_RECURRENCE_SPAN;
constexpr int WAVES = 8;
constexpr int RPW = SPAN / WAVES;  // steps of a wave

struct Args {
  int64_t batch, steps, features;
  Strides z, v, o, y, gz, gv, go;
  const int32_t* lengths;
  int64_t tiles, feature_tiles;  // tiles = batch * feature_tiles, one a workgroup's features
  int spans;
  unsigned long long* maps;  // (tiles, spans, 64 CPL) words of the chain
  unsigned* ticket;
};

__device__ __forceinline__ int64_t length_of(const Args& p, int64_t b) {
  if (p.lengths == nullptr) return p.steps;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.steps ? p.steps : n;
}

// The product p of gates of which `least` is the smallest.  One that underflows
// stays above zero where they all are: it would make no number of an infinite
// state, which a run of open gates keeps.
__device__ __forceinline__ float product_of_gates(float p, float least) {
  return fmaxf(p, fminf(least, __uint_as_float(1)));  // (1: the smallest number above zero)
}
__device__ __forceinline__ float compose_gates(float a, float b) { return product_of_gates(a * b, fminf(a, b)); }

// A span's map in a word of the chain: A >= 0 with its sign bit set (a word of
// zeros: not there yet) and H.  A = 0 says that H is the leaving state itself, so
// a closed gate's zero goes as CLOSED, a number that no product of gates is.
constexpr unsigned CLOSED = 0x40000000u;
__device__ __forceinline__ unsigned long long map_word(float A, float H) {
  const unsigned a = (A == 0.f ? CLOSED : __float_as_uint(A)) | 0x80000000u;
  return (unsigned long long)(__float_as_uint(H)) << 32 | a;
}
__device__ __forceinline__ unsigned long long state_word(float h) {
  return (unsigned long long)(__float_as_uint(h)) << 32 | 0x80000000u;
}
__device__ __forceinline__ void put_word(unsigned long long* p, unsigned long long w) {
  __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long get_word(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The state that enters span k of the chain (k >= 1), for the lane's features:
// the maps of spans k - 1, k - 2, ... composed until a known state.  words: the
// lane's first word of span 0; a span's words are `pitch` apart.
template <int CPL>
__device__ void look_back(const unsigned long long* words, int64_t pitch, int k, float (&h)[CPL]) {
  constexpr int AHEAD = 4;
  float a[CPL];
  bool done[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) a[c] = 1.f, h[c] = 0.f, done[c] = false;
  int j = k - 1;
  for (int tries = 0; j >= 0 && tries < (1 << 24); ++tries) {
    unsigned long long w[AHEAD][CPL];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
      for (int c = 0; c < CPL; ++c) w[i][c] = get_word(words + (j - i > 0 ? j - i : 0) * pitch + c);
    bool there = true, all = false;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      bool valid = true, ended = true;
#pragma unroll
      for (int c = 0; c < CPL; ++c) valid = valid && (unsigned(w[i][c]) >> 31) != 0;
      there = there && !all && j >= 0 && __all(valid);
      if (there) {
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          const unsigned bits = unsigned(w[i][c]) & 0x7fffffffu;
          const float H = __uint_as_float(unsigned(w[i][c] >> 32));
          if (!done[c]) h[c] += a[c] * H;
          a[c] = compose_gates(a[c], bits == CLOSED ? 0.f : __uint_as_float(bits));
          done[c] = done[c] || unsigned(w[i][c]) == 0x80000000u;
          ended = ended && done[c];
        }
        all = __all(ended);
        --j;
      }
    }
    if (all) return;
    if (!there) __builtin_amdgcn_s_sleep(1);
  }
  if (j < 0) return;
#pragma unroll
  for (int c = 0; c < CPL; ++c) h[c] = __uint_as_float(0x7fc00000u);  // (never: see above)
}

// What a workgroup works on.
struct Place {
  int64_t b, tile;  // batch entry
  int span;         // place in the chain, 0 first
  uint32_t c;       // the lane's first feature
};

// CHAIN: spans by ticket, else one span a sequence (steps <= SPAN).
template <int CPL, bool CHAIN>
__device__ __forceinline__ Place place_of(const Args& p, unsigned* slot) {
  int64_t id = blockIdx.x;
  if constexpr (CHAIN) {
    if (threadIdx.x == 0) *slot = atomicAdd(p.ticket, 1u);
    __syncthreads();
    id = uint32_t(__builtin_amdgcn_readfirstlane(int(*slot)));  // (one for all: addresses stay in scalar registers)
  }
  Place q;
  q.tile = id % p.tiles;
  q.span = int(id / p.tiles);
  q.b = q.tile / p.feature_tiles;
  // Lanes past the end take the last CPL features too, with the same results:
  // they store the same values to the same places, so no lane is masked.
  const uint32_t c = uint32_t(q.tile % p.feature_tiles) * (64 * CPL) + (threadIdx.x & 63) * CPL;
  q.c = min(c, uint32_t(p.features) - CPL);
  return q;
}

template <class T, int CPL>
using raw_t = typename pack_of<T, CPL>::raw;

// The lane's features of a row.  (Scalar row address, 32-bit lane offset.)
template <class T, int CPL>
__device__ __forceinline__ raw_t<T, CPL> get(const T* row, uint32_t c) {
  return *reinterpret_cast<const pack_t<T, CPL>*>(reinterpret_cast<const char*>(row) + uint32_t(c * sizeof(T)));
}
template <class T, int CPL>
__device__ __forceinline__ void put(T* row, uint32_t c, const float (&v)[CPL]) {
  store_n<CPL>(reinterpret_cast<T*>(reinterpret_cast<char*>(row) + uint32_t(c * sizeof(T))), CPL, v);
}

// A value that the compiler cannot tell from a new one.
template <class V>
__device__ __forceinline__ void hide(V& v) {
  uint32_t w = 0;
  static_assert(sizeof(V) <= 4, "one register");
  __builtin_memcpy(&w, &v, sizeof(V));
  asm volatile("" : "+v"(w));
  __builtin_memcpy(&v, &w, sizeof(V));
}

// R rows of an array from row t on, one load each; past `rows` the last of them again.
template <bool FULL, class T, int CPL, int R>
__device__ __forceinline__ void get_rows(const T* p, Strides s, int64_t b, int64_t t, uint32_t c, int rows,
                                         raw_t<T, CPL> (&out)[R]) {
  const T* row = p + at(s, b, t);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    out[i] = get<T, CPL>(row, c);
    if (FULL || i + 1 < rows) row += s.t;
  }
}

template <class T, int CPL>
__device__ __forceinline__ void put_zeros(T* p, Strides s, int64_t b, int64_t t, int64_t end, uint32_t c) {
  for (; t < end; ++t) put<T, CPL>(p + at(s, b, t), c, {});
}

// R rows a wave.  GATED: with o.
template <class T, int CPL, int R, bool CHAIN, bool GATED>
__global__ void __launch_bounds__(64 * WAVES)
recurrence_kernel(Args p, const T* z, const T* v, const T* o, const float* h_zero, T* y, float* h_out, float* states) {
  __shared__ float mapA[WAVES][64 * CPL], mapH[WAVES][64 * CPL], enter[64 * CPL];
  __shared__ unsigned slot;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const Place q = place_of<CPL, CHAIN>(p, &slot);
  const int64_t n = length_of(p, q.b), span0 = int64_t(q.span) * SPAN, t0 = span0 + wave * R;
  const int64_t end = min(t0 + R, p.steps);
  if (span0 >= n && q.span > 0) {  // past the end (the first span goes on for the states)
    put_zeros<T, CPL>(y, p.y, q.b, t0, end, q.c);
    return;
  }
  const int rows = int(max<int64_t>(0, min<int64_t>(n - t0, R)));  // live rows of this wave
  const auto body = [&](auto full_) {  // full: all rows of all waves are live
    constexpr bool FULL = decltype(full_)::value;
    raw_t<T, CPL> zr[R], vr[R], orw[R];
    float s[R][CPL], bv[R][CPL];
    float A[CPL], H[CPL], h[CPL], least[CPL];
#pragma unroll
    for (int c = 0; c < CPL; ++c) A[c] = least[c] = 1.f, H[c] = 0.f, h[c] = 0.f;
    if (FULL || rows > 0) {
      get_rows<FULL, T, CPL, R>(z, p.z, q.b, t0, q.c, rows, zr);
      get_rows<FULL, T, CPL, R>(v, p.v, q.b, t0, q.c, rows, vr);
      if constexpr (GATED) get_rows<FULL, T, CPL, R>(o, p.o, q.b, t0, q.c, rows, orw);
    }
    if (q.span == 0 && h_zero != nullptr) {
#pragma unroll
      for (int c = 0; c < CPL; ++c) h[c] = h_zero[q.b * p.features + q.c + c];
    }
    if (FULL || rows > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          float gn;
          logistic<T>(float(zr[i][c]), s[i][c], gn);
          bv[i][c] = gn * float(vr[i][c]);
          if (!FULL && i >= rows) s[i][c] = 1.f, bv[i][c] = 0.f;
          A[c] *= s[i][c], least[c] = fminf(least[c], s[i][c]);
          H[c] = s[i][c] * H[c] + bv[i][c];
        }
#pragma unroll
      for (int c = 0; c < CPL; ++c) A[c] = product_of_gates(A[c], least[c]);
    }
    // the state that enters this wave's rows
    if (waves > 1) {
#pragma unroll
      for (int c = 0; c < CPL; ++c) mapA[wave][lane * CPL + c] = A[c], mapH[wave][lane * CPL + c] = H[c];
      __syncthreads();
      if constexpr (CHAIN) {
        if (wave == 0) {
          float tA[CPL], tH[CPL];
#pragma unroll
          for (int c = 0; c < CPL; ++c) {
            tA[c] = A[c], tH[c] = H[c];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) {
              const float a = mapA[i][lane * CPL + c];
              tH[c] = a * tH[c] + mapH[i][lane * CPL + c];
              tA[c] = compose_gates(tA[c], a);
            }
          }
          const int64_t pitch = 64 * CPL;
          unsigned long long* words = p.maps + q.tile * p.spans * pitch + lane * CPL;
          if (q.span > 0) {
#pragma unroll
            for (int c = 0; c < CPL; ++c) put_word(words + q.span * pitch + c, map_word(tA[c], tH[c]));
            look_back<CPL>(words, pitch, q.span, h);
          }
#pragma unroll
          for (int c = 0; c < CPL; ++c) {
            put_word(words + q.span * pitch + c, state_word(tA[c] * h[c] + tH[c]));
            enter[lane * CPL + c] = h[c];
          }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CPL; ++c) h[c] = enter[lane * CPL + c];
      }
    }
    if (states != nullptr && wave == 0) put<float, CPL>(states + (q.b * p.spans + q.span) * p.features, q.c, h);
    for (int i = 0; i < wave; ++i)
#pragma unroll
      for (int c = 0; c < CPL; ++c) h[c] = mapA[i][lane * CPL + c] * h[c] + mapH[i][lane * CPL + c];
    T* row = y + at(p.y, q.b, t0);
    if (FULL || rows > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float r[CPL];
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          h[c] = s[i][c] * h[c] + bv[i][c];
          r[c] = h[c];
          if constexpr (GATED) {
            const float x = float(orw[i][c]);
            r[c] *= x * logistic<T>(x);
          }
        }
        if (FULL || i < rows) {  // (past them h stands still; leaving the loop instead keeps it from being unrolled)
          put<T, CPL>(row, q.c, r);
          row += p.y.t;
        }
      }
    }
    if (!FULL) put_zeros<T, CPL>(y, p.y, q.b, t0 + rows, end, q.c);
    // the wave of the last live step (the first wave where there is none) has the state that leaves
    if (n == 0 ? wave == 0 : rows > 0 && t0 + rows == n) {
      if (h_out != nullptr) put<float, CPL>(h_out + q.b * p.features, q.c, h);
      if (states != nullptr)
        for (int k = q.span + 1; k < p.spans; ++k)
          put<float, CPL>(states + (q.b * p.spans + k) * p.features, q.c, h);
    }
  };
  if (span0 + waves * R <= n)
    body(std::true_type());
  else
    body(std::false_type());
}

// The backward; spans of the chain count from the last live one.
template <class T, int CPL, int R, bool CHAIN, bool GATED>
__global__ void __launch_bounds__(64 * WAVES)
recurrence_adj_kernel(Args p, const T* z, const T* v, const T* o, const float* states, const T* g_y, const float* g_h,
                      T* g_z, T* g_v, T* g_o, float* g_hzero) {
  __shared__ float mapA[WAVES][64 * CPL], mapH[WAVES][64 * CPL], mapG[WAVES][64 * CPL], enter[64 * CPL];
  __shared__ unsigned slot;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const Place q = place_of<CPL, CHAIN>(p, &slot);
  const int64_t n = length_of(p, q.b);
  const int live_spans = int((n + SPAN - 1) / SPAN);
  const int place = q.span;                                              // in the chain, while it is live
  const int span = place < live_spans ? live_spans - 1 - place : place;  // of the sequence
  const int64_t span0 = int64_t(span) * SPAN, t0 = span0 + wave * R, end = min(t0 + R, p.steps);
  const auto zeros_from = [&](int64_t t) {
    put_zeros<T, CPL>(g_z, p.gz, q.b, t, end, q.c);
    put_zeros<T, CPL>(g_v, p.gv, q.b, t, end, q.c);
    if constexpr (GATED) put_zeros<T, CPL>(g_o, p.go, q.b, t, end, q.c);
  };
  if (place >= live_spans) {
    zeros_from(t0);
    if (n == 0 && place == 0 && wave == 0 && g_hzero != nullptr) {
      float e[CPL];
#pragma unroll
      for (int c = 0; c < CPL; ++c) e[c] = g_h != nullptr ? g_h[q.b * p.features + q.c + c] : 0.f;
      put<float, CPL>(g_hzero + q.b * p.features, q.c, e);
    }
    return;
  }
  const int rows = int(max<int64_t>(0, min<int64_t>(n - t0, R)));
  const auto body = [&](auto full_) {  // full: all rows of all waves are live
    constexpr bool FULL = decltype(full_)::value;
    raw_t<T, CPL> zr[R], vr[R], orw[R], gr[R];
    float s[R][CPL], sn[R][CPL], b[R][CPL];  // b: then the state before the row
    float h[CPL], e[CPL], A[CPL], H[CPL], G[CPL], least[CPL];
    if (FULL || rows > 0) {
      get_rows<FULL, T, CPL, R>(z, p.z, q.b, t0, q.c, rows, zr);
      get_rows<FULL, T, CPL, R>(v, p.v, q.b, t0, q.c, rows, vr);
      get_rows<FULL, T, CPL, R>(g_y, p.y, q.b, t0, q.c, rows, gr);
      if constexpr (GATED) get_rows<FULL, T, CPL, R>(o, p.o, q.b, t0, q.c, rows, orw);
    }
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
      h[c] = states[(q.b * p.spans + span) * p.features + q.c + c];
      e[c] = place == 0 && g_h != nullptr ? g_h[q.b * p.features + q.c + c] : 0.f;
      A[c] = least[c] = 1.f, H[c] = 0.f, G[c] = 0.f;
    }
    if (FULL || rows > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          logistic<T>(float(zr[i][c]), s[i][c], sn[i][c]);
          b[i][c] = sn[i][c] * float(vr[i][c]);
          if (!FULL && i >= rows) s[i][c] = 1.f, sn[i][c] = b[i][c] = 0.f;
          A[c] *= s[i][c], least[c] = fminf(least[c], s[i][c]);
          H[c] = s[i][c] * H[c] + b[i][c];
        }
#pragma unroll
      for (int c = 0; c < CPL; ++c) A[c] = product_of_gates(A[c], least[c]);
#pragma unroll
      for (int i = R - 1; i >= 0; --i) {
        if (!FULL && i >= rows) continue;
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          float g = float(gr[i][c]);
          if constexpr (GATED) {
            const float x = float(orw[i][c]);
            g *= x * logistic<T>(x);
          }
          G[c] = s[i][c] * (g + G[c]);
        }
      }
      // (o's logistic is taken again below: kept, its 32 registers spill)
      if constexpr (GATED) {
#pragma unroll
        for (int i = 0; i < R; ++i) hide(orw[i]);
      }
    }
    if (waves > 1) {
#pragma unroll
      for (int c = 0; c < CPL; ++c)
        mapA[wave][lane * CPL + c] = A[c], mapH[wave][lane * CPL + c] = H[c], mapG[wave][lane * CPL + c] = G[c];
      __syncthreads();
      if constexpr (CHAIN) {
        if (wave == 0) {
          float tA[CPL], tG[CPL];
#pragma unroll
          for (int c = 0; c < CPL; ++c) {
            tA[c] = 1.f, tG[c] = 0.f;
#pragma unroll
            for (int i = WAVES - 1; i >= 0; --i) {
              const float a = mapA[i][lane * CPL + c];
              tG[c] = a * tG[c] + mapG[i][lane * CPL + c];
              tA[c] = compose_gates(tA[c], a);
            }
          }
          const int64_t pitch = 64 * CPL;
          unsigned long long* words = p.maps + q.tile * p.spans * pitch + lane * CPL;
          if (place > 0) {
#pragma unroll
            for (int c = 0; c < CPL; ++c) put_word(words + place * pitch + c, map_word(tA[c], tG[c]));
            look_back<CPL>(words, pitch, place, e);
          }
#pragma unroll
          for (int c = 0; c < CPL; ++c) {
            put_word(words + place * pitch + c, state_word(tA[c] * e[c] + tG[c]));
            enter[lane * CPL + c] = e[c];
          }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CPL; ++c) e[c] = enter[lane * CPL + c];
      }
    }
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
      for (int i = 0; i < wave; ++i) h[c] = mapA[i][lane * CPL + c] * h[c] + mapH[i][lane * CPL + c];
      for (int i = waves - 1; i > wave; --i) e[c] = mapA[i][lane * CPL + c] * e[c] + mapG[i][lane * CPL + c];
    }
    if (FULL || rows > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          const float next = s[i][c] * h[c] + b[i][c];
          b[i][c] = h[c];
          h[c] = next;
        }
      T *rz = g_z + at(p.gz, q.b, t0 + rows), *rv = g_v + at(p.gv, q.b, t0 + rows);
      T* ro = GATED ? g_o + at(p.go, q.b, t0 + rows) : nullptr;
#pragma unroll
      for (int i = R - 1; i >= 0; --i) {
        if (!FULL && i >= rows) continue;  // (such a row leaves e as it is)
        float gz[CPL], gv[CPL], go[CPL];
#pragma unroll
        for (int c = 0; c < CPL; ++c) {
          const float vv = float(vr[i][c]);
          float g = float(gr[i][c]);
          if constexpr (GATED) {
            const float x = float(orw[i][c]), so = logistic<T>(x), xs = x * so;
            go[c] = g * (s[i][c] * b[i][c] + sn[i][c] * vv) * (so + xs * (1.f - so));
            g *= xs;
          }
          const float d = g + e[c];
          gv[c] = d * sn[i][c];
          e[c] = s[i][c] * d;
          gz[c] = gv[c] * s[i][c] * (b[i][c] - vv);
        }
        rz -= p.gz.t, rv -= p.gv.t;
        put<T, CPL>(rz, q.c, gz);
        put<T, CPL>(rv, q.c, gv);
        if constexpr (GATED) {
          ro -= p.go.t;
          put<T, CPL>(ro, q.c, go);
        }
      }
    }
    if (!FULL) zeros_from(t0 + rows);
    if (span == 0 && wave == 0 && g_hzero != nullptr) put<float, CPL>(g_hzero + q.b * p.features, q.c, e);
  };
  if (span0 + waves * R <= n)
    body(std::true_type());
  else
    body(std::false_type());
}

// h_out = h_zero (g_hzero = g_h) where there are no steps.
__global__ void __launch_bounds__(256) copy_state_kernel(const float* in, float* out, int64_t n) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) out[i] = in != nullptr ? in[i] : 0.f;
}

// The chain's words and its ticket start from zero.  (Four stores a thread: a
// kernel, as a recorded memset does not replay rightly.)
__global__ void __launch_bounds__(256) clear_kernel(uint4* p, int64_t n) {
  const int64_t i = int64_t(blockIdx.x) * 1024 + threadIdx.x;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j * 256 < n) p[i + j * 256] = uint4{0, 0, 0, 0};
}

Args args_of(const dtst_recurrence_desc& d, const int32_t* lengths, int cpl) {
  auto st = [](const int64_t (&s)[2]) { return Strides{s[0], s[1]}; };
  Args p{d.batch, d.steps, d.features, st(d.z_stride), st(d.v_stride), st(d.o_stride), st(d.y_stride),
         st(d.g_z_stride), st(d.g_v_stride), st(d.g_o_stride), lengths, 0, 0, 0, nullptr, nullptr};
  p.feature_tiles = (d.features + 64 * cpl - 1) / (64 * cpl);
  p.tiles = p.feature_tiles * d.batch;
  p.spans = int((d.steps + SPAN - 1) / SPAN);
  return p;
}

// Features of a lane: two, but one in the backward of 32 bits (two would hold
// more registers than there are) and where two leave half of the CUs idle (2 x
// 128 x 1000 bf16: backward 11 against 9 us; 2 x 1024 x 2048, 256 workgroups: 22
// against 23).
// The last lanes of a tile of 128 step back over features of the same tile.  A
// single feature left over would be computed with its neighbour, which another
// workgroup has too and may have updated in place already: such a number of
// features is taken one a lane.
int lane_features(const dtst_recurrence_desc& d, bool adj) {
  const int64_t spans = (d.steps + SPAN - 1) / SPAN;
  const bool fills = d.batch * ((d.features + 127) / 128) * spans > 128;
  return fills && d.features % 128 != 1 && !(adj && d.type == DTST_F32) ? 2 : 1;
}

template <class F>
int by_type(int type, F&& f) {
  if (type == DTST_F32) return f(float());
  if (type == DTST_BF16) return f(bf16_t());
  return f(f16_t());
}

int copy_state(const float* in, float* out, int64_t n, hipStream_t s) {
  if (out == nullptr || out == in) return hipSuccess;
  hipLaunchKernelGGL(copy_state_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0, s, in, out, n);
  return hipGetLastError();
}

// Clears the chain's words and ticket where there is one, then calls
// f(args, element, CPL, R, CHAIN, GATED, workgroups, threads): spans by ticket
// where a sequence has several; one row a wave for one step (its registers and
// loads are then one row's).
template <bool ADJ, class F>
int by_form(const dtst_recurrence_desc& d, const int32_t* lengths, bool with_o, void* workspace, hipStream_t s, F&& f) {
  using std::integral_constant;
  using std::false_type;
  using std::true_type;
  return by_type(d.type, [&](auto t) {
    const auto rest = [&](auto cpl, auto gated) {
      Args p = args_of(d, lengths, cpl.value);
      if (p.spans > 1) {
        const int64_t bytes = 64 + p.tiles * p.spans * 64 * cpl.value * 8;
        p.ticket = static_cast<unsigned*>(workspace);
        p.maps = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + 64);
        hipLaunchKernelGGL(clear_kernel, dim3(unsigned((bytes / 16 + 1023) / 1024)), dim3(256), 0, s,
                           static_cast<uint4*>(workspace), bytes / 16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return int(e);
        return f(p, t, cpl, integral_constant<int, RPW>(), true_type(), gated, unsigned(p.tiles * p.spans), 64 * WAVES);
      }
      if (p.steps == 1)
        return f(p, t, cpl, integral_constant<int, 1>(), false_type(), gated, unsigned(p.tiles), 64);
      return f(p, t, cpl, integral_constant<int, RPW>(), false_type(), gated, unsigned(p.tiles),
               64 * int((p.steps + RPW - 1) / RPW));
    };
    const auto with_gate = [&](auto cpl) { return with_o ? rest(cpl, true_type()) : rest(cpl, false_type()); };
    if constexpr (!(ADJ && std::is_same_v<decltype(t), float>))
      if (lane_features(d, ADJ) == 2) return with_gate(integral_constant<int, 2>());
    return with_gate(integral_constant<int, 1>());
  });
}

}  // namespace

size_t recurrence_workspace(int64_t batch, int64_t steps, int64_t features, int) {
  if (steps <= SPAN) return 0;
  // (tiles of 128 features; those of 64 have no more words)
  return 64 + size_t(batch * ((features + 127) / 128)) * ((steps + SPAN - 1) / SPAN) * 128 * 8;
}

int launch_recurrence(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o, const float* h_zero,
                      const int32_t* lengths, void* y, float* h_out, float* states, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.steps == 0) return copy_state(h_zero, h_out, d.batch * d.features, s);
  return by_form<false>(d, lengths, o != nullptr, workspace, s,
                 [&](const Args& p, auto t, auto cpl, auto r, auto chain, auto gated, unsigned groups, int threads) {
                   using T = decltype(t);
                   hipLaunchKernelGGL((recurrence_kernel<T, decltype(cpl)::value, decltype(r)::value,
                                                         decltype(chain)::value, decltype(gated)::value>),
                                      dim3(groups), dim3(threads), 0, s, p, static_cast<const T*>(z),
                                      static_cast<const T*>(v), static_cast<const T*>(o), h_zero, static_cast<T*>(y),
                                      h_out, states);
                   return int(hipGetLastError());
                 });
}

int launch_recurrence_adj(const dtst_recurrence_desc& d, const void* z, const void* v, const void* o,
                          const int32_t* lengths, const float* states, const void* g_y, const float* g_h, void* g_z,
                          void* g_v, void* g_o, float* g_hzero, void* workspace, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.steps == 0) return copy_state(g_h, g_hzero, d.batch * d.features, s);
  return by_form<true>(d, lengths, o != nullptr, workspace, s,
                 [&](const Args& p, auto t, auto cpl, auto r, auto chain, auto gated, unsigned groups, int threads) {
                   using T = decltype(t);
                   hipLaunchKernelGGL((recurrence_adj_kernel<T, decltype(cpl)::value, decltype(r)::value,
                                                             decltype(chain)::value, decltype(gated)::value>),
                                      dim3(groups), dim3(threads), 0, s, p, static_cast<const T*>(z),
                                      static_cast<const T*>(v), static_cast<const T*>(o), states,
                                      static_cast<const T*>(g_y), g_h, static_cast<T*>(g_z), static_cast<T*>(g_v),
                                      static_cast<T*>(g_o), g_hzero);
                   return int(hipGetLastError());
                 });
}

}  // namespace dtst
