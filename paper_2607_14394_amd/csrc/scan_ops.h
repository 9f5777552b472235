// What the state-space scan's two directions share: the step size of a raw value,
// the decay of a run of steps, and the arrays' places.
#pragma once

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {

constexpr int SCAN_SPAN = DTST_SCAN_SPAN;
constexpr float LOG2E = 1.44269502162933349609375f;

// D = log(1 + exp(d)) = max(d, 0) + log(1 + e), e = exp(-|d|), of a d of type T.
// 1 + e rounds e's low bits off; what it lost, c, goes back in (to first order, whose
// error is c e / (1 + e), 2^-24 of the result).
template <class T>
__device__ __forceinline__ float softplus(float d) {
  constexpr float ln2 = 0.693147180559945309f;
  const float e = exp_minus<T>(fabsf(d));
  const float u = 1.f + e, c = e - (u - 1.f);
  return fmaxf(d, 0.f) + fmaf(__builtin_amdgcn_logf(u), ln2, c);
}

// exp(a D) of a run of steps whose D come to `sum`, the largest being `most`; a2 =
// a log2(e).  One that underflows though no step's does stays above zero: it would
// make no number of an infinite state, which the steps one by one keep.  A sum past
// 32 bits is their largest, of which a = 0 makes 1 as of every step.  (A D that is no
// number shows in the run's end.)
__device__ __forceinline__ float run_decay(float a2, float sum, float most) {
  const float A = __builtin_amdgcn_exp2f(a2 * fminf(sum, 3.402823466e38f));
  return a2 * most >= -126.f ? fmaxf(A, __uint_as_float(1)) : A;
}

struct ScanArgs {
  int64_t batch, steps, features;
  int states;
  Strides x, delta, b, c, o, y, gx, gdelta, gb, gc, go;
  const int32_t* lengths;
  int segments;          // of a sequence
  int64_t segment;       // steps of each but the last, a multiple of SCAN_SPAN
  int64_t tiles, spans;  // of 64 features; of SCAN_SPAN steps
};

__device__ __forceinline__ int64_t scan_length(const ScanArgs& p, int64_t b) {
  if (p.lengths == nullptr) return p.steps;
  const int64_t n = p.lengths[b];
  return n < 0 ? 0 : n > p.steps ? p.steps : n;
}

// A lane's offset in bytes, which the compiler cannot tell from any other: it would
// fold it into each row's address, two registers and an instruction a row.
__device__ __forceinline__ uint32_t lane_offset(uint32_t bytes) {
  asm volatile("" : "+v"(bytes));
  return bytes;
}

// The lane's value of a row.  (Scalar row address, 32-bit lane offset.)
template <class T>
__device__ __forceinline__ T get(const T* row, uint32_t offset) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + offset);
}
template <class T>
__device__ __forceinline__ void put(T* row, uint32_t offset, float v) {
  *reinterpret_cast<T*>(reinterpret_cast<char*>(row) + offset) = T(v);
}
// Of R rows from row t on; FULL: all there, else past `rows` the last of them again.
template <bool FULL, int R, class T>
__device__ __forceinline__ void get_rows(const T* p, Strides s, int64_t e, int64_t t, int rows, uint32_t offset,
                                         T (&out)[R]) {
  const T* row = p + at(s, e, t);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    out[i] = get(row, offset);
    if (FULL || i + 1 < rows) row += s.t;
  }
}

// Waves a SIMD that the forward's kernel of so many states is built for: as its registers
// allow.
constexpr int scan_waves(int states) { return states <= 8 ? 4 : states <= 32 ? 3 : 2; }

struct ScanPointers {
  const void *x, *delta, *b, *c, *o;
  const float *a, *skip, *h_zero;
  void* y;
  float *h_out, *states, *carry;
};
template <class T>
int launch_scan_type(const ScanArgs& p, const ScanPointers& q, hipStream_t s);

ScanArgs scan_args(const dtst_scan_desc& d, const int32_t* lengths, bool adj);
// Turns the ends in carry (batch, segments, states + 2, features: the state's end
// from zero, the sum and the largest of the segment's D; none of the last segment's,
// in reverse of the first's) into what enters.
int launch_scan_carry(const ScanArgs& p, const float* a, const float* first, float* carry, bool reverse, void* stream);
int launch_copy_states(const float* in, float* out, int64_t n, void* stream);

}  // namespace dtst
