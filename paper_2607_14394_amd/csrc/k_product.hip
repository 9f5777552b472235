// Product of 8-bit arrays with a power-of-two scale for each 128 of the summed
// axis (dtst_product):  c[i,j] = sum_l a[i,l] b[j,l] + bias[j].
//
// A code is a bf16 number without loss, also times its scale, so the operands go
// to v_mfma_f32_16x16x32_bf16, whose sums are exact to 32 bits; the 8-bit
// instruction keeps only 13 bits below the largest of eight neighbouring
// products.  Two codes and their scale make two bf16 in one instruction.  Lane l
// holds row l % 16 of both operands and 8 of each 32 of the summed axis (any
// eight, as long as they are the same for both).  With b as the first operand a
// lane ends with four neighbouring columns 4 (l / 16) + r of row l % 16 of c.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16_t v8b __attribute__((ext_vector_type(8)));
typedef bf16_t v2b __attribute__((ext_vector_type(2)));

// Eight codes times their scale.
__device__ __forceinline__ v8b widen(uint32_t lo, uint32_t hi, float scale) {
  const v2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const v2b b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const v2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const v2b d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return v8b{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 2^(s - 127)
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fc00000u : s << 23);
}

struct Operands {
  const uint8_t *a, *b;
  const uint8_t *sa, *sb;
  int64_t m, n, k, ld_a, ld_sa, ld_b, ld_sb, ld_c;
  const float* bias;
  int accumulate;
};

// Four neighbouring columns of a row of c, `left` of them inside.
template <class TC>
__device__ __forceinline__ void put_c(TC* c, int64_t left, v4f v, const float* bias, int accumulate) {
  float o[4], e[4];
  if (bias != nullptr) {
    load_n<4>(bias, left, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += e[i];
  }
  if (accumulate) {
    load_n<4>(c, left, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += e[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = v[i];
  store_n<4>(c, left, o);
}

// A wave takes 32 x 32 of c, a workgroup 64 x 64, straight from global memory.
template <class TC>
__global__ void __launch_bounds__(256)
product_direct_kernel(Operands p, TC* c, int n_tiles) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t m0 = int64_t(blockIdx.x / n_tiles) * 64 + (wave >> 1) * 32;
  const int64_t n0 = int64_t(blockIdx.x % n_tiles) * 64 + (wave & 1) * 32;
  const int r = lane & 15, g = lane >> 4;
  const uint8_t *pa[2], *pb[2], *psa[2], *psb[2];
  v4f acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    // rows past the end read the last one; their results are not stored
    const int64_t ra = min(m0 + i * 16 + r, p.m - 1), rb = min(n0 + i * 16 + r, p.n - 1);
    pa[i] = p.a + ra * p.ld_a + g * 32;
    pb[i] = p.b + rb * p.ld_b + g * 32;
    psa[i] = p.sa + ra * p.ld_sa;
    psb[i] = p.sb + rb * p.ld_sb;
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  for (int64_t k = 0; k < p.k; k += 128) {
    v8b fa[2][4], fb[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float sa = scale_value(psa[i][k >> 7]), sb = scale_value(psb[i][k >> 7]);
      const uint4 *qa = reinterpret_cast<const uint4*>(pa[i] + k), *qb = reinterpret_cast<const uint4*>(pb[i] + k);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 x = qa[h], y = qb[h];
        fa[i][2 * h] = widen(x.x, x.y, sa), fa[i][2 * h + 1] = widen(x.z, x.w, sa);
        fb[i][2 * h] = widen(y.x, y.y, sb), fb[i][2 * h + 1] = widen(y.z, y.w, sb);
      }
    }
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][h], fa[i][h], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t row = m0 + i * 16 + r;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t col = n0 + j * 16 + g * 4;
      if (row < p.m && col < p.n)
        put_c(c + row * p.ld_c + col, p.n - col, acc[i][j], p.bias == nullptr ? nullptr : p.bias + col, p.accumulate);
    }
  }
}

template <class TC>
int launch(const Operands& p, void* c, hipStream_t s) {
  const int64_t mt = (p.m + 63) / 64, nt = (p.n + 63) / 64;
  hipLaunchKernelGGL(product_direct_kernel<TC>, dim3(unsigned(mt * nt)), dim3(256), 0, s, p, static_cast<TC*>(c),
                     int(nt));
  return hipGetLastError();
}

}  // namespace

size_t product_workspace(int64_t, int64_t, int64_t) { return 0; }

int launch_product(const dtst_product_desc& d, const void* a, const void* a_scale, const void* b, const void* b_scale,
                   const float* bias, void* c, void*, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Operands p{static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(b),
                   static_cast<const uint8_t*>(a_scale), static_cast<const uint8_t*>(b_scale),
                   d.m, d.n, d.k, d.ld_a, d.ld_a_scale, d.ld_b, d.ld_b_scale, d.ld_c, bias, d.accumulate};
  if (d.c_type == DTST_F32) return launch<float>(p, c, s);
  if (d.c_type == DTST_BF16) return launch<bf16_t>(p, c, s);
  return launch<f16_t>(p, c, s);
}

}  // namespace dtst
