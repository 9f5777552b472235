// Product of 8-bit arrays with a power-of-two scale for each 128 of the summed
// axis (dtst_product):  c[i,j] = sum_l a[i,l] b[j,l] + bias[j].
//
// Two forms of the matrix products.  Exact: a code times its scale is a bf16
// number without loss, so the operands are widened (two codes an instruction,
// the scale with it) for v_mfma_f32_16x16x32_bf16, whose sums are exact to 32
// bits.  Short (dtst_product_desc::short_sums): v_mfma_scale_f32_16x16x128_f8f6f4
// takes 128 codes at once and the scales' powers of two as an operand, at twice
// the rate, but keeps only 13 bits below the largest of eight neighbouring
// products.  In both, lane l holds row l % 16 of the operands and a quarter of
// the 128 codes (any quarter, as long as it is the same for both); with b as the
// first operand a lane ends with four neighbouring columns 4 (l / 16) + r of row
// l % 16 of c.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
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

// 2^(s - 127); s = 255 is no number.
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

// ---- few rows of a ----------------------------------------------------------
//
// Up to 16 MT rows: bound by reading b once.  A workgroup takes 16 rows of b;
// its waves take every eighth block of 128 codes, straight from global memory,
// and their sums meet in LDS in a fixed order.
constexpr int FEW_WAVES = 8;

template <class TC, int MT>
__global__ void __launch_bounds__(64 * FEW_WAVES)
product_few_kernel(Operands p, TC* c) {
  __shared__ v4f sums[FEW_WAVES][MT][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t n0 = int64_t(blockIdx.x) * 16;
  // rows past the end read the last one; their results are not stored
  const int64_t rb = min(n0 + r, p.n - 1);
  const uint8_t *pb = p.b + rb * p.ld_b + g * 32, *psb = p.sb + rb * p.ld_sb;
  const uint8_t *pa[MT], *psa[MT];
  v4f acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t ra = min(int64_t(i * 16 + r), p.m - 1);
    pa[i] = p.a + ra * p.ld_a + g * 32;
    psa[i] = p.sa + ra * p.ld_sa;
    acc[i] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  const int nk = int((p.k + 127) / 128);
  for (int kb = wave; kb < nk; kb += FEW_WAVES) {
    const uint4* qb = reinterpret_cast<const uint4*>(pb + int64_t(kb) * 128);
    const uint4 y0 = qb[0], y1 = qb[1];
    const float sb = scale_value(psb[kb]);
    uint4 x[MT][2];
    float sa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint4* qa = reinterpret_cast<const uint4*>(pa[i] + int64_t(kb) * 128);
      x[i][0] = qa[0], x[i][1] = qa[1];
      sa[i] = scale_value(psa[i][kb]);
    }
    const v8b fb[4] = {widen(y0.x, y0.y, sb), widen(y0.z, y0.w, sb), widen(y1.x, y1.y, sb), widen(y1.z, y1.w, sb)};
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[2 * h], widen(x[i][h].x, x[i][h].y, sa[i]), acc[i], 0, 0, 0);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[2 * h + 1], widen(x[i][h].z, x[i][h].w, sa[i]), acc[i], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < MT; i += FEW_WAVES) {
    v4f v = sums[0][i][lane];
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) v += sums[w][i][lane];
    const int64_t row = i * 16 + r, col = n0 + g * 4;
    if (row < p.m && col < p.n)
      put_c(c + row * p.ld_c + col, p.n - col, v, p.bias == nullptr ? nullptr : p.bias + col, p.accumulate);
  }
}

// ---- tiles ------------------------------------------------------------------
//
// A workgroup of WM x WN waves takes BM x BN of c, a wave TM x TN tiles of 16 x
// 16.  Each 128 codes of the summed axis are a stage: the rows' 128 bytes go
// straight from global memory to LDS (16 bytes a lane, no registers), STAGES - 1
// stages ahead of the products.  A row's 16-byte chunk i lies at place
// i ^ (row % 8), so the 8 lanes that read one chunk of 8 rows meet 8 different
// places.  Scale bytes come by four stages at a time, a word a row.
constexpr int ROW = 128;

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)(p)));
}

// 64 lanes' 16 (4) bytes at base + off to LDS at `to` + 16 (4) times the lane.
// (The compiler does not see the load: whoever reads the bytes waits for it.)
__device__ __forceinline__ void fetch16(const uint8_t* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void fetch4(const uint8_t* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
// At most N of the wave's loads are still on their way, and none of its reads
// of LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}

template <bool SHORT, int WM, int WN, int TM, int TN, int STAGES, class TC>
__global__ void __launch_bounds__(64 * WM * WN)
product_tile_kernel(Operands p, TC* c, int m_tiles, int n_tiles) {
  constexpr int WAVES = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, STAGE = (BM + BN) * ROW;
  constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;  // loads of a wave and stage: 8 rows each
  static_assert(LA * 8 * WAVES == BM && LB * 8 * WAVES == BN, "whole loads");
  constexpr int SCALES = (BM + BN) * 4;
  extern __shared__ uint8_t lds[];  // STAGES stages, then two groups of scale words
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r = lane & 15, g = lane >> 4;

  // Workgroups go to the 8 dies in turn: a die gets neighbouring tiles, in bands
  // of 8 tile rows, so that its cache holds their operands.
  int id = blockIdx.x;
  const int all = m_tiles * n_tiles;
  if (all >= 64) {
    const int die = id % 8, per = all / 8, extra = all % 8;
    id = die * per + min(die, extra) + id / 8;
  }
  const int band = id / (8 * n_tiles), band_rows = min(8, m_tiles - band * 8), in_band = id - band * 8 * n_tiles;
  const int64_t m0 = int64_t(band * 8 + in_band % band_rows) * BM, n0 = int64_t(in_band / band_rows) * BN;

  // Where this lane's loads start: row wave * L + .. of each operand.  Rows past
  // the end read the last one; their results are not stored.
  const uint8_t *base_a = p.a + m0 * p.ld_a, *base_b = p.b + n0 * p.ld_b;
  const int chunk = (lane & 7) ^ (lane >> 3);
  uint32_t off_a[LA], off_b[LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int64_t row = min<int64_t>((wave * LA + i) * 8 + (lane >> 3), p.m - 1 - m0);
    off_a[i] = uint32_t(row * p.ld_a) + chunk * 16;
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int64_t row = min<int64_t>((wave * LB + i) * 8 + (lane >> 3), p.n - 1 - n0);
    off_b[i] = uint32_t(row * p.ld_b) + chunk * 16;
  }
  // scale words: 64 rows a load, the waves in turn
  constexpr int SL = (BM + BN) / 64, SPW = (SL + WAVES - 1) / WAVES;
  uint32_t off_s[SPW];
#pragma unroll
  for (int i = 0; i < SPW; ++i) {
    const int row = (wave + i * WAVES) * 64 + lane;
    off_s[i] = row < BM ? uint32_t(min<int64_t>(row, p.m - 1 - m0) * p.ld_sa)
                        : uint32_t(min<int64_t>(row - BM, p.n - 1 - n0) * p.ld_sb);
  }
  const uint8_t *base_sa = p.sa + m0 * p.ld_sa, *base_sb = p.sb + n0 * p.ld_sb;

  const uint32_t lds0 = lds_address(lds);
  const auto fetch = [&](int kb) {
    const uint32_t to = lds0 + (kb % STAGES) * STAGE;
    if (kb % 4 == 0) {
#pragma unroll
      for (int i = 0; i < SPW; ++i) {
        const int part = wave + i * WAVES;
        if (part < SL)
          fetch4((part * 64 < BM ? base_sa : base_sb) + kb, off_s[i],
                 lds0 + STAGES * STAGE + (kb / 4 % 2) * SCALES + part * 256);
      }
    }
#pragma unroll
    for (int i = 0; i < LA; ++i) fetch16(base_a + int64_t(kb) * ROW, off_a[i], to + (wave * LA + i) * 1024);
#pragma unroll
    for (int i = 0; i < LB; ++i)
      fetch16(base_b + int64_t(kb) * ROW, off_b[i], to + BM * ROW + (wave * LB + i) * 1024);
  };

  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  const int wm = wave / WN, wn = wave % WN;
  const int place = r * ROW + ((g ^ (r & 7)) << 4);  // chunk g of row r; chunk g + 4 lies at ^ 64
  const int nk = int((p.k + 127) / 128);
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < nk) fetch(s);
  for (int kb = 0; kb < nk; ++kb) {
    // this stage's loads are done when only those of the STAGES - 2 later ones are left
    if (kb + STAGES - 2 < nk)
      wait_loads<(LA + LB) * (STAGES - 2)>();
    else
      wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    if (kb + STAGES - 1 < nk) fetch(kb + STAGES - 1);  // over the stage that every wave has left
    const uint8_t* at_a = lds + (kb % STAGES) * STAGE + wm * TM * 16 * ROW;
    const uint8_t* at_b = lds + (kb % STAGES) * STAGE + BM * ROW + wn * TN * 16 * ROW;
    const uint8_t* at_sa = lds + STAGES * STAGE + (kb / 4 % 2) * SCALES + (wm * TM * 16 + r) * 4 + kb % 4;
    const uint8_t* at_sb = lds + STAGES * STAGE + (kb / 4 % 2) * SCALES + (BM + wn * TN * 16 + r) * 4 + kb % 4;
    if constexpr (SHORT) {
      v8i fb[TN];
      int sb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const v4i lo = *reinterpret_cast<const v4i*>(at_b + j * 16 * ROW + place);
        const v4i hi = *reinterpret_cast<const v4i*>(at_b + j * 16 * ROW + (place ^ 64));
        fb[j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        sb[j] = at_sb[j * 64];
      }
      // row tiles one ahead of the products
      v8i fa[2];
      int sa[2];
      const auto read_a = [&](int i) {
        const v4i lo = *reinterpret_cast<const v4i*>(at_a + i * 16 * ROW + place);
        const v4i hi = *reinterpret_cast<const v4i*>(at_a + i * 16 * ROW + (place ^ 64));
        fa[i & 1] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        sa[i & 1] = at_sa[i * 64];
      };
      read_a(0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i + 1 < TM) read_a(i + 1);
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i & 1], acc[i][j], 0, 0, 0, sb[j], 0,
                                                                        sa[i & 1]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      float sa[TM], sb[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = scale_value(at_sb[j * 64]);
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = scale_value(at_sa[i * 64]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // half of the quarter at a time: fewer registers
        v8b fb[TN][2];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const v4i x = *reinterpret_cast<const v4i*>(at_b + j * 16 * ROW + (place ^ (h * 64)));
          fb[j][0] = widen(x[0], x[1], sb[j]), fb[j][1] = widen(x[2], x[3], sb[j]);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const v4i x = *reinterpret_cast<const v4i*>(at_a + i * 16 * ROW + (place ^ (h * 64)));
          const v8b fa[2] = {widen(x[0], x[1], sa[i]), widen(x[2], x[3], sa[i])};
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < TN; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][e], fa[e], acc[i][j], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t row = m0 + (wm * TM + i) * 16 + r;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t col = n0 + (wn * TN + j) * 16 + g * 4;
      if (row < p.m && col < p.n)
        put_c(c + row * p.ld_c + col, p.n - col, acc[i][j], p.bias == nullptr ? nullptr : p.bias + col, p.accumulate);
    }
  }
}

template <class TC, int MT>
int launch_few(const Operands& p, void* c, hipStream_t s) {
  hipLaunchKernelGGL((product_few_kernel<TC, MT>), dim3(unsigned((p.n + 15) / 16)), dim3(64 * FEW_WAVES), 0, s, p,
                     static_cast<TC*>(c));
  return hipGetLastError();
}

template <bool SHORT, int WM, int WN, int TM, int TN, int STAGES, class TC>
int launch_tile(const Operands& p, void* c, hipStream_t s) {
  constexpr int BM = WM * TM * 16, BN = WN * TN * 16;
  const int64_t mt = (p.m + BM - 1) / BM, nt = (p.n + BN - 1) / BN;
  constexpr size_t lds = size_t(STAGES) * (BM + BN) * ROW + 2 * (BM + BN) * 4;
  auto* fn = product_tile_kernel<SHORT, WM, WN, TM, TN, STAGES, TC>;
  if (lds > 65536) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(fn, dim3(unsigned(mt * nt)), dim3(64 * WM * WN), lds, s, p, static_cast<TC*>(c), int(mt), int(nt));
  return hipGetLastError();
}

template <class TC>
int launch(const Operands& p, int short_sums, void* c, hipStream_t s) {
  if (p.m <= 16) return launch_few<TC, 1>(p, c, s);
  if (p.m <= 32) return launch_few<TC, 2>(p, c, s);
  if (p.m <= 64) return launch_few<TC, 4>(p, c, s);
  const auto tiles = [&](int64_t bm, int64_t bn) { return ((p.m + bm - 1) / bm) * ((p.n + bn - 1) / bn); };
  if (short_sums) {
    if (tiles(256, 256) >= 200) return launch_tile<true, 2, 2, 8, 8, 2, TC>(p, c, s);
    if (tiles(128, 128) >= 200) return launch_tile<true, 2, 2, 4, 4, 2, TC>(p, c, s);
    return launch_tile<true, 2, 2, 2, 2, 4, TC>(p, c, s);
  }
  if (tiles(256, 256) >= 200) return launch_tile<false, 2, 4, 8, 4, 2, TC>(p, c, s);
  if (tiles(128, 128) >= 200) return launch_tile<false, 2, 2, 4, 4, 2, TC>(p, c, s);
  return launch_tile<false, 2, 2, 2, 2, 4, TC>(p, c, s);
}

}  // namespace

size_t product_workspace(int64_t, int64_t, int64_t) { return 0; }

int launch_product(const dtst_product_desc& d, const void* a, const void* a_scale, const void* b, const void* b_scale,
                   const float* bias, void* c, void*, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Operands p{static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(b),
                   static_cast<const uint8_t*>(a_scale), static_cast<const uint8_t*>(b_scale),
                   d.m, d.n, d.k, d.ld_a, d.ld_a_scale, d.ld_b, d.ld_b_scale, d.ld_c, bias, d.accumulate};
  if (d.c_type == DTST_F32) return launch<float>(p, d.short_sums, c, s);
  if (d.c_type == DTST_BF16) return launch<bf16_t>(p, d.short_sums, c, s);
  return launch<f16_t>(p, d.short_sums, c, s);
}

}  // namespace dtst
