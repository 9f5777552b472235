// Product of 8-bit arrays with a power-of-two scale for each 128 of the summed
// axis (dtst_product):  c[i,j] = sum_l a[i,l] b[j,l] + bias[j].
//
// A code times its scale is a bf16 number without loss, so the operands are
// widened (two codes an instruction, the scale with it) for
// v_mfma_f32_16x16x32_bf16, whose sums are exact to 32 bits.
// (v_mfma_scale_f32_16x16x128_f8f6f4 takes 128 codes and the scales' powers of
// two at once, at twice the rate, but its sum of eight neighbouring products keeps
// 13 bits below the largest: too few for the 32-bit states of a recurrence on the
// results, which move by 3e-3.)  Lane l holds row l % 16 of the operands and a
// quarter of the 128 codes (any quarter, as long as it is the same for both); with
// b as the first operand a lane ends with four neighbouring columns 4 (l / 16) + r
// of row l % 16 of c.
//
// Large products are bound by the matrix cores and what feeds them: 8192^3 716 to
// 753 us, by the card (1530 to 1460 TFLOP/s; the cores are busy 67% of the time;
// without the widening, two codes an instruction in between, 12 to 15% less).
// Smaller ones wait for their first loads and their stores.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "seq_internal.h"
#include "seq_ops.h"

namespace dtst {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
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

// 2^(s - 127), s = 1 .. 254, of a byte read a tile ago.  (The empty statement
// keeps the shift here: next to the read it would wait for it.)
__device__ __forceinline__ float scale_value(int s) {
  asm volatile("" : "+v"(s));
  return __int_as_float(s << 23);
}

struct Operands {
  const uint8_t *a, *b;
  const uint8_t *sa, *sb;
  int64_t m, n, k, ld_a, ld_sa, ld_b, ld_sb, ld_c;
  const float* bias;
  int accumulate;
};

// A workgroup takes BM x BN of c.  WM x WN waves hold it, each TM x TN tiles of 16
// x 16; KS such groups take a part of the summed axis each and add up in LDS at
// the end.  Each 128 codes of the summed axis are a stage: the rows' 128 bytes go
// straight from global memory to LDS (16 bytes a lane, no registers), STAGES - 1
// stages ahead of the products.  A row's 16-byte chunk i lies at place
// i ^ (row % 8), so the 8 lanes that read one chunk of 8 rows meet 8 different
// places.  Scale bytes come by four stages at a time, a word a row.
constexpr int ROW = 128;

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)(p)));
}

// 64 lanes' 16 bytes at base + off (4 bytes at p) to LDS at `to` + 16 (4) times
// the lane.  (The compiler does not see the load: whoever reads the bytes waits
// for it.  m0 is no register that it keeps values in: it writes m0 itself where an
// instruction of its own takes it.)
__device__ __forceinline__ void fetch16(const uint8_t* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void fetch4(const uint8_t* p, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(to), "v"(p) : "memory");
}
// At most N of the wave's loads are still on their way, and none of its reads
// of LDS.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(N) : "memory");
}

// Tile row and column of a workgroup.  Workgroups go to the 8 dies in turn: a die
// gets neighbouring tiles, in bands of 8 tile rows, so that its cache holds their
// operands.  (readfirstlane: the addresses that follow belong in scalar registers)
__device__ __forceinline__ void tile_of(int m_tiles, int n_tiles, int& tm, int& tn) {
  int id = blockIdx.x;
  const int all = m_tiles * n_tiles;
  if (all >= 64) {
    const int die = id % 8, per = all / 8, extra = all % 8;
    id = die * per + min(die, extra) + id / 8;
  }
  const int band = id / (8 * n_tiles), band_rows = min(8, m_tiles - band * 8), in_band = id - band * 8 * n_tiles;
  tm = __builtin_amdgcn_readfirstlane(band * 8 + in_band % band_rows);
  tn = __builtin_amdgcn_readfirstlane(in_band / band_rows);
}

// A wave's TM x TN tiles of sums to c from (row0, col0) on: 16 rows at a time
// through the wave's own strip of LDS, so that a lane stores eight neighbouring
// columns and a row's lanes whole lines.
constexpr int strip_pitch(int tn) { return tn * 16 + 4; }  // (8 rows' accesses of 16 bytes meet all banks)
constexpr int strip_floats(int tn) { return 16 * strip_pitch(tn); }

template <int TM, int TN, class TC>
__device__ __forceinline__ void put_tiles(const Operands& p, TC* c, const v4f (&acc)[TM][TN], int64_t row0, int64_t col0,
                                          int lane, float* strip) {
  constexpr int PITCH = strip_pitch(TN);
  const int r = lane & 15, g = lane >> 4;
  constexpr int PARTS_C = (TN + 1) / 2;  // eights of a strip's columns that a lane takes
  float bias[PARTS_C][8];                // (read once: inside the loop each read would hold up a store)
#pragma unroll
  for (int e = 0; e < PARTS_C; ++e) {
    const int64_t col = col0 + (e * 64 + lane) % (TN * 2) * 8;
    if (p.bias != nullptr) {
      load_n<8>(p.bias + col, p.n - col, bias[e]);
    } else {
#pragma unroll
      for (int h = 0; h < 8; ++h) bias[e][h] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j) *reinterpret_cast<v4f*>(strip + r * PITCH + j * 16 + g * 4) = acc[i][j];
    wave_sync();  // (the strip's values go from lane to lane)
#pragma unroll
    for (int e = 0; e < PARTS_C; ++e) {
      const int at = (e * 64 + lane) / (TN * 2), c8 = (e * 64 + lane) % (TN * 2) * 8;
      if (TN % 2 != 0 && at >= 16) continue;
      float v[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v4f x = *reinterpret_cast<const v4f*>(strip + at * PITCH + c8 + h * 4);
#pragma unroll
        for (int l = 0; l < 4; ++l) v[4 * h + l] = x[l] + bias[e][4 * h + l];
      }
      const int64_t row = row0 + i * 16 + at, col = col0 + c8;
      if (row < p.m && col < p.n) {
        TC* to = c + row * p.ld_c + col;
        if (p.accumulate) {
          float old[8];
          load_n<8>(to, p.n - col, old);
#pragma unroll
          for (int h = 0; h < 8; ++h) v[h] += old[h];
        }
        store_n<8>(to, p.n - col, v);
      }
    }
    wave_sync();
  }
}

template <int WM, int WN, int TM, int TN, int STAGES, int KS, class TC>
__global__ void __launch_bounds__(64 * WM * WN * KS)
product_tile_kernel(Operands p, TC* c, int m_tiles, int n_tiles) {
  constexpr int WAVES = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, STAGE = (BM + BN) * ROW;
  constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;  // loads of a wave and stage: 8 rows each
  static_assert(LA * 8 * WAVES == BM && LB * 8 * WAVES == BN, "whole loads");
  constexpr int SL = (BM + BN + 63) / 64, SPW = (SL + WAVES - 1) / WAVES;  // scale words: 64 rows a load, waves in turn
  constexpr int SCALES = SL * 256;
  constexpr int GROUP = STAGES * STAGE + 2 * SCALES;  // LDS of a group: its stages, then two groups of scale words
  static_assert((KS - 1) * BM * BN * 4 <= KS * GROUP, "the sums fit over the stages");
  extern __shared__ uint8_t lds_all[];
  const int any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wave = any_wave % WAVES, group = any_wave / WAVES;
  uint8_t* lds = lds_all + group * GROUP;
  const int r = lane & 15, g = lane >> 4;

  int tile_m, tile_n;
  tile_of(m_tiles, n_tiles, tile_m, tile_n);
  const int64_t m0 = int64_t(tile_m) * BM, n0 = int64_t(tile_n) * BN;

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
  const uint8_t* scale_rows[SPW];  // this lane's row of scales for each load
#pragma unroll
  for (int i = 0; i < SPW; ++i) {
    const int row = (wave + i * WAVES) * 64 + lane;
    scale_rows[i] = row < BM ? p.sa + min(m0 + row, p.m - 1) * p.ld_sa : p.sb + min(n0 + row - BM, p.n - 1) * p.ld_sb;
  }

  // this group's blocks of 128: nk from block k0 on, the first of them number
  // k_odd of its scale word; every group meets at `steps` barriers
  const int blocks = int((p.k + 127) / 128);
  const int steps = (blocks + KS - 1) / KS;
  const int k0 = group * steps, nk = KS == 1 ? blocks : min(max(blocks - k0, 0), steps);
  const int k_odd = KS == 1 ? 0 : k0 % 4;
  base_a += int64_t(k0) * ROW, base_b += int64_t(k0) * ROW;

  const uint32_t lds0 = lds_address(lds);
  // the scale words (at a word's first stage) and part i of n of a stage's loads
  const auto fetch_scales = [&](int kb) {
    if ((k_odd + kb) % 4 == 0 || (KS > 1 && kb == 0)) {
#pragma unroll
      for (int i = 0; i < SPW; ++i) {
        const int part = wave + i * WAVES;
        if (part < SL) fetch4(scale_rows[i] + (k0 + kb) / 4 * 4, lds0 + STAGES * STAGE + ((k_odd + kb) / 4 % 2) * SCALES + part * 256);
      }
    }
  };
  const auto fetch = [&](int kb, int i, int n) {
    const uint32_t to = lds0 + (kb % STAGES) * STAGE;
#pragma unroll
    for (int l = (LA + LB) * i / n; l < (LA + LB) * (i + 1) / n; ++l) {
      if (l < LA)
        fetch16(base_a + int64_t(kb) * ROW, off_a[l], to + (wave * LA + l) * 1024);
      else
        fetch16(base_b + int64_t(kb) * ROW, off_b[l - LA], to + BM * ROW + (wave * LB + l - LA) * 1024);
    }
  };

  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  const int wm = wave / WN, wn = wave % WN;
  const int place = r * ROW + ((g ^ (r & 7)) << 4);  // chunk g of row r; chunk g + 4 lies at ^ 64
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < nk) fetch_scales(s), fetch(s, 0, 1);
  for (int kb = 0; kb < steps; ++kb) {
    // this stage's loads are done when only those of the STAGES - 2 later ones are left
    if (kb + STAGES - 2 < nk)
      wait_loads<(LA + LB) * (STAGES - 2)>();
    else
      wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    // The loads go over the stage that every wave has left, spread over the first
    // half of the products: in one go they would hold up the first reads of LDS.
    constexpr int PARTS = TM >= 4 ? TM / 2 : 1;
    const int ahead = kb + STAGES - 1;
    if (ahead < nk) {
      fetch_scales(ahead);
      if (PARTS == 1) fetch(ahead, 0, 1);
    }
    if (KS > 1 && kb >= nk) continue;
    const uint8_t* at_a = lds + (kb % STAGES) * STAGE + wm * TM * 16 * ROW;
    const uint8_t* at_b = lds + (kb % STAGES) * STAGE + BM * ROW + wn * TN * 16 * ROW;
    const int word = (k_odd + kb) / 4, byte = (k_odd + kb) % 4;
    const uint8_t* at_sa = lds + STAGES * STAGE + word % 2 * SCALES + (wm * TM * 16 + r) * 4 + byte;
    const uint8_t* at_sb = lds + STAGES * STAGE + word % 2 * SCALES + (BM + wn * TN * 16 + r) * 4 + byte;
    // A lane's 32 codes of a row are two halves of 16.  Products of a row tile go
    // with the widening of the next one, and in the first half with that of b's
    // second: a product takes the issue of four instructions, so that between two
    // of them others are free.  Codes are read a tile before they are widened.
    constexpr int Q = 2 * TM;  // (half, row tile) in turn
    v8b fa[2][2], fb[2][TN][2];
    v4i xa[2], xb;
    int ba[2], bb[TN];  // scale bytes of the codes read
    const auto read_a = [&](int q) {
      xa[q & 1] = *reinterpret_cast<const v4i*>(at_a + q % TM * 16 * ROW + (place ^ (q / TM * 64)));
      ba[q & 1] = at_sa[q % TM * 64];
    };
    const auto widen_a = [&](int q) {
      const float s = scale_value(ba[q & 1]);
      fa[q & 1][0] = widen(xa[q & 1][0], xa[q & 1][1], s), fa[q & 1][1] = widen(xa[q & 1][2], xa[q & 1][3], s);
    };
    const auto widen_b = [&](int h, int j, const v4i& x) {
      const float s = scale_value(bb[j]);
      fb[h][j][0] = widen(x[0], x[1], s), fb[h][j][1] = widen(x[2], x[3], s);
    };
    const auto read_b = [&](int h, int j) {
      return *reinterpret_cast<const v4i*>(at_b + j * 16 * ROW + (place ^ (h * 64)));
    };
    {
      v4i x[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) x[j] = read_b(0, j), bb[j] = at_sb[j * 64];
      read_a(0);
      read_a(1);
#pragma unroll
      for (int j = 0; j < TN; ++j) widen_b(0, j, x[j]);
      widen_a(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    // b's second half: tile j is read at step first_b[j] and widened at the next
    constexpr int STEP_B = TM >= TN + 1 ? 1 : 0;  // a tile a step, or all of them in the last step of the first half
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int h = q / TM, i = q % TM;
      v4i late[TN];
      if (STEP_B == 1 && h == 0 && i >= 1 && i <= TN) widen_b(1, i - 1, xb);
      if (STEP_B == 1 && h == 0 && i < TN) xb = read_b(1, i);
      if (STEP_B == 0 && q == TM - 1) {
#pragma unroll
        for (int j = 0; j < TN; ++j) late[j] = read_b(1, j);
      }
      if (q + 1 < Q) widen_a(q + 1);
      if (q + 2 < Q) read_a(q + 2);  // (over the codes of tile q)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[h][j][e], fa[q & 1][e], acc[i][j], 0, 0, 0);
      if (STEP_B == 0 && q == TM - 1) {
#pragma unroll
        for (int j = 0; j < TN; ++j) widen_b(1, j, late[j]);
      }
      // one product, then up to three of the others
#pragma unroll
      for (int e = 0; e < 2 * TN; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (PARTS > 1 && h == 0 && i < PARTS && ahead < nk) fetch(ahead, i, PARTS);
    }
  }
  __syncthreads();
  if constexpr (KS > 1) {
    v4f* sums = reinterpret_cast<v4f*>(lds_all) + wave * 64 + lane;  // (group - 1, tile, wave, lane)
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) sums[(((group - 1) * TM + i) * TN + j) * WAVES * 64] = acc[i][j];
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < KS - 1; ++k)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] += sums[((k * TM + i) * TN + j) * WAVES * 64];
  }
  static_assert((KS - 1) * BM * BN * 4 + WAVES * strip_floats(TN) * 4 <= KS * GROUP, "the strips fit beside the sums");
  put_tiles<TM, TN>(p, c, acc, m0 + wm * TM * 16, n0 + wn * TN * 16, lane,
                    reinterpret_cast<float*>(lds_all + (KS - 1) * BM * BN * 4) + wave * strip_floats(TN));
}

// Raises a kernel's limit of dynamic LDS on the current device, once (the call
// takes as long as a launch).
hipError_t allow_lds(const void* fn, size_t bytes, std::atomic<uint64_t>& done) {
  if (bytes <= 65536) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <int WM, int WN, int TM, int TN, int STAGES, int KS, class TC>
int launch_tile(const Operands& p, void* c, hipStream_t s) {
  constexpr int BM = WM * TM * 16, BN = WN * TN * 16;
  const int64_t mt = (p.m + BM - 1) / BM, nt = (p.n + BN - 1) / BN;
  constexpr size_t lds = KS * (size_t(STAGES) * (BM + BN) * ROW + 2 * ((BM + BN + 63) / 64 * 256));
  auto* fn = product_tile_kernel<WM, WN, TM, TN, STAGES, KS, TC>;
  static std::atomic<uint64_t> allowed{0};  // devices whose limit for this kernel is raised (one bit each, 64 of them)
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(fn), lds, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(fn, dim3(unsigned(mt * nt)), dim3(64 * WM * WN * KS), lds, s, p, static_cast<TC*>(c), int(mt), int(nt));
  return hipGetLastError();
}

// The tile.  A card of 256 CUs is short of workgroups long before it is short of
// products, so small results take the smallest tile that still leaves one
// workgroup a CU, its waves dividing the summed axis (KS).  Measured, in us:
//                        16 x 32  32 x 32  64 x 32  64 x 64  128 x 64  128 x 128    without KS
//   4 x 4608 x 2048          4.1      4.6      5.8      8.2
//   48 x 4608 x 2048         7.2      8.5      6.3      7.8
//   512 x 512 x 8192        15.0     10.9     15.8     21.4
//   4096 x 64 x 2048         7.0      5.0      6.2      8.0
//   1024 x 1024 x 8192                        30.7     22.6      33.3
//   1900 x 1000 x 2048                                 16.6      13.6       18.6          18.4
//   1400 x 1400 x 8192                                 44.0      38.5       54.7          59.1
//   2048 x 2048 x 2048                                           25.3       21.5          23.9
//   2048 x 2048 x 512                                                       11.3          10.4
// (64 x 64 by two waves, each all of a's rows: four of 32 x 32, which widen more,
// take 3% longer, one that widens least 25%, and fewer groups of more stages 2 to 8%.)
// Larger ones take the tile whose rounds of workgroups over the card cost least,
// at the rates that full rounds reach (at_once: workgroups that the card holds;
// where a CU holds two, the last round of a few overlaps the one before).  Every
// wave widens the rows that it reads, which large tiles do least:
//                        128 x 64  128 x 128  128 x 192  128 x 256  192 x 192  192 x 256  256 x 256
//   2048 x 2048 x 2048       23.6       26.3                  31.0
//   4096 x 1536 x 2048       36.6       35.6       29.0       34.1       35.8
//   4096 x 2048 x 4608       88.5       72.9                  65.4       69.0       78.4
//   4608 x 2048 x 4096       95.9       93.2       86.2                             71.2       88.6
//   8192 x 8192 x 8192                   956                   893        907        847        759
struct Tile {
  int64_t bm, bn, at_once;
  double rate;  // TFLOP/s of full rounds
};

double cost(const Operands& p, const Tile& t) {
  const int64_t tiles = ((p.m + t.bm - 1) / t.bm) * ((p.n + t.bn - 1) / t.bn);
  const double whole = double((tiles + t.at_once - 1) / t.at_once), part = double(tiles) / double(t.at_once);
  const double rounds = t.at_once > 256 && tiles > t.at_once ? (whole + part) / 2 : whole;
  return rounds * double(t.at_once * t.bm * t.bn) / t.rate;
}

template <class TC>
int launch(const Operands& p, void* c, hipStream_t s) {
  const auto tiles = [&](int64_t bm, int64_t bn) { return ((p.m + bm - 1) / bm) * ((p.n + bn - 1) / bn); };
  if (tiles(16, 32) <= 256) return launch_tile<1, 1, 1, 2, 3, 8, TC>(p, c, s);
  if (tiles(32, 32) <= 256) return launch_tile<1, 1, 2, 2, 2, 8, TC>(p, c, s);
  if (tiles(64, 32) <= 256) return launch_tile<2, 1, 2, 2, 3, 4, TC>(p, c, s);
  if (tiles(64, 64) <= 256) return launch_tile<1, 2, 4, 2, 2, 4, TC>(p, c, s);
  if (tiles(128, 64) <= 256) return launch_tile<2, 2, 4, 2, 2, 2, TC>(p, c, s);
  if (tiles(128, 128) <= 256 && p.k >= 1024) return launch_tile<2, 2, 4, 4, 2, 2, TC>(p, c, s);
  const Tile forms[] = {{128, 64, 512, 800},   {128, 128, 512, 1080}, {128, 192, 256, 1050}, {128, 256, 256, 1200},
                        {192, 192, 256, 1180}, {192, 256, 256, 1340}, {256, 256, 256, 1450}};
  int best = 0;
  for (int i = 1; i < 7; ++i)
    if (cost(p, forms[i]) < cost(p, forms[best])) best = i;
  switch (best) {
    case 0: return launch_tile<2, 2, 4, 2, 3, 1, TC>(p, c, s);
    case 1: return launch_tile<2, 2, 4, 4, 2, 1, TC>(p, c, s);
    case 2: return launch_tile<2, 4, 4, 3, 2, 1, TC>(p, c, s);
    case 3: return launch_tile<2, 4, 4, 4, 2, 1, TC>(p, c, s);
    case 4: return launch_tile<2, 4, 6, 3, 2, 1, TC>(p, c, s);
    case 5: return launch_tile<2, 4, 6, 4, 2, 1, TC>(p, c, s);
    default: return launch_tile<2, 4, 8, 4, 2, 1, TC>(p, c, s);
  }
}

}  // namespace

int launch_product(const dtst_product_desc& d, const void* a, const void* a_scale, const void* b, const void* b_scale,
                   const float* bias, void* c, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const Operands p{static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(b),
                   static_cast<const uint8_t*>(a_scale), static_cast<const uint8_t*>(b_scale),
                   d.m, d.n, d.k, d.ld_a, d.ld_a_scale, d.ld_b, d.ld_b_scale, d.ld_c, bias, d.accumulate};
  if (d.c_type == DTST_F32) return launch<float>(p, c, s);
  if (d.c_type == DTST_BF16) return launch<bf16_t>(p, c, s);
  return launch<f16_t>(p, c, s);
}

}  // namespace dtst
