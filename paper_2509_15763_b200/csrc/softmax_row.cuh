// The softmax of one 128-column score row held in a thread's registers, as the tcgen05 attention kernels take it: a thread owns a
// query row, reads its scores of a key tile from tensor memory and writes the weights back as bf16.
#pragma once
#include "sm100_ptx.cuh"

namespace ug {
namespace {

using namespace sm100;

constexpr int kCols = 128;  // score columns per thread and tile

// kNan: a NaN among them is the maximum.
template <bool kNan = false>
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  if constexpr (kNan)
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  else
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <bool kNan = false>
__device__ __forceinline__ float max2(float a, float b) {
  return kNan ? max3<true>(a, b, b) : fmaxf(a, b);
}

// Bit e of the result: column 32 * c + e lies inside [lo, hi].
__device__ __forceinline__ uint32_t chunk_mask(int lo, int hi, int c) {
  const int a = max(lo - 32 * c, 0), b = min(hi - 32 * c, 31);
  return a > b ? 0u : ((0xffffffffu >> (31 - b)) & (0xffffffffu << a));
}

// Hidden columns (outside [lo, hi]) of a row of raw scores become -inf.
__device__ __forceinline__ void mask_row(uint32_t (&sc)[kCols], int lo, int hi) {
#pragma unroll
  for (int c = 0; c < kCols / 32; ++c) {
    const uint32_t bits = chunk_mask(lo, hi, c);
#pragma unroll
    for (int e = 0; e < 32; ++e) sc[c * 32 + e] = (bits >> e) & 1u ? sc[c * 32 + e] : 0xff800000u;
  }
}

// Row maximum of the raw scores of one tile.
template <bool kNan = false>
__device__ __forceinline__ float row_max(const uint32_t (&sc)[kCols]) {
  float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
  for (int e = 0; e < kCols; e += 8) {
    m0 = max3<kNan>(m0, __uint_as_float(sc[e]), __uint_as_float(sc[e + 1]));
    m1 = max3<kNan>(m1, __uint_as_float(sc[e + 2]), __uint_as_float(sc[e + 3]));
    m2 = max3<kNan>(m2, __uint_as_float(sc[e + 4]), __uint_as_float(sc[e + 5]));
    m3 = max3<kNan>(m3, __uint_as_float(sc[e + 6]), __uint_as_float(sc[e + 7]));
  }
  return max2<kNan>(max2<kNan>(m0, m1), max2<kNan>(m2, m3));
}

// Half a pass over a row of raw scores (columns 64 * kHalf .. + 63): p = 2^(s * scale_log2 - m) written to
// TMEM as bf16 pairs; returns the sum of the half row.  The first half also leaves the maximum raw score of
// the WHOLE row in mx, so that the caller knows whether m still serves before it hands any of P over.
// m must be finite; a score of -inf gives p = 0 (or about 2^-126 where the exponential is taken on the FMA
// pipe).  The special-function unit (16 exponentials per clock and SM) bounds this loop, so kEmuNum of every
// kEmuDen column pairs go to the FMA pipe (ex2_fma2) and the maximum rides along on the ALU pipe.
constexpr int kEmuNum = 2, kEmuDen = 8;
template <int kHalf, bool kNan = false>
__device__ __forceinline__ float row_exp(const uint32_t (&sc)[kCols], uint32_t t_p, float scale_log2, float m, float& mx) {
  uint64_t l01 = f32x2(0.f, 0.f), l23 = l01;
  const uint64_t scale2 = f32x2(scale_log2, scale_log2), negm2 = f32x2(-m, -m);
  float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
  for (int c = kHalf * (kCols / 64); c < (kHalf + 1) * (kCols / 64); ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const int i0 = c * 32 + e;
      float x[4];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int pair = i0 / 2 + q;
        f32x2_split(fma2(f32x2(__uint_as_float(sc[i0 + 2 * q]), __uint_as_float(sc[i0 + 2 * q + 1])), scale2, negm2),
                    x[2 * q], x[2 * q + 1]);
        if ((pair * kEmuNum) % kEmuDen < kEmuNum) {
          ex2_fma2(x[2 * q], x[2 * q + 1]);
        } else {
          x[2 * q] = ex2(x[2 * q]);
          x[2 * q + 1] = ex2(x[2 * q + 1]);
        }
      }
      if (kHalf == 0) {  // the maximum of both halves: 8 columns per 4 exponentials
        const int j0 = 2 * i0;
        m0 = max3<kNan>(m0, __uint_as_float(sc[j0]), __uint_as_float(sc[j0 + 1]));
        m1 = max3<kNan>(m1, __uint_as_float(sc[j0 + 2]), __uint_as_float(sc[j0 + 3]));
        m0 = max3<kNan>(m0, __uint_as_float(sc[j0 + 4]), __uint_as_float(sc[j0 + 5]));
        m1 = max3<kNan>(m1, __uint_as_float(sc[j0 + 6]), __uint_as_float(sc[j0 + 7]));
      }
      l01 = add2(l01, f32x2(x[0], x[1]));
      l23 = add2(l23, f32x2(x[2], x[3]));
      pk[e / 2] = pack_bf16(x[0], x[1]);
      pk[e / 2 + 1] = pack_bf16(x[2], x[3]);
    }
    tmem_st(t_p + c * 16, pk);
  }
  if (kHalf == 0) mx = max2<kNan>(m0, m1);
  float l0, l1, l2, l3;
  f32x2_split(l01, l0, l1);
  f32x2_split(l23, l2, l3);
  return (l0 + l1) + (l2 + l3);
}

}  // namespace
}  // namespace ug
