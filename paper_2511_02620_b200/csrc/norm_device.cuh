// What the norms share: sums over a row, its factor, and the way from a row in registers to h and codes.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "mx_device.cuh"
#include "mx_kernels.h"

namespace difr {

constexpr int kNormMaxThreads = 512;

// Sum over the threads of a row, the same value in all of them.  A row of more than one warp has the CTA to itself.
// Eight terms at a time are added in fp32 (five roundings at most), their sums in fp64, where nothing more is lost: values
// next to a border of the 4-bit format depend on the sum's last bits.
__device__ __forceinline__ float row_sum(double v, double* part, int warps) {
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) v += shfl_xor_double(v, m);
  if (warps == 1) return (float)v;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < warps; ++i) s += part[i];
  return (float)s;
}

// 1 / sqrt(mean + eps) and a factor to apply first.  Squares of values above 1.8e19 leave fp32's range, those of values
// below 1.1e-19 its normal numbers, which shows where eps is smaller still: such a row is measured by `again` in units of
// 2^80 or 2^-80, eps with it.  Where eps alone takes the sum out of range, a quarter of both stays inside.  A row with a
// NaN is NaN throughout; one with an infinity is NaN there and zero elsewhere, as the formula has it.
template <typename F>
__device__ __forceinline__ float2 row_scale(float ss, float inv_d, float eps, F again) {
  const float mean = __fmul_rn(ss, inv_d);  // (a value of its own: no fma)
  const float m = __fadd_rn(mean, eps);
  const bool huge = ss > 3.0e38f;
  if (huge || m < 0x1p-100f) {
    const float unit = huge ? 0x1p-80f : 0x1p80f;
    const float root = rsqrtf(__fadd_rn(__fmul_rn(again(unit), inv_d), eps * unit * unit));
    // (half of the unit each: small values of a huge row stay normal numbers as long as their y is one)
    const float part = huge ? 0x1p-40f : 0x1p40f;
    return make_float2(part, part * root);
  }
  if (m > 3.0e38f) return make_float2(1.f, 0.5f * rsqrtf(__fadd_rn(0.25f * mean, 0.25f * eps)));
  return make_float2(1.f, rsqrtf(m));
}

// Sum over a thread's part of a row of the squares of its values times `unit`.
template <typename X, int VPT>
__device__ __forceinline__ double row_squares(const Vec8<X> (&v)[VPT], float unit) {
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    float2 a = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 e = unit == 1.f ? v[j].pair(i) : fmul2(v[j].pair(i), make_float2(unit, unit));
      a = ffma2(e, e, a);
    }
    sum += (double)(a.x + a.y);
  }
  return sum;
}

// y = v f weight of a row in registers (thread t of tpr holds the vectors j tpr + t), to h and / or codes and scales.
// OFFSET: p.weight_offset is added to the weights.
template <typename X, int VPT, int FMT, bool AL, bool OFFSET, typename P>
__device__ __forceinline__ void emit_norm(const P& p, const Vec8<X> (&v)[VPT], float2 f, int64_t row, int t, int tpr, X* stage) {
  const X* w = static_cast<const X*>(p.weight);
  __nv_bfloat16* h = static_cast<__nv_bfloat16*>(p.h) + row * p.ldh;
  const int nvec_mx = FMT ? (int)mx_blocks(p.d) * 4 : 0;
  unsigned char* scales = p.scales + (FMT ? mx_scale_offset(row, 0, mx_words(p.d)) : 0);
  unsigned char* codes = p.codes + (FMT ? row * mx_pitch_bytes(FMT, p.d) : 0);
  const bool rescaled = f.x != 1.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = j * tpr + t;
    Vec8<X> g[1];
    RowVectors<X, 1, AL> fg;
    fetch_row(fg, w, i, 0, p.d);
    finish_row(g, fg, w, i, 0, p.d, stage);
    float2 y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float2 a = v[j].pair(k);
      if (rescaled) a = fmul2(a, make_float2(f.x, f.x));
      float2 gain = g[0].pair(k);
      if constexpr (OFFSET) gain = fadd2(gain, make_float2(p.weight_offset, p.weight_offset));
      y[k] = fmul2(fmul2(a, make_float2(f.y, f.y)), gain);
    }
    if (p.h != nullptr) {
      Vec8<__nv_bfloat16> o;
#pragma unroll
      for (int k = 0; k < 4; ++k) o.set_pair(k, y[k]);
      store_row<__nv_bfloat16, AL>(o, h, i, p.d, reinterpret_cast<__nv_bfloat16*>(stage));
    }
    if constexpr (FMT != 0) {
      const bool past = i >= nvec_mx;
      // (the columns behind the row are zeros: values and weights were filled with them)
      uint32_t c[2];
      const uint32_t word = mx_quantize8<FMT>(y, past, c);
      if (!past) {
        if (FMT == kMx8)
          *reinterpret_cast<uint2*>(codes + i * 8) = make_uint2(c[0], c[1]);
        else
          *reinterpret_cast<uint32_t*>(codes + i * 4) = c[0];
        if ((t & 15) == 0) *reinterpret_cast<uint32_t*>(scales + (i >> 4) * kSfWordBytes) = word;
      }
    }
  }
}

}  // namespace difr
