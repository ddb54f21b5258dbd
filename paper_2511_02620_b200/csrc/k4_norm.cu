// Final root-mean-square norm with the residual's addition:
//
//   r = round(x + residual)                       (the residual stream, rounded to the inputs' type)
//   y = r / sqrt(mean(r^2) + eps) * weight        (fp32; the mean over the row's d elements)
//   h = bf16(y)  and / or  codes, scales = microscaled(y)
//
// A row stays in registers between the sum of its squares and the scaling, so every element is read once and every
// result written once: the kernel is bound by those bytes.  One row belongs to a group of whole warps (a thread holds
// 8 * VPT elements, 16 bytes of bf16 at a time); short rows share a CTA.  The sum runs in fp32 in a fixed order
// (per thread, shuffles, warps in order), so results do not depend on the launch.  y is rounded once, whatever asks
// for it: the microscaled codes are taken from the fp32 value, not from h.
#include <cuda_runtime.h>

#include "mx_device.cuh"
#include "mx_kernels.h"

namespace difr {

constexpr int kNormMaxThreads = 1024;

// Sum over the threads of a row, the same value in all of them.  `part`: one float per warp of the CTA.
__device__ __forceinline__ float row_sum(float v, float* part, int first_warp, int warps) {
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  if (warps == 1) return v;
  __syncthreads();  // (the array may still be read for an earlier sum)
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
  for (int i = 0; i < warps; ++i) s += part[first_warp + i];
  return s;
}

template <typename X, int VPT>
__global__ void __launch_bounds__(VPT == 1 ? 512 : kNormMaxThreads) rms_norm(const NormParams p) {
  __shared__ float part[kNormMaxThreads / 32];
  const int tpr = p.threads_per_row;
  const int in_cta = threadIdx.x / tpr;  // (tpr is a multiple of 32: uniform over a warp)
  const int t = threadIdx.x - in_cta * tpr;
  const int64_t row = (int64_t)blockIdx.x * p.rows_per_cta + in_cta;
  const bool live = row < p.T;
  const X* x = static_cast<const X*>(p.x) + (live ? row * p.ldx : 0);
  const X* res = static_cast<const X*>(p.residual) + (live && p.residual ? row * p.ld_residual : 0);

  float v[VPT][8];
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int e0 = (j * tpr + t) * 8;
    const int d = live ? p.d : 0;
    load8<X>(x, e0, d, p.vec_x, v[j]);
  }
  if (p.residual != nullptr) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int e0 = (j * tpr + t) * 8;
      float r[8];
      load8<X>(res, e0, live ? p.d : 0, p.vec_residual, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = to_float<X>(from_float<X>(v[j][i] + r[i]));
      if (p.residual_out != nullptr && live)
        store8<X>(static_cast<X*>(p.residual_out) + row * p.ld_residual_out, e0, p.d, p.vec_residual_out, v[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(v[j][i], v[j][i], ss);
  const int first_warp = in_cta * (tpr >> 5);
  ss = row_sum(ss, part, first_warp, tpr >> 5);
  float pre = 1.f, rstd;
  // Squares of values above 1.8e19 leave fp32's range: such a row is measured again in units of 2^80.  (A row with a NaN
  // is NaN throughout, one with an infinity is NaN there and zero elsewhere, as the formula has it.)  The vote keeps the barriers of row_sum uniform.
  const bool over = ss > 3.0e38f;
  rstd = 1.f / sqrtf(ss / (float)p.d + p.eps);
  if (__syncthreads_or(over)) {
    float s2 = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = v[j][i] * 0x1p-80f;
        s2 = fmaf(a, a, s2);
      }
    s2 = row_sum(s2, part, first_warp, tpr >> 5);
    if (over) {
      pre = 0x1p-80f;
      rstd = 1.f / sqrtf(s2 / (float)p.d);
    }
  }
  if (!live) return;  // whole warps; no barrier follows

  const X* w = static_cast<const X*>(p.weight);
  __nv_bfloat16* h = static_cast<__nv_bfloat16*>(p.h);
  const int64_t words = mx_words(p.d);
  const int nvec = p.fmt ? (int)mx_blocks(p.d) * 4 : (p.d + 7) / 8;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int vec = j * tpr + t, e0 = vec * 8;
    float g[8];
    load8<X>(w, e0, p.d, p.vec_weight, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] * pre * rstd * g[i];
    if (h != nullptr && e0 < p.d) store8<__nv_bfloat16>(h + row * p.ldh, e0, p.d, p.vec_h, v[j]);
    if (p.fmt != 0) {
      // elements past the row must be zeros, not 0 * infinity
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e0 + i >= p.d) v[j][i] = 0.f;
      uint32_t c[2];
      uint32_t word;
      const bool past = vec >= nvec;
      if (p.fmt == kMx8) {
        word = mx_quantize8<kMx8>(v[j], past, c);
        if (!past) *reinterpret_cast<uint2*>(p.codes + row * mx_pitch_bytes(kMx8, p.d) + e0) = make_uint2(c[0], c[1]);
      } else {
        word = mx_quantize8<kMx4>(v[j], past, c);
        if (!past) *reinterpret_cast<uint32_t*>(p.codes + row * mx_pitch_bytes(kMx4, p.d) + (e0 >> 1)) = c[0];
      }
      if ((t & 15) == 0 && vec < nvec)
        *reinterpret_cast<uint32_t*>(p.scales + mx_scale_offset(row, vec >> 4, words)) = word;
    }
  }
}

template <typename X>
static cudaError_t launch_typed(NormParams p, cudaStream_t stream) {
  // threads per row: whole warps that cover the row (to whole blocks of 32 elements) at VPT vectors each
  const int nvec = (p.d + 31) / 32 * 4;
  int vpt = nvec <= 512 ? 1 : nvec <= 2048 ? 2 : 4;
  p.threads_per_row = ((nvec + vpt - 1) / vpt + 31) / 32 * 32;
  p.rows_per_cta = p.threads_per_row >= 256 ? 1 : 256 / p.threads_per_row;
  if (p.T < p.rows_per_cta) p.rows_per_cta = (int)p.T;
  const int64_t grid = (p.T + p.rows_per_cta - 1) / p.rows_per_cta;
  const int threads = p.threads_per_row * p.rows_per_cta;
  if (vpt == 1)
    rms_norm<X, 1><<<(unsigned)grid, threads, 0, stream>>>(p);
  else if (vpt == 2)
    rms_norm<X, 2><<<(unsigned)grid, threads, 0, stream>>>(p);
  else
    rms_norm<X, 4><<<(unsigned)grid, threads, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_rms_norm(const NormParams& p, int dtype, cudaStream_t stream) {
  switch (dtype) {
    case kBf16: return launch_typed<__nv_bfloat16>(p, stream);
    case kF16: return launch_typed<__half>(p, stream);
    default: return launch_typed<float>(p, stream);
  }
}

}  // namespace difr
