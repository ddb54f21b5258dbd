// Final root-mean-square norm with the residual's addition:
//
//   r = round(x + residual)                       (the residual stream, rounded to the inputs' type)
//   y = r / sqrt(mean(r^2) + eps) * weight        (fp32; the mean over the row's d elements)
//   h = bf16(y)  and / or  codes, scales = microscaled(y)
//
// A row stays in registers between the sum of its squares and the scaling, so every element is read once and every
// result written once: the kernel is bound by those bytes, as long as it spends few instructions per element (elements
// are kept as they lie in memory, 8 per load, and worked on in pairs).  A row belongs to a group of whole warps.  Of the
// rows off the 16-byte boundaries (odd d, odd strides) 16-bit ones on 8 or 4 bytes are read, on 8 bytes written, directly in
// such pieces; the others are turned through shared memory.  The sum runs in a fixed order (per thread, shuffles, warps
// in order) that d, the type and whether all rows lie on 16-byte boundaries fix, not the batch.  y is rounded once,
// whatever asks for it: the codes are taken from the fp32 value, not from h.
// Measured in bf16 with residual, stream and h: 65536 x 2048 161 us, 6.7 TB/s of necessary bytes (238 us while an element
// cost 45 instructions); 8192 x 5120 56 us; to 8 bits without h 52 us.
#include <cuda_runtime.h>

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

// Rounded sum of two vectors.
template <typename X>
__device__ __forceinline__ void add_rounded(Vec8<X>& a, const Vec8<X>& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a.set_pair(i, fadd2(a.pair(i), b.pair(i)));
}

// Threads that an SM holds: as many as registers for VPT vectors allow.  Short rows without codes (one vector a thread, d up
// to 256) need all 2048 to have enough loads in flight: 2^20 rows of 128 in bf16 172 us at 32 registers, 195 at 38.
constexpr int norm_min_ctas(int vpt, int fmt, bool al) { return vpt == 8 ? 1 : vpt == 1 && fmt == 0 && al ? 4 : 2; }

template <typename X, int VPT, bool RES, int FMT, bool AL>
__global__ void __launch_bounds__(kNormMaxThreads, norm_min_ctas(VPT, FMT, AL)) rms_norm(const NormParams p) {
  __shared__ double part[2][kNormMaxThreads / 32];
  __shared__ uint4 stage_all[AL ? 1 : kNormMaxThreads * sizeof(X) / 2];  // 256 elements per warp
  X* stage = reinterpret_cast<X*>(stage_all) + (AL ? 0 : (threadIdx.x >> 5) * 256);
  const int tpr = p.threads_per_row, warps = tpr >> 5;
  const int in_cta = p.rows_per_cta == 1 ? 0 : (int)threadIdx.x >> 5;  // short rows: one warp each
  const int t = p.rows_per_cta == 1 ? (int)threadIdx.x : (int)threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * p.rows_per_cta + in_cta;
  if (row >= p.T) return;  // only where a row is a warp: no barrier is missed

  const X* x = static_cast<const X*>(p.x) + row * p.ldx;
  const X* res = static_cast<const X*>(p.residual) + row * p.ld_residual;
  Vec8<X> v[VPT];
  {
    RowVectors<X, VPT, AL> fx, fr;
    fetch_row(fx, x, t, tpr, p.d);
    if (RES) fetch_row(fr, res, t, tpr, p.d);
    finish_row(v, fx, x, t, tpr, p.d, stage);
    if (RES) {
      Vec8<X> r[VPT];
      finish_row(r, fr, res, t, tpr, p.d, stage);
      X* to = static_cast<X*>(p.residual_out) + row * p.ld_residual_out;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        add_rounded<X>(v[j], r[j]);
        if (p.residual_out != nullptr) store_row<X, AL>(v[j], to, j * tpr + t, p.d, stage);
      }
    }
  }
  auto squares = [&](float unit) {
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
  };
  const float2 f = row_scale(row_sum(squares(1.f), part[0], warps), p.inv_d, p.eps,
                             [&](float unit) { return row_sum(squares(unit), part[1], warps); });

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
      y[k] = fmul2(fmul2(a, make_float2(f.y, f.y)), g[0].pair(k));
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

template <typename X, int VPT, bool RES, bool AL>
static void launch_format(const NormParams& p, unsigned grid, int threads, cudaStream_t stream) {
  if (p.fmt == kMx8)
    rms_norm<X, VPT, RES, kMx8, AL><<<grid, threads, 0, stream>>>(p);
  else if (p.fmt == kMx4)
    rms_norm<X, VPT, RES, kMx4, AL><<<grid, threads, 0, stream>>>(p);
  else
    rms_norm<X, VPT, RES, 0, AL><<<grid, threads, 0, stream>>>(p);
}
template <typename X, int VPT>
static void launch_vec(const NormParams& p, unsigned grid, int threads, cudaStream_t stream) {
  if (p.vec) {
    if (p.residual != nullptr)
      launch_format<X, VPT, true, true>(p, grid, threads, stream);
    else
      launch_format<X, VPT, false, true>(p, grid, threads, stream);
  } else {
    if (p.residual != nullptr)
      launch_format<X, VPT, true, false>(p, grid, threads, stream);
    else
      launch_format<X, VPT, false, false>(p, grid, threads, stream);
  }
}

template <typename X>
static cudaError_t launch_typed(NormParams p, cudaStream_t stream) {
  // Vectors per thread, whatever the number of rows, so that a row's result does not depend on its batch: four (fp32: two,
  // the same registers), for more loads in flight and fewer barriers per byte: T = 16384, d = 4096 in bf16 took 45.9 us
  // at four, 48.3 at two, 47.3 at eight.  Rows off the 16-byte boundaries need the registers for their pieces: one.
  const int nvec = (p.d + 127) / 128 * 16;  // to whole scale words
  int vpt = !p.vec ? 1 : sizeof(X) == 4 ? 2 : 4;
  while (vpt > 1 && nvec <= 32 * vpt / 2) vpt /= 2;
  while ((nvec + vpt - 1) / vpt > kNormMaxThreads) vpt *= 2;
  p.threads_per_row = ((nvec + vpt - 1) / vpt + 31) / 32 * 32;
  p.rows_per_cta = p.threads_per_row == 32 ? 4 : 1;
  const unsigned grid = (unsigned)((p.T + p.rows_per_cta - 1) / p.rows_per_cta);
  const int threads = p.threads_per_row * p.rows_per_cta;
  if (vpt == 1)
    launch_vec<X, 1>(p, grid, threads, stream);
  else if (vpt == 2)
    launch_vec<X, 2>(p, grid, threads, stream);
  else if (vpt == 4)
    launch_vec<X, 4>(p, grid, threads, stream);
  else
    launch_vec<X, 8>(p, grid, threads, stream);
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
