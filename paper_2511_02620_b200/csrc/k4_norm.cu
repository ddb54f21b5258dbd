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
#include "norm_device.cuh"

namespace difr {

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
  auto squares = [&](float unit) { return row_squares<X, VPT>(v, unit); };
  const float2 f = row_scale(row_sum(squares(1.f), part[0], warps), p.inv_d, p.eps,
                             [&](float unit) { return row_sum(squares(unit), part[1], warps); });

  emit_norm<X, VPT, FMT, AL, false>(p, v, f, row, t, tpr, stage);
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
