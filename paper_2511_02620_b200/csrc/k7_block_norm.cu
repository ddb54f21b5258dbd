// The norms before and after a block, with its gate and residual scale:
//
//   n = x / sqrt(mean(x^2) + post_eps) * (post_weight + offset)     (n = x without post_weight)
//   r = round(beta * residual + alpha * (gate * n))                 (the residual stream, rounded to the inputs' type)
//   y = r / sqrt(mean(r^2) + eps) * (weight + offset)
//   h = bf16(y)  and / or  codes, scales = microscaled(y)
//
// One pass over the row, as in the final norm: x stays in registers as it lies in memory, becomes r there, and r stays for
// the second norm.  The residual and a gate are loaded together with x, so that their bytes are in flight while the first
// sum is taken.  Bound by its bytes: 65536 x 2048 in bf16 with a gate per channel 204 to 215 us (166 of bytes).  Sums, their order and
// the handling of rows at the ends of fp32 are the final norm's.
#include <cuda_runtime.h>

#include "mx_device.cuh"
#include "mx_kernels.h"
#include "norm_device.cuh"
#include "step_kernels.h"

namespace difr {

// A thread holds VPT vectors of x, of the residual and of the gate.  Two (fp32: one) and at most 64 registers a thread: 65536 x
// 2048 in bf16 with a gate per channel took 206 us, 219 without the limit, 224 at four vectors, 266 at one.
template <typename X, int VPT, int FMT, bool GATE, bool AL>
__global__ void __launch_bounds__(kNormMaxThreads, VPT <= 2 ? 2 : 1) block_norm(const BlockNormParams p) {
  __shared__ double part[4][kNormMaxThreads / 32];
  __shared__ uint4 stage_all[AL ? 1 : kNormMaxThreads * sizeof(X) / 2];  // 256 elements per warp
  X* stage = reinterpret_cast<X*>(stage_all) + (AL ? 0 : (threadIdx.x >> 5) * 256);
  const int tpr = p.threads_per_row, warps = tpr >> 5;
  const int in_cta = p.rows_per_cta == 1 ? 0 : (int)threadIdx.x >> 5;  // short rows: one warp each
  const int t = p.rows_per_cta == 1 ? (int)threadIdx.x : (int)threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * p.rows_per_cta + in_cta;
  if (row >= p.T) return;  // only where a row is a warp: no barrier is missed

  const X* x = static_cast<const X*>(p.x) + row * p.ldx;
  const X* res = static_cast<const X*>(p.residual) + row * p.ld_residual;
  const X* gate = static_cast<const X*>(p.gate) + row * p.ld_gate;
  const X* post = static_cast<const X*>(p.post_weight);
  Vec8<X> v[VPT];
  {
    RowVectors<X, VPT, AL> fx, fr;
    RowVectors<X, GATE ? VPT : 1, AL> fg;
    fetch_row(fx, x, t, tpr, p.d);
    fetch_row(fr, res, t, tpr, p.d);
    if (GATE) fetch_row(fg, gate, t, tpr, p.d);
    finish_row(v, fx, x, t, tpr, p.d, stage);
    float2 f = make_float2(1.f, 1.f);
    if (post != nullptr)
      f = row_scale(row_sum(row_squares<X, VPT>(v, 1.f), part[0], warps), p.inv_d, p.post_eps,
                    [&](float unit) { return row_sum(row_squares<X, VPT>(v, unit), part[1], warps); });
    Vec8<X> r[VPT], g[GATE ? VPT : 1];
    finish_row(r, fr, res, t, tpr, p.d, stage);
    if (GATE) finish_row(g, fg, gate, t, tpr, p.d, stage);
    X* to = static_cast<X*>(p.residual_out) + row * p.ld_residual_out;
    const float2 beta = make_float2(p.beta, p.beta);
    const float2 alpha = make_float2(p.alpha, p.alpha);
    const float2 offset = make_float2(p.weight_offset, p.weight_offset);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      Vec8<X> w[1];
      if (post != nullptr) {
        RowVectors<X, 1, AL> fw;
        fetch_row(fw, post, j * tpr + t, 0, p.d);
        finish_row(w, fw, post, j * tpr + t, 0, p.d, stage);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float2 a = v[j].pair(i);
        if (post != nullptr) {
          if (f.x != 1.f) a = fmul2(a, make_float2(f.x, f.x));
          a = fmul2(fmul2(a, make_float2(f.y, f.y)), fadd2(w[0].pair(i), offset));
        }
        if (GATE) a = fmul2(a, g[j].pair(i));
        // (alpha last, as the formula has it: its product with the root or with x may leave fp32 where n does not)
        v[j].set_pair(i, ffma2(beta, r[j].pair(i), fmul2(a, alpha)));
      }
      if (p.residual_out != nullptr) store_row<X, AL>(v[j], to, j * tpr + t, p.d, stage);
    }
  }
  if (p.weight == nullptr) return;  // only the stream is wanted
  const float2 f = row_scale(row_sum(row_squares<X, VPT>(v, 1.f), part[2], warps), p.inv_d, p.eps,
                             [&](float unit) { return row_sum(row_squares<X, VPT>(v, unit), part[3], warps); });
  emit_norm<X, VPT, FMT, AL, true>(p, v, f, row, t, tpr, stage);
}

template <typename X, int VPT, int FMT>
static void launch_format(const BlockNormParams& p, unsigned grid, int threads, cudaStream_t stream) {
  if (p.vec) {
    if (p.gate != nullptr)
      block_norm<X, VPT, FMT, true, true><<<grid, threads, 0, stream>>>(p);
    else
      block_norm<X, VPT, FMT, false, true><<<grid, threads, 0, stream>>>(p);
  } else if constexpr (VPT != 4) {
    if (p.gate != nullptr)
      block_norm<X, VPT, FMT, true, false><<<grid, threads, 0, stream>>>(p);
    else
      block_norm<X, VPT, FMT, false, false><<<grid, threads, 0, stream>>>(p);
  }
}
template <typename X, int VPT>
static void launch_vec(const BlockNormParams& p, unsigned grid, int threads, cudaStream_t stream) {
  if (p.fmt == kMx8)
    launch_format<X, VPT, kMx8>(p, grid, threads, stream);
  else if (p.fmt == kMx4)
    launch_format<X, VPT, kMx4>(p, grid, threads, stream);
  else
    launch_format<X, VPT, 0>(p, grid, threads, stream);
}

template <typename X>
static cudaError_t launch_typed(BlockNormParams p, cudaStream_t stream) {
  // Vectors per thread by the row alone, so that a row's result does not depend on its batch.
  const int nvec = (p.d + 127) / 128 * 16;  // to whole scale words
  int vpt = !p.vec ? 1 : sizeof(X) == 4 ? 1 : 2;
  while (vpt > 1 && nvec <= 32 * vpt / 2) vpt /= 2;
  while ((nvec + vpt - 1) / vpt > kNormMaxThreads) vpt *= 2;
  if (!p.vec && vpt == 4) vpt = 8;  // (not built: rows of more than 8192 off the 16-byte boundaries)
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

cudaError_t launch_block_norm(const BlockNormParams& p, int dtype, cudaStream_t stream) {
  switch (dtype) {
    case kBf16: return launch_typed<__nv_bfloat16>(p, stream);
    case kF16: return launch_typed<__half>(p, stream);
    default: return launch_typed<float>(p, stream);
  }
}

}  // namespace difr
