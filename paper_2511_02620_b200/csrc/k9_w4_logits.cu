// LM-head product of bf16 hidden states with 4-bit weights:
//
//   l[t, v] = sum over groups g of scale[v, g] * sum over k in g of h[t, k] code[v, k]
//
// A warp an id, a lane 32 codes (16 bytes) at a time, eight tokens in registers; fp32 throughout.
#include <cuda_runtime.h>

#include "step_kernels.h"
#include "w4_device.cuh"

namespace difr {

constexpr int kW4LogitWarps = 8, kW4Tokens = 8;

__device__ __forceinline__ float finite_or_nan(float x) { return fmaf(0.f, x, x); }

template <typename OUT>
__global__ void __launch_bounds__(kW4LogitWarps * 32) w4_logits(const W4LogitsParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t v = (int64_t)blockIdx.x * kW4LogitWarps + warp;
  if (v >= p.V) return;
  const int64_t pitch = w4_pitch_bytes(p.d);
  const uint4* codes = reinterpret_cast<const uint4*>(p.codes + v * pitch);
  const __nv_bfloat16* scales = p.scales + v * w4_scale_pitch(p.d, p.group);
  const int blocks = (int)(pitch / 16);
  for (int t0 = blockIdx.y * kW4Tokens; t0 < p.T; t0 += gridDim.y * kW4Tokens) {
    float acc[kW4Tokens] = {};
    for (int b = lane; b < blocks; b += 32) {
      const uint4 c = codes[b];
      const float s = finite_or_nan(__bfloat162float(scales[b * 32 / p.group]));
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
      float sum[kW4Tokens] = {};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 two = w4_pair(w[i >> 2], i & 3);
        const int k = b * 32 + 2 * i;
#pragma unroll
        for (int j = 0; j < kW4Tokens; ++j) {
          if (t0 + j >= p.T) break;
          const __nv_bfloat16* h = p.h + (int64_t)(t0 + j) * p.ldh;
          if (k < p.d) sum[j] = fmaf(two.x, finite_or_nan(__bfloat162float(h[k])), sum[j]);
          if (k + 1 < p.d) sum[j] = fmaf(two.y, finite_or_nan(__bfloat162float(h[k + 1])), sum[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < kW4Tokens; ++j) acc[j] = fmaf(s, sum[j], acc[j]);
    }
#pragma unroll
    for (int j = 0; j < kW4Tokens; ++j) {
#pragma unroll
      for (int m = 16; m >= 1; m >>= 1) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], m);
      if (lane == j && t0 + j < p.T)
        static_cast<OUT*>(p.logits)[(int64_t)(t0 + j) * p.ld + v] = from_float<OUT>(acc[j]);
    }
  }
}

cudaError_t launch_w4_logits(const W4LogitsParams& p, int dtype, cudaStream_t stream) {
  const int tiles = (p.T + kW4Tokens - 1) / kW4Tokens;
  const dim3 grid((unsigned)((p.V + kW4LogitWarps - 1) / kW4LogitWarps), (unsigned)(tiles < 64 ? tiles : 64));
  if (dtype == kBf16)
    w4_logits<__nv_bfloat16><<<grid, kW4LogitWarps * 32, 0, stream>>>(p);
  else
    w4_logits<float><<<grid, kW4LogitWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace difr
