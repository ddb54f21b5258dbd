// C ABI of a decoding step's operators: the block norm.  Argument checks and launches; nothing here computes.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/difr.h"
#include "difr_host.h"
#include "mx_device.cuh"
#include "step_kernels.h"

namespace {

using namespace difr;

// Streaming multiprocessors of the current device; DIFR_ERR_ARCH for another architecture.
difr_status device_sms(int* sms) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> cached[kMaxDevices];  // 0: not asked yet, -1: another architecture
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return DIFR_ERR_CUDA;
  const bool slot = dev >= 0 && dev < kMaxDevices;
  int n = slot ? cached[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return DIFR_ERR_CUDA;
    if (major != 10) n = -1;
    if (slot) cached[dev].store(n, std::memory_order_relaxed);
  }
  if (n < 0) return DIFR_ERR_ARCH;
  *sms = n;
  return DIFR_OK;
}

}  // namespace

extern "C" {

difr_status difr_block_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const difr_block* block,
                            const void* weight, int32_t dtype, int64_t T, int64_t d, float eps, const difr_norm_out* out,
                            difr_stream_t stream) {
  if (!out || !block || !known_dtype(dtype) || T < 0 || d <= 0 || !(eps > 0.f) || !isfinite(eps)) return DIFR_ERR_INVALID_ARG;
  if (!isfinite(block->scale) || !isfinite(block->residual_scale) || !isfinite(block->weight_offset))
    return DIFR_ERR_INVALID_ARG;
  if (block->post_weight && (!(block->post_eps > 0.f) || !isfinite(block->post_eps))) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 && !known_format(out->mx_format)) return DIFR_ERR_INVALID_ARG;
  if (T > kMaxRows || d > kNormMaxD) return DIFR_ERR_SHAPE;
  if (T == 0) return DIFR_OK;
  if (!x || !residual) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 ? (!out->codes || !out->scales) : (out->codes || out->scales)) return DIFR_ERR_INVALID_ARG;
  const bool normed = out->h || out->mx_format != 0;
  if (normed ? !weight : (weight || !out->residual)) return DIFR_ERR_INVALID_ARG;
  const int64_t ld_gate = block->gate ? block->ld_gate : 0;
  if (ldx < d || ld_residual < d || (ld_gate != 0 && ld_gate < d) || (out->residual && out->ld_residual < d) ||
      (out->h && out->ldh < d))
    return DIFR_ERR_INVALID_ARG;
  if (ldx > kMaxLd || ld_residual > kMaxLd || ld_gate > kMaxLd || (out->residual && out->ld_residual > kMaxLd) ||
      (out->h && out->ldh > kMaxLd))
    return DIFR_ERR_SHAPE;
  const int eb = elem_bytes(dtype);
  if (!aligned_to(x, eb) || !aligned_to(residual, eb) || !aligned_to(weight, eb) || !aligned_to(block->post_weight, eb) ||
      !aligned_to(block->gate, eb) || (out->residual && !aligned_to(out->residual, eb)) || (out->h && !aligned_to(out->h, 2)))
    return DIFR_ERR_ALIGN;
  if (out->mx_format != 0 && (!aligned16(out->codes) || !aligned16(out->scales))) return DIFR_ERR_ALIGN;
  int sms = 0;
  const difr_status ds = device_sms(&sms);
  if (ds != DIFR_OK) return ds;
  BlockNormParams p;
  memset(&p, 0, sizeof p);
  p.x = x; p.residual = residual; p.post_weight = block->post_weight; p.gate = block->gate; p.weight = weight;
  p.residual_out = out->residual; p.h = out->h;
  p.codes = static_cast<unsigned char*>(out->codes); p.scales = static_cast<unsigned char*>(out->scales);
  p.T = T; p.ldx = ldx; p.ld_residual = ld_residual; p.ld_gate = ld_gate;
  p.ld_residual_out = out->ld_residual; p.ldh = out->ldh;
  p.d = (int)d; p.fmt = out->mx_format; p.eps = eps; p.post_eps = block->post_eps; p.inv_d = 1.f / (float)d;
  p.alpha = block->scale; p.beta = block->residual_scale; p.weight_offset = block->weight_offset;
  p.vec = d % 8 == 0 && vector_rows(x, ldx, dtype) && vector_rows(residual, ld_residual, dtype) && aligned16(weight) &&
          aligned16(block->post_weight) && vector_rows(block->gate, ld_gate, dtype) &&
          (!out->residual || vector_rows(out->residual, out->ld_residual, dtype)) &&
          (!out->h || vector_rows(out->h, out->ldh, DIFR_BF16));
  return launch_block_norm(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

}  // extern "C"
