// Microscaled formats: values -> codes and scales, and back.
//
// Both are bound by their bytes.  A warp takes a part of a row, a lane 8 consecutive values at a time (16 bytes of
// bf16); the four lanes of a block find its maximum with two shuffles and the sixteen lanes of four blocks put their
// scale bytes together, so that scales leave as whole 32-bit words.  Four vectors per lane are loaded before the first
// is used.
#include <cuda_runtime.h>

#include "mx_device.cuh"
#include "mx_kernels.h"

namespace difr {

constexpr int kCvtWarps = 8;    // rows per CTA
constexpr int kCvtUnroll = 4;   // vectors of 8 values per lane
constexpr int kCvtElems = 32 * 8 * kCvtUnroll;  // of a row, per CTA

template <typename X, int FMT>
__global__ void __launch_bounds__(kCvtWarps * 32) mx_quantize(const MxConvertParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kCvtWarps + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  const X* in = static_cast<const X*>(p.in) + row * p.ld;
  unsigned char* codes = p.codes + row * mx_pitch_bytes(FMT, p.d);
  const int64_t words = mx_words(p.d);
  const int nvec = (int)mx_blocks(p.d) * 4;
  const int vec0 = (int)blockIdx.y * (kCvtElems / 8) + lane;
  float v[kCvtUnroll][8];
#pragma unroll
  for (int j = 0; j < kCvtUnroll; ++j) load8<X>(in, (vec0 + j * 32) * 8, p.d, p.vec, v[j]);
#pragma unroll
  for (int j = 0; j < kCvtUnroll; ++j) {
    const int vec = vec0 + j * 32;
    const bool past = vec >= nvec;
    uint32_t c[2];
    const uint32_t word = mx_quantize8<FMT>(v[j], past, c);
    if (!past) {
      if (FMT == kMx8)
        *reinterpret_cast<uint2*>(codes + (int64_t)vec * 8) = make_uint2(c[0], c[1]);
      else
        *reinterpret_cast<uint32_t*>(codes + (int64_t)vec * 4) = c[0];
      if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(p.scales + mx_scale_offset(row, vec >> 4, words)) = word;
    }
  }
}

template <typename X, int FMT>
__global__ void __launch_bounds__(kCvtWarps * 32) mx_dequantize(const MxConvertParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kCvtWarps + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  X* out = static_cast<X*>(p.out) + row * p.ld;
  const unsigned char* codes = p.codes + row * mx_pitch_bytes(FMT, p.d);
  const int64_t words = mx_words(p.d);
  const int nvec = (p.d + 7) / 8;
  const int vec0 = (int)blockIdx.y * (kCvtElems / 8) + lane;
  uint2 c[kCvtUnroll];
  uint32_t byte[kCvtUnroll];
#pragma unroll
  for (int j = 0; j < kCvtUnroll; ++j) {
    const int vec = vec0 + j * 32;
    c[j] = make_uint2(0u, 0u);
    byte[j] = 0u;
    if (vec < nvec) {
      if (FMT == kMx8)
        c[j] = *reinterpret_cast<const uint2*>(codes + (int64_t)vec * 8);
      else
        c[j].x = *reinterpret_cast<const uint32_t*>(codes + (int64_t)vec * 4);
      byte[j] = p.scales[mx_scale_offset(row, vec >> 4, words) + ((vec >> 2) & 3)];
    }
  }
#pragma unroll
  for (int j = 0; j < kCvtUnroll; ++j) {
    const int vec = vec0 + j * 32;
    if (vec >= nvec) break;
    const float s = mx_scale_value(byte[j]);
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 two;
      if (FMT == kMx8)
        two = cvt_e4m3x2_to_float2(((i < 2 ? c[j].x : c[j].y) >> (16 * (i & 1))) & 0xFFFFu);
      else
        two = cvt_e2m1x2_to_float2((c[j].x >> (8 * i)) & 0xFFu);
      v[2 * i] = two.x * s;
      v[2 * i + 1] = two.y * s;
    }
    store8<X>(out, vec * 8, p.d, p.vec, v);
  }
}

static dim3 cvt_grid(const MxConvertParams& p) {
  return dim3((unsigned)((p.rows + kCvtWarps - 1) / kCvtWarps), (unsigned)((p.d + kCvtElems - 1) / kCvtElems));
}

template <typename X>
static cudaError_t quantize_typed(const MxConvertParams& p, cudaStream_t stream) {
  if (p.fmt == kMx8)
    mx_quantize<X, kMx8><<<cvt_grid(p), kCvtWarps * 32, 0, stream>>>(p);
  else
    mx_quantize<X, kMx4><<<cvt_grid(p), kCvtWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_mx_quantize(const MxConvertParams& p, int dtype, cudaStream_t stream) {
  switch (dtype) {
    case kBf16: return quantize_typed<__nv_bfloat16>(p, stream);
    case kF16: return quantize_typed<__half>(p, stream);
    default: return quantize_typed<float>(p, stream);
  }
}

template <typename X>
static cudaError_t dequantize_typed(const MxConvertParams& p, cudaStream_t stream) {
  if (p.fmt == kMx8)
    mx_dequantize<X, kMx8><<<cvt_grid(p), kCvtWarps * 32, 0, stream>>>(p);
  else
    mx_dequantize<X, kMx4><<<cvt_grid(p), kCvtWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_mx_dequantize(const MxConvertParams& p, int dtype, cudaStream_t stream) {
  return dtype == kBf16 ? dequantize_typed<__nv_bfloat16>(p, stream) : dequantize_typed<float>(p, stream);
}

}  // namespace difr
