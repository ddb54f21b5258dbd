// 4-bit weights with group scales: values -> codes and scales, and back.
//
//   scale = bf16(largest magnitude of the group / 7), below 2^-126: 0;  code = value / scale to the nearest integer, ties to
//   even.  A seventh rounded to eight bits leaves quotients under 7.03, so that codes stay within -7 .. 7.
//
// Laid out like the microscaled conversions: a warp takes a part of a row, a lane 8 consecutive values at a time; a group is
// 4, 8 or 16 neighbouring lanes, its maximum two to four shuffles away.  Both directions are bound by their bytes as long as
// few instructions are spent per value: 128256 x 4096 in bf16 takes 276 us to codes, 520 with the way back (409 of bytes).
#include <cuda_runtime.h>

#include "step_kernels.h"
#include "w4_device.cuh"

namespace difr {

constexpr int kW4Warps = 8;    // rows per CTA
constexpr int kW4Unroll = 4;   // vectors of 8 values per lane
constexpr int kW4Vecs = 32 * kW4Unroll;  // of a row, per CTA

// bf16(amax / 7), exactly rounded (nearest, ties to even), as its bits; 0x7FC0 for a group with a NaN or an infinity.
__device__ __forceinline__ uint32_t w4_scale_bits(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 0x7FC0u;
  const float amax = __uint_as_float(amax_bits);
  // a seventh within an ulp, cut to bf16; the midpoint above it times seven is a short number and decides
  const uint32_t low = __float_as_uint(amax * (1.f / 7.f)) >> 16;
  const float seven_mid = 7.f * __uint_as_float((low << 16) | 0x8000u);
  const uint32_t bits = low + (amax > seven_mid || (amax == seven_mid && (low & 1u)) ? 1u : 0u);
  return bits < 0x80u ? 0u : bits;
}

// The bits of a half of a packed result, through a statement that the optimiser does not look into: with a plain cast
// nvcc 12.9.86 drew the last four bits of some of the eight from another byte of the pair.
__device__ __forceinline__ uint32_t opaque_bits(float x) {
  uint32_t r;
  asm("mov.b32 %0, %1;" : "=r"(r) : "f"(x));
  return r;
}

// Codes of eight 16-bit values.  A quotient of 16-bit numbers that is no tie is at least 2^-14 away from one, so quotients a
// little too small and a little too large round to the same integer except at ties, where they round to both neighbours.  On
// 1.5 * 2^23 the sum of the two holds the integer in the same bits one exponent higher, where a unit is 2: the addition itself
// rounds a tie's odd sum to the even neighbour.  The eight integers + 8 are then digits of a number to the base 16.
__device__ __forceinline__ uint32_t codes_of_halves(const float2 (&v)[4], float inv) {
  const float2 small = make_float2(inv * (1.f - 0x1p-22f), inv * (1.f - 0x1p-22f));
  const float2 large = make_float2(inv * (1.f + 0x1p-22f), inv * (1.f + 0x1p-22f));
  const float2 magic = make_float2(12582912.f, 12582912.f);
  uint32_t word = 0;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    const float2 u = fadd2(ffma2(v[i], small, magic), ffma2(v[i], large, magic));
    word = (word * 16u + opaque_bits(u.y)) * 16u + opaque_bits(u.x);
  }
  constexpr uint32_t base = 0x4BC00000u - 8u;  // the bits of 2 * 1.5 * 2^23, and the 8 that is added to each
  return (word - base * 0x11111111u) ^ 0x88888888u;
}
// Codes of eight fp32 values, whose quotients may lie next to a tie.  1.5 * 2^23: the sum's last bits are the integer nearest
// to value * inv; what is left of the value, which is exact, shows where inv's rounding took the wrong side of a border, and the
// ties.
__device__ __forceinline__ uint32_t codes_of_floats(const float2 (&v)[4], float inv, float scale) {
  const uint32_t half = __float_as_uint(0.5f * scale);
  uint32_t word = 0;
#pragma unroll
  for (int i = 3; i >= 0; --i) {
    const float2 t = ffma2(v[i], make_float2(inv, inv), make_float2(12582912.f, 12582912.f));
    const float2 q = fadd2(t, make_float2(-12582912.f, -12582912.f));
    const float2 r = ffma2(q, make_float2(-scale, -scale), v[i]);
    const uint32_t a = opaque_bits(t.x), b = opaque_bits(t.y);
    // (a tie moves away from an odd integer: half of the scale less its last bit; magnitudes compare like their bits)
    const uint32_t ra = opaque_bits(r.x), rb = opaque_bits(r.y);
    const uint32_t ca = a + ((ra & 0x7FFFFFFFu) > half - (a & 1u) ? (uint32_t)((int)ra >> 31) | 1u : 0u);
    const uint32_t cb = b + ((rb & 0x7FFFFFFFu) > half - (b & 1u) ? (uint32_t)((int)rb >> 31) | 1u : 0u);
    word = (word << 8) | ((cb & 15u) << 4) | (ca & 15u);
  }
  return word;
}

template <typename X, int GROUP, bool AL>
__global__ void __launch_bounds__(kW4Warps * 32) w4_quantize(const W4ConvertParams p) {
  __shared__ uint4 stage_all[AL ? 1 : kW4Warps * 32 * sizeof(X) / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  X* stage = reinterpret_cast<X*>(stage_all) + (AL ? 0 : warp * 256);
  const int64_t row = (int64_t)blockIdx.x * kW4Warps + warp;
  if (row >= p.rows) return;
  const int nvec = (int)(w4_pitch_bytes(p.d) / 4);  // words of codes
  const int64_t spitch = w4_scale_pitch(p.d, GROUP);
  const int nvec_scales = (int)(spitch * (GROUP / 8));  // the scales behind the last group are zeros
  const int vec0 = (int)blockIdx.y * kW4Vecs + lane;
  uint32_t* codes = reinterpret_cast<uint32_t*>(p.codes + row * w4_pitch_bytes(p.d));
  __nv_bfloat16* scales = p.scales + row * spitch;
  Vec8<X> raw[kW4Unroll];
  const X* in = static_cast<const X*>(p.in) + row * p.ld;
  RowVectors<X, kW4Unroll, AL> fetched;
  fetch_row(fetched, in, vec0, 32, p.d);
  finish_row(raw, fetched, in, vec0, 32, p.d, stage);
#pragma unroll
  for (int j = 0; j < kW4Unroll; ++j) {
    const int vec = vec0 + j * 32;
    if (vec - lane >= nvec_scales && vec - lane >= nvec) break;  // uniform over the warp
    float2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = raw[j].pair(i);
    // (magnitudes compare like their bits, and a NaN's bits are above every number's)
    float f = max3_abs(v[0].x, v[0].y, v[1].x);
    f = max3_abs(f, v[1].y, v[2].x);
    f = max3_abs(f, v[2].y, v[3].x);
    f = max3_abs(f, v[3].y, 0.f);
    uint32_t m = __float_as_uint(f);
#pragma unroll
    for (int s = 1; s < GROUP / 8; s <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
    const uint32_t bits = w4_scale_bits(m);
    const float scale = __uint_as_float(bits << 16);
    const bool number = bits != 0u && bits != 0x7FC0u;
    const uint32_t word = !number ? 0u : sizeof(X) == 2 ? codes_of_halves(v, 1.f / scale) : codes_of_floats(v, 1.f / scale, scale);
    if (vec < nvec) codes[vec] = word;
    if (vec < nvec_scales && (lane & (GROUP / 8 - 1)) == 0)
      scales[vec / (GROUP / 8)] = __ushort_as_bfloat16((unsigned short)bits);
  }
}

template <typename X, bool AL>
__global__ void __launch_bounds__(kW4Warps * 32) w4_dequantize(const W4ConvertParams p) {
  __shared__ uint4 stage_all[AL ? 1 : kW4Warps * 32 * sizeof(X) / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  X* stage = reinterpret_cast<X*>(stage_all) + (AL ? 0 : warp * 256);
  const int64_t row = (int64_t)blockIdx.x * kW4Warps + warp;
  if (row >= p.rows) return;
  X* out = static_cast<X*>(p.out) + row * p.ld;
  const int nvec = (p.d + 7) / 8;
  const int vec0 = (int)blockIdx.y * kW4Vecs + lane;
  const int vecs_per_group = p.group / 8;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(p.codes + row * w4_pitch_bytes(p.d));
  const __nv_bfloat16* scales = p.scales + row * w4_scale_pitch(p.d, p.group);
  uint32_t c[kW4Unroll];
  float s[kW4Unroll];
#pragma unroll
  for (int j = 0; j < kW4Unroll; ++j) {
    const int vec = vec0 + j * 32;
    c[j] = vec < nvec ? codes[vec] : 0u;
    s[j] = vec < nvec ? __bfloat162float(scales[vec / vecs_per_group]) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < kW4Unroll; ++j) {
    const int vec = vec0 + j * 32;
    if (vec - lane >= nvec) break;  // uniform over the warp
    Vec8<X> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.set_pair(i, fmul2(w4_pair(c[j], i), make_float2(s[j], s[j])));
    store_row<X, AL>(o, out, vec, p.d, stage);
  }
}

static dim3 w4_grid(const W4ConvertParams& p, int64_t vecs) {
  return dim3((unsigned)((p.rows + kW4Warps - 1) / kW4Warps), (unsigned)((vecs + kW4Vecs - 1) / kW4Vecs));
}

template <typename X, int GROUP>
static cudaError_t quantize_group(const W4ConvertParams& p, cudaStream_t stream) {
  const int64_t words = w4_pitch_bytes(p.d) / 4, scales = w4_scale_pitch(p.d, GROUP) * (GROUP / 8);
  const dim3 grid = w4_grid(p, words > scales ? words : scales);
  if (p.vec)
    w4_quantize<X, GROUP, true><<<grid, kW4Warps * 32, 0, stream>>>(p);
  else
    w4_quantize<X, GROUP, false><<<grid, kW4Warps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}
template <typename X>
static cudaError_t quantize_typed(const W4ConvertParams& p, cudaStream_t stream) {
  return p.group == 32 ? quantize_group<X, 32>(p, stream)
                       : p.group == 64 ? quantize_group<X, 64>(p, stream) : quantize_group<X, 128>(p, stream);
}

cudaError_t launch_w4_quantize(const W4ConvertParams& p, int dtype, cudaStream_t stream) {
  switch (dtype) {
    case kBf16: return quantize_typed<__nv_bfloat16>(p, stream);
    case kF16: return quantize_typed<__half>(p, stream);
    default: return quantize_typed<float>(p, stream);
  }
}

template <typename X>
static cudaError_t dequantize_typed(const W4ConvertParams& p, cudaStream_t stream) {
  const dim3 grid = w4_grid(p, (p.d + 7) / 8);
  if (p.vec)
    w4_dequantize<X, true><<<grid, kW4Warps * 32, 0, stream>>>(p);
  else
    w4_dequantize<X, false><<<grid, kW4Warps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_w4_dequantize(const W4ConvertParams& p, int dtype, cudaStream_t stream) {
  return dtype == kBf16 ? dequantize_typed<__nv_bfloat16>(p, stream) : dequantize_typed<float>(p, stream);
}

}  // namespace difr
