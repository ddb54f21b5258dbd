// Device-side building blocks of the microscaled formats and of the block-scaled tensor-core product.
//
// A microscaled tensor [rows, d] keeps blocks of 32 values along a row: every value is a code of an 8-bit (e4m3,
// largest 448 = 1.75 * 2^8) or 4-bit (e2m1, largest 6 = 1.5 * 2^2) floating-point format, every block has one
// power-of-two scale, stored as its exponent + 127 in a byte (255: the block held a NaN or an infinity).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "difr_device.cuh"

namespace difr {

constexpr int kMx8 = 8, kMx4 = 4;  // bits per code; the values of difr_mx_format
constexpr int kMxBlock = 32;
constexpr int kSfWordRows = 128, kSfWordBytes = 512;  // a scale word: four scales of each of 128 rows

__host__ __device__ constexpr int mx_emax(int fmt) { return fmt == kMx8 ? 8 : 2; }
__host__ __device__ __forceinline__ int64_t mx_blocks(int64_t d) { return (d + kMxBlock - 1) / kMxBlock; }
__host__ __device__ __forceinline__ int64_t mx_words(int64_t d) { return (mx_blocks(d) + 3) / 4; }
__host__ __device__ __forceinline__ int64_t mx_pitch_bytes(int fmt, int64_t d) {
  return mx_blocks(d) * kMxBlock * fmt / 8;
}
// Byte offset of the four scales of blocks 4 w .. 4 w + 3 of a row: what the tensor core reads as a 128 x 4 block is
// 512 consecutive bytes, 16 per lane (row % 32), 4 of them per quarter (row / 32) of the 128 rows.
__device__ __forceinline__ int64_t mx_scale_offset(int64_t row, int64_t w, int64_t words) {
  return ((row >> 7) * words + w) * kSfWordBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// Scale byte of a block from the bits of its largest magnitude: exponent floor(log2 amax) - emax, at least -127.  The
// exponent field of an fp32 is floor(log2) + 127 for normal numbers; zero and subnormal maxima end at the smallest
// scale, where their codes are still exact or round to zero.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - mx_emax(FMT), 0);
}
// 2^(127 - byte), what a value is multiplied by before it is rounded: exact, since it is a power of two.  0 for the
// blocks that are not numbers: their codes are then written as 0 (0 * infinity is NaN, so they are cleared apart).
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) {
  return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}
// 2^(byte - 127); NaN for 255 (whose bits would be infinity's).
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
  uint32_t bits = byte << 23;
  if (byte == 0u) bits = 0x00400000u;
  if (byte == 255u) bits = 0x7FC00000u;
  return __uint_as_float(bits);
}

// Rounding to the formats: nearest, ties to even, magnitudes above the largest become the largest.
__device__ __forceinline__ uint32_t cvt_e4m3x4(float a0, float a1, float a2, float a3) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(lo) : "f"(a0), "f"(a1));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(hi) : "f"(a2), "f"(a3));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ uint32_t cvt_e2m1x8(const float2 (&a)[4]) {
  uint32_t r;
  asm("{\n"
      ".reg .b8 b0, b1, b2, b3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      "mov.b32 %0, {b0, b1, b2, b3};\n"
      "}\n"
      : "=r"(r)
      : "f"(a[0].x), "f"(a[0].y), "f"(a[1].x), "f"(a[1].y), "f"(a[2].x), "f"(a[2].y), "f"(a[3].x), "f"(a[3].y));
  return r;
}
// Codes back to values (exact in fp16: e4m3 and e2m1 are subsets of it).
__device__ __forceinline__ float2 half2_bits_to_float2(uint32_t h2) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h2));
}
__device__ __forceinline__ float2 cvt_e4m3x2_to_float2(uint32_t two_codes) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)two_codes));
  return half2_bits_to_float2(h2);
}
__device__ __forceinline__ float2 cvt_e2m1x2_to_float2(uint32_t two_codes) {
  uint32_t h2;
  asm("{\n"
      ".reg .b8 b;\n"
      "cvt.u8.u32 b, %1;\n"
      "cvt.rn.f16x2.e2m1x2 %0, b;\n"
      "}\n"
      : "=r"(h2)
      : "r"(two_codes));
  return half2_bits_to_float2(h2);
}

// max(|a|, |b|, |c|); a NaN among them is what comes out.
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 fmul2(float2 a, float2 b) {
  unsigned long long d;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(d)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&d);
}

// Quantises 8 consecutive values held by each lane.  A block of 32 is four neighbouring lanes (lane % 4 == 0 starts
// one), a scale word (four blocks) sixteen; every lane of the warp takes part, lanes past the row hold zeros.  `codes`
// receives 8 codes (4 or 8 bytes), the returned word is the four scale bytes of the lane's sixteen.
template <int FMT>
__device__ __forceinline__ uint32_t mx_quantize8(const float2 (&v)[4], bool past_end, uint32_t (&codes)[2]) {
  // (magnitudes compare like their bits, and a NaN's bits are above every number's)
  float f = max3_abs(v[0].x, v[0].y, v[1].x);
  f = max3_abs(f, v[1].y, v[2].x);
  f = max3_abs(f, v[2].y, v[3].x);
  f = max3_abs(f, v[3].y, 0.f);
  uint32_t m = __float_as_uint(f);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const uint32_t byte = past_end ? 0u : mx_scale_byte<FMT>(m);
  const float inv = mx_inverse_scale(byte);
  float2 q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = fmul2(v[i], make_float2(inv, inv));
  if (FMT == kMx8) {
    codes[0] = cvt_e4m3x4(q[0].x, q[0].y, q[1].x, q[1].y);
    codes[1] = cvt_e4m3x4(q[2].x, q[2].y, q[3].x, q[3].y);
  } else {
    codes[0] = cvt_e2m1x8(q);
    codes[1] = 0;
  }
  if (byte == 255u) codes[0] = codes[1] = 0;
  uint32_t word = byte << (((threadIdx.x >> 2) & 3) * 8);
  word |= __shfl_xor_sync(0xffffffffu, word, 4);
  word |= __shfl_xor_sync(0xffffffffu, word, 8);
  return word;
}

// ---------------------------------------------------------------- element types of inputs and outputs
template <typename X>
__device__ __forceinline__ X from_float(float x);
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }

// Eight consecutive elements as they lie in memory, on a 16-byte boundary.  (Plain loads, not the read-only path: a call
// may write its result over its input.)
template <typename X>
struct Vec8 {
  uint4 q[sizeof(X) / 2];
  __device__ __forceinline__ void load(const X* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(X* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = q[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (int)sizeof(X) / 2; ++i) q[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ uint32_t word(int i) const {
    const uint4& a = q[i >> 2];
    return (i & 3) == 0 ? a.x : (i & 3) == 1 ? a.y : (i & 3) == 2 ? a.z : a.w;
  }
  __device__ __forceinline__ void set_word(int i, uint32_t w) {
    uint4& a = q[i >> 2];
    if ((i & 3) == 0) a.x = w;
    else if ((i & 3) == 1) a.y = w;
    else if ((i & 3) == 2) a.z = w;
    else a.w = w;
  }
  // elements 2 i and 2 i + 1
  __device__ __forceinline__ float2 pair(int i) const;
  __device__ __forceinline__ void set_pair(int i, float2 v);
};
template <>
__device__ __forceinline__ float2 Vec8<__nv_bfloat16>::pair(int i) const {
  const uint32_t w = word(i);
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float2 Vec8<__half>::pair(int i) const {
  return half2_bits_to_float2(word(i));
}
template <>
__device__ __forceinline__ float2 Vec8<float>::pair(int i) const {
  return make_float2(__uint_as_float(word(2 * i)), __uint_as_float(word(2 * i + 1)));
}
template <>
__device__ __forceinline__ void Vec8<__nv_bfloat16>::set_pair(int i, float2 v) {
  __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
  set_word(i, *reinterpret_cast<uint32_t*>(&b));
}
template <>
__device__ __forceinline__ void Vec8<__half>::set_pair(int i, float2 v) {
  __half2 b = __floats2half2_rn(v.x, v.y);
  set_word(i, *reinterpret_cast<uint32_t*>(&b));
}
template <>
__device__ __forceinline__ void Vec8<float>::set_pair(int i, float2 v) {
  set_word(2 * i, __float_as_uint(v.x));
  set_word(2 * i + 1, __float_as_uint(v.y));
}

// Rows off the 16-byte boundaries (odd d, odd strides).  16-bit rows on 8 or 4 bytes are read, on 8 bytes written, by lanes
// that hold eight neighbours each (norm of 20000 x 4100 with all outputs 186 us, 226 by way of shared memory).  Others a warp
// moves as units that the row's start allows, neighbouring lanes neighbouring units, and turns its 256 elements through
// `stage`; only the end of a row is checked element by element.  All loads of a thread go out before the first is turned.
struct RawUnits {
  uint32_t w[8];  // two, four or eight units of a lane
};
template <typename X, typename U>
__device__ __forceinline__ void fetch_units(RawUnits& raw, const X* from, int lane) {
  constexpr int kUnits = 8 * (int)sizeof(X) / (int)sizeof(U);
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    const U one = reinterpret_cast<const U*>(from)[k * 32 + lane];
    if constexpr (sizeof(U) == 8) {
      raw.w[2 * k] = one.x;
      raw.w[2 * k + 1] = one.y;
    } else if constexpr (sizeof(U) == 4) {
      raw.w[k] = *reinterpret_cast<const uint32_t*>(&one);
    } else {
      raw.w[k] = *reinterpret_cast<const uint16_t*>(&one);
    }
  }
}
template <typename X, typename U>
__device__ __forceinline__ void place_units(const RawUnits& raw, X* to, int lane) {
  constexpr int kUnits = 8 * (int)sizeof(X) / (int)sizeof(U);
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    if constexpr (sizeof(U) == 8)
      reinterpret_cast<uint2*>(to)[k * 32 + lane] = make_uint2(raw.w[2 * k], raw.w[2 * k + 1]);
    else if constexpr (sizeof(U) == 4)
      reinterpret_cast<uint32_t*>(to)[k * 32 + lane] = raw.w[k];
    else
      reinterpret_cast<uint16_t*>(to)[k * 32 + lane] = (uint16_t)raw.w[k];
  }
}
// 16-bit rows on 8 or 4 bytes need no turning: a lane's eight elements are two or four units of its own.
template <typename X>
__device__ __forceinline__ int direct_bytes(const X* row) {  // 0: not such a row
  const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(row) & 7u;
  return sizeof(X) != 2 ? 0 : at == 0 ? 8 : at == 4 ? 4 : 0;
}
template <typename X>
__device__ __forceinline__ void fetch_direct(RawUnits& raw, const X* from, int n, int bytes) {  // n elements are there
  if (n >= 8) {
    if (bytes == 8) {
      const uint2 a = reinterpret_cast<const uint2*>(from)[0], b = reinterpret_cast<const uint2*>(from)[1];
      raw.w[0] = a.x; raw.w[1] = a.y; raw.w[2] = b.x; raw.w[3] = b.y;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) raw.w[i] = reinterpret_cast<const uint32_t*>(from)[i];
    }
  } else {
    const uint16_t* one = reinterpret_cast<const uint16_t*>(from);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      raw.w[i] = (2 * i < n ? one[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)one[2 * i + 1] << 16 : 0u);
  }
}
// (On 4 bytes four stores a lane, a quarter of every line each, take longer than the turn: 71.6 us against 68.4 for
// 64000 x 1750 from 8 bits.)
template <typename X>
__device__ __forceinline__ void store_direct(const Vec8<X>& v, X* to, int n) {  // rows on 8 bytes
  if (n >= 8) {
    reinterpret_cast<uint2*>(to)[0] = make_uint2(v.word(0), v.word(1));
    reinterpret_cast<uint2*>(to)[1] = make_uint2(v.word(2), v.word(3));
  } else {
    uint16_t* one = reinterpret_cast<uint16_t*>(to);
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) one[i] = (uint16_t)(v.word(i >> 1) >> (16 * (i & 1)));
  }
}

// The units a warp moves its 256 elements e0 .. by: 8, 4 or 2 bytes, 0 for single elements with a check each (the end of
// a row).  The same in all lanes.
template <typename X>
__device__ __forceinline__ int unit_bytes(const X* row, int e0, int d) {
  if (e0 + 256 > d) return 0;
  const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(row) & 7u;
  return at == 0 ? 8 : (at == 4 ? 4 : (int)sizeof(X));
}

// Vectors vec0 + j stride (j < N) of a row of d elements, one per lane, zeros past its end; vec0 - lane is the same in
// all lanes.  AL: the row starts on a 16-byte boundary and d is a multiple of 8.  In two steps, so that a caller can
// start more rows before it needs the first: fetch_row, then finish_row.
template <typename X, int N, bool AL>
struct RowVectors {
  Vec8<X> v[AL ? N : 1];
  RawUnits raw[AL ? 1 : N];
};
template <typename X, int N, bool AL>
__device__ __forceinline__ void fetch_row(RowVectors<X, N, AL>& f, const X* row, int vec0, int stride, int d) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int i = vec0 + j * stride;
    if constexpr (AL) {
      if (i * 8 < d) f.v[j].load(row + i * 8); else f.v[j].zero();
    } else {
      const int e0 = (i - lane) * 8;
      const int direct = direct_bytes(row);
      const int bytes = unit_bytes(row, e0, d);
      if (sizeof(X) == 2 && direct != 0) {
        fetch_direct<X>(f.raw[j], row + i * 8, d - i * 8, direct);
      } else if (bytes == 8) {
        fetch_units<X, uint2>(f.raw[j], row + e0, lane);
      } else if (bytes == 4) {
        fetch_units<X, uint32_t>(f.raw[j], row + e0, lane);
      } else if (sizeof(X) == 2 && bytes == 2) {
        fetch_units<X, X>(f.raw[j], row + e0, lane);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int e = e0 + k * 32 + lane;
          const X one = e < d ? row[e] : from_float<X>(0.f);
          if constexpr (sizeof(X) == 4)
            f.raw[j].w[k] = *reinterpret_cast<const uint32_t*>(&one);
          else
            f.raw[j].w[k] = *reinterpret_cast<const uint16_t*>(&one);
        }
      }
    }
  }
}
template <typename X, int N, bool AL>
__device__ __forceinline__ void finish_row(Vec8<X> (&v)[N], const RowVectors<X, N, AL>& f, const X* row, int vec0,
                                           int stride, int d, X* stage) {
  if constexpr (AL) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = f.v[j];
  } else {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (sizeof(X) == 2 && direct_bytes(row) != 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j].set_word(k, f.raw[j].w[k]);
        continue;
      }
      const int bytes = unit_bytes(row, (vec0 + j * stride - lane) * 8, d);
      if (bytes == 8)
        place_units<X, uint2>(f.raw[j], stage, lane);
      else if (bytes == 4 && sizeof(X) == 2)
        place_units<X, uint32_t>(f.raw[j], stage, lane);
      else
        place_units<X, X>(f.raw[j], stage, lane);  // (fp32: the same units as for 4 bytes)
      __syncwarp();
      v[j].load(stage + lane * 8);
      __syncwarp();
    }
  }
}
// The way back for one vector per lane.
template <typename X, bool AL>
__device__ __forceinline__ void store_row(const Vec8<X>& v, X* row, int vec, int d, X* stage) {
  if constexpr (AL) {
    if (vec * 8 < d) v.store(row + vec * 8);
  } else {
    const int lane = threadIdx.x & 31;
    if (sizeof(X) == 2 && direct_bytes(row) == 8) {
      store_direct<X>(v, row + vec * 8, d - vec * 8);
      return;
    }
    const int e0 = (vec - lane) * 8;
    const int bytes = unit_bytes(row, e0, d);
    RawUnits raw;
    v.store(stage + lane * 8);
    __syncwarp();
    if (bytes == 8) {
      fetch_units<X, uint2>(raw, stage, lane);
      place_units<X, uint2>(raw, row + e0, lane);
    } else if (bytes == 4) {
      fetch_units<X, uint32_t>(raw, stage, lane);
      place_units<X, uint32_t>(raw, row + e0, lane);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int at = k * 32 + lane;
        if (e0 + at < d) row[e0 + at] = stage[at];
      }
    }
    __syncwarp();
  }
}

// ------------------------------------------------------- PTX: TMA and tcgen05 of the block-scaled product
// Waits at CTA scope: for phases that a copy or a commit completes (what they order lies in shared memory and TMEM, and
// is read by the tensor core).  mbar_peek_cta only looks, mbar_test_cta lets the hardware suspend the thread for a while.
__device__ __forceinline__ bool mbar_peek_cta(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_test_cta(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// The bounded wait at CTA scope; `seen`: the barrier's phase was already seen to be complete.
__device__ __forceinline__ bool mbar_wait_cta(uint32_t bar, uint32_t parity, bool seen, volatile int* abort_flag,
                                              long long limit_cycles = kWaitCycles) {
  if (seen || mbar_test_cta(bar, parity)) return true;
  const long long t0 = clock64();
  while (true) {
    if (mbar_test_cta(bar, parity)) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit_cycles) {
      *abort_flag = 1;
      return false;
    }
  }
}

// Three-dimensional form of tma_load_2d_pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst_smem, const void* tmap, int x, int y, int z,
                                                 uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%2, %3, %4}], [%5], %6;"
      ::"r"(dst_smem), "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
      : "memory");
}

// Tile store: shared memory (rows of the box one after another) -> global memory; what lies outside the tensor is left out.
__device__ __forceinline__ void tma_store_2d(const void* tmap, int x, int y, uint32_t src_smem, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.global.shared::cta.bulk_group.L2::cache_hint [%0, {%1, %2}], [%3], %4;"
      ::"l"(tmap), "r"(x), "r"(y), "r"(src_smem), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// At most N of this thread's committed stores still read shared memory.
template <int N>
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Makes this thread's shared-memory writes visible to the copies that follow.
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// The same, and whether `ok` held for all of its threads.
__device__ __forceinline__ bool named_barrier_and(int id, int threads, bool ok) {
  uint32_t all;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %3, 0;\n"
      "barrier.cta.red.and.pred q, %1, %2, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(all)
      : "r"(id), "r"(threads), "r"((uint32_t)ok)
      : "memory");
  return all != 0;
}
__device__ __forceinline__ uint64_t l2_policy_evict_first() {
  uint64_t pol;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
  return pol;
}

// Programmatic launches: a kernel may be made ready while the one before it in the stream still runs; it reads and
// writes memory only behind grid_wait(), which returns once that kernel has completed.  grid_release() lets the next one
// be made ready.
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Copies one scale word (32 lanes x 16 bytes, in each CTA of the pair from its own shared memory) to four TMEM
// columns, repeated in all four lane quarters.  Issued by the thread that issues the MMAs; a following MMA sees it.
__device__ __forceinline__ void tmem_copy_scales_pair(uint32_t taddr, uint64_t sdesc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(sdesc) : "memory");
}
// Shared-memory descriptor of a scale word: no swizzle, 8 x 16-byte core matrices 128 bytes apart.
__device__ __forceinline__ uint64_t umma_desc_scales(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(128 >> 4) << 16;
  d |= (uint64_t)(128 >> 4) << 32;
  d |= (uint64_t)1 << 46;  // descriptor version of sm_100
  return d;
}

// Instruction descriptor of the block-scaled kinds: fp32 accumulator, both operands K-major, power-of-two scales.
// The operands' type field is 0 for e4m3 among the 8-bit formats and 1 for e2m1 of the 4-bit kind.
template <int FMT>
__host__ __device__ constexpr uint32_t umma_idesc_mx(int M, int N) {
  return (FMT == kMx8 ? 0u : ((1u << 7) | (1u << 10))) | ((uint32_t)(N >> 3) << 17) | (1u << 23) |
         ((uint32_t)(M >> 4) << 24);
}
// Which byte of the scales' 32-bit TMEM cells the MMA starts with, for both operands.
__host__ __device__ constexpr uint32_t umma_idesc_scale_byte(uint32_t b) { return (b << 4) | (b << 29); }

// D[tmem] (+)= (A * scales_a) (B * scales_b)^T, 256 x N x 32 bytes of codes along K, issued by one thread of the
// pair's first CTA.  Each CTA's TMEM holds the scales of its own 128 rows of A and of all N rows of B.
template <int FMT>
__device__ __forceinline__ void umma_mx_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                             uint32_t tmem_sa, uint32_t tmem_sb, uint32_t accumulate) {
  if (FMT == kMx8) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n"
        "}\n"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(tmem_sa), "r"(tmem_sb)
        : "memory");
  } else {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n"
        "}\n"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(tmem_sa), "r"(tmem_sb)
        : "memory");
  }
}

// 32 lanes x 32 consecutive fp32 columns, and the wait for it (see tmem_ld_32x16 and tmem_ld_wait).
__device__ __forceinline__ void tmem_ld_32x32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_wait32(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                 "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                 "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                 "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

}  // namespace difr
