// Device-side building blocks of 4-bit weights with group scales.
//
// A tensor [rows, d]: every value is an integer code -8 .. 7 in two's complement times the bf16 scale of its group (32, 64
// or 128 values along a row).  Codes two to a byte, the even column in the low half, rows of whole 32 columns; scales in
// rows of whole 8.
#pragma once
#include "mx_device.cuh"

namespace difr {

__host__ __device__ __forceinline__ int64_t w4_pitch_bytes(int64_t d) { return (d + 31) / 32 * 16; }
__host__ __device__ __forceinline__ int64_t w4_scale_pitch(int64_t d, int group) { return ((d + group - 1) / group + 7) / 8 * 8; }

// Values 2 i and 2 i + 1 of the eight codes of a word.  ((code ^ 8) + 2^23) as fp32 bits, 2^23 + 8 taken off.  (The logic as
// one instruction, its constants in registers: it takes one immediate only.)
__device__ __forceinline__ float2 w4_pair(uint32_t word, int i) {
  uint32_t a, b, magic;
  asm("mov.b32 %0, 0x4B000008;" : "=r"(magic));
  asm("lop3.b32 %0, %1, 15, %2, 0x6A;" : "=r"(a) : "r"(word >> (8 * i)), "r"(magic));  // (a & b) ^ c
  asm("lop3.b32 %0, %1, 15, %2, 0x6A;" : "=r"(b) : "r"(word >> (8 * i + 4)), "r"(magic));
  return fadd2(make_float2(__uint_as_float(a), __uint_as_float(b)), make_float2(-8388616.f, -8388616.f));
}

}  // namespace difr
