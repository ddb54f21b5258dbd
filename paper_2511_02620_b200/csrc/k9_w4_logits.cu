// LM-head product of bf16 hidden states with 4-bit weights:
//
//   l[t, v] = sum over k of h[t, k] code[v, k] scale[v, group of k]
//
// on the fp16 tensor cores, with exact products.  A code has four bits and a bf16 scale eight: with its sign a weight has
// at most eleven, which is what fp16 holds, and a bf16 hidden state has eight.  What fp16 lacks is range, so both operands
// go in with a power of two of their own: a token's row of h times 2^(14 - exponent of its largest value), prepared by
// `w4_prepare` in the workspace, an id's weights times 2^(10 - exponent of its largest scale).  The epilogue takes both
// back.  What is smaller than 2^-31 of its row's largest hidden state, or in a group whose scale is below 2^-27 of its id's
// largest, loses bits below 2^-39 (2^-35) of that largest.
//
// Weights: a thread turns words of eight codes into four pairs of fp16.  (word shifted & 0x03C003C0) ^ 0x4E004E00 are two
// numbers 24 + code, and one fma with (S, -24 S), S the scale, makes them code * S, exactly: 24 S has ten bits.  A pair is the
// codes k and k + 4 of its word.
//
// Two kernels, by the number of tokens alone; both take the vocabulary as the MMA's M side, read W once per token tile and
// give the same bits (an MMA adds the same sixteen products in either).
//
// Up to 16 tokens, `w4_few`: a warp takes 32 ids along all of k with mma.sync.  It brings its own codes and scales by TMA, two
// stages of two steps ahead, and meets nobody.  One token x 128256 x 4096 takes 62 to 64 us (43 of bytes), 16 tokens 84; a step
// of 16 ids is 167 instructions, 13 of them for each word of codes that becomes fp16.  (The other kernel takes 104 for one token.)
//
// More tokens, `w4_logits`: tcgen05.mma takes its A operand from TMEM, where the converted weights go; a lane is an id.  CTAs
// run as persistent pairs (cta_group::2) on tiles of 256 ids x BN tokens: each CTA loads and converts its own 128 ids and loads
// half of the tile's tokens, and the pair's first CTA issues the MMAs.  A step is 128 values of k: 64 TMEM columns of
// converted weights (a slot), a stage of h; a stage of codes is two steps.  TMEM: two accumulators and the slots; with BN =
// 256 the accumulators overlap by 128 columns, which the epilogue reads first.  4096 tokens x 128256 x 4096 take 2700 us in
// short runs (1.59 PFLOP/s), 2950 to 3150 sustained under the power cap (1.37 to 1.46); 64 tokens 109 to 115, which is about 1000
// clocks at 1965 MHz for each step of seven tiles.  Warps issue in 51 of 100 cycles then, DRAM is at 32 %: the chain of a step
// sets the time, of which no link was measured by itself.
//
// The tensor cores drop what lies below an accumulator's last bit, towards zero: logits lose 3e-6 of their size at d = 4096.  Parts of
// 1024 (2048) values added in fp32 bring that to 7e-7 (1.4e-6) at every d.  It was built, with the sums of a tile of 256 tokens in
// shared memory, and left out: 4096 tokens x 128256 x 4096 to bf16 3250 us with parts of 2048 for 3020, 777 x 32003 x 1749 to fp32
// 137 for 111 with parts of 1024, one token 66 for 62.
// Warps: 0 TMA of h, 1 MMA, 2 TMEM allocation, 3 TMA of codes, 4..11 epilogue (two per lane quarter, half of the tile's columns
// each), 12..19 conversion (two per lane quarter, even and odd steps, counted on from tile to tile).
//
// The order of k.  In mma.sync lane t of four holds, of a block of 128 values, the 32 at 32 t, four words, and an MMA adds pairs
// q = 0 and 1, or 2 and 3, of all four lanes' words w.  TMEM columns and h follow that: pair q of word w of lane t is column
// 8 (2 w + q / 2) + 4 (q & 1) + t of a step.  Where the last block has 64 values at most, lane t holds the 16 at 16 t, two words.
#include <cuda.h>
#include <cuda_runtime.h>
#include <string.h>

#include <type_traits>

#include "difr_kernels.h"
#include "logit_tiles.cuh"
#include "step_kernels.h"
#include "w4_device.cuh"

namespace difr {

constexpr int kW4EpiWarp0 = 4, kW4EpiWarps = 8, kW4CvtWarp0 = 12, kW4CvtWarps = 8;
constexpr int kW4Threads = 32 * (kW4CvtWarp0 + kW4CvtWarps);
constexpr int kW4TmemCols = 512;
constexpr int kW4Step = 128;        // values of k
constexpr int kW4SlotCols = 64;     // of a step: 128 fp16 a lane
constexpr int kW4CodeBytes = 128 * 128;  // a stage of codes: two steps of 128 ids

template <int BN>
struct W4Tile {
  static constexpr int tokens = BN;
  static constexpr int h_box = BN / 2 * 128;   // 64 values of half of the tokens
  static constexpr int h_bytes = 2 * h_box;
  static constexpr int bar_bytes = 1024;
  static constexpr int out_buffers = BN == 256 ? 3 : 0;
  static constexpr int out_bytes = 2 * out_buffers * kLogitOutBytes;
  static constexpr int h_stages = BN == 256 ? 4 : BN == 128 ? 5 : BN == 64 ? 6 : 8;
  static constexpr int fit = (227 * 1024 - 1024 - bar_bytes - out_bytes - h_stages * h_bytes) / kW4CodeBytes;
  static constexpr int c_stages = fit > 12 ? 12 : fit;
  static constexpr int smem_bytes = h_stages * h_bytes + c_stages * kW4CodeBytes + out_bytes + bar_bytes + 1024;
  static constexpr bool overlap = BN == 256;
  static constexpr int shared_cols = overlap ? 128 : 0;
  static constexpr int acc_stride = BN - shared_cols;
  static constexpr int slot_col0 = 2 * BN - shared_cols;
  static constexpr int fit_slots = (kW4TmemCols - slot_col0) / kW4SlotCols;
  static constexpr int slots = fit_slots > 4 ? 4 : fit_slots;
  // epilogue: columns per TMEM load, loads per accumulator, loads per half that cover the shared columns
  static constexpr int chunk = BN >= 64 ? 32 : 16;
  static constexpr int chunks = BN / chunk;
  static constexpr int shared_loads = shared_cols / (2 * chunk);
  static_assert(c_stages >= 3 && slots >= 2, "pipeline depth");
  static_assert((slots & (slots - 1)) == 0, "steps are counted modulo 2^32");
  static_assert(slots >= 2, "the steps of a conversion warp are two apart");
};

// Instruction descriptor: dense, fp32 accumulator, fp16 A and B, both K-major.
__host__ __device__ constexpr uint32_t umma_idesc_f16(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// D[tmem] (+)= A[tmem] * B[smem]^T over 16 values of k, 256 x N, issued by one thread of the pair's first CTA: each CTA's
// TMEM holds its own 128 rows of A, each CTA's shared memory half of B's rows.
__device__ __forceinline__ void umma_f16_tmem_pair(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc,
                                                   uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 32 lanes x 32 consecutive columns, and the wait for the thread's stores.
__device__ __forceinline__ void tmem_st_32x32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// An arrival that publishes no memory of this thread.  (A releasing one waits for every load that the thread has under way.)
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t bar_cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster_addr) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// ------------------------------------------------------------------ hidden states
// A row of h as fp16 times 2^e, e = 14 - exponent of its largest value, in pairs in the order of k told above, zeros to whole
// 64; and -10 - e, the token's share of what the epilogue takes back.  A row with a NaN or an infinity is NaN.  For
// `w4_few` the 16 bytes of a word's four pairs lie together: [block][word][token][lane].
// One CTA a token, a thread eight values at a time; the second reading finds them in L1.
constexpr int kPrepareMax = 1024;
__device__ __forceinline__ void load_eight(uint32_t (&v)[4], const unsigned short* h, int k, int d, bool vec) {
  if (vec && k + 8 <= d) {
    const uint4 q = *reinterpret_cast<const uint4*>(h + k);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = (k + 2 * i < d ? h[k + 2 * i] : 0u) | (k + 2 * i + 1 < d ? (uint32_t)h[k + 2 * i + 1] << 16 : 0u);
  }
}
__global__ void __launch_bounds__(kPrepareMax) w4_prepare(const W4LogitsParams p) {
  __shared__ uint32_t part[kPrepareMax / 32];
  grid_release();
  const int64_t token = blockIdx.x;
  const unsigned short* h = reinterpret_cast<const unsigned short*>(p.h) + token * p.ldh;
  const int d = p.d, eights = p.h16_pitch / 8;
  uint32_t top = 0;  // magnitudes of bf16 compare like their bits, and a NaN's or an infinity's are above every number's
  for (int i = threadIdx.x; i < eights; i += blockDim.x) {
    uint32_t v[4];
    load_eight(v, h, i * 8, d, p.h_vec);
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, max(v[j] & 0x7FFFu, (v[j] >> 16) & 0x7FFFu));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
  for (int w = 0; w < (int)blockDim.x / 32; ++w) top = max(top, part[w]);
  const bool broken = top >= 0x7F80u;
  const int e = broken || top == 0u ? 0 : 14 - (max((int)(top >> 7), 1) - 127);
  const float f1 = __int_as_float((127 + e / 2) << 23), f2 = __int_as_float((127 + e - e / 2) << 23);  // (|e| <= 141)
  if (threadIdx.x == 0) p.token_exp[token] = -10 - e;
  for (int i = threadIdx.x; i < eights; i += blockDim.x) {
    uint32_t v[4], pair[4];
    load_eight(v, h, i * 8, d, p.h_vec);
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // values q and q + 4
      const uint32_t a = (q & 1) ? v[q >> 1] & 0xFFFF0000u : v[q >> 1] << 16;
      const uint32_t b = (q & 1) ? v[2 + (q >> 1)] & 0xFFFF0000u : v[2 + (q >> 1)] << 16;
      __half2 two = __floats2half2_rn(__uint_as_float(a) * f1 * f2, __uint_as_float(b) * f1 * f2);
      if (broken) two = __half2half2(__ushort_as_half((unsigned short)0x7FFF));
      pair[q] = *reinterpret_cast<uint32_t*>(&two);
    }
    const int block = i >> 4, in = i & 15;
    const bool half = p.half_last && block == p.k_steps - 1;
    const int t = half ? in >> 1 : in >> 2, w = half ? in & 1 : in & 3;
    if (p.few) {
      reinterpret_cast<uint4*>(p.h16)[(((int64_t)block * 4 + w) * p.T + token) * 4 + t] = make_uint4(pair[0], pair[1], pair[2], pair[3]);
    } else {
      uint32_t* to = reinterpret_cast<uint32_t*>(p.h16) + token * (p.h16_pitch / 2) + block * 64 + 16 * w + t;
#pragma unroll
      for (int q = 0; q < 4; ++q) to[8 * (q >> 1) + 4 * (q & 1)] = pair[q];
    }
  }
}

// ------------------------------------------------------------------ scales
// Largest exponent field (times 2^7) of eight scales and `top`, NaN and infinities left out.
__device__ __forceinline__ uint32_t fold_scales(uint4 s, uint32_t top) {
  const uint32_t w[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = w[k] & 0x7F80u, hi = (w[k] >> 16) & 0x7F80u;
    if (lo != 0x7F80u) top = max(top, lo);
    if (hi != 0x7F80u) top = max(top, hi);
  }
  return top;
}
// The exponent (floor log2) that is, 0 where no scale counts; scales below 2^-126 count as zero.
__device__ __forceinline__ int scale_exponent(uint32_t top) { return top == 0u ? 0 : (int)(top >> 7) - 127; }
// Of a row's scales i0, i0 + step .. (eights).
__device__ __forceinline__ uint32_t fold_row(const __nv_bfloat16* scales, int i0, int step, int n8, uint32_t top) {
  constexpr int U = 4;
  for (int i = i0; i < n8; i += U * step) {
    uint4 s[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      s[u] = i + u * step < n8 ? __ldg(reinterpret_cast<const uint4*>(scales) + i + u * step) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < U; ++u) top = fold_scales(s[u], top);
  }
  return top;
}
// A scale times 2^(10 - exponent) as a pair of fp16.  That power as two factors: one would leave fp32 for tiny scales.  (An
// infinity ends as NaN: 24 times it is taken off.)
__device__ __forceinline__ float2 scale_factors(int exponent) {
  const int shift = 10 - exponent;
  return make_float2(__int_as_float((127 + shift / 2) << 23), __int_as_float((127 + shift - shift / 2) << 23));
}
__device__ __forceinline__ __half2 normal_scale(uint32_t bits16, float2 by) {
  return __float2half2_rn(__uint_as_float(bits16 << 16) * by.x * by.y);
}
// The scales of a step as they lie there, and one for each 32 of its 128 values.  (Two functions: what is done with a load
// right behind it waits for it there and then.  Spread out when it came in, a step of conversion took 1570 clocks.)
__device__ __forceinline__ uint2 load_step_scales(const __nv_bfloat16* scales, int step, int group) {
  uint2 raw = make_uint2(0u, 0u);
  if (group == 128)
    raw.x = __ldg(reinterpret_cast<const unsigned short*>(scales) + step);
  else if (group == 64)
    raw.x = __ldg(reinterpret_cast<const uint32_t*>(scales) + step);
  else
    raw = __ldg(reinterpret_cast<const uint2*>(scales) + step);
  return raw;
}
__device__ __forceinline__ uint2 spread_step_scales(uint2 raw, int group) {
  if (group == 32) return raw;
  const uint32_t lo = __byte_perm(raw.x, 0, 0x1010), hi = group == 128 ? lo : __byte_perm(raw.x, 0, 0x3232);
  return make_uint2(lo, hi);
}
// Eight codes -> four pairs of fp16.  (The logic as one instruction with both constants in registers: it takes one immediate
// only, and left to itself the compiler spent 14 of them on a word, which set the pace.  Shifts to the left go as products,
// so that they share a pipe with the fma and not with the logic.)
struct ConvertBits {
  uint32_t mask, magic;
};
__device__ __forceinline__ ConvertBits convert_bits() {
  ConvertBits b;
  asm volatile("mov.b32 %0, 0x03C003C0;" : "=r"(b.mask));
  asm volatile("mov.b32 %0, 0x4E004E00;" : "=r"(b.magic));
  return b;
}
// Pairs 2 e and 2 e + 1 of a word.
__device__ __forceinline__ void convert_half(uint32_t w, int e, __half2 scale, __half2 offset, ConvertBits k, uint32_t* out) {
  const uint32_t at[2] = {e == 0 ? w * 64u : w >> 2, e == 0 ? w * 4u : w >> 6};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t bits;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(bits) : "r"(at[i]), "r"(k.mask), "r"(k.magic));  // (a & b) ^ c
    const __half2 v = __hfma2(*reinterpret_cast<const __half2*>(&bits), scale, offset);
    out[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}
__device__ __forceinline__ void convert_word(uint32_t w, __half2 scale, __half2 offset, ConvertBits k, uint32_t* out) {
  convert_half(w, 0, scale, offset, k, out);
  convert_half(w, 1, scale, offset, k, out + 2);
}

// x times 2^e, e from -276 to 230, rounded once: where 2^e is no normal number, by way of fp64.
__device__ __forceinline__ float times_power(float x, int e) {
  if (e >= -126 && e <= 127) return x * __int_as_float((127 + e) << 23);
  return (float)((double)x * __hiloint2double((1023 + e) << 20, 0));
}
// Takes the powers of two back: r[j] times 2^(ids's exponent + token's).  `mine`: the exponent of token t0 + lane.
template <int N>
__device__ __forceinline__ void take_back(uint32_t (&r)[N], int id_exp, int mine) {
  const int lo = __reduce_min_sync(0xffffffffu, mine) + __reduce_min_sync(0xffffffffu, id_exp);
  const int hi = __reduce_max_sync(0xffffffffu, mine) + __reduce_max_sync(0xffffffffu, id_exp);
  if (lo >= -126 && hi <= 127) {
    const int bits = (127 + id_exp) << 23, more = mine << 23;
#pragma unroll
    for (int j = 0; j < N; ++j)
      r[j] = __float_as_uint(__uint_as_float(r[j]) * __int_as_float(bits + __shfl_sync(0xffffffffu, more, j)));
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      r[j] = __float_as_uint(times_power(__uint_as_float(r[j]), id_exp + __shfl_sync(0xffffffffu, mine, j)));
  }
}

// ------------------------------------------------------------------ up to 16 tokens
constexpr int kFewWarps = 2, kFewIds = kW4FewIds, kFewTiles = kFewIds / 16;
constexpr int kFewStages = 2, kFewStageBytes = kFewIds * 128;          // codes of two steps
constexpr int kFewScaleSlots = 4, kFewScaleBytes = kFewIds * 16;       // eight scales of each id
constexpr int kFewWarpBytes = kFewStages * kFewStageBytes + kFewScaleSlots * kFewScaleBytes;
constexpr int kFewSmem = kFewWarps * kFewWarpBytes + kFewWarps * kFewStages * 8 + 1024;  // + barriers, alignment

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t ld_shared_2(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void tma_load_2d_hint(uint32_t dst_smem, const void* tmap, int x, int y, uint32_t bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
      ::"r"(dst_smem), "l"(tmap), "r"(x), "r"(y), "r"(bar), "l"(policy)
      : "memory");
}

// The first of the ids of lanes 4 g .. 4 g + 3 among the warp's, the others 8 further each.
__device__ __forceinline__ int few_row(int g) { return ((g & 1) << 2) | (g >> 1); }
// A lane's logits (ids v, v + 8 ..) on their way out.  Not ok: a wait ran out, they are NaN and copies in flight get time to land.
template <int NT, typename OUT>
__device__ __forceinline__ void few_finish(const W4LogitsParams& p, const float (&acc)[kFewTiles][NT][4],
                                           const int (&id_exp)[2 * kFewTiles], bool ok, int64_t v_first, int t) {
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) { }
    if ((threadIdx.x & 31) == 0 && p.device_status != nullptr) *p.device_status = kStatusTimeout;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int token = n * 8 + 2 * t + j;
      if (token < p.T) {
        const int token_exp = ok ? p.token_exp[token] : 0;
        OUT* out = static_cast<OUT*>(p.logits) + (int64_t)token * p.ld;
#pragma unroll
        for (int r = 0; r < 2 * kFewTiles; ++r) {
          const int64_t v = v_first + 8 * r;
          const float value = ok ? acc[r >> 1][n][2 * (r & 1) + j] : __int_as_float(0x7FC00000);
          if (v < p.V) out[v] = from_float<OUT>(times_power(value, id_exp[r] + token_exp));
        }
      }
    }
}

// NT: tiles of eight tokens.
template <int NT, typename OUT>
__global__ void __launch_bounds__(32 * kFewWarps)
w4_few(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_s,
       const __grid_constant__ W4LogitsParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t code_ring = smem_base + (uint32_t)(warp * kFewStages * kFewStageBytes);
  const uint32_t scale_ring = smem_base + (uint32_t)(kFewWarps * kFewStages * kFewStageBytes + warp * kFewScaleSlots * kFewScaleBytes);
  const uint32_t bars = smem_base + (uint32_t)(kFewWarps * kFewWarpBytes + warp * kFewStages * 8);
  volatile int* abort_flag = &abort_word;
  if (threadIdx.x == 0) abort_word = 0;
  if (lane == 0) {
    for (int s = 0; s < kFewStages; ++s) mbar_init(bars + 8u * (uint32_t)s, 1);
    mbar_fence_init();
  }
  __syncthreads();
  const int64_t v0 = ((int64_t)blockIdx.x * kFewWarps + warp) * kFewIds;
  if (v0 >= p.V) return;  // (nothing below waits for another warp)

  const int n_stages = (p.k_steps + 1) / 2;
  const int scale_shift = p.group == 128 ? 2 : p.group == 64 ? 1 : 0;  // a scale is for 2^shift chunks of 32 codes
  const uint64_t policy = p.w_once ? l2_policy_evict_first() : l2_policy_evict_normal();
  int next = 0, next_slot = 0;  // stage to fetch, its place
  auto fetch = [&]() {
    if (lane == 0) {
      const uint32_t bar = bars + 8u * (uint32_t)next_slot;
      // (a slot of eight scales is for 2^shift stages)
      const int slot = next >> scale_shift;
      const bool with_scales = slot << scale_shift == next;
      mbar_arrive_expect_tx(bar, (uint32_t)(kFewStageBytes + (with_scales ? kFewScaleBytes : 0)));
      tma_load_2d_hint(code_ring + (uint32_t)(next_slot * kFewStageBytes), &tmap_w, next * 128, (int)v0, bar, policy);
      if (with_scales)
        tma_load_2d_hint(scale_ring + (uint32_t)(slot % kFewScaleSlots * kFewScaleBytes), &tmap_s, slot * 8, (int)v0, bar, policy);
    }
    ++next;
    if (++next_slot == kFewStages) next_slot = 0;
  };
  for (int s = 0; s < kFewStages && s < n_stages; ++s) fetch();
  // ids of this lane's two rows of the MMA: neighbours among the 16 bytes that eight lanes read at once lie in different halves
  // of the swizzled 128-byte lines
  const int at0 = few_row(g);
  const int64_t spitch = w4_scale_pitch(p.d, p.group);
  float2 by[2 * kFewTiles];
  int id_exp[2 * kFewTiles];
  {
    const int n8 = (int)(spitch / 8);
    auto scale_row = [&](int r) { return p.scales + min(v0 + at0 + 8 * r, (int64_t)p.V - 1) * spitch; };
    uint4 some[2 * kFewTiles];  // (all rows' first loads before the first is looked at)
#pragma unroll
    for (int r = 0; r < 2 * kFewTiles; ++r)
      some[r] = t < n8 ? __ldg(reinterpret_cast<const uint4*>(scale_row(r)) + t) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int r = 0; r < 2 * kFewTiles; ++r) {
      uint32_t top = fold_row(scale_row(r), t + 4, 4, n8, fold_scales(some[r], 0u));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      id_exp[r] = scale_exponent(top);
      by[r] = scale_factors(id_exp[r]);
    }
  }
  grid_wait();  // h comes from the kernel before
  // [block][word][token][lane]; lanes without a token read another one's, for columns that nobody looks at
  const unsigned char* h[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) h[n] = reinterpret_cast<const unsigned char*>(p.h16) + (min(n * 8 + g, p.T - 1) * 4 + t) * 16;
  const uint32_t h_word = (uint32_t)p.T * 64u;
  float acc[kFewTiles][NT][4] = {};
  const __half2 minus24 = __float2half2_rn(-24.f);
  const ConvertBits k = convert_bits();
  // One step: codes and scales of this lane's ids, and h, of which `words` words are there.  `between`: called behind the first of
  // the tiles.
  auto take = [&](const uint4 (&c)[2 * kFewTiles], const uint32_t (&s)[2 * kFewTiles], auto words, auto between) {
    constexpr int W = decltype(words)::value;
    uint4 b[NT][W];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int w = 0; w < W; ++w) b[n][w] = *reinterpret_cast<const uint4*>(h[n] + w * h_word);
      h[n] += 4 * h_word;
    }
#pragma unroll
    for (int m = 0; m < kFewTiles; ++m) {
      const __half2 scale0 = normal_scale(s[2 * m], by[2 * m]), scale1 = normal_scale(s[2 * m + 1], by[2 * m + 1]);
      const __half2 offset0 = __hmul2(scale0, minus24), offset1 = __hmul2(scale1, minus24);
      const uint32_t w0[4] = {c[2 * m].x, c[2 * m].y, c[2 * m].z, c[2 * m].w};
      const uint32_t w1[4] = {c[2 * m + 1].x, c[2 * m + 1].y, c[2 * m + 1].z, c[2 * m + 1].w};
#pragma unroll
      for (int w = 0; w < W; ++w) {
        uint32_t a[4], a8[4];
        convert_word(w0[w], scale0, offset0, k, a);
        convert_word(w1[w], scale1, offset1, k, a8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_f16(acc[m][n], a[0], a8[0], a[1], a8[1], b[n][w].x, b[n][w].y);
          mma_f16(acc[m][n], a[2], a8[2], a[3], a8[3], b[n][w].z, b[n][w].w);
        }
      }
      if (m == 0) between();
    }
  };
  auto nothing = []() {};
  // of a stage: the line of this lane's first id (the others 8 lines further each), 16 bytes for each of eight chunks of 32
  // codes; of a slot of scales its first id's
  const uint32_t line = code_ring + (uint32_t)(at0 * 128), swizzle = (uint32_t)at0;
  const uint32_t scale_line = scale_ring + (uint32_t)(at0 * 16);
  uint4 c[2 * kFewTiles];
  uint32_t s[2 * kFewTiles];
  auto load = [&](uint32_t stage_line, int chunk, uint32_t row_chunk) {
    const uint32_t x = stage_line + (((uint32_t)chunk ^ swizzle) << 4);
    const uint32_t i = row_chunk >> scale_shift;
    const uint32_t y = scale_line + (i >> 3) % kFewScaleSlots * kFewScaleBytes + (i & 7u) * 2u;
#pragma unroll
    for (int r = 0; r < 2 * kFewTiles; ++r) {
      c[r] = ld_shared_16(x + 1024u * (uint32_t)r);
      s[r] = ld_shared_2(y + 128u * (uint32_t)r);
    }
  };
  const uint32_t none = (uint32_t)p.h16_pitch & 63u;  // 0, which the compiler does not know: rows of h16 are whole 64 values
  bool ok = true;
  const int whole = (p.k_steps - (p.half_last ? 1 : 0)) / 2;  // stages of two whole steps
  int slot = 0;
  uint32_t phase = 0;
  for (int i = 0; i < whole; ++i) {
    ok = __all_sync(0xffffffffu, mbar_wait_cta(bars + 8u * (uint32_t)slot, phase, false, abort_flag));
    if (!ok) break;
    const uint32_t from = line + (uint32_t)(slot * kFewStageBytes);
    load(from, t, (uint32_t)(8 * i + t));
    take(c, s, std::integral_constant<int, 4>(), nothing);
    load(from, t + 4, (uint32_t)(8 * i + 4 + t));
    // The stage may be filled again once all lanes' reads of it have returned.  Nothing but their values shows that here: the
    // arrival in fetch() is waited for by nobody, and a read held up behind others of its SM can be overtaken by a copy from L2.
    // So the refill hangs on a vote over what was read.  With one tile of tokens it waits until half of that has been worked on,
    // so that nothing waits for the reads (one token 63.5 us, 69.8 with the vote right behind them); with two the reads have
    // returned by then anyway, and the loop is better in one piece (16 tokens 82 us, 94 the other way).
    auto refill = [&]() {
      uint32_t seen = 0;
#pragma unroll
      for (int r = 0; r < 2 * kFewTiles; ++r) seen |= c[r].x | s[r];
      if (__all_sync(0xffffffffu, (seen & none) == 0u) && next < n_stages) fetch();
    };
    if constexpr (NT == 1) {
      take(c, s, std::integral_constant<int, 4>(), refill);
    } else {
      refill();
      take(c, s, std::integral_constant<int, 4>(), nothing);
    }
    if (++slot == kFewStages) { slot = 0; phase ^= 1u; }
  }
  if (ok && whole < n_stages) {  // a whole step, a half one, or both
    ok = __all_sync(0xffffffffu, mbar_wait_cta(bars + 8u * (uint32_t)slot, phase, false, abort_flag));
    const uint32_t from = line + (uint32_t)(slot * kFewStageBytes);
    int step = 2 * whole;
    if (ok && step < p.k_steps - (p.half_last ? 1 : 0)) {
      load(from, t, (uint32_t)(4 * step + t));
      take(c, s, std::integral_constant<int, 4>(), nothing);
      ++step;
    }
    if (ok && step < p.k_steps) {  // lanes t and t + 1 share a chunk, eight bytes each
      load(from, (step & 1) * 4 + (t >> 1), (uint32_t)(4 * step + (t >> 1)));
      if (t & 1) {
#pragma unroll
        for (int r = 0; r < 2 * kFewTiles; ++r) {
          c[r].x = c[r].z;
          c[r].y = c[r].w;
        }
      }
      take(c, s, std::integral_constant<int, 2>(), nothing);
    }
  }
  few_finish<NT, OUT>(p, acc, id_exp, ok, v0 + at0, t);
}

// What w4_few ends with where a wait runs out, without a product: its warps, the barrier of each never arrived at.
template <int NT, typename OUT>
__global__ void __launch_bounds__(32 * kFewWarps)
w4_few_wait_selftest(const __grid_constant__ W4LogitsParams p, long long limit_cycles) {
  __shared__ uint64_t bars[kFewWarps];
  __shared__ int abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  if (threadIdx.x == 0) abort_word = 0;
  if (lane == 0) {
    mbar_init(smem_u32(&bars[warp]), 1);
    mbar_fence_init();
  }
  __syncthreads();
  const int64_t v0 = ((int64_t)blockIdx.x * kFewWarps + warp) * kFewIds;
  if (v0 >= p.V) return;
  const bool ok = __all_sync(0xffffffffu, mbar_wait_cta(smem_u32(&bars[warp]), 0, false, &abort_word, limit_cycles));
  const float acc[kFewTiles][NT][4] = {};
  const int id_exp[2 * kFewTiles] = {};
  few_finish<NT, OUT>(p, acc, id_exp, ok, v0 + few_row(g), t);
}

// ------------------------------------------------------------------ more tokens
template <int BN, typename OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kW4Threads, 1)
w4_logits(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_h,
          const __grid_constant__ CUtensorMap tmap_h_last, const __grid_constant__ CUtensorMap tmap_out,
          const __grid_constant__ W4LogitsParams p) {
  using Tl = W4Tile<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t smem_base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - raw_addr);

  // Both CTAs of a pair lay out their barriers at the same offsets.
  //   h_full[s]   first CTA's copy is used: 1 arrival (its producer) + the bytes of both CTAs' loads
  //   h_empty[s]  each CTA's own copy: 1 arrival, the commit of the MMAs that read the stage, delivered to both
  //   c_full[s]   own: 1 arrival + the bytes of the CTA's codes;  c_empty[s] own: one arrival per conversion warp
  //   a_full[s]   first CTA's copy is used: one arrival per conversion warp of the step, of both CTAs
  //   a_empty[s]  each CTA's own copy: the commit of the MMAs that read the slot, delivered to both
  //   acc_full[a], acc_free[a]  as in the microscaled product
  constexpr int HS = Tl::h_stages, CS = Tl::c_stages, AS = Tl::slots;
  const uint32_t h_base = smem_base, c_base = smem_base + HS * Tl::h_bytes;
  uint8_t* out_pieces = smem + HS * Tl::h_bytes + CS * kW4CodeBytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(out_pieces + Tl::out_bytes);
  const uint32_t bar0 = smem_u32(bars);
  auto h_full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
  auto h_empty = [&](int s) { return bar0 + 8u * (uint32_t)(HS + s); };
  auto c_full = [&](int s) { return bar0 + 8u * (uint32_t)(2 * HS + s); };
  auto c_empty = [&](int s) { return bar0 + 8u * (uint32_t)(2 * HS + CS + s); };
  auto a_full = [&](int s) { return bar0 + 8u * (uint32_t)(2 * HS + 2 * CS + s); };
  auto a_empty = [&](int s) { return bar0 + 8u * (uint32_t)(2 * HS + 2 * CS + AS + s); };
  auto acc_full = [&](int a) { return bar0 + 8u * (uint32_t)(2 * HS + 2 * CS + 2 * AS + a); };
  auto acc_free = [&](int a) { return bar0 + 8u * (uint32_t)(2 * HS + 2 * CS + 2 * AS + 2 + a); };
  constexpr int kBars = 2 * HS + 2 * CS + 2 * AS + 4;
  static_assert(kBars * 8 + 8 <= Tl::bar_bytes, "barrier block");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t cta = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  const int n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < HS; ++s) {
      mbar_init(h_full(s), 1);
      mbar_init(h_empty(s), 1);
    }
    for (int s = 0; s < CS; ++s) {
      mbar_init(c_full(s), 1);
      mbar_init(c_empty(s), kW4CvtWarps);
    }
    for (int s = 0; s < AS; ++s) {
      mbar_init(a_full(s), kW4CvtWarps);  // four warps of a step, of two CTAs
      mbar_init(a_empty(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full(a), 1);
      mbar_init(acc_free(a), 2 * kW4EpiWarps);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmap_w);
    tma_prefetch_desc(&tmap_h);
    tma_prefetch_desc(&tmap_h_last);
  }
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(tmem_slot), kW4TmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  TileWalk walk(p, pair, n_pairs);
  const int c_steps = (p.k_steps + 1) / 2;  // stages of codes per tile

  // (The kernel may start while `w4_prepare` runs; what that writes, h and the tokens' exponents, is read behind grid_wait().
  // Codes and scales were there before it.)
  if (warp == 0) {
    // ------------------------------------------------------------ TMA of h
    grid_wait();
    const uint64_t keep = l2_policy_evict_last();
    const uint32_t full0_base = map_to_cta(h_full(0), 0);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    int vt, tt;
    while (ok && walk.next(vt, tt)) {
      const bool last = tt == p.n_tt - 1;
      const int half = last ? p.last_tokens / 2 : BN / 2;
      const void* tmap_tokens = last ? &tmap_h_last : &tmap_h;
      const int h_row = tt * BN + (int)cta * half;
      for (int k = 0; k < p.k_steps; ++k) {
        if (!__all_sync(0xffffffffu, mbar_wait(h_empty(stage), phase ^ 1u, abort_flag))) { ok = false; break; }
        if (elect_one()) {
          // (the second box of the last step may lie behind the row: it reads zeros)
          if (cta == 0) mbar_arrive_expect_tx(h_full(stage), 2u * 2u * (uint32_t)half * 128u);
          const uint32_t full0 = full0_base + 8u * (uint32_t)stage;
          const uint32_t dst = h_base + (uint32_t)(stage * Tl::h_bytes);
          tma_load_2d_pair(dst, tmap_tokens, k * kW4Step, h_row, full0, keep);
          tma_load_2d_pair(dst + Tl::h_box, tmap_tokens, k * kW4Step + 64, h_row, full0, keep);
        }
        __syncwarp();
        if (++stage == HS) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 3) {
    // ---------------------------------------------------------- TMA of codes
    const uint64_t stream = p.w_once ? l2_policy_evict_first() : l2_policy_evict_normal();
    const uint32_t full_base = map_to_cta(c_full(0), cta);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    int vt, tt;
    while (ok && walk.next(vt, tt)) {
      const int w_row = vt * kLogitPairM + (int)cta * 128;
      for (int k = 0; k < c_steps; ++k) {
        if (!__all_sync(0xffffffffu, mbar_wait(c_empty(stage), phase ^ 1u, abort_flag))) { ok = false; break; }
        if (elect_one()) {
          mbar_arrive_expect_tx(c_full(stage), (uint32_t)kW4CodeBytes);
          tma_load_2d_pair(c_base + (uint32_t)(stage * kW4CodeBytes), &tmap_w, k * 128, w_row, full_base + 8u * (uint32_t)stage,
                           stream);
        }
        __syncwarp();
        if (++stage == CS) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    if (cta == 0) {
      const uint64_t desc0 = umma_desc_k_major_sw128(h_base);
      const uint32_t desc_hi = (uint32_t)(desc0 >> 32), desc_lo0 = (uint32_t)desc0;
      int stage = 0, slot = 0, acc = 0;
      uint32_t phase = 0, slot_phase = 0, n_tile = 0;
      bool ok = true;
      int vt, tt;
      for (; ok && walk.next(vt, tt); ++n_tile) {
        const uint32_t idesc = umma_idesc_f16(kLogitPairM, tt == p.n_tt - 1 ? p.last_tokens : BN);
        // Separate accumulators: the tile before last has been read.  Overlapping ones: the shared columns of the last
        // tile have been read (every epilogue warp had then finished the tile before it).
        if (Tl::overlap) {
          if (n_tile >= 1 && !__all_sync(0xffffffffu, mbar_wait(acc_free(acc ^ 1), ((n_tile - 1) >> 1) & 1u, abort_flag))) {
            ok = false;
            break;
          }
        } else {
          if (n_tile >= 2 && !__all_sync(0xffffffffu, mbar_wait(acc_free(acc), ((n_tile - 2) >> 1) & 1u, abort_flag))) {
            ok = false;
            break;
          }
        }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * Tl::acc_stride);
        // (a last token tile narrower than the others has its boxes closer together in the stage all the same)
        uint32_t accumulate = 0;
        for (int k = 0; k < p.k_steps; ++k) {
          if (!__all_sync(0xffffffffu, mbar_wait(h_full(stage), phase, abort_flag))) { ok = false; break; }
          if (!__all_sync(0xffffffffu, mbar_wait(a_full(slot), slot_phase, abort_flag))) { ok = false; break; }
          tc_fence_after();
          const int n_mma = p.half_last && k + 1 == p.k_steps ? 4 : 8;
          const uint32_t b_lo = desc_lo0 + ((uint32_t)(stage * Tl::h_bytes) >> 4);
          const uint32_t a_tmem = tmem_base + (uint32_t)(Tl::slot_col0 + slot * kW4SlotCols);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < kW4Step / 16; ++kk) {
              if (kk < n_mma) {
                const uint64_t b_desc =
                    ((uint64_t)desc_hi << 32) | (b_lo + (uint32_t)(kk >> 2) * (Tl::h_box >> 4) + 2u * (uint32_t)(kk & 3));
                umma_f16_tmem_pair(d_tmem, a_tmem + 8u * (uint32_t)kk, b_desc, idesc, kk == 0 ? accumulate : 1u);
              }
            }
            umma_commit_pair(h_empty(stage), 3);
            umma_commit_pair(a_empty(slot), 3);
          }
          __syncwarp();
          accumulate = 1;
          if (++stage == HS) { stage = 0; phase ^= 1u; }
          if (++slot == AS) { slot = 0; slot_phase ^= 1u; }
        }
        if (ok && elect_one()) umma_commit_pair(acc_full(acc), 3);
        __syncwarp();
        acc ^= 1;
      }
    }
  } else if (warp >= kW4CvtWarp0) {
    // -------------------------------------------------------------- conversion
    const int quarter = warp & 3;  // the TMEM lane quarter this warp may write
    const int odd = (warp - kW4CvtWarp0) >> 2;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const int r = quarter * 32 + lane;  // row of the CTA's 128
    const uint32_t row_smem = c_base + (uint32_t)r * 128u, swizzle = (uint32_t)(r & 7);
    const uint32_t full0_base = map_to_cta(a_full(0), 0);
    const int64_t spitch = w4_scale_pitch(p.d, p.group);
    const __half2 minus24 = __float2half2_rn(-24.f);
    const ConvertBits bits = convert_bits();
    int stage = 0;
    uint32_t phase = 0, step0 = 0;  // steps of the tiles before
    bool ok = true;
    int vt, tt;
    while (ok && walk.next(vt, tt)) {
      const int v = min(vt * kLogitPairM + (int)cta * 128 + r, p.V - 1);
      const __nv_bfloat16* scales = p.scales + (int64_t)v * spitch;
      const float2 by = scale_factors(scale_exponent(fold_row(scales, 0, 1, (int)(spitch / 8), 0u)));
      // The steps of a warp are two apart, from tile to tile as well: a wait for a slot tells its phases apart only while this warp
      // knows the phase before the awaited one to be complete, from its own last wait, and with two slots that is two steps back.
      const int first = odd ^ (int)(step0 & 1u);
      uint2 raw = first < p.k_steps ? load_step_scales(scales, first, p.group) : make_uint2(0u, 0u);
      for (int k = 0; k < c_steps; ++k) {
        const int step = 2 * k + first;
        if (!__all_sync(0xffffffffu, mbar_wait_cta(c_full(stage), phase, false, abort_flag))) { ok = false; break; }
        if (step < p.k_steps) {
          const uint32_t from = row_smem + (uint32_t)(stage * kW4CodeBytes);
          uint4 c[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) c[j] = ld_shared_16(from + ((((uint32_t)(first * 4 + j)) ^ swizzle) << 4));
          const bool half_step = p.half_last && step == p.k_steps - 1;
          uint2 here = spread_step_scales(raw, p.group);
          if (step + 2 < p.k_steps) raw = load_step_scales(scales, step + 2, p.group);
          if (half_step) {  // lane t of mma.sync: the 16 codes at 16 t
            here = make_uint2(__byte_perm(here.x, 0, 0x1010), __byte_perm(here.x, 0, 0x3232));
            c[3].x = c[1].z; c[3].y = c[1].w;
            c[2].x = c[1].x; c[2].y = c[1].y;
            c[1].x = c[0].z; c[1].y = c[0].w;
          }
          __half2 s[4], off[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t two = t < 2 ? here.x : here.y;
            s[t] = normal_scale((t & 1) == 0 ? two : two >> 16, by);
            off[t] = __hmul2(s[t], minus24);
          }
          const uint32_t g = step0 + (uint32_t)step;
          const uint32_t slot = g % (uint32_t)AS, slot_phase = (g / (uint32_t)AS) & 1u;
          const uint32_t to = tmem_base + lane_addr + (uint32_t)Tl::slot_col0 + slot * kW4SlotCols;
#pragma unroll
          for (int half = 0; half < 2; ++half) {  // words 2 half and 2 half + 1 of the four chunks
            uint32_t out[32];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                uint32_t four[4];
                convert_word(half == 0 ? (w == 0 ? c[t].x : c[t].y) : (w == 0 ? c[t].z : c[t].w), s[t], off[t], bits, four);
#pragma unroll
                for (int q = 0; q < 4; ++q) out[8 * (2 * w + (q >> 1)) + 4 * (q & 1) + t] = four[q];
              }
            }
            if (half == 0) {
              if (!__all_sync(0xffffffffu, mbar_wait_cta(a_empty((int)slot), slot_phase ^ 1u, false, abort_flag))) {
                ok = false;
                break;
              }
              tc_fence_after();
            }
            tmem_st_32x32(to + 32u * (uint32_t)half, out);  // (the second half of a half step: columns that no MMA reads)
          }
          if (!ok) break;
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_relaxed(full0_base + 8u * slot);  // (TMEM writes are ordered by the fence above)
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(c_empty(stage));
        if (++stage == CS) { stage = 0; phase ^= 1u; }
      }
      step0 += (uint32_t)p.k_steps;
    }
  } else if (warp >= kW4EpiWarp0) {
    // ---------------------------------------------------------------- epilogue
    grid_wait();
    const int quarter = warp & 3;  // the TMEM lane quarter this warp may read
    const int half = (warp - kW4EpiWarp0) >> 2;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const int64_t spitch = w4_scale_pitch(p.d, p.group);
    int acc = 0;
    uint32_t acc_phase = 0;
    OutPieces<OUT> pieces;
    pieces.buf = reinterpret_cast<OUT*>(out_pieces + half * (Tl::out_bytes / 2));
    pieces.next = 0;
    pieces.policy = l2_policy_evict_first();
    int vt, tt;
    bool given_up = false;
    while (walk.next(vt, tt)) {
      const int v = vt * kLogitPairM + (int)cta * 128 + quarter * 32 + lane;
      const int id_exp = scale_exponent(fold_row(p.scales + (int64_t)min(v, p.V - 1) * spitch, 0, 1, (int)(spitch / 8), 0u));
      const bool ok = mbar_wait_cta(acc_full(acc), acc_phase, false, abort_flag);
      __syncwarp();
      tc_fence_after();
      const uint32_t free_bar = map_to_cta(acc_free(acc), 0);
      // A tile store cuts rows at whole 16 bytes only: where the last ids end inside such a piece, they leave by plain
      // stores.
      const int v_block = v - quarter * 32 - lane;
      const bool by_tile = BN == 256 && p.tile_stores &&
                           (v_block + 128 <= p.V || p.V % (16 / (int)sizeof(OUT)) == 0);
      constexpr int kLoads = (Tl::chunks + 1) / 2;
      // where the accumulators overlap, the shared columns are read first, all of them before the first store
      constexpr int kFirst = Tl::overlap ? Tl::shared_loads : 1;
      uint32_t r[kFirst][Tl::chunk];
      auto load = [&](int c, int n) {
#pragma unroll
        for (int q = 0; q < kFirst; ++q) {
          const int ch = epi_chunk<Tl>(c + q, half, acc);
          if (q < n && ch >= 0 && tt * BN + ch * Tl::chunk < p.T) {
            const uint32_t taddr = tmem_base + lane_addr + (uint32_t)(acc * Tl::acc_stride + ch * Tl::chunk);
            if constexpr (Tl::chunk == 32) tmem_ld_32x32(taddr, r[q]); else tmem_ld_32x16(taddr, r[q]);
          }
        }
#pragma unroll
        for (int q = 0; q < kFirst; ++q) {
          if constexpr (Tl::chunk == 32) tmem_ld_wait32(r[q]); else tmem_ld_wait(r[q]);
        }
      };
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_nofence(free_bar);
      };
      if (ok) {
        load(0, kFirst);
        if (Tl::overlap || kLoads == 1) release();
      }
      // (the warps of a half meet at barriers below, so they give up together or not at all)
      given_up = BN == 256 ? !named_barrier_and(1 + half, 128, ok) : !__all_sync(0xffffffffu, ok);
      if (given_up) break;
#pragma unroll 1
      for (int c = 0; c < kLoads;) {
        const int n_here = c == 0 ? kFirst : 1;
#pragma unroll
        for (int q = 0; q < kFirst; ++q) {
          const int ch = epi_chunk<Tl>(c + q, half, acc);
          const int t0 = tt * BN + ch * Tl::chunk;
          if (q < n_here && ch >= 0 && t0 < p.T) {
            const int t = t0 + (lane & (Tl::chunk - 1));
            take_back<Tl::chunk>(r[q], id_exp, t < p.T ? p.token_exp[t] : 0);
            if constexpr (BN == 256) {
              if (by_tile) {
                pieces.template store<Tl::out_buffers>(p, &tmap_out, r[q], t0, v_block, quarter, lane, half);
                continue;
              }
            }
            store_chunk<Tl::chunk>(p, r[q], t0, v, static_cast<OUT*>(nullptr));
          }
        }
        c += n_here;
        if (c < kLoads) {
          load(c, 1);
          if (!Tl::overlap && c == kLoads - 1) release();
        }
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
    if (BN == 256 && p.tile_stores) bulk_wait_all();  // the pieces stay until they have left
    if (given_up) fill_given_up<Tl, OUT>(p, walk, vt, tt, acc, half, (int)cta * 128 + quarter * 32 + lane);
  }

  __syncwarp();
  if (*abort_flag) {
    // a wait ran out somewhere: give copies and MMAs still in flight time to land before TMEM is released
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000LL) { }
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, kW4TmemCols);
  }
  if (threadIdx.x == 0 && *abort_flag && p.device_status != nullptr) *p.device_status = kStatusTimeout;
}

// ------------------------------------------------------------------ launcher
// `w4_prepare`, and the kernel that may start while it runs.
template <typename... P, typename... A>
static cudaError_t launch_after_prepare(const W4LogitsParams& p, void (*kernel)(P...), int grid, int threads, int smem,
                                        cudaStream_t stream, const A&... args) {
  const int eights = p.h16_pitch / 8;
  w4_prepare<<<p.T, eights >= kPrepareMax ? kPrepareMax : (eights + 31) / 32 * 32, 0, stream>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)grid, 1, 1);
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  memset(&attr, 0, sizeof attr);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int BN, typename OUT>
static cudaError_t launch_tile(const CUtensorMap& w, const CUtensorMap& h, const CUtensorMap& hl, const CUtensorMap& out,
                               const W4LogitsParams& p, int grid, cudaStream_t stream) {
  const cudaError_t e =
      cudaFuncSetAttribute(w4_logits<BN, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, W4Tile<BN>::smem_bytes);
  if (e != cudaSuccess) return e;
  return launch_after_prepare(p, w4_logits<BN, OUT>, grid, kW4Threads, W4Tile<BN>::smem_bytes, stream, w, h, hl, out, p);
}

template <typename OUT>
static cudaError_t launch_typed(int bn, const CUtensorMap& w, const CUtensorMap& h, const CUtensorMap& hl,
                                const CUtensorMap& out, const W4LogitsParams& p, int grid, cudaStream_t stream) {
  switch (bn) {
    case 32: return launch_tile<32, OUT>(w, h, hl, out, p, grid, stream);
    case 64: return launch_tile<64, OUT>(w, h, hl, out, p, grid, stream);
    case 128: return launch_tile<128, OUT>(w, h, hl, out, p, grid, stream);
    case 256: return launch_tile<256, OUT>(w, h, hl, out, p, grid, stream);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_w4_logits(int tokens_per_tile, int dtype, const CUtensorMap& w, const CUtensorMap& h,
                             const CUtensorMap& h_last, const CUtensorMap& out, const W4LogitsParams& p, int grid,
                             cudaStream_t stream) {
  return dtype == kBf16 ? launch_typed<__nv_bfloat16>(tokens_per_tile, w, h, h_last, out, p, grid, stream)
                        : launch_typed<float>(tokens_per_tile, w, h, h_last, out, p, grid, stream);
}

template <int NT, typename OUT>
static cudaError_t launch_few(const CUtensorMap& w, const CUtensorMap& s, const W4LogitsParams& p, cudaStream_t stream) {
  const cudaError_t e = cudaFuncSetAttribute(w4_few<NT, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
  if (e != cudaSuccess) return e;
  const int grid = (int)((p.V + (int64_t)kFewIds * kFewWarps - 1) / (kFewIds * kFewWarps));
  return launch_after_prepare(p, w4_few<NT, OUT>, grid, 32 * kFewWarps, kFewSmem, stream, w, s, p);
}
cudaError_t launch_w4_few(int dtype, const CUtensorMap& w, const CUtensorMap& s, const W4LogitsParams& p, cudaStream_t stream) {
  if (dtype == kBf16)
    return p.T <= 8 ? launch_few<1, __nv_bfloat16>(w, s, p, stream) : launch_few<2, __nv_bfloat16>(w, s, p, stream);
  return p.T <= 8 ? launch_few<1, float>(w, s, p, stream) : launch_few<2, float>(w, s, p, stream);
}

template <typename OUT>
static cudaError_t launch_selftest(int bn, const W4LogitsParams& p, int done, long long limit, int grid, cudaStream_t stream) {
  if (p.few) {
    if (done > 0) return cudaSuccess;  // (a warp has one tile)
    const int few_grid = (int)((p.V + (int64_t)kFewIds * kFewWarps - 1) / (kFewIds * kFewWarps));
    if (p.T <= 8)
      w4_few_wait_selftest<1, OUT><<<few_grid, 32 * kFewWarps, 0, stream>>>(p, limit);
    else
      w4_few_wait_selftest<2, OUT><<<few_grid, 32 * kFewWarps, 0, stream>>>(p, limit);
    return cudaGetLastError();
  }
  switch (bn) {
    case 32: logit_wait_selftest<W4Tile<32>, OUT><<<grid, kLogitEpiThreads, 0, stream>>>(p, done, limit); break;
    case 64: logit_wait_selftest<W4Tile<64>, OUT><<<grid, kLogitEpiThreads, 0, stream>>>(p, done, limit); break;
    case 128: logit_wait_selftest<W4Tile<128>, OUT><<<grid, kLogitEpiThreads, 0, stream>>>(p, done, limit); break;
    default: logit_wait_selftest<W4Tile<256>, OUT><<<grid, kLogitEpiThreads, 0, stream>>>(p, done, limit); break;
  }
  return cudaGetLastError();
}
cudaError_t launch_w4_wait_selftest(int tokens_per_tile, int dtype, const W4LogitsParams& p, int done_tiles,
                                    long long limit_cycles, int grid, cudaStream_t stream) {
  return dtype == kBf16 ? launch_selftest<__nv_bfloat16>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream)
                        : launch_selftest<float>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream);
}

}  // namespace difr
