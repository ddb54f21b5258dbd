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
// The vocabulary is the MMA's M side, as in the microscaled product.  Weights become fp16 on their way from shared memory to
// TMEM, where the MMA takes its A operand from: a lane is an id, a thread turns words of eight codes into four pairs.
// (word shifted & 0x03C003C0) ^ 0x4E004E00 are two numbers 24 + code in fp16, and one fma with (S, -24 S), S the scale, makes
// them code * S, exactly: 24 S has ten bits.  A pair is the codes k and k + 4 of its eight, so `w4_prepare` lays out h in the
// order 0 4 1 5 2 6 3 7.
//
// CTAs run as persistent pairs (cta_group::2) on tiles of 256 ids x BN tokens: each CTA loads and converts its own 128 ids and
// loads half of the tile's tokens, and the pair's first CTA issues the MMAs.  A step is 128 values of k: 64 TMEM columns of
// converted weights (a slot), a stage of h; a stage of codes is two steps.
//
// TMEM: two accumulators and the slots.  With BN = 256 the accumulators overlap by 128 columns, which the epilogue reads first.
//
// Warps: 0 TMA of h, 1 MMA, 2 TMEM allocation, 3 TMA of codes, 4..11 epilogue (two per lane quarter, half of the tile's columns
// each), 12..19 conversion (two per lane quarter, even and odd steps).
#include <cuda.h>
#include <cuda_runtime.h>
#include <string.h>

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
__device__ __forceinline__ uint4 ld_shared_16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

// ------------------------------------------------------------------ hidden states
// A row of h as fp16 times 2^e, e = 14 - exponent of its largest value, k in the order 0 4 1 5 2 6 3 7 of each eight, zeros
// to whole 64; and -10 - e, the token's share of what the epilogue takes back.  A row with a NaN or an infinity is NaN.
constexpr int kPrepareThreads = 256;
__global__ void __launch_bounds__(kPrepareThreads) w4_prepare(const W4LogitsParams p) {
  __shared__ uint32_t part[kPrepareThreads / 32];
  grid_release();
  const int64_t t = blockIdx.x;
  const unsigned short* h = reinterpret_cast<const unsigned short*>(p.h) + t * p.ldh;
  const int d = p.d;
  uint32_t top = 0;  // magnitudes of bf16 compare like their bits, and a NaN's or an infinity's are above every number's
  for (int k = threadIdx.x; k < d; k += kPrepareThreads) top = max(top, (uint32_t)h[k] & 0x7FFFu);
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPrepareThreads / 32; ++w) top = max(top, part[w]);
  const bool broken = top >= 0x7F80u;
  const int e = broken || top == 0u ? 0 : 14 - (max((int)(top >> 7), 1) - 127);
  const float f1 = __int_as_float((127 + e / 2) << 23), f2 = __int_as_float((127 + e - e / 2) << 23);  // (|e| <= 141)
  if (threadIdx.x == 0) p.token_exp[t] = -10 - e;
  __half* out = p.h16 + t * p.h16_pitch;
  for (int i = threadIdx.x; i < p.h16_pitch / 2; i += kPrepareThreads) {
    // the pair at 2 i holds k = 8 (i / 4) + i % 4 and the one four further
    const int k = (i >> 2) * 8 + (i & 3);
    const float a = k < d ? __uint_as_float((uint32_t)h[k] << 16) * f1 * f2 : 0.f;
    const float b = k + 4 < d ? __uint_as_float((uint32_t)h[k + 4] << 16) * f1 * f2 : 0.f;
    __half2 two = __floats2half2_rn(a, b);
    if (broken) two = __half2half2(__ushort_as_half((unsigned short)0x7FFF));
    reinterpret_cast<__half2*>(out)[i] = two;
  }
}

// ------------------------------------------------------------------ scales
// Exponent (floor log2) of the largest magnitude among a row's finite scales, 0 where there is none; scales below 2^-126
// count as zero.
__device__ __forceinline__ int row_exponent(const __nv_bfloat16* scales, int n8) {
  uint32_t top = 0;
  for (int i = 0; i < n8; ++i) {
    const uint4 s = __ldg(reinterpret_cast<const uint4*>(scales) + i);
    const uint32_t w[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t lo = w[k] & 0x7F80u, hi = (w[k] >> 16) & 0x7F80u;
      if (lo != 0x7F80u) top = max(top, lo);
      if (hi != 0x7F80u) top = max(top, hi);
    }
  }
  return top == 0u ? 0 : (int)(top >> 7) - 127;
}
// A scale times 2^(10 - exponent) as a pair of fp16; NaN for a NaN or an infinity.
__device__ __forceinline__ __half2 normal_scale(uint32_t bits16, int shift) {
  const int e = (int)((bits16 >> 7) & 255u);
  float s = e == 0 || e + shift <= 0 ? 0.f : __uint_as_float((bits16 << 16) + ((uint32_t)shift << 23));
  if (e == 255) s = __int_as_float(0x7FC00000);
  return __half2half2(__float2half_rn(s));
}
// The scales of a step, one for each 32 of its 128 values.
__device__ __forceinline__ uint2 step_scales(const __nv_bfloat16* scales, int step, int group) {
  if (group == 128) {
    const uint32_t one = __ldg(reinterpret_cast<const unsigned short*>(scales) + step);
    return make_uint2(one | (one << 16), one | (one << 16));
  }
  if (group == 64) {
    const uint32_t two = __ldg(reinterpret_cast<const uint32_t*>(scales) + step);
    return make_uint2(__byte_perm(two, 0, 0x1010), __byte_perm(two, 0, 0x3232));
  }
  return __ldg(reinterpret_cast<const uint2*>(scales) + step);
}
// Eight codes -> four pairs of fp16.
__device__ __forceinline__ void convert_word(uint32_t w, __half2 scale, __half2 offset, uint32_t* out) {
  const uint32_t at[4] = {w << 6, w << 2, w >> 2, w >> 6};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bits = (at[i] & 0x03C003C0u) ^ 0x4E004E00u;
    const __half2 v = __hfma2(*reinterpret_cast<const __half2*>(&bits), scale, offset);
    out[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
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
#pragma unroll 1
    for (int j = 0; j < N; ++j) {
      const int e = id_exp + __shfl_sync(0xffffffffu, mine, j);
      // (from -276 to 230: three factors, the sum's rounding to a subnormal last)
      const int a = max(-120, min(120, e)), b = max(-120, min(120, e - a)), c = e - a - b;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i == j)
          r[i] = __float_as_uint(__uint_as_float(r[i]) * __int_as_float((127 + a) << 23) * __int_as_float((127 + b) << 23) *
                                 __int_as_float((127 + c) << 23));
    }
  }
}

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
          const int n_mma = k + 1 < p.k_steps ? kW4Step / 16 : p.last_mmas;
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
    int stage = 0;
    uint32_t phase = 0, step0 = 0;  // steps of the tiles before
    bool ok = true;
    int vt, tt;
    while (ok && walk.next(vt, tt)) {
      const int v = min(vt * kLogitPairM + (int)cta * 128 + r, p.V - 1);
      const __nv_bfloat16* scales = p.scales + (int64_t)v * spitch;
      const int shift = 10 - row_exponent(scales, (int)(spitch / 8));
      uint2 sc = odd < p.k_steps ? step_scales(scales, odd, p.group) : make_uint2(0u, 0u);
      for (int k = 0; k < c_steps; ++k) {
        const int step = 2 * k + odd;
        if (!__all_sync(0xffffffffu, mbar_wait_cta(c_full(stage), phase, false, abort_flag))) { ok = false; break; }
        if (step < p.k_steps) {
          const uint32_t from = row_smem + (uint32_t)(stage * kW4CodeBytes);
          uint4 c[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) c[j] = ld_shared_16(from + ((((uint32_t)(odd * 4 + j)) ^ swizzle) << 4));
          const uint2 here = sc;
          if (step + 2 < p.k_steps) sc = step_scales(scales, step + 2, p.group);
          const uint32_t g = step0 + (uint32_t)step;
          const uint32_t slot = g % (uint32_t)AS, slot_phase = (g / (uint32_t)AS) & 1u;
          const uint32_t to = tmem_base + lane_addr + (uint32_t)Tl::slot_col0 + slot * kW4SlotCols;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t out[32];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t two = half == 0 ? here.x : here.y;
              const __half2 s = normal_scale(j == 0 ? two & 0xFFFFu : two >> 16, shift);
              const __half2 off = __hmul2(s, minus24);
              const uint4& q = c[half * 2 + j];
              convert_word(q.x, s, off, out + 16 * j);
              convert_word(q.y, s, off, out + 16 * j + 4);
              convert_word(q.z, s, off, out + 16 * j + 8);
              convert_word(q.w, s, off, out + 16 * j + 12);
            }
            if (half == 0) {
              if (!__all_sync(0xffffffffu, mbar_wait_cta(a_empty((int)slot), slot_phase ^ 1u, false, abort_flag))) {
                ok = false;
                break;
              }
              tc_fence_after();
            }
            tmem_st_32x32(to + 32u * (uint32_t)half, out);
          }
          if (!ok) break;
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_nofence(full0_base + 8u * slot);  // (TMEM writes are ordered by the fence above)
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
      const int id_exp = row_exponent(p.scales + (int64_t)min(v, p.V - 1) * spitch, (int)(spitch / 8));
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
template <int BN, typename OUT>
static cudaError_t launch_tile(const CUtensorMap& w, const CUtensorMap& h, const CUtensorMap& hl, const CUtensorMap& out,
                               const W4LogitsParams& p, int grid, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(w4_logits<BN, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, W4Tile<BN>::smem_bytes);
  if (e != cudaSuccess) return e;
  w4_prepare<<<p.T, kPrepareThreads, 0, stream>>>(p);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)grid, 1, 1);
  cfg.blockDim = dim3(kW4Threads, 1, 1);
  cfg.dynamicSmemBytes = W4Tile<BN>::smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  memset(&attr, 0, sizeof attr);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, w4_logits<BN, OUT>, w, h, hl, out, p);
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

}  // namespace difr
