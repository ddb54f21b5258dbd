// LM-head product on microscaled operands:
//
//   l[t, v] = sum over blocks b of 2^(e_h[t,b] + e_W[v,b]) * sum over k in b of h[t,k] W[v,k]
//
// tcgen05.mma with block scales (kind::mxf8f6f4 for e4m3, kind::mxf4 for e2m1) multiplies the codes, applies both
// power-of-two scales and accumulates in fp32 in TMEM; the accumulator leaves as fp32 or bf16.
//
// The vocabulary is the MMA's M side and the tokens its N side: N goes from 16 (a decoding step, bound by the bytes of
// W) to 256 (re-scoring a batch, bound by the tensor pipe or by the logits' bytes), and a lane of the accumulator is a
// vocabulary id, so the 32 lanes of a warp hold 32 neighbouring logits of one token at a time.
//
// CTAs run as persistent pairs (cta_group::2) on tiles of 256 ids x BN tokens: each CTA loads its own 128 rows of W
// and half of the tile's tokens, and the pair's first CTA issues the MMAs.  A stage is a slice of 128 bytes of codes
// along the hidden dimension (128 or 256 values) with its scale words (four blocks of 128 rows each): those of the
// CTA's own 128 ids and, in both CTAs, those of all BN tokens.  tcgen05.cp puts the words into TMEM, where the MMAs
// read them.
//
// TMEM: two accumulators and each stage's scales.  With BN = 256 two accumulators would take all 512 columns, so they
// overlap by 64 (e4m3) or 128 (e2m1): the epilogue reads the shared columns first, and the next tile's MMAs start as
// soon as it has.  (Fewer columns of scales than stages were slower: the MMA warp then had to wait for the readers of a
// slot, and its own loop, not the tensor pipe, set the pace: 520 clocks a stage where the MMAs take 512.)
//
// Measured: one token x 128256 x 4096 in 4 bits 46 us (6.1 TB/s); 4096 tokens 848 to 892 us in bf16, 4.8 to 5.1 PFLOP/s at the
// power cap (1.2 to 1.4 GHz, tensor pipe 83 % active); 4096 x 152064 x 5120 in 8 bits 2400 to 2510 us with bf16 logits, 2.5 to
// 2.66 PFLOP/s (95 % active), 2610 to 2710 us with fp32 ones.  Tiles go in rounds over all pairs, not in stretches per pair:
// the latter's W slabs leave L2, 3604 us.
//
// Warps: 0 TMA, 1 MMA, 2 TMEM allocation, 4..11 epilogue (two per lane quarter, half of the tile's columns each).
#include <cuda.h>
#include <cuda_runtime.h>
#include <string.h>

#include "difr_kernels.h"
#include "mx_device.cuh"
#include "mx_kernels.h"

namespace difr {

constexpr int kMxEpiWarp0 = 4, kMxEpiWarps = 8;
constexpr int kMxThreads = 32 * (kMxEpiWarp0 + kMxEpiWarps);
constexpr int kMxSlice = 128;  // bytes of codes per row and stage
constexpr int kMxMmaBytes = 32;
constexpr int kMxTmemCols = 512;

template <int FMT, int BN>
struct MxTile {
  static constexpr int words = FMT == kMx8 ? 1 : 2;       // scale words per slice (128 values each)
  static constexpr int row_blocks = BN > 128 ? 2 : 1;     // 128-token blocks of scales
  static constexpr int a_bytes = 128 * kMxSlice;
  static constexpr int b_bytes = BN / 2 * kMxSlice;
  static constexpr int sa_bytes = words * kSfWordBytes;
  static constexpr int sb_bytes = words * row_blocks * kSfWordBytes;
  static constexpr int load_bytes = a_bytes + b_bytes + sa_bytes + sb_bytes;
  static constexpr int stage_bytes = (load_bytes + 1023) / 1024 * 1024;
  static constexpr int bar_bytes = 512;
  // 256-token tiles leave through shared memory: out_buffers pieces in flight for each half of the epilogue
  static constexpr int out_buffers = BN == 256 ? 3 : 0;
  static constexpr int out_bytes = 2 * out_buffers * kMxOutBytes;
  static constexpr int fit = (227 * 1024 - 1024 - bar_bytes - out_bytes) / stage_bytes;
  static constexpr int stages = fit > 12 ? 12 : fit;
  static constexpr int smem_bytes = stages * stage_bytes + out_bytes + bar_bytes + 1024;  // + slack for 1024-byte alignment
  // TMEM columns: two accumulators, and a slot of scales per stage
  static constexpr int sa_cols = 4 * words, sb_cols = 4 * words * row_blocks;
  static constexpr int sf_cols = sa_cols + sb_cols;
  static constexpr bool overlap = BN == 256;
  static constexpr int shared_cols = !overlap ? 0 : sf_cols * stages > 64 ? 128 : 64;
  static constexpr int acc_stride = BN - shared_cols;
  static constexpr int sf_col0 = 2 * BN - shared_cols;
  // epilogue: columns per TMEM load, loads per accumulator, loads per half that cover the shared columns
  static constexpr int chunk = BN >= 64 ? 32 : 16;
  static constexpr int chunks = BN / chunk;
  static constexpr int shared_loads = shared_cols / (2 * chunk);
  static_assert(sf_col0 + stages * sf_cols <= kMxTmemCols, "TMEM columns");
  static_assert(stages >= 4, "pipeline depth");
};

// Which chunk of the accumulator the `i`-th load of an epilogue half takes (-1: none).  Overlapping accumulators start
// with the shared columns: the last ones of accumulator 0, the first ones of accumulator 1.
template <int FMT, int BN>
__device__ __forceinline__ int epi_chunk(int i, int half, int acc) {
  using Tl = MxTile<FMT, BN>;
  if (Tl::overlap) {
    constexpr int shared = 2 * Tl::shared_loads, rest = Tl::chunks - shared;
    if (i < Tl::shared_loads) return (acc == 0 ? rest : 0) + half * Tl::shared_loads + i;
    return (acc == 0 ? 0 : shared) + half * (rest / 2) + i - Tl::shared_loads;
  }
  const int c = i * 2 + half;
  return c < Tl::chunks ? c : -1;
}

// Token columns of one TMEM load -> logits.  r[j] is the logit of id `v` (this lane's) for token t0 + j.
template <int N>
__device__ __forceinline__ void store_chunk(const MxLogitsParams& p, const uint32_t (&r)[N], int t0, int v, float*) {
  float* dst = static_cast<float*>(p.logits) + (int64_t)t0 * p.ld + v;
  const bool ok = v < p.V;
  const int n = p.T - t0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (j < n && ok) __stcs(dst, __uint_as_float(r[j]));
    dst += p.ld;
  }
}
template <int N>
__device__ __forceinline__ void store_chunk(const MxLogitsParams& p, const uint32_t (&r)[N], int t0, int v,
                                            __nv_bfloat16*) {
  __nv_bfloat16* base = static_cast<__nv_bfloat16*>(p.logits) + (int64_t)t0 * p.ld;
  const int n = p.T - t0;
  if (p.pack_pairs) {
    // neighbouring lanes trade: the even one takes ids v, v + 1 of token j, the odd one ids v - 1, v of token j + 1
    const bool odd = (v & 1) != 0;
    const int v0 = v & ~1;
    __nv_bfloat16* dst = base + v0 + (odd ? p.ld : 0);
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      const float a = __uint_as_float(r[j]), b = __uint_as_float(r[j + 1]);
      const float got = __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
      __nv_bfloat162 two = odd ? __floats2bfloat162_rn(got, b) : __floats2bfloat162_rn(a, got);
      if (j + (odd ? 1 : 0) < n) {
        if (v0 + 1 < p.V)
          __stcs(reinterpret_cast<uint32_t*>(dst), *reinterpret_cast<uint32_t*>(&two));
        else if (v0 < p.V)
          *dst = two.x;
      }
      dst += 2 * p.ld;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n && v < p.V) base[(int64_t)j * p.ld + v] = __float2bfloat16_rn(__uint_as_float(r[j]));
  }
}

// The staged way out of a 32-token chunk, for the four warps (128 ids) of an epilogue half: through pieces in shared
// memory that leave by TMA, whole rows of 128 ids at a time.  (Stored from registers, a warp's 32 ids of one token
// are a request of 128 or 64 bytes each, and the requests, not the bytes, were what the epilogue took its time for.)
template <typename OUT>
struct OutPieces {
  static constexpr int kTokens = mx_out_tokens((int)sizeof(OUT));
  OUT* buf;        // this half's pieces
  int next;        // the one to fill
  uint64_t policy;

  template <int BUFFERS>
  __device__ __forceinline__ void store(const MxLogitsParams& p, const CUtensorMap* map, const uint32_t (&r)[32], int t0,
                                        int v_block, int quarter, int lane, int half) {
    const bool issuer = quarter == 0 && lane == 0;
#pragma unroll
    for (int k = 0; k < 32 / kTokens; ++k) {
      if (t0 + k * kTokens >= p.T) break;  // the same in all four warps
      if (issuer) bulk_wait_read<BUFFERS - 1>();  // the store that last left from this piece has read it
      named_barrier(1 + half, 128);
      OUT* dst = buf + next * (kMxOutBytes / (int)sizeof(OUT));
#pragma unroll
      for (int j = 0; j < kTokens; ++j)
        dst[j * 128 + quarter * 32 + lane] = from_float<OUT>(__uint_as_float(r[k * kTokens + j]));
      fence_async_shared();
      named_barrier(1 + half, 128);
      if (issuer) {
        if (v_block < p.V) tma_store_2d(map, v_block, t0 + k * kTokens, smem_u32(dst), policy);
        bulk_commit();
      }
      if (++next == BUFFERS) next = 0;
    }
  }
};

// The tiles of one pair.  Tiles are numbered in groups of token tiles (a group's tokens stay in L2 while W passes by),
// inside a group along the vocabulary, inside that along the group's token tiles, and are dealt out in rounds of one
// tile per pair: the pairs that run at the same time share a few rows of W.  From round to round the deal shifts by
// `shift` pairs, chosen so that the narrower last token tiles reach all pairs alike.
struct TileWalk {
  const MxLogitsParams& p;
  const int pair, n_pairs;
  int round0, turn;  // first tile of the round, pair that is dealt to first

  __device__ __forceinline__ TileWalk(const MxLogitsParams& params, int pr, int n)
      : p(params), pair(pr), n_pairs(n), round0(0), turn(0) {}
  __device__ __forceinline__ bool next(int& vt, int& tt) {
    const int at = pair - turn;
    const int i = round0 + (at < 0 ? at + n_pairs : at);
    if (i >= p.n_tiles) return false;
    round0 += n_pairs;
    turn += p.shift;
    if (turn >= n_pairs) turn -= n_pairs;
    const int per_group = p.group * p.n_vt;
    const int g = i / per_group;
    const int rem = i - g * per_group;
    const int first = g * p.group;
    const int cnt = min(p.group, p.n_tt - first);
    vt = rem / cnt;
    tt = first + rem - vt * cnt;
    return true;
  }
};

// After a wait that ran out: the warp's part of tile (vt, tt) and of the pair's next ones becomes NaN, so that no caller
// takes what the buffer held before for logits.  `lane_id`: this lane's id inside a vocabulary tile.
template <int FMT, int BN, typename OUT>
__device__ __forceinline__ void fill_given_up(const MxLogitsParams& p, TileWalk& walk, int vt, int tt, int acc, int half,
                                              int lane_id) {
  using Tl = MxTile<FMT, BN>;
  const OUT nan = from_float<OUT>(__int_as_float(0x7FC00000));
  do {
    const int v = vt * kMxPairM + lane_id;
#pragma unroll 1
    for (int i = 0; i < (Tl::chunks + 1) / 2; ++i) {
      const int ch = epi_chunk<FMT, BN>(i, half, acc);
      const int t0 = tt * BN + ch * Tl::chunk;
      if (ch < 0 || v >= p.V) continue;
#pragma unroll 1
      for (int t = t0; t < t0 + Tl::chunk && t < p.T; ++t) static_cast<OUT*>(p.logits)[(int64_t)t * p.ld + v] = nan;
    }
    acc ^= 1;
  } while (walk.next(vt, tt));
}

template <int FMT, int BN, typename OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMxThreads, 1)
mx_logits(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_h,
          const __grid_constant__ CUtensorMap tmap_h_last, const __grid_constant__ CUtensorMap tmap_sw,
          const __grid_constant__ CUtensorMap tmap_sh, const __grid_constant__ CUtensorMap tmap_out,
          const __grid_constant__ MxLogitsParams p) {
  using Tl = MxTile<FMT, BN>;
  constexpr int kStages = Tl::stages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t smem_base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - raw_addr);

  // Both CTAs of a pair lay out their barriers at the same offsets.
  //   full[s]     first CTA's copy is used: 1 arrival (its producer) + the bytes of both CTAs' loads
  //   empty[s]    each CTA's own copy: 1 arrival, the commit of the MMAs that read the stage, delivered to both
  //   acc_full[a] each CTA's own copy: 1 arrival, the commit after a tile's last MMA, delivered to both
  //   acc_free[a] first CTA's copy is used: one arrival per epilogue warp of both CTAs, after its last load of the
  //               accumulator, or, where the accumulators overlap, after its load of shared columns
  const uint32_t bar0 = smem_base + kStages * Tl::stage_bytes + Tl::out_bytes;
  uint8_t* out_pieces = smem + kStages * Tl::stage_bytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(out_pieces + Tl::out_bytes);
  auto full_bar = [&](int s) { return bar0 + 8u * (uint32_t)s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (uint32_t)(kStages + s); };
  auto acc_full_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * kStages + a); };
  auto acc_free_bar = [&](int a) { return bar0 + 8u * (uint32_t)(2 * kStages + 2 + a); };
  static_assert((2 * kStages + 4) * 8 + 8 <= Tl::bar_bytes, "barrier block");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kStages + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t cta = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  const int n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full_bar(a), 1);
      mbar_init(acc_free_bar(a), 2 * kMxEpiWarps);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmap_w);
    tma_prefetch_desc(&tmap_h);
    tma_prefetch_desc(&tmap_h_last);
    tma_prefetch_desc(&tmap_sw);
    tma_prefetch_desc(&tmap_sh);
  }
  // (TMEM is taken only now: a CTA that held it while it waited could keep it from the kernel it waits for)
  grid_wait();
  grid_release();
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(tmem_slot), kMxTmemCols);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_arrive();
  cluster_wait();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  TileWalk walk(p, pair, n_pairs);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    const uint64_t keep = l2_policy_evict_last(), stream = p.w_once ? l2_policy_evict_first() : l2_policy_evict_normal();
    const uint32_t full0_base = map_to_cta(full_bar(0), 0);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    int vt, tt;
    while (ok && walk.next(vt, tt)) {
      const bool last = tt == p.n_tt - 1;
      const int half = last ? p.last_tokens / 2 : BN / 2;
      const uint32_t bytes = (uint32_t)(Tl::load_bytes - (BN / 2 - half) * kMxSlice);
      const void* tmap_tokens = last ? &tmap_h_last : &tmap_h;
      const int w_row = vt * kMxPairM + (int)cta * 128;
      const int h_row = tt * BN + (int)cta * half;
      for (int k = 0; k < p.k_steps; ++k) {
        if (!__all_sync(0xffffffffu, mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag))) { ok = false; break; }
        if (elect_one()) {
          if (cta == 0) mbar_arrive_expect_tx(full_bar(stage), 2u * bytes);
          const uint32_t full0 = full0_base + 8u * (uint32_t)stage;
          const uint32_t dst = smem_base + (uint32_t)(stage * Tl::stage_bytes);
          tma_load_2d_pair(dst, &tmap_w, k * kMxSlice, w_row, full0, stream);
          tma_load_2d_pair(dst + Tl::a_bytes, tmap_tokens, k * kMxSlice, h_row, full0, keep);
          tma_load_3d_pair(dst + Tl::a_bytes + Tl::b_bytes, &tmap_sw, 0, k * Tl::words, w_row >> 7, full0, stream);
          tma_load_3d_pair(dst + Tl::a_bytes + Tl::b_bytes + Tl::sa_bytes, &tmap_sh, 0, k * Tl::words,
                           (tt * BN) >> 7, full0, keep);
        }
        __syncwarp();
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issuer
    if (cta == 0) {
      const uint64_t desc0 = umma_desc_k_major_sw128(smem_base);
      const uint32_t desc_hi = (uint32_t)(desc0 >> 32), desc_lo0 = (uint32_t)desc0;
      const uint64_t sdesc0 = umma_desc_scales(smem_base);
      const uint32_t sdesc_hi = (uint32_t)(sdesc0 >> 32), sdesc_lo0 = (uint32_t)sdesc0;
      int stage = 0, acc = 0;
      uint32_t phase = 0, n_tile = 0;
      bool full_seen = false;
      bool ok = true;
      int vt, tt;
      for (; ok && walk.next(vt, tt); ++n_tile) {
        const uint32_t idesc = umma_idesc_mx<FMT>(kMxPairM, tt == p.n_tt - 1 ? p.last_tokens : BN);
        // Separate accumulators: the tile before last has been read.  Overlapping ones: the shared columns of the last
        // tile have been read (every epilogue warp had then finished the tile before it).
        if (Tl::overlap) {
          if (n_tile >= 1 && !__all_sync(0xffffffffu, mbar_wait(acc_free_bar(acc ^ 1), ((n_tile - 1) >> 1) & 1u,
                                                                abort_flag))) { ok = false; break; }
        } else {
          if (n_tile >= 2 && !__all_sync(0xffffffffu, mbar_wait(acc_free_bar(acc), ((n_tile - 2) >> 1) & 1u,
                                                                abort_flag))) { ok = false; break; }
        }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + (uint32_t)(acc * Tl::acc_stride);
        uint32_t accumulate = 0;
        for (int k = 0; k < p.k_steps; ++k) {
          if (!__all_sync(0xffffffffu, mbar_wait_cta(full_bar(stage), phase, full_seen, abort_flag))) { ok = false; break; }
          // a look at the next stage: its answer is there by the time it is needed
          {
            const bool wrap = stage + 1 == kStages;
            full_seen = mbar_peek_cta(full_bar(wrap ? 0 : stage + 1), wrap ? phase ^ 1u : phase);
          }
          tc_fence_after();
          const int n_mma = k + 1 < p.k_steps ? kMxSlice / kMxMmaBytes : p.last_mmas;
          const uint32_t at = (uint32_t)(stage * Tl::stage_bytes) >> 4;
          const uint32_t a_lo = desc_lo0 + at, b_lo = a_lo + (Tl::a_bytes >> 4);
          const uint32_t sa_lo = sdesc_lo0 + at + ((Tl::a_bytes + Tl::b_bytes) >> 4);
          const uint32_t sb_lo = sa_lo + (Tl::sa_bytes >> 4);
          // (a stage has its own columns for scales, free again when the stage is)
          const uint32_t sa = tmem_base + (uint32_t)(Tl::sf_col0 + stage * Tl::sf_cols);
          const uint32_t sb = sa + Tl::sa_cols;
          if (elect_one()) {
#pragma unroll
            for (int w = 0; w < Tl::words; ++w) {
              tmem_copy_scales_pair(sa + 4u * w, ((uint64_t)sdesc_hi << 32) | (sa_lo + (uint32_t)w * (kSfWordBytes >> 4)));
#pragma unroll
              for (int b = 0; b < Tl::row_blocks; ++b)
                tmem_copy_scales_pair(sb + 4u * (w * Tl::row_blocks + b),
                                      ((uint64_t)sdesc_hi << 32) |
                                          (sb_lo + (uint32_t)(b * Tl::words + w) * (kSfWordBytes >> 4)));
            }
#pragma unroll
            for (int kk = 0; kk < kMxSlice / kMxMmaBytes; ++kk) {
              if (kk < n_mma) {
                // 32 values per MMA and one scale (e4m3), or 64 and two (e2m1)
                const int w = FMT == kMx8 ? 0 : kk >> 1;
                const uint32_t id = FMT == kMx8 ? (uint32_t)kk : 2u * (kk & 1);
                const uint64_t a_desc = ((uint64_t)desc_hi << 32) | (a_lo + 2u * kk);
                const uint64_t b_desc = ((uint64_t)desc_hi << 32) | (b_lo + 2u * kk);
                umma_mx_pair<FMT>(d_tmem, a_desc, b_desc, idesc | umma_idesc_scale_byte(id), sa + 4u * w,
                                  sb + 4u * w * Tl::row_blocks, kk == 0 ? accumulate : 1u);
              }
            }
            umma_commit_pair(empty_bar(stage), 3);
          }
          __syncwarp();
          accumulate = 1;
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
        if (ok && elect_one()) umma_commit_pair(acc_full_bar(acc), 3);
        __syncwarp();
        acc ^= 1;
      }
    }
  } else if (warp >= kMxEpiWarp0) {
    // ---------------------------------------------------------------- epilogue
    const int quarter = warp & 3;  // the TMEM lane quarter this warp may read
    const int half = (warp - kMxEpiWarp0) >> 2;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    int acc = 0;
    uint32_t acc_phase = 0;
    OutPieces<OUT> pieces;
    pieces.buf = reinterpret_cast<OUT*>(out_pieces + half * (Tl::out_bytes / 2));
    pieces.next = 0;
    pieces.policy = l2_policy_evict_first();
    int vt, tt;
    bool given_up = false;
    while (walk.next(vt, tt)) {
      const bool ok = mbar_wait_cta(acc_full_bar(acc), acc_phase, false, abort_flag);
      __syncwarp();
      tc_fence_after();
      const int v = vt * kMxPairM + (int)cta * 128 + quarter * 32 + lane;
      const uint32_t free_bar = map_to_cta(acc_free_bar(acc), 0);
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
          const int ch = epi_chunk<FMT, BN>(c + q, half, acc);
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
          const int ch = epi_chunk<FMT, BN>(c + q, half, acc);
          const int t0 = tt * BN + ch * Tl::chunk;
          if (q < n_here && ch >= 0 && t0 < p.T) {
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
    if (given_up) fill_given_up<FMT, BN, OUT>(p, walk, vt, tt, acc, half, (int)cta * 128 + quarter * 32 + lane);
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
    tmem_dealloc_pair(tmem_base, kMxTmemCols);
  }
  if (threadIdx.x == 0 && *abort_flag && p.device_status != nullptr) *p.device_status = kStatusTimeout;
}

// The way out of the epilogue after waits that ran out, without a product: a CTA is the eight epilogue warps, its first
// `done_tiles` tiles count as finished, and the barrier of the next one is never arrived at.  With tiles of 256 tokens one
// warp of each half sees its barrier complete, so that it is the others that make it give up.
template <int FMT, int BN, typename OUT>
__global__ void __launch_bounds__(32 * kMxEpiWarps)
mx_wait_selftest(const __grid_constant__ MxLogitsParams p, int done_tiles, long long limit_cycles) {
  __shared__ uint64_t bars[2];  // never complete, complete
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bars[0]), 1);
    mbar_init(smem_u32(&bars[1]), 1);
    abort_word = 0;
    mbar_fence_init();
    mbar_arrive(smem_u32(&bars[1]));
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int half = warp >> 2, quarter = warp & 3;
  TileWalk walk(p, blockIdx.x >> 1, gridDim.x >> 1);
  int vt, tt;
  for (int k = 0; k <= done_tiles; ++k)
    if (!walk.next(vt, tt)) return;  // all tiles of the pair are finished, in all of its threads
  const bool ok = mbar_wait_cta(smem_u32(&bars[BN == 256 && quarter == 1 ? 1 : 0]), 0, false, abort_flag, limit_cycles);
  __syncwarp();
  const bool given_up = BN == 256 ? !named_barrier_and(1 + half, 128, ok) : !__all_sync(0xffffffffu, ok);
  if (given_up)
    fill_given_up<FMT, BN, OUT>(p, walk, vt, tt, done_tiles & 1, half, (int)(blockIdx.x & 1) * 128 + quarter * 32 + lane);
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.device_status != nullptr) *p.device_status = kStatusTimeout;
}

// ------------------------------------------------------------------ launcher
template <int FMT, int BN, typename OUT>
static cudaError_t launch_tile(const CUtensorMap& w, const CUtensorMap& h, const CUtensorMap& hl, const CUtensorMap& sw,
                               const CUtensorMap& sh, const CUtensorMap& out, const MxLogitsParams& p, int grid, cudaStream_t stream) {
  const cudaError_t e = cudaFuncSetAttribute(mx_logits<FMT, BN, OUT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             MxTile<FMT, BN>::smem_bytes);
  if (e != cudaSuccess) return e;
  // (a programmatic launch: a CTA is set up while the kernel before it ends; with the policy of a head that is read once a
  // decoding step of 128256 x 4096 in 4 bits takes 46 us instead of 49 for it)
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)grid, 1, 1);
  cfg.blockDim = dim3(kMxThreads, 1, 1);
  cfg.dynamicSmemBytes = MxTile<FMT, BN>::smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  memset(&attr, 0, sizeof attr);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, mx_logits<FMT, BN, OUT>, w, h, hl, sw, sh, out, p);
}

template <int FMT, typename OUT>
static cudaError_t launch_typed(int bn, const CUtensorMap& w, const CUtensorMap& h, const CUtensorMap& hl, const CUtensorMap& sw,
                                const CUtensorMap& sh, const CUtensorMap& out, const MxLogitsParams& p, int grid, cudaStream_t stream) {
  switch (bn) {
    case 16: return launch_tile<FMT, 16, OUT>(w, h, hl, sw, sh, out, p, grid, stream);
    case 32: return launch_tile<FMT, 32, OUT>(w, h, hl, sw, sh, out, p, grid, stream);
    case 64: return launch_tile<FMT, 64, OUT>(w, h, hl, sw, sh, out, p, grid, stream);
    case 128: return launch_tile<FMT, 128, OUT>(w, h, hl, sw, sh, out, p, grid, stream);
    case 256: return launch_tile<FMT, 256, OUT>(w, h, hl, sw, sh, out, p, grid, stream);
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_mx_logits(int fmt, int tokens_per_tile, int dtype, const CUtensorMap& w, const CUtensorMap& h,
                             const CUtensorMap& hl, const CUtensorMap& sw, const CUtensorMap& sh, const CUtensorMap& out, const MxLogitsParams& p, int grid,
                             cudaStream_t stream) {
  if (fmt == kMx8)
    return dtype == kBf16 ? launch_typed<kMx8, __nv_bfloat16>(tokens_per_tile, w, h, hl, sw, sh, out, p, grid, stream)
                          : launch_typed<kMx8, float>(tokens_per_tile, w, h, hl, sw, sh, out, p, grid, stream);
  return dtype == kBf16 ? launch_typed<kMx4, __nv_bfloat16>(tokens_per_tile, w, h, hl, sw, sh, out, p, grid, stream)
                        : launch_typed<kMx4, float>(tokens_per_tile, w, h, hl, sw, sh, out, p, grid, stream);
}

template <int FMT, typename OUT>
static cudaError_t launch_selftest(int bn, const MxLogitsParams& p, int done, long long limit, int grid, cudaStream_t stream) {
  constexpr int threads = 32 * kMxEpiWarps;
  switch (bn) {
    case 16: mx_wait_selftest<FMT, 16, OUT><<<grid, threads, 0, stream>>>(p, done, limit); break;
    case 32: mx_wait_selftest<FMT, 32, OUT><<<grid, threads, 0, stream>>>(p, done, limit); break;
    case 64: mx_wait_selftest<FMT, 64, OUT><<<grid, threads, 0, stream>>>(p, done, limit); break;
    case 128: mx_wait_selftest<FMT, 128, OUT><<<grid, threads, 0, stream>>>(p, done, limit); break;
    default: mx_wait_selftest<FMT, 256, OUT><<<grid, threads, 0, stream>>>(p, done, limit); break;
  }
  return cudaGetLastError();
}

cudaError_t launch_mx_wait_selftest(int fmt, int tokens_per_tile, int dtype, const MxLogitsParams& p, int done_tiles,
                                    long long limit_cycles, int grid, cudaStream_t stream) {
  if (fmt == kMx8)
    return dtype == kBf16 ? launch_selftest<kMx8, __nv_bfloat16>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream)
                          : launch_selftest<kMx8, float>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream);
  return dtype == kBf16 ? launch_selftest<kMx4, __nv_bfloat16>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream)
                        : launch_selftest<kMx4, float>(tokens_per_tile, p, done_tiles, limit_cycles, grid, stream);
}

// Pairs the device keeps resident at once: one CTA per SM, the same for every variant (each takes the whole TMEM).
int mx_logits_max_resident_pairs() {
  using Tl = MxTile<kMx4, 256>;
  if (cudaFuncSetAttribute(mx_logits<kMx4, 256, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, Tl::smem_bytes) !=
      cudaSuccess)
    return 0;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3(2 * 148, 1, 1);
  cfg.blockDim = dim3(kMxThreads, 1, 1);
  cfg.dynamicSmemBytes = Tl::smem_bytes;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 2;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, mx_logits<kMx4, 256, float>, &cfg) != cudaSuccess) return 0;
  return n;
}

}  // namespace difr
