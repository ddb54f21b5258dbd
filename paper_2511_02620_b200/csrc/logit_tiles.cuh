// What the products that make logits on CTA pairs share: the tiles of a pair, the order in which its epilogue reads an
// accumulator, and the ways out of it.  `Tl` describes a kernel's tile: tokens, overlap, shared_loads, chunk, chunks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mx_device.cuh"
#include "mx_kernels.h"

namespace difr {

// Which chunk of the accumulator the `i`-th load of an epilogue half takes (-1: none).  Overlapping accumulators start
// with the shared columns: the last ones of accumulator 0, the first ones of accumulator 1.
template <typename Tl>
__device__ __forceinline__ int epi_chunk(int i, int half, int acc) {
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
__device__ __forceinline__ void store_chunk(const LogitTiles& p, const uint32_t (&r)[N], int t0, int v, float*) {
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
__device__ __forceinline__ void store_chunk(const LogitTiles& p, const uint32_t (&r)[N], int t0, int v,
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
  static constexpr int kTokens = logit_out_tokens((int)sizeof(OUT));
  OUT* buf;        // this half's pieces
  int next;        // the one to fill
  uint64_t policy;

  template <int BUFFERS>
  __device__ __forceinline__ void store(const LogitTiles& p, const CUtensorMap* map, const uint32_t (&r)[32], int t0,
                                        int v_block, int quarter, int lane, int half) {
    const bool issuer = quarter == 0 && lane == 0;
#pragma unroll
    for (int k = 0; k < 32 / kTokens; ++k) {
      if (t0 + k * kTokens >= p.T) break;  // the same in all four warps
      if (issuer) bulk_wait_read<BUFFERS - 1>();  // the store that last left from this piece has read it
      named_barrier(1 + half, 128);
      OUT* dst = buf + next * (kLogitOutBytes / (int)sizeof(OUT));
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
  const LogitTiles& p;
  const int pair, n_pairs;
  int round0, turn;  // first tile of the round, pair that is dealt to first

  __device__ __forceinline__ TileWalk(const LogitTiles& params, int pr, int n)
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
template <typename Tl, typename OUT>
__device__ __forceinline__ void fill_given_up(const LogitTiles& p, TileWalk& walk, int vt, int tt, int acc, int half,
                                              int lane_id) {
  const OUT nan = from_float<OUT>(__int_as_float(0x7FC00000));
  do {
    const int v = vt * kLogitPairM + lane_id;
#pragma unroll 1
    for (int i = 0; i < (Tl::chunks + 1) / 2; ++i) {
      const int ch = epi_chunk<Tl>(i, half, acc);
      const int t0 = tt * Tl::tokens + ch * Tl::chunk;
      if (ch < 0 || v >= p.V) continue;
#pragma unroll 1
      for (int t = t0; t < t0 + Tl::chunk && t < p.T; ++t) static_cast<OUT*>(p.logits)[(int64_t)t * p.ld + v] = nan;
    }
    acc ^= 1;
  } while (walk.next(vt, tt));
}

// The way out of the epilogue after waits that ran out, without a product: a CTA is the eight epilogue warps, its first
// `done_tiles` tiles count as finished, and the barrier of the next one is never arrived at.  With tiles of 256 tokens one
// warp of each half sees its barrier complete, so that it is the others that make it give up.
constexpr int kLogitEpiThreads = 256;
template <typename Tl, typename OUT>
__global__ void __launch_bounds__(kLogitEpiThreads)
logit_wait_selftest(const __grid_constant__ LogitTiles p, int done_tiles, long long limit_cycles) {
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
  const bool ok = mbar_wait_cta(smem_u32(&bars[Tl::tokens == 256 && quarter == 1 ? 1 : 0]), 0, false, abort_flag, limit_cycles);
  __syncwarp();
  const bool given_up = Tl::tokens == 256 ? !named_barrier_and(1 + half, 128, ok) : !__all_sync(0xffffffffu, ok);
  if (given_up)
    fill_given_up<Tl, OUT>(p, walk, vt, tt, done_tiles & 1, half, (int)(blockIdx.x & 1) * 128 + quarter * 32 + lane);
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.device_status != nullptr) *p.device_status = kStatusTimeout;
}

}  // namespace difr
