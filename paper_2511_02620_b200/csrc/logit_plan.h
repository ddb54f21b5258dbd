// Host side of the products that make logits: how they are cut into tiles, the tensor map of the logits.
#pragma once
#include <atomic>

#include "difr_host.h"
#include "mx_kernels.h"

namespace difr {

// Streaming multiprocessors and resident CTA pairs of the current device; DIFR_ERR_ARCH for another architecture.
inline difr_status device_pairs(int* pairs) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> cached[kMaxDevices];  // 0: not asked yet, -1: another architecture, otherwise pairs
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return DIFR_ERR_CUDA;
  const bool slot = dev >= 0 && dev < kMaxDevices;
  int n = slot ? cached[dev].load(std::memory_order_relaxed) : 0;
  if (n == 0) {
    int major = 0, sms = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return DIFR_ERR_CUDA;
    n = -1;
    if (major == 10) {
      n = mx_logits_max_resident_pairs();
      if (n <= 0) return DIFR_ERR_CUDA;
      if (n > sms / 2) n = sms / 2;
    }
    if (slot) cached[dev].store(n, std::memory_order_relaxed);
  }
  if (n < 0) return DIFR_ERR_ARCH;
  *pairs = n;
  return DIFR_OK;
}

inline int common_divisor(int a, int b) {
  while (b != 0) {
    const int r = a % b;
    a = b;
    b = r;
  }
  return a;
}

// The logits [T, V] as the epilogue stores them: pieces of 128 ids x some tokens.
inline bool logits_tmap(CUtensorMap* map, void* base, int32_t dtype, int64_t T, int64_t V, int64_t ld) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)V, (cuuint64_t)T};
  const cuuint64_t strides[1] = {(cuuint64_t)(ld * elem_bytes(dtype))};
  const cuuint32_t box[2] = {128, (cuuint32_t)logit_out_tokens(elem_bytes(dtype))};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, dtype == DIFR_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline int logit_tile_tokens(int64_t T, int min_tokens) {
  // the smallest width that holds all tokens, tiles of 256 beyond 128
  int bn = min_tokens;
  while (bn < 256 && bn < T) bn *= 2;
  return bn;
}
inline bool too_many_tiles(int64_t T, int64_t V, int min_tokens) {  // their numbers are 32-bit
  const int bn = logit_tile_tokens(T, min_tokens);
  return (V + kLogitPairM - 1) / kLogitPairM * ((T + bn - 1) / bn) > (int64_t)1 << 29;
}
// How T >= 1 tokens x V ids are cut into tiles, of min_tokens (16 or 32) to 256 tokens; `h_pitch`: bytes of a token as the
// kernel loads it, `w_bytes`: all of W's.
inline void plan_logit_tiles(int64_t T, int64_t V, int64_t h_pitch, int64_t w_bytes, int min_tokens, void* logits,
                                    int32_t dtype, int64_t ld, int32_t* device_status, int pairs, LogitTiles* p,
                                    int* tokens_per_tile, int* grid) {
  int bn = logit_tile_tokens(T, min_tokens);
  const int64_t n_vt = (V + kLogitPairM - 1) / kLogitPairM;
  // Where tiles of 256 leave half of the pairs idle, tiles of 128: twice as many, each about half as long (1024 x 1000 x
  // 8192 in 8 bits, 16 tiles: 20 us instead of 26; 600 x 3000 x 6000, 36 tiles: 17.3 instead of 22).  Otherwise W would
  // only be loaded twice as often (777 x 32000 x 1749: 60 us instead of 52).
  if (bn == 256 && n_vt * ((T + 255) / 256) <= pairs / 2) bn = 128;
  const int64_t n_tt = (T + bn - 1) / bn;
  p->logits = logits; p->ld = ld; p->device_status = device_status;
  p->T = (int)T; p->V = (int)V;
  p->n_vt = (int)n_vt; p->n_tt = (int)n_tt;
  p->n_tiles = (int)(n_vt * n_tt);
  // the last token tile is only as wide as its tokens (in steps of what the MMA takes)
  p->last_tokens = (int)((T - (n_tt - 1) * bn + min_tokens - 1) / min_tokens * min_tokens);
  // tokens of a raster group: about 32 MB of them, a quarter of L2, so that they stay there while W passes
  int64_t group = ((int64_t)32 << 20) / ((int64_t)bn * h_pitch);
  if (group < 1) group = 1;
  if (group > n_tt) group = n_tt;
  p->group = (int)group;
  p->w_once = n_tt == 1 && w_bytes > ((int64_t)96 << 20);
  p->pack_pairs = dtype == DIFR_BF16 && ld % 2 == 0 && aligned_to(logits, 4);
  p->tile_stores = bn == 256 && vector_rows(logits, ld, dtype) && ld <= ((int64_t)1 << 36);
  const int n_pairs = p->n_tiles < pairs ? p->n_tiles : pairs;
  // a pair's token tiles follow each other in steps of n_pairs - shift: prime to their number, all come in turn
  p->shift = 0;
  if (n_pairs > 1)
    while (p->shift < n_pairs - 1 && common_divisor(n_pairs - p->shift, p->group) != 1) ++p->shift;
  *tokens_per_tile = bn;
  *grid = 2 * n_pairs;
}

}  // namespace difr
