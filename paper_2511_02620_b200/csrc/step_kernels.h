// Parameter blocks and launchers of a decoding step's operators: block norm, 4-bit weights with group scales, verification of
// drafted tokens (host-visible part).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "mx_kernels.h"

namespace difr {

struct BlockNormParams {
  const void* x;            // [T][ldx]
  const void* residual;     // [T][ld_residual]
  const void* post_weight;  // [d], nullable: no norm after the block
  const void* gate;         // [T][ld_gate], nullable; ld_gate 0: one row for all tokens
  const void* weight;       // [d], nullable: only the stream is wanted
  void* residual_out;       // [T][ld_residual_out], nullable
  void* h;                  // bf16 [T][ldh], nullable
  unsigned char* codes;     // nullable: microscaled output
  unsigned char* scales;
  int64_t T, ldx, ld_residual, ld_gate, ld_residual_out, ldh;
  int d, fmt;
  float eps, post_eps, inv_d, alpha, beta, weight_offset;
  int threads_per_row, rows_per_cta;
  bool vec;                 // all rows start on 16-byte boundaries and d is a multiple of 8
};
cudaError_t launch_block_norm(const BlockNormParams& p, int dtype, cudaStream_t stream);

struct W4ConvertParams {
  const void* in;         // quantise: [rows][ld]
  void* out;              // dequantise: [rows][ld]
  unsigned char* codes;
  __nv_bfloat16* scales;
  int64_t rows, ld;
  int d, group;
  bool vec;               // the rows of `in` / `out` start on 16-byte boundaries and d is a multiple of 8
};
cudaError_t launch_w4_quantize(const W4ConvertParams& p, int dtype, cudaStream_t stream);
cudaError_t launch_w4_dequantize(const W4ConvertParams& p, int dtype, cudaStream_t stream);

struct W4LogitsParams : LogitTiles {
  const __nv_bfloat16* h;  // [T][ldh]
  const __nv_bfloat16* scales;
  __half* h16;             // [T][h16_pitch], workspace: h as the tensor cores take it
  int* token_exp;          // [T], workspace: what the epilogue takes back of it
  int64_t ldh;
  int d, group, h16_pitch;
  int k_steps;             // of 128 values
  bool h_vec;              // h's rows start on 16-byte boundaries
  bool half_last;          // the last one has 64 at most
  bool few;                // launch_w4_few: only the sizes, buffers and strides of the tiles' part are used
};
// Tokens that go through `w4_few`.  128256 x 4096, us, few / tiles: one token 62 / 104, 16 84 / 105, 17 128 / 105; 151936 x 2048
// 43 / 72, 55 / 72, 74 / 73.  (Of 3000 ids, where the tiles are fewer than the pairs, 25 / 20 at four tokens, 29 / 21 at 16.)
constexpr int kW4Few = 16;
constexpr int kW4FewIds = 32;  // ids of a warp
// maps: codes in boxes of 128 bytes x kW4FewIds rows, scales in boxes of 8 x kW4FewIds rows
cudaError_t launch_w4_few(int dtype, const CUtensorMap& w, const CUtensorMap& s, const W4LogitsParams& p, cudaStream_t stream);
// `tokens_per_tile`: 32, 64, 128 or 256; maps: codes, h16, h16 for the last token tile, logits (used with tile_stores only).
cudaError_t launch_w4_logits(int tokens_per_tile, int dtype, const CUtensorMap& w, const CUtensorMap& h,
                             const CUtensorMap& h_last, const CUtensorMap& out, const W4LogitsParams& p, int grid,
                             cudaStream_t stream);
// Validation aid: how the product of `p` ends where a wait runs out; nothing is computed.
cudaError_t launch_w4_wait_selftest(int tokens_per_tile, int dtype, const W4LogitsParams& p, int done_tiles,
                                    long long limit_cycles, int grid, cudaStream_t stream);

struct VerifyParams {
  const void* logits;            // [n_drafts + B][ld]
  const float* probs;            // [n_drafts][ld_probs], nullable
  const int32_t* drafted;        // [n_drafts]
  const int32_t* offsets;        // [B + 1]
  const uint32_t* accept_words;  // [n_drafts]
  const uint32_t* sample_words;  // [B]
  const float* temperatures;     // [B], nullable
  int32_t* tokens;               // [B][max_drafts + 1]
  int32_t* n_accepted;           // [B]
  float* p_draft;                // [n_drafts], nullable
  uint32_t* status;              // [B], nullable
  float4* records;               // [n_drafts + B][chunks]: largest logit, sum of exponentials, first id of the largest
  float4* picks;                 // [B]: largest logit of the row to sample, how it is sampled, accepted drafts
  int64_t ld, ld_probs;
  float temperature;
  int B, n_drafts, V, max_drafts, chunks;
  int first_request;             // of a launch
};
constexpr int kVerifyMaxDrafts = 255;
constexpr int kVerifyChunkVecs = 1024;  // 16-byte vectors of logits per record
// the bits of difr_drafts_out.status
constexpr uint32_t kDraftBadToken = 1, kDraftBadRow = 2, kDraftBadOffsets = 4, kDraftBadTemperature = 8;
cudaError_t launch_verify_drafts(const VerifyParams& p, int dtype, cudaStream_t stream);

}  // namespace difr
