// Parameter blocks and launchers of the norm, the microscaled formats and their product (host-visible part).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace difr {

// Element types of inputs and outputs: the values of difr_dtype.
constexpr int kBf16 = 0, kF16 = 1, kF32 = 2;

struct NormParams {
  const void* x;         // [T][ldx]
  const void* residual;  // [T][ld_residual], nullable
  const void* weight;    // [d]
  void* residual_out;    // [T][ld_residual_out], nullable: x + residual, rounded to the inputs' type
  void* h;               // bf16 [T][ldh], nullable
  unsigned char* codes;  // nullable: microscaled output
  unsigned char* scales;
  int64_t T, ldx, ld_residual, ld_residual_out, ldh;
  int d, fmt;
  float eps, inv_d;
  int threads_per_row, rows_per_cta;
  bool vec;              // all rows start on 16-byte boundaries and d is a multiple of 8
};
constexpr int kNormMaxD = 32768;
cudaError_t launch_rms_norm(const NormParams& p, int dtype, cudaStream_t stream);

struct MxConvertParams {
  const void* in;        // quantise: [rows][ld]
  void* out;             // dequantise: [rows][ld]
  unsigned char* codes;
  unsigned char* scales;
  int64_t rows, ld;
  int d, fmt;
  bool vec;              // the rows of `in` / `out` start on 16-byte boundaries and d is a multiple of 8
};
cudaError_t launch_mx_quantize(const MxConvertParams& p, int dtype, cudaStream_t stream);
cudaError_t launch_mx_dequantize(const MxConvertParams& p, int dtype, cudaStream_t stream);

struct MxLogitsParams {
  void* logits;          // [T][ld]
  int64_t ld;
  int32_t* device_status;
  int T, V;
  int k_steps;           // 128-byte slices of a row of codes
  int last_mmas;         // MMAs (32 bytes of codes each) of the last slice
  int n_vt, n_tt;        // vocabulary tiles of 256 ids, token tiles
  int group;             // token tiles per raster group
  int last_tokens;       // width of the last token tile, a multiple of 16
  int n_tiles;
  int shift;             // of the deal, per round
  bool pack_pairs;       // bf16 logits, plain stores: two neighbouring ids leave in one 4-byte store
  bool w_once;           // one token tile, and a W that does not fit L2: its rows need not stay there
  bool tile_stores;      // the rows of the logits start on 16-byte boundaries: tiles leave by TMA (256-token tiles only)
};
constexpr int kMxPairM = 256;  // vocabulary ids per tile of a CTA pair
constexpr int kMxOutBytes = 8192;                            // a piece of a tile on its way out: 128 ids x
constexpr int mx_out_tokens(int elem) { return kMxOutBytes / (128 * elem); }  // 16 (fp32) or 32 (bf16) tokens
// `tokens_per_tile`: 16, 32, 64, 128 or 256; maps: codes of W, of h, of h for the last token tile, scales of W
// and of h, logits (used with tile_stores only).
cudaError_t launch_mx_logits(int fmt, int tokens_per_tile, int dtype, const CUtensorMap& w, const CUtensorMap& h,
                             const CUtensorMap& h_last, const CUtensorMap& sw, const CUtensorMap& sh, const CUtensorMap& out, const MxLogitsParams& p, int grid,
                             cudaStream_t stream);
// The end of the product after waits that ran out, with nothing computed: see difr_selftest_mx_wait.
cudaError_t launch_mx_wait_selftest(int fmt, int tokens_per_tile, int dtype, const MxLogitsParams& p, int done_tiles,
                                    long long limit_cycles, int grid, cudaStream_t stream);
int mx_logits_max_resident_pairs();

}  // namespace difr
