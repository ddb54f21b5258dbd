// C ABI of the operators around the LM head: the final norm, the microscaled formats and the product on them.
// Argument checks, tensor maps and launches; nothing here computes.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/difr.h"
#include "difr_host.h"
#include "mx_device.cuh"
#include "mx_kernels.h"

namespace {

using namespace difr;

constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxD = (int64_t)1 << 20, kMaxLd = (int64_t)1 << 40;

int elem_bytes(int32_t dtype) { return dtype == DIFR_F32 ? 4 : 2; }
bool known_dtype(int32_t dtype) { return dtype == DIFR_BF16 || dtype == DIFR_F16 || dtype == DIFR_F32; }
bool known_format(int32_t f) { return f == DIFR_MX8 || f == DIFR_MX4; }
bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) == 0; }
// rows of `ld` elements that all start on 16-byte boundaries
bool vector_rows(const void* p, int64_t ld, int32_t dtype) {
  return aligned16(p) && (ld * elem_bytes(dtype)) % 16 == 0;
}

// Streaming multiprocessors and resident CTA pairs of the current device; DIFR_ERR_ARCH for another architecture.
difr_status device_pairs(int* pairs) {
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

int common_divisor(int a, int b) {
  while (b != 0) {
    const int r = a % b;
    a = b;
    b = r;
  }
  return a;
}

// Codes of a microscaled tensor as bytes: box of 128 bytes (128-byte swizzle) x box_rows rows.
bool codes_tmap(CUtensorMap* map, const void* base, int fmt, int64_t rows, int64_t d, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const int64_t pitch = mx_pitch_bytes(fmt, d);
  const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Its scales: [row blocks of 128][words][512 bytes], box of box_words x box_blocks whole words.
bool scales_tmap(CUtensorMap* map, const void* base, int64_t rows, int64_t d, int box_words, int box_blocks) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const int64_t words = mx_words(d), blocks = (rows + kSfWordRows - 1) / kSfWordRows;
  const cuuint64_t dims[3] = {(cuuint64_t)(kSfWordBytes / 4), (cuuint64_t)words, (cuuint64_t)blocks};
  const cuuint64_t strides[2] = {(cuuint64_t)kSfWordBytes, (cuuint64_t)(words * kSfWordBytes)};
  const cuuint32_t box[3] = {(cuuint32_t)(kSfWordBytes / 4), (cuuint32_t)box_words, (cuuint32_t)box_blocks};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The logits [T, V] as the epilogue stores them: pieces of 128 ids x some tokens.
bool logits_tmap(CUtensorMap* map, void* base, int32_t dtype, int64_t T, int64_t V, int64_t ld) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)V, (cuuint64_t)T};
  const cuuint64_t strides[1] = {(cuuint64_t)(ld * elem_bytes(dtype))};
  const cuuint32_t box[2] = {128, (cuuint32_t)mx_out_tokens(elem_bytes(dtype))};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, dtype == DIFR_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool mx_supported(int64_t rows, int64_t d) { return rows <= kMaxRows && d <= kMaxD; }

// (empty batches carry no buffers: the pointers are looked at only where there are rows)
difr_status convert_checks(const void* codes, const void* scales, int32_t format, int64_t rows, int64_t d,
                           const void* plain, int32_t dtype, int64_t ld) {
  if (!known_format(format) || !known_dtype(dtype) || rows < 0 || d <= 0 || ld < d) return DIFR_ERR_INVALID_ARG;
  if (!mx_supported(rows, d) || ld > kMaxLd) return DIFR_ERR_SHAPE;
  if (rows == 0) return DIFR_OK;
  if (!codes || !scales || !plain) return DIFR_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(scales) || !aligned_to(plain, elem_bytes(dtype))) return DIFR_ERR_ALIGN;
  return DIFR_OK;
}

difr_status product_checks(int32_t format, int64_t T, int64_t d, int64_t V, int32_t dtype, int64_t ld) {
  if (!known_format(format) || (dtype != DIFR_F32 && dtype != DIFR_BF16)) return DIFR_ERR_INVALID_ARG;
  if (T < 0 || d <= 0 || V <= 0 || ld < V) return DIFR_ERR_INVALID_ARG;
  if (!mx_supported(T, d) || V > kMaxRows || ld > kMaxLd) return DIFR_ERR_SHAPE;
  return DIFR_OK;
}

// How a product of T >= 1 tokens is cut into tiles: the kernel's parameters, tokens per tile, grid.
difr_status mx_plan(int32_t format, int64_t T, int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld,
                    int32_t* device_status, MxLogitsParams* out, int* tokens_per_tile, int* grid) {
  // tokens per tile: the smallest width that holds all tokens, tiles of 256 beyond 128
  int bn = 16;
  while (bn < 256 && bn < T) bn *= 2;
  const int64_t n_vt = (V + kMxPairM - 1) / kMxPairM;
  if (n_vt * ((T + bn - 1) / bn) > (int64_t)1 << 29) return DIFR_ERR_SHAPE;  // tile numbers are 32-bit
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  // Where tiles of 256 leave half of the pairs idle, tiles of 128: twice as many, each about half as long (1024 x 1000 x
  // 8192 in 8 bits, 16 tiles: 20 us instead of 26; 600 x 3000 x 6000, 36 tiles: 17.3 instead of 22).  Otherwise W would
  // only be loaded twice as often (777 x 32000 x 1749: 60 us instead of 52).
  if (bn == 256 && n_vt * ((T + 255) / 256) <= pairs / 2) bn = 128;
  const int64_t n_tt = (T + bn - 1) / bn;
  MxLogitsParams p;
  memset(&p, 0, sizeof p);
  const int64_t pitch = mx_pitch_bytes(format, d);
  p.logits = logits; p.ld = ld; p.device_status = device_status;
  p.T = (int)T; p.V = (int)V;
  p.k_steps = (int)((pitch + 127) / 128);
  p.last_mmas = (int)((pitch - (int64_t)(p.k_steps - 1) * 128 + 31) / 32);
  p.n_vt = (int)n_vt; p.n_tt = (int)n_tt;
  p.n_tiles = (int)(n_vt * n_tt);
  // the last token tile is only as wide as its tokens (in steps of 16, what the MMA takes)
  p.last_tokens = (int)((T - (n_tt - 1) * bn + 15) / 16 * 16);
  // tokens of a raster group: about 32 MB of codes, a quarter of L2, so that they stay there while W passes
  const int64_t per_tile = (int64_t)bn * pitch;
  int64_t group = ((int64_t)32 << 20) / per_tile;
  if (group < 1) group = 1;
  if (group > n_tt) group = n_tt;
  p.group = (int)group;
  // W is read once where there is one token tile; one that L2 cannot keep for the next call either (96 of its 126 MB) goes
  // by it.  Codes of d = 2048 in 8 bits, read again in every call, 48 tokens: 260 MB 51.9 us by it, 53.4 otherwise; 112 MB
  // 27.2 and 27.9; 80 MB 16.6 and 17.3, but there it also puts out what other kernels keep in L2.  One token: 0 to 4 %.
  p.w_once = n_tt == 1 && V * pitch > ((int64_t)96 << 20);
  p.pack_pairs = dtype == DIFR_BF16 && ld % 2 == 0 && aligned_to(logits, 4);
  p.tile_stores = bn == 256 && vector_rows(logits, ld, dtype) && ld <= ((int64_t)1 << 36);
  const int n_pairs = p.n_tiles < pairs ? p.n_tiles : pairs;
  // a pair's token tiles follow each other in steps of n_pairs - shift: prime to their number, all come in turn
  if (n_pairs > 1)
    while (p.shift < n_pairs - 1 && common_divisor(n_pairs - p.shift, p.group) != 1) ++p.shift;
  *out = p;
  *tokens_per_tile = bn;
  *grid = 2 * n_pairs;
  return DIFR_OK;
}

}  // namespace

extern "C" {

size_t difr_mx_codes_bytes(int32_t format, int64_t rows, int64_t d) {
  if (!known_format(format) || rows < 1 || d < 1 || !mx_supported(rows, d)) return 0;
  return (size_t)rows * (size_t)mx_pitch_bytes(format, d);
}

size_t difr_mx_scales_bytes(int64_t rows, int64_t d) {
  if (rows < 1 || d < 1 || !mx_supported(rows, d)) return 0;
  return (size_t)((rows + kSfWordRows - 1) / kSfWordRows) * (size_t)mx_words(d) * (size_t)kSfWordBytes;
}

difr_status difr_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t d, int64_t ldx, int32_t format,
                             void* codes, void* scales, difr_stream_t stream) {
  const difr_status st = convert_checks(codes, scales, format, rows, d, x, dtype, ldx);
  if (st != DIFR_OK || rows == 0) return st;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  MxConvertParams p;
  memset(&p, 0, sizeof p);
  p.in = x; p.codes = static_cast<unsigned char*>(codes); p.scales = static_cast<unsigned char*>(scales);
  p.rows = rows; p.ld = ldx; p.d = (int)d; p.fmt = format; p.vec = d % 8 == 0 && vector_rows(x, ldx, dtype);
  return launch_mx_quantize(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

difr_status difr_mx_dequantize(const void* codes, const void* scales, int32_t format, int64_t rows, int64_t d,
                               void* out, int32_t dtype, int64_t ldo, difr_stream_t stream) {
  const difr_status st = convert_checks(codes, scales, format, rows, d, out, dtype, ldo);
  if (st != DIFR_OK) return st;
  if (dtype == DIFR_F16) return DIFR_ERR_INVALID_ARG;  // its range ends far inside the formats'
  if (rows == 0) return DIFR_OK;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  MxConvertParams p;
  memset(&p, 0, sizeof p);
  p.out = out;
  p.codes = static_cast<unsigned char*>(const_cast<void*>(codes));
  p.scales = static_cast<unsigned char*>(const_cast<void*>(scales));
  p.rows = rows; p.ld = ldo; p.d = (int)d; p.fmt = format; p.vec = d % 8 == 0 && vector_rows(out, ldo, dtype);
  return launch_mx_dequantize(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK
                                                                                              : DIFR_ERR_CUDA;
}

difr_status difr_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const void* weight,
                          int32_t dtype, int64_t T, int64_t d, float eps, const difr_norm_out* out,
                          difr_stream_t stream) {
  if (!out || !known_dtype(dtype) || T < 0 || d <= 0 || !(eps > 0.f) || !isfinite(eps)) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 && !known_format(out->mx_format)) return DIFR_ERR_INVALID_ARG;
  if (T > kMaxRows || d > kNormMaxD) return DIFR_ERR_SHAPE;
  if (T == 0) return DIFR_OK;
  if (!x || !weight) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 ? (!out->codes || !out->scales) : (out->codes || out->scales)) return DIFR_ERR_INVALID_ARG;
  if (!out->h && out->mx_format == 0) return DIFR_ERR_INVALID_ARG;
  if (out->residual && !residual) return DIFR_ERR_INVALID_ARG;
  if (ldx < d || (residual && ld_residual < d) || (out->residual && out->ld_residual < d) || (out->h && out->ldh < d))
    return DIFR_ERR_INVALID_ARG;
  if (ldx > kMaxLd || (residual && ld_residual > kMaxLd) ||
      (out->residual && out->ld_residual > kMaxLd) || (out->h && out->ldh > kMaxLd))
    return DIFR_ERR_SHAPE;
  const int eb = elem_bytes(dtype);
  if (!aligned_to(x, eb) || !aligned_to(weight, eb) || (residual && !aligned_to(residual, eb)) ||
      (out->residual && !aligned_to(out->residual, eb)) || (out->h && !aligned_to(out->h, 2)))
    return DIFR_ERR_ALIGN;
  if (out->mx_format != 0 && (!aligned16(out->codes) || !aligned16(out->scales))) return DIFR_ERR_ALIGN;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  NormParams p;
  memset(&p, 0, sizeof p);
  p.x = x; p.residual = residual; p.weight = weight; p.residual_out = out->residual; p.h = out->h;
  p.codes = static_cast<unsigned char*>(out->codes); p.scales = static_cast<unsigned char*>(out->scales);
  p.T = T; p.ldx = ldx; p.ld_residual = ld_residual; p.ld_residual_out = out->ld_residual; p.ldh = out->ldh;
  p.d = (int)d; p.fmt = out->mx_format; p.eps = eps; p.inv_d = 1.f / (float)d;
  p.vec = d % 8 == 0 && vector_rows(x, ldx, dtype) && aligned16(weight) &&
          (!residual || vector_rows(residual, ld_residual, dtype)) &&
          (!out->residual || vector_rows(out->residual, out->ld_residual, dtype)) &&
          (!out->h || vector_rows(out->h, out->ldh, DIFR_BF16));
  return launch_rms_norm(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

difr_status difr_mx_logits(const void* h_codes, const void* h_scales, const void* W_codes, const void* W_scales,
                           int32_t format, int64_t T, int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld,
                           int32_t* device_status, difr_stream_t stream) {
  const difr_status st = product_checks(format, T, d, V, dtype, ld);
  if (st != DIFR_OK || T == 0) return st;
  if (!h_codes || !h_scales || !W_codes || !W_scales || !logits) return DIFR_ERR_INVALID_ARG;
  if (!aligned16(h_codes) || !aligned16(h_scales) || !aligned16(W_codes) || !aligned16(W_scales) ||
      !aligned_to(logits, elem_bytes(dtype)))
    return DIFR_ERR_ALIGN;
  MxLogitsParams p;
  int bn = 0, grid = 0;
  const difr_status plan = mx_plan(format, T, d, V, logits, dtype, ld, device_status, &p, &bn, &grid);
  if (plan != DIFR_OK) return plan;
  const int words = format == DIFR_MX8 ? 1 : 2;
  CUtensorMap tw, th, th_last, tsw, tsh;
  if (!codes_tmap(&tw, W_codes, format, V, d, 128) || !codes_tmap(&th, h_codes, format, T, d, bn / 2) ||
      !scales_tmap(&tsw, W_scales, V, d, words, 1) || !scales_tmap(&tsh, h_scales, T, d, words, bn > 128 ? 2 : 1))
    return DIFR_ERR_CUDA;
  th_last = th;
  if (p.last_tokens != bn && !codes_tmap(&th_last, h_codes, format, T, d, p.last_tokens / 2)) return DIFR_ERR_CUDA;
  CUtensorMap tout;
  memset(&tout, 0, sizeof tout);
  if (p.tile_stores && !logits_tmap(&tout, logits, dtype, T, V, ld)) return DIFR_ERR_CUDA;
  return launch_mx_logits(format, bn, dtype, tw, th, th_last, tsw, tsh, tout, p, grid, reinterpret_cast<cudaStream_t>(stream)) ==
                 cudaSuccess
             ? DIFR_OK
             : DIFR_ERR_CUDA;
}

difr_status difr_selftest_mx_wait(int32_t format, int64_t T, int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld,
                                  int32_t done_tiles, int64_t limit_cycles, int32_t* device_status,
                                  difr_stream_t stream) {
  if (done_tiles < 0 || limit_cycles < 1 || limit_cycles > 1000000000LL) return DIFR_ERR_INVALID_ARG;
  const difr_status st = product_checks(format, T, d, V, dtype, ld);
  if (st != DIFR_OK || T == 0) return st;
  if (!logits) return DIFR_ERR_INVALID_ARG;
  if (!aligned_to(logits, elem_bytes(dtype))) return DIFR_ERR_ALIGN;
  MxLogitsParams p;
  int bn = 0, grid = 0;
  const difr_status plan = mx_plan(format, T, d, V, logits, dtype, ld, device_status, &p, &bn, &grid);
  if (plan != DIFR_OK) return plan;
  return launch_mx_wait_selftest(format, bn, dtype, p, done_tiles, (long long)limit_cycles, grid,
                                 reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess
             ? DIFR_OK
             : DIFR_ERR_CUDA;
}

}  // extern "C"
