// C ABI of a decoding step's operators: block norm, 4-bit weights with group scales, verification of drafted tokens.
// Argument checks and launches; nothing here computes.
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include "../../include/difr.h"
#include "difr_host.h"
#include "logit_plan.h"
#include "mx_device.cuh"
#include "step_kernels.h"
#include "w4_device.cuh"

namespace {

using namespace difr;

bool known_group(int32_t g) { return g == 32 || g == 64 || g == 128; }

difr_status w4_convert_checks(const void* codes, const void* scales, int32_t group, int64_t rows, int64_t d, const void* plain,
                              int32_t dtype, int64_t ld) {
  if (!known_group(group) || !known_dtype(dtype) || rows < 0 || d <= 0 || ld < d) return DIFR_ERR_INVALID_ARG;
  if (rows > kMaxRows || d > kMaxD || ld > kMaxLd) return DIFR_ERR_SHAPE;
  if (rows == 0) return DIFR_OK;
  if (!codes || !scales || !plain) return DIFR_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(scales) || !aligned_to(plain, elem_bytes(dtype))) return DIFR_ERR_ALIGN;
  return DIFR_OK;
}

W4ConvertParams w4_convert_params(const void* codes, const void* scales, int32_t group, int64_t rows, int64_t d,
                                  const void* plain, int32_t dtype, int64_t ld) {
  W4ConvertParams p;
  memset(&p, 0, sizeof p);
  p.codes = static_cast<unsigned char*>(const_cast<void*>(codes));
  p.scales = static_cast<__nv_bfloat16*>(const_cast<void*>(scales));
  p.rows = rows; p.ld = ld; p.d = (int)d; p.group = group;
  p.vec = d % 8 == 0 && vector_rows(plain, ld, dtype);
  return p;
}

// Workspace of the product: exponents of the tokens, then h as fp16 in rows of whole 64 values.
int64_t w4_h16_pitch(int64_t d) { return (d + 63) / 64 * 64; }
int64_t w4_exponent_bytes(int64_t T) { return (T * 4 + 255) / 256 * 256; }

// Tensor map of rows of bytes (codes) or fp16 (h): boxes of 128 bytes (128-byte swizzle) x box_rows rows.
bool rows_tmap(CUtensorMap* map, const void* base, CUtensorMapDataType type, int elem, int64_t rows, int64_t cols, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(cols * elem)};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scales: boxes of eight of kW4FewIds rows.
bool scales_tmap(CUtensorMap* map, const void* base, int64_t rows, int64_t spitch) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)spitch, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(spitch * 2)};
  const cuuint32_t box[2] = {8, kW4FewIds};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

difr_status w4_product_checks(int64_t T, int64_t d, int64_t V, int32_t dtype, int64_t ld) {
  if (dtype != DIFR_F32 && dtype != DIFR_BF16) return DIFR_ERR_INVALID_ARG;
  if (T < 0 || d <= 0 || V <= 0 || ld < V) return DIFR_ERR_INVALID_ARG;
  if (T > kMaxRows || d > kMaxD || V > kMaxRows || ld > kMaxLd) return DIFR_ERR_SHAPE;
  return DIFR_OK;
}

// How a product of T >= 1 tokens is cut up: what of the kernel's parameters the sizes and the logits decide, tokens per tile, grid.
difr_status w4_plan(int64_t T, int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld, int32_t* device_status,
                    W4LogitsParams* p, int* bn, int* grid) {
  if (too_many_tiles(T, V, 32)) return DIFR_ERR_SHAPE;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  memset(p, 0, sizeof *p);
  const int64_t h16_pitch = w4_h16_pitch(d);
  plan_logit_tiles(T, V, h16_pitch * 2, V * w4_pitch_bytes(d), 32, logits, dtype, ld, device_status, pairs, p, bn, grid);
  p->d = (int)d; p->h16_pitch = (int)h16_pitch;
  p->k_steps = (int)((d + 127) / 128);
  p->half_last = d - (int64_t)(p->k_steps - 1) * 128 <= 64;
  p->few = T <= kW4Few;
  return DIFR_OK;
}

// Records of a row: its vectors, of which the first may begin before the row.
int64_t verify_chunks(int64_t V, int elem) {
  const int64_t n = 16 / elem;
  return ((V + 2 * (n - 1)) / n + kVerifyChunkVecs - 1) / kVerifyChunkVecs;
}
bool verify_supported(int64_t B, int64_t n_drafts, int64_t V) {
  return n_drafts + B <= kMaxRows && V <= ((int64_t)1 << 27) && B <= ((int64_t)1 << 27);
}

}  // namespace

extern "C" {

difr_status difr_block_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const difr_block* block,
                            const void* weight, int32_t dtype, int64_t T, int64_t d, float eps, const difr_norm_out* out,
                            difr_stream_t stream) {
  if (!out || !block || !known_dtype(dtype) || T < 0 || d <= 0 || !(eps > 0.f) || !isfinite(eps)) return DIFR_ERR_INVALID_ARG;
  if (!isfinite(block->scale) || !isfinite(block->residual_scale) || !isfinite(block->weight_offset))
    return DIFR_ERR_INVALID_ARG;
  if (block->post_weight && (!(block->post_eps > 0.f) || !isfinite(block->post_eps))) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 && !known_format(out->mx_format)) return DIFR_ERR_INVALID_ARG;
  if (T > kMaxRows || d > kNormMaxD) return DIFR_ERR_SHAPE;
  if (T == 0) return DIFR_OK;
  if (!x || !residual) return DIFR_ERR_INVALID_ARG;
  if (out->mx_format != 0 ? (!out->codes || !out->scales) : (out->codes || out->scales)) return DIFR_ERR_INVALID_ARG;
  const bool normed = out->h || out->mx_format != 0;
  if (normed ? !weight : (weight || !out->residual)) return DIFR_ERR_INVALID_ARG;
  const int64_t ld_gate = block->gate ? block->ld_gate : 0;
  if (ldx < d || ld_residual < d || (ld_gate != 0 && ld_gate < d) || (out->residual && out->ld_residual < d) ||
      (out->h && out->ldh < d))
    return DIFR_ERR_INVALID_ARG;
  if (ldx > kMaxLd || ld_residual > kMaxLd || ld_gate > kMaxLd || (out->residual && out->ld_residual > kMaxLd) ||
      (out->h && out->ldh > kMaxLd))
    return DIFR_ERR_SHAPE;
  const int eb = elem_bytes(dtype);
  if (!aligned_to(x, eb) || !aligned_to(residual, eb) || !aligned_to(weight, eb) || !aligned_to(block->post_weight, eb) ||
      !aligned_to(block->gate, eb) || (out->residual && !aligned_to(out->residual, eb)) || (out->h && !aligned_to(out->h, 2)))
    return DIFR_ERR_ALIGN;
  if (out->mx_format != 0 && (!aligned16(out->codes) || !aligned16(out->scales))) return DIFR_ERR_ALIGN;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  BlockNormParams p;
  memset(&p, 0, sizeof p);
  p.x = x; p.residual = residual; p.post_weight = block->post_weight; p.gate = block->gate; p.weight = weight;
  p.residual_out = out->residual; p.h = out->h;
  p.codes = static_cast<unsigned char*>(out->codes); p.scales = static_cast<unsigned char*>(out->scales);
  p.T = T; p.ldx = ldx; p.ld_residual = ld_residual; p.ld_gate = ld_gate;
  p.ld_residual_out = out->ld_residual; p.ldh = out->ldh;
  p.d = (int)d; p.fmt = out->mx_format; p.eps = eps; p.post_eps = block->post_eps; p.inv_d = 1.f / (float)d;
  p.alpha = block->scale; p.beta = block->residual_scale; p.weight_offset = block->weight_offset;
  p.vec = d % 8 == 0 && vector_rows(x, ldx, dtype) && vector_rows(residual, ld_residual, dtype) && aligned16(weight) &&
          aligned16(block->post_weight) && vector_rows(block->gate, ld_gate, dtype) &&
          (!out->residual || vector_rows(out->residual, out->ld_residual, dtype)) &&
          (!out->h || vector_rows(out->h, out->ldh, DIFR_BF16));
  return launch_block_norm(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

size_t difr_w4_codes_bytes(int64_t rows, int64_t d) {
  if (rows < 1 || d < 1 || rows > kMaxRows || d > kMaxD) return 0;
  return (size_t)rows * (size_t)w4_pitch_bytes(d);
}

size_t difr_w4_scales_bytes(int64_t rows, int64_t d, int32_t group) {
  if (rows < 1 || d < 1 || rows > kMaxRows || d > kMaxD || !known_group(group)) return 0;
  return (size_t)rows * (size_t)w4_scale_pitch(d, group) * 2;
}

difr_status difr_w4_quantize(const void* x, int32_t dtype, int64_t rows, int64_t d, int64_t ldx, int32_t group, void* codes,
                             void* scales, difr_stream_t stream) {
  const difr_status st = w4_convert_checks(codes, scales, group, rows, d, x, dtype, ldx);
  if (st != DIFR_OK || rows == 0) return st;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  W4ConvertParams p = w4_convert_params(codes, scales, group, rows, d, x, dtype, ldx);
  p.in = x;
  return launch_w4_quantize(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

difr_status difr_w4_dequantize(const void* codes, const void* scales, int32_t group, int64_t rows, int64_t d, void* out,
                               int32_t dtype, int64_t ldo, difr_stream_t stream) {
  const difr_status st = w4_convert_checks(codes, scales, group, rows, d, out, dtype, ldo);
  if (st != DIFR_OK) return st;
  if (dtype == DIFR_F16) return DIFR_ERR_INVALID_ARG;  // a bf16 scale's range is not fp16's
  if (rows == 0) return DIFR_OK;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  W4ConvertParams p = w4_convert_params(codes, scales, group, rows, d, out, dtype, ldo);
  p.out = out;
  return launch_w4_dequantize(p, dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

size_t difr_w4_workspace_bytes(int64_t T, int64_t d) {
  if (T < 1 || d < 1 || T > kMaxRows || d > kMaxD) return 0;
  return (size_t)(w4_exponent_bytes(T) + T * w4_h16_pitch(d) * 2);
}

difr_status difr_w4_logits(const void* h, int64_t ldh, const void* W_codes, const void* W_scales, int32_t group, int64_t T,
                           int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld, void* workspace,
                           size_t workspace_bytes, int32_t* device_status, difr_stream_t stream) {
  if (!known_group(group) || ldh < d) return DIFR_ERR_INVALID_ARG;
  const difr_status st = w4_product_checks(T, d, V, dtype, ld);
  if (st != DIFR_OK) return st;
  if (ldh > kMaxLd) return DIFR_ERR_SHAPE;
  if (T == 0) return DIFR_OK;
  if (!h || !W_codes || !W_scales || !logits) return DIFR_ERR_INVALID_ARG;
  if (!aligned_to(h, 2) || !aligned16(W_codes) || !aligned16(W_scales) || !aligned_to(logits, elem_bytes(dtype)) ||
      !aligned_to(device_status, 4) || !aligned16(workspace))
    return DIFR_ERR_ALIGN;
  if (!workspace || workspace_bytes < difr_w4_workspace_bytes(T, d)) return DIFR_ERR_WORKSPACE;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  W4LogitsParams p;
  int bn = 0, grid = 0;
  const difr_status plan = w4_plan(T, d, V, logits, dtype, ld, device_status, &p, &bn, &grid);
  if (plan != DIFR_OK) return plan;
  const int64_t pitch = w4_pitch_bytes(d), h16_pitch = w4_h16_pitch(d);
  p.h = static_cast<const __nv_bfloat16*>(h);
  p.scales = static_cast<const __nv_bfloat16*>(W_scales);
  p.token_exp = static_cast<int*>(workspace);
  p.h16 = reinterpret_cast<__half*>(static_cast<char*>(workspace) + w4_exponent_bytes(T));
  p.ldh = ldh; p.group = group;
  p.h_vec = vector_rows(h, ldh, DIFR_BF16);
  CUtensorMap tw, th, th_last, tout;
  if (p.few) {
    if (!rows_tmap(&tw, W_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, V, pitch, kW4FewIds) || !scales_tmap(&th, W_scales, V, w4_scale_pitch(d, group)))
      return DIFR_ERR_CUDA;
    return launch_w4_few(dtype, tw, th, p, s) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
  }
  if (!rows_tmap(&tw, W_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, V, pitch, 128) ||
      !rows_tmap(&th, p.h16, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, T, h16_pitch, bn / 2))
    return DIFR_ERR_CUDA;
  th_last = th;
  if (p.last_tokens != bn && !rows_tmap(&th_last, p.h16, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, T, h16_pitch, p.last_tokens / 2))
    return DIFR_ERR_CUDA;
  memset(&tout, 0, sizeof tout);
  if (p.tile_stores && !logits_tmap(&tout, logits, dtype, T, V, ld)) return DIFR_ERR_CUDA;
  return launch_w4_logits(bn, dtype, tw, th, th_last, tout, p, grid, s) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

difr_status difr_selftest_w4_wait(int64_t T, int64_t d, int64_t V, void* logits, int32_t dtype, int64_t ld, int32_t done_tiles,
                                  int64_t limit_cycles, int32_t* device_status, difr_stream_t stream) {
  if (done_tiles < 0 || limit_cycles < 1 || limit_cycles > 1000000000LL) return DIFR_ERR_INVALID_ARG;
  const difr_status st = w4_product_checks(T, d, V, dtype, ld);
  if (st != DIFR_OK || T == 0) return st;
  if (!logits) return DIFR_ERR_INVALID_ARG;
  if (!aligned_to(logits, elem_bytes(dtype)) || !aligned_to(device_status, 4)) return DIFR_ERR_ALIGN;
  W4LogitsParams p;
  int bn = 0, grid = 0;
  const difr_status plan = w4_plan(T, d, V, logits, dtype, ld, device_status, &p, &bn, &grid);
  if (plan != DIFR_OK) return plan;
  return launch_w4_wait_selftest(bn, dtype, p, done_tiles, (long long)limit_cycles, grid, reinterpret_cast<cudaStream_t>(stream)) ==
                 cudaSuccess
             ? DIFR_OK
             : DIFR_ERR_CUDA;
}

size_t difr_verify_workspace_bytes(int64_t B, int64_t n_drafts, int64_t V) {
  if (B < 1 || n_drafts < 0 || V < 1 || B > kMaxRows || n_drafts > kMaxRows || !verify_supported(B, n_drafts, V)) return 0;
  return ((size_t)(n_drafts + B) * (size_t)verify_chunks(V, 4) + (size_t)B) * sizeof(float4);
}

difr_status difr_verify_drafts(const difr_drafts* in, int64_t B, int64_t n_drafts, int64_t V, const difr_drafts_out* out,
                               difr_stream_t stream) {
  if (!in || !out || !known_dtype(in->dtype) || B < 0 || n_drafts < 0 || V <= 0) return DIFR_ERR_INVALID_ARG;
  if (in->max_drafts < 0 || in->max_drafts > kVerifyMaxDrafts) return DIFR_ERR_INVALID_ARG;
  if (!in->temperatures && (!(in->temperature >= 0.f) || !isfinite(in->temperature))) return DIFR_ERR_INVALID_ARG;
  if (in->ld < V || (in->draft_probs && in->ld_draft < V)) return DIFR_ERR_INVALID_ARG;
  if (B > kMaxRows || n_drafts > kMaxRows || !verify_supported(B, n_drafts, V) || in->ld > kMaxLd ||
      (in->draft_probs && in->ld_draft > kMaxLd))
    return DIFR_ERR_SHAPE;
  if (B == 0) return DIFR_OK;
  if (!in->logits || !in->offsets || !in->sample_words || !out->tokens || !out->n_accepted) return DIFR_ERR_INVALID_ARG;
  if (n_drafts > 0 && (!in->draft_tokens || !in->accept_words)) return DIFR_ERR_INVALID_ARG;
  if (!aligned_to(in->logits, elem_bytes(in->dtype)) || !aligned_to(in->draft_probs, 4) || !aligned_to(in->draft_tokens, 4) ||
      !aligned_to(in->offsets, 4) || !aligned_to(in->accept_words, 4) || !aligned_to(in->sample_words, 4) ||
      !aligned_to(in->temperatures, 4) || !aligned_to(out->tokens, 4) || !aligned_to(out->n_accepted, 4) ||
      !aligned_to(out->p_draft, 4) || !aligned_to(out->status, 4) || !aligned16(out->workspace))
    return DIFR_ERR_ALIGN;
  VerifyParams p;
  memset(&p, 0, sizeof p);
  p.chunks = (int)verify_chunks(V, elem_bytes(in->dtype));
  if (!out->workspace || out->workspace_bytes < difr_verify_workspace_bytes(B, n_drafts, V))
    return DIFR_ERR_WORKSPACE;
  int pairs = 0;
  const difr_status ds = device_pairs(&pairs);
  if (ds != DIFR_OK) return ds;
  p.logits = in->logits; p.probs = in->draft_probs; p.drafted = in->draft_tokens; p.offsets = in->offsets;
  p.accept_words = in->accept_words; p.sample_words = in->sample_words;
  p.temperatures = in->temperatures; p.temperature = in->temperature;
  p.tokens = out->tokens; p.n_accepted = out->n_accepted; p.p_draft = out->p_draft; p.status = out->status;
  p.picks = static_cast<float4*>(out->workspace);
  p.records = p.picks + B;
  p.ld = in->ld; p.ld_probs = in->ld_draft;
  p.B = (int)B; p.n_drafts = (int)n_drafts; p.V = (int)V; p.max_drafts = in->max_drafts;
  return launch_verify_drafts(p, in->dtype, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? DIFR_OK : DIFR_ERR_CUDA;
}

}  // extern "C"
