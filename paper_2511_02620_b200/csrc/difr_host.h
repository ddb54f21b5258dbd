// Host-side helpers shared by the files that implement the C entry points.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/difr.h"

namespace difr {

// Largest rows, hidden sizes and row strides of the operators around the LM head.
constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxD = (int64_t)1 << 20, kMaxLd = (int64_t)1 << 40;

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = nullptr;
  if (fn == nullptr) {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(sym);
  }
  return fn;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned_to(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(n - 1)) == 0; }
inline int elem_bytes(int32_t dtype) { return dtype == DIFR_F32 ? 4 : 2; }
inline bool known_dtype(int32_t dtype) { return dtype == DIFR_BF16 || dtype == DIFR_F16 || dtype == DIFR_F32; }
inline bool known_format(int32_t f) { return f == DIFR_MX8 || f == DIFR_MX4; }
// rows of `ld` elements that all start on 16-byte boundaries
inline bool vector_rows(const void* p, int64_t ld, int32_t dtype) {
  return aligned16(p) && (ld * elem_bytes(dtype)) % 16 == 0;
}

}  // namespace difr
