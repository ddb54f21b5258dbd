// Verification of drafted tokens against the target's logits, from given random words.  Per request, with n drafted tokens
// x_j, target rows l_j (j = 0 .. n), p_j = softmax(l_j / Temp), draft probabilities q_j (1 at x_j where none are given):
//
//   x_j is accepted iff mu_j q_j(x_j) < p_j(x_j);  m = the first refused one (n: none)
//   the next token is the first id i with sum over k <= i of r(k) > nu sum of r,
//   r = max(p_m - q_m, 0) (p_m itself where that is zero everywhere), or p_n where nothing was refused
//
// Five kernels.  `draft_rows` reads every row once, a CTA a chunk of it, and leaves (largest logit, sum of exponentials, first
// id of the largest) per chunk in fp32: bound by the logits' bytes.  `draft_merge`, a CTA a request, joins the records and
// walks the drafts.  Of the row a request ends at `draft_sums` takes the sums of chunks of ids, of the exponentials first where a
// residual needs the row's sum before it can be added up, and `draft_pick` finds the token in the chunk that holds the target.
// Whole numbers hang on these comparisons, so what decides is in fp64: exponentials of the sampled row, and the row sum of a
// draft whose acceptance lies within fp32's error of the border, which `draft_merge` then takes again.  (As one kernel with a
// cluster of CTAs a request, the sampling spent its time at the clusters' barriers: 151 us and more for 192 requests of 151936
// ids, where all five now take 177 with an L2 flushed between calls, 61 of them bytes.)
#include <cuda_runtime.h>
#include <string.h>

#include "mx_device.cuh"
#include "step_kernels.h"

namespace difr {

constexpr int kRowThreads = 256, kRowVecs = kVerifyChunkVecs / kRowThreads;
constexpr int kMergeThreads = 256;
constexpr int kSumThreads = 256, kSumWarps = kSumThreads / 32, kSumIds = 8192;  // ids of a chunk of sums
constexpr double kLog2e = 1.4426950408889634, kLn2 = 0.6931471805599453;
// Relative error allowed for a row sum from fp32 terms: an exponent is off by 2^-23 times itself (terms beyond 2^-40 of the
// sum do not count), ex2 by 2^-22, sums of 1024 vectors by a few 2^-24: under 2^-17 in all.
constexpr double kNearBorder = 1.0 / 65536;

// The larger one; NaN where one is NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// The request that target row `row` belongs to: the last b with offsets[b] + b <= row.
__device__ __forceinline__ int request_of_row(const int32_t* offsets, int B, int64_t row) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)offsets[mid] + mid <= row) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Sixteen bytes of logits as they lie in memory: a thread keeps four of them, unpacked where they are used, so that 2048
// threads fit an SM.
template <typename X>
struct LogitVec;
template <>
struct LogitVec<float> {
  static constexpr int n = 4;
  static constexpr uint32_t none = 0xFF800000u;  // -infinity
  static __device__ __forceinline__ float get(const uint4& q, int i) {
    return __uint_as_float(i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w);
  }
  static __device__ __forceinline__ float largest(const uint4& q) {
    return max_nan(max_nan(get(q, 0), get(q, 1)), max_nan(get(q, 2), get(q, 3)));
  }
};
template <typename H2>
__device__ __forceinline__ H2 as_pair(uint32_t w) { return *reinterpret_cast<const H2*>(&w); }
__device__ __forceinline__ uint32_t vec_word(const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; }
template <>
struct LogitVec<__nv_bfloat16> {
  static constexpr int n = 8;
  static constexpr uint32_t none = 0xFF80FF80u;
  static __device__ __forceinline__ float get(const uint4& q, int i) {
    const uint32_t w = vec_word(q, i >> 1);
    return __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
  }
  static __device__ __forceinline__ float largest(const uint4& q) {
    using H2 = __nv_bfloat162;
    const H2 m = __hmax2_nan(__hmax2_nan(as_pair<H2>(q.x), as_pair<H2>(q.y)), __hmax2_nan(as_pair<H2>(q.z), as_pair<H2>(q.w)));
    return max_nan(__low2float(m), __high2float(m));
  }
};
template <>
struct LogitVec<__half> {
  static constexpr int n = 8;
  static constexpr uint32_t none = 0xFC00FC00u;
  static __device__ __forceinline__ float get(const uint4& q, int i) {
    const __half2 h = as_pair<__half2>(vec_word(q, i >> 1));
    return (i & 1) ? __high2float(h) : __low2float(h);
  }
  static __device__ __forceinline__ float largest(const uint4& q) {
    using H2 = __half2;
    const H2 m = __hmax2_nan(__hmax2_nan(as_pair<H2>(q.x), as_pair<H2>(q.y)), __hmax2_nan(as_pair<H2>(q.z), as_pair<H2>(q.w)));
    return max_nan(__low2float(m), __high2float(m));
  }
};

template <typename X>
__global__ void __launch_bounds__(kRowThreads, 8) draft_rows(const VerifyParams p) {
  using L = LogitVec<X>;
  constexpr int N = L::n;
  __shared__ float2 part[kRowThreads / 32];
  __shared__ int part_id[kRowThreads / 32];
  const int64_t row = blockIdx.x;
  const int chunk = blockIdx.y;
  const X* l = static_cast<const X*>(p.logits) + row * p.ld;
  // vectors lie on 16-byte boundaries of memory: the first one of a row may begin before it
  const int before = (int)((reinterpret_cast<uintptr_t>(l) & 15u) / sizeof(X));
  const int first = chunk * kVerifyChunkVecs * N + (int)threadIdx.x * N - before;  // of this thread; kRowThreads N further each
  // (`draft_merge` overwrites it for every draft of a request that it looks at)
  if (p.p_draft != nullptr && chunk == 0 && threadIdx.x == 0 && row < p.n_drafts) p.p_draft[row] = __int_as_float(0x7FC00000);
  uint4 v[kRowVecs];
  const float none = __int_as_float(0xFF800000);
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k) {
    const int e0 = first + k * kRowThreads * N;
    if (e0 >= 0 && e0 + N <= p.V) {
      v[k] = __ldg(reinterpret_cast<const uint4*>(l + e0));
    } else {
      uint32_t w[4] = {L::none, L::none, L::none, L::none};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (e0 + i < 0 || e0 + i >= p.V) continue;
        if constexpr (sizeof(X) == 4) {
          w[i] = reinterpret_cast<const uint32_t*>(l)[e0 + i];
        } else {
          const uint32_t one = reinterpret_cast<const uint16_t*>(l)[e0 + i];
          w[i >> 1] = (i & 1) ? (w[i >> 1] & 0xFFFFu) | one << 16 : (w[i >> 1] & 0xFFFF0000u) | one;
        }
      }
      v[k] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  float temperature = p.temperature;
  if (p.temperatures != nullptr) temperature = p.temperatures[request_of_row(p.offsets, p.B, row)];
  float m = L::largest(v[0]);
#pragma unroll
  for (int k = 1; k < kRowVecs; ++k) m = max_nan(m, L::largest(v[k]));
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
  float sum = 0.f;
  int id = 0x7fffffff;
  const float c = temperature > 0.f ? fminf((float)kLog2e / temperature, 3.4e38f) : 0.f;
  if (temperature > 0.f) {
    if (m > none) {  // (also false for NaN, which decides by itself)
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kRowVecs; ++k)
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          // (the difference first: a product of its own would round at the size of the logits)
          const float2 z = fmul2(fadd2(make_float2(L::get(v[k], i), L::get(v[k], i + 1)), make_float2(-m, -m)), make_float2(c, c));
          s2 = fadd2(s2, make_float2(ex2_approx(z.x), ex2_approx(z.y)));
        }
      sum = s2.x + s2.y;
    }
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
  } else {
#pragma unroll
    for (int k = kRowVecs - 1; k >= 0; --k)
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (L::get(v[k], i) == m) id = first + k * kRowThreads * N + i;
    id = __reduce_min_sync(0xffffffffu, id);
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) {
    part[warp] = make_float2(m, sum);
    part_id[warp] = id;
  }
  __syncthreads();
  if (warp == 0) {
    const bool there = lane < kRowThreads / 32;
    const float2 mine = there ? part[lane] : make_float2(none, 0.f);
    id = there ? part_id[lane] : 0x7fffffff;
    m = mine.x;
#pragma unroll
    for (int s = 4; s >= 1; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
    sum = mine.x > none ? mine.y * ex2_approx((mine.x - m) * c) : 0.f;
#pragma unroll
    for (int s = 4; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (mine.x != m) id = 0x7fffffff;
    id = __reduce_min_sync(0xffffffffu, id);
    if (lane == 0) p.records[row * p.chunks + chunk] = make_float4(m, sum, __int_as_float(id), 0.f);
  }
}

// 2^y for y <= 0 in fp64 (0 below 2^-1000): 2^(n / 256) from the table, the rest by the series of 2^f = exp(f ln 2), |f| <=
// 2^-9, to its fourth power: off by 2^-54 and the roundings.
constexpr int kExpTable = 256;
__device__ __forceinline__ void fill_exp_table(double* table) {
  for (int i = threadIdx.x; i < kExpTable; i += blockDim.x) table[i] = exp2((double)i / kExpTable);
}
__device__ __forceinline__ double exp2_neg(double y, const double* table) {
  const double magic = 6755399441055744.0 / kExpTable;  // 1.5 * 2^52 / 256: rounds to whole 256ths
  const double t = y + magic;
  const int n = __double2loint(t);
  const double f = y - (t - magic);
  constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4;
  double s = fma(f, c4, c3);
  s = fma(f, s, c2);
  s = fma(f, s, c1);
  s = fma(f, s, 1.0);
  s *= table[n & (kExpTable - 1)];
  // (the exponent goes into the upper word; y's, compared there too, is that of -1000 or beyond)
  s = __hiloint2double(__double2hiint(s) + ((n >> 8) << 20), __double2loint(s));
  return (uint32_t)__double2hiint(y) >= 0xC08F4000u ? 0.0 : s;
}

enum DraftState : int { kRefused = 0, kAccepted = 1, kNear = 2, kBroken = 3 };

__device__ __forceinline__ double uniform(uint32_t word) { return ((double)word + 0.5) * (1.0 / 4294967296.0); }
__device__ __forceinline__ double draft_q(const VerifyParams& p, int draft, int x) {
  if (p.probs == nullptr) return 1.0;
  return x >= 0 && x < p.V ? (double)p.probs[(int64_t)draft * p.ld_probs + x] : 0.0;
}
// The terms that a token is sampled by: exponentials of a row, one id left out or none, or what the draft leaves of the
// probabilities.
template <typename X>
struct SampledRow {
  const X* row;
  const float* q_row;  // null: exponentials
  const double* table;
  double m, c, inv_z;
  int without;         // -1: none; exponentials only

  __device__ __forceinline__ double exponential(float l) const { return exp2_neg(((double)l - m) * c, table); }
  template <bool RES>
  __device__ __forceinline__ double term(float l, float q) const {
    const double e = exponential(l);
    if (!RES) return e;
    const double r = fma(e, inv_z, -(double)q);
    return r > 0.0 ? r : 0.0;  // (0 for a NaN too)
  }
  // Eight ids of each lane from i0 on, 32 apart; what is behind the range has no probability.
  struct Some {
    float l[8], q[8];
  };
  template <bool RES>
  __device__ __forceinline__ void load(Some& s, int i0, int to) const {
    const int lane = threadIdx.x & 31;
    if (i0 + 256 <= to) {
      const X* l = row + i0 + lane;
#pragma unroll
      for (int u = 0; u < 8; ++u) s.l[u] = (float)l[32 * u];
      if (RES) {
        const float* q = q_row + i0 + lane;
#pragma unroll
        for (int u = 0; u < 8; ++u) s.q[u] = q[32 * u];
      }
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + lane + 32 * u;
        s.l[u] = i < to ? (float)row[i] : __int_as_float(0xFF800000);
        if (RES) s.q[u] = i < to ? q_row[i] : 0.f;
      }
    }
    if (!RES && (unsigned)(without - i0) < 256u) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + lane + 32 * u == without) s.l[u] = __int_as_float(0xFF800000);
    }
  }
  template <bool RES>
  __device__ __forceinline__ double terms(const Some& s) const {
    double a = 0.0, b = 0.0;
#pragma unroll
    for (int u = 0; u < 8; u += 2) {
      a += term<RES>(s.l[u], s.q[u]);
      b += term<RES>(s.l[u + 1], s.q[u + 1]);
    }
    return a + b;
  }
  // Sum over the ids from .. to, in all lanes of the warp; the next ids are under way while some are worked on.  `first` holds
  // the first ones.
  template <bool RES>
  __device__ __forceinline__ double sum(int from, int to, Some& first) const {
    double acc = 0.0;
    for (int i0 = from; i0 < to; i0 += 512) {
      Some second;
      if (i0 + 256 < to) load<RES>(second, i0 + 256, to);
      acc += terms<RES>(first);
      if (i0 + 512 < to) load<RES>(first, i0 + 512, to);
      if (i0 + 256 < to) acc += terms<RES>(second);
    }
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) acc += shfl_xor_double(acc, s);
    return acc;
  }
  template <bool RES>
  __device__ __forceinline__ double sum(int from, int to) const {
    Some first;
    load<RES>(first, from, to);
    return sum<RES>(from, to, first);
  }
  __device__ __forceinline__ double sum(int from, int to) const {
    return q_row != nullptr ? sum<true>(from, to) : sum<false>(from, to);
  }
};

// Of a request: what is sampled, by mode.
enum PickMode : int { kPickNone = 0, kPickRow = 1, kPickWithout = 2, kPickResidual = 3 };

__device__ __forceinline__ double scale_of(float temperature) { return kLog2e / (double)temperature; }
__device__ __forceinline__ float temperature_of(const VerifyParams& p, int b) {
  return p.temperatures != nullptr ? p.temperatures[b] : p.temperature;
}

// Joins the records of a request's rows, a warp a row, and walks its drafts.
template <typename X>
__global__ void __launch_bounds__(kMergeThreads) draft_merge(const VerifyParams p) {
  __shared__ double table[kExpTable];
  __shared__ double warp_sums[kMergeThreads / 32];
  __shared__ float row_max[kVerifyMaxDrafts + 1];
  __shared__ int row_id[kVerifyMaxDrafts + 1];
  __shared__ int state[kVerifyMaxDrafts + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x;
  const float none = __int_as_float(0xFF800000);
  fill_exp_table(table);
  const int o0 = p.offsets[b], o1 = p.offsets[b + 1];
  const float temperature = temperature_of(p, b);
  __syncthreads();
  grid_wait();
  grid_release();
  uint32_t status = 0;
  if (o0 < 0 || o1 < o0 || o1 > p.n_drafts || o1 - o0 > p.max_drafts) status |= kDraftBadOffsets;
  if (!(temperature >= 0.f) || temperature > 3.4e38f) status |= kDraftBadTemperature;
  int32_t* tokens = p.tokens + (int64_t)b * (p.max_drafts + 1);
  int m = 0, mode = kPickNone;
  if (status == 0) {  // the same in the whole CTA
    const int n = o1 - o0;
    const int64_t row0 = (int64_t)o0 + b;
    const bool greedy = temperature == 0.f;
    const double c = greedy ? 0.0 : scale_of(temperature);
    const X* logits = static_cast<const X*>(p.logits);
    int broken_ids = 0;
    for (int j = warp; j <= n; j += kMergeThreads / 32) {
      const float4* rec = p.records + (row0 + j) * p.chunks;
      const int x = j < n ? p.drafted[o0 + j] : -1;
      const bool known = x >= 0 && x < p.V;
      const float lx = known ? (float)logits[(row0 + j) * p.ld + x] : 0.f;
      const double bound = j < n ? uniform(p.accept_words[o0 + j]) * draft_q(p, o0 + j, x) : 0.0;
      float top = none;
      for (int k = lane; k < p.chunks; k += 32) top = max_nan(top, rec[k].x);
#pragma unroll
      for (int s = 16; s >= 1; s >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, s));
      const bool fine = top > none && top < -none;
      double sum = 0.0;
      int id = 0x7fffffff;
      for (int k = lane; k < p.chunks; k += 32) {
        const float4 r = rec[k];
        if (r.x > none) sum += (double)r.y * exp2_neg(((double)r.x - (double)top) * c, table);
        if (r.x == top) id = min(id, __float_as_int(r.z));
      }
#pragma unroll
      for (int s = 16; s >= 1; s >>= 1) sum += shfl_xor_double(sum, s);
      id = __reduce_min_sync(0xffffffffu, id);
      int st = fine ? kRefused : kBroken;
      double pd = __longlong_as_double(0x7FF8000000000000LL);
      if (j < n) {
        if (!known) broken_ids = 1;
        if (fine) {
          pd = !known ? 0.0 : greedy ? (x == id ? 1.0 : 0.0) : exp2_neg(((double)lx - (double)top) * c, table) / sum;
          if (bound < pd) st = kAccepted;
          if (!greedy && known && fabs(bound - pd) <= kNearBorder * pd) st = kNear;
        }
        if (lane == 0 && p.p_draft != nullptr) p.p_draft[o0 + j] = (float)pd;
      }
      if (lane == 0) {
        row_max[j] = top;
        row_id[j] = id;
        state[j] = st;
      }
    }
    broken_ids = __syncthreads_or(broken_ids);
    if (broken_ids) status |= kDraftBadToken;
    bool broken = false;
    for (; m < n; ++m) {
      int st = state[m];
      if (st == kNear) {
        const SampledRow<X> r = {logits + (row0 + m) * p.ld, nullptr, table, (double)row_max[m], c, 1.0, -1};
        const int per_warp = (p.V + kMergeThreads / 32 - 1) / (kMergeThreads / 32);
        const int from = min(p.V, warp * per_warp);
        const double acc = r.sum(from, min(p.V, from + per_warp));
        __syncthreads();
        if (lane == 0) warp_sums[warp] = acc;
        __syncthreads();
        double z = 0.0;
        for (int w = 0; w < kMergeThreads / 32; ++w) z += warp_sums[w];
        const int x = p.drafted[o0 + m];
        st = uniform(p.accept_words[o0 + m]) * draft_q(p, o0 + m, x) < r.exponential((float)r.row[x]) / z ? kAccepted : kRefused;
      }
      if (st == kAccepted) continue;
      broken = st == kBroken;
      break;
    }
    if (m == n) broken = state[n] == kBroken;
    if (broken) status |= kDraftBadRow;
    for (int j = threadIdx.x; j <= p.max_drafts; j += kMergeThreads)
      tokens[j] = j < m ? p.drafted[o0 + j] : j == m && greedy && !broken ? row_id[m] : -1;
    if (!greedy && !broken) mode = m == n ? kPickRow : p.probs == nullptr ? kPickWithout : kPickResidual;
    if (threadIdx.x == 0) p.picks[b] = make_float4(row_max[m], __int_as_float(mode), __int_as_float(m), 0.f);
  } else {
    for (int j = threadIdx.x; j <= p.max_drafts; j += kMergeThreads) tokens[j] = -1;
    if (threadIdx.x == 0) p.picks[b] = make_float4(0.f, __int_as_float(kPickNone), __int_as_float(0), 0.f);
  }
  if (threadIdx.x == 0) {
    p.n_accepted[b] = m;
    if (p.status != nullptr) p.status[b] = status;
  }
}

// The row that request b samples; its sums of chunks lie where the records of its rows did, (exponentials, terms) each.
template <typename X>
__device__ __forceinline__ SampledRow<X> sampled_row(const VerifyParams& p, int b, float4 pick, const double* table, double2** sums) {
  const int o0 = p.offsets[b], m = __float_as_int(pick.z), mode = __float_as_int(pick.y);
  const int64_t row0 = (int64_t)o0 + b;
  *sums = reinterpret_cast<double2*>(p.records + row0 * p.chunks);
  const int x = mode == kPickWithout ? p.drafted[o0 + m] : -1;
  return {static_cast<const X*>(p.logits) + (row0 + m) * p.ld,
          mode == kPickResidual ? p.probs + (int64_t)(o0 + m) * p.ld_probs : nullptr, table, (double)pick.x,
          scale_of(temperature_of(p, b)), 1.0, x >= 0 && x < p.V ? x : -1};
}
// The row's sum, the same in all lanes of all warps: the chunks' in their order by lanes, then the lanes'.
__device__ __forceinline__ double sum_of_chunks(const double2* sums, int n) {
  double z = 0.0;
  for (int k = threadIdx.x & 31; k < n; k += 32) z += sums[k].x;
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) z += shfl_xor_double(z, s);
  return z;
}

// A chunk's sum.  TERMS: of the terms; otherwise of the exponentials, where a residual needs them.
template <typename X, bool TERMS>
__global__ void __launch_bounds__(kSumThreads, 4) draft_sums(const VerifyParams p) {
  __shared__ double table[kExpTable];
  __shared__ double warp_sums[kSumWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = p.first_request + blockIdx.y, chunk = blockIdx.x, n_chunks = gridDim.x;
  fill_exp_table(table);
  __syncthreads();
  grid_wait();
  grid_release();
  const float4 pick = p.picks[b];
  const int mode = __float_as_int(pick.y);
  if (TERMS ? mode == kPickNone : mode != kPickResidual) return;
  double2* sums;
  SampledRow<X> r = sampled_row<X>(p, b, pick, table, &sums);
  if (!TERMS) r.q_row = nullptr;
  const int from = min(chunk * kSumIds + warp * (kSumIds / kSumWarps), p.V), to = min(from + kSumIds / kSumWarps, p.V);
  typename SampledRow<X>::Some some;
  double acc;
  if (TERMS && mode == kPickResidual) {
    r.template load<true>(some, from, to);  // (under way before the row's sum is put together)
    r.inv_z = 1.0 / sum_of_chunks(sums, n_chunks);
    acc = r.template sum<true>(from, to, some);
  } else {
    acc = r.template sum<false>(from, to);
  }
  if (lane == 0) warp_sums[warp] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int w = 0; w < kSumWarps; ++w) s += warp_sums[w];
    if (TERMS) sums[chunk].y = s; else sums[chunk].x = s;
  }
}

// The token: the chunk that holds the target sum, in it the warp's range, which all warps share out once more, and in that the
// warp that walks its part.  Each time the last range with a sum at all where rounding has the target beyond every one.
template <typename X>
__global__ void __launch_bounds__(kSumThreads) draft_pick(const VerifyParams p) {
  __shared__ double table[kExpTable];
  __shared__ double warp_sums[2][kSumWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x;
  const int n_chunks = (p.V + kSumIds - 1) / kSumIds;
  fill_exp_table(table);
  __syncthreads();
  grid_wait();
  const float4 pick = p.picks[b];
  const int mode = __float_as_int(pick.y), m = __float_as_int(pick.z);
  if (mode == kPickNone) return;
  double2* sums;
  SampledRow<X> r = sampled_row<X>(p, b, pick, table, &sums);
  int32_t* token = p.tokens + (int64_t)b * (p.max_drafts + 1) + m;
  // (lanes take the chunks' sums, so that their loads go out together; the row's sum is the one that the residual was taken by)
  double total = 0.0, z = 0.0;
  for (int k = lane; k < n_chunks; k += 32) {
    total += sums[k].y;
    z += sums[k].x;
  }
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) {
    total += shfl_xor_double(total, s);
    z += shfl_xor_double(z, s);
  }
  const bool left = total > 0.0;
  if (!left && mode == kPickWithout) {  // all of the probability was the drafted token's
    if (threadIdx.x == 0) *token = r.without;
    return;
  }
  if (!left) {  // the draft leaves nothing: the target's own probabilities
    r.q_row = nullptr;
    total = z;
  } else if (mode == kPickResidual) {
    r.inv_z = 1.0 / z;
  }
  const double target = uniform(p.sample_words[b]) * total;
  int from = 0, to = p.V;
  double run = 0.0;
  {
    // 32 chunks at a time: the last with a sum that begins at or before the target
    double before = 0.0;
    int chunk = 0;
    bool any = false;
    for (int k0 = 0; k0 < n_chunks; k0 += 32) {
      const int k = k0 + lane;
      const double own = k < n_chunks ? (left ? sums[k].y : sums[k].x) : 0.0;
      double scan = own;
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, scan, s);
        if (lane >= s) scan += o;
      }
      const double begin = before + scan - own;
      const unsigned some = __ballot_sync(0xffffffffu, own > 0.0), good = __ballot_sync(0xffffffffu, own > 0.0 && begin <= target);
      if (good != 0 || (!any && some != 0)) {
        const int who = good != 0 ? 31 - __clz(good) : __ffs(some) - 1;
        chunk = k0 + who;
        run = __shfl_sync(0xffffffffu, begin, who);
        any = true;
      }
      before += __shfl_sync(0xffffffffu, scan, 31);
    }
    from = chunk * kSumIds;
    to = min(p.V, from + kSumIds);
  }
#pragma unroll 1
  for (int level = 0; level < 2; ++level) {
    const int part = (to - from + kSumWarps - 1) / kSumWarps;
    const int p_first = min(to, from + warp * part);
    const double acc = r.sum(p_first, min(to, p_first + part));
    if (lane == 0) warp_sums[level][warp] = acc;
    __syncthreads();
    int found = -1;
    double found_run = run;
    for (int w = 0; w < kSumWarps; ++w) {
      const double s = warp_sums[level][w];
      if (s > 0.0 && (found < 0 || run <= target)) {
        found = w;
        found_run = run;
      }
      run += s;
    }
    from = min(to, from + max(found, 0) * part);
    to = min(to, from + part);
    run = found_run;
    if (level == 1 && warp != found) from = to;  // one warp walks
  }
  int at = -1;
  constexpr int U = 4;  // neighbours a lane
  for (int i0 = from; i0 < to; i0 += 32 * U) {
    double v[U], own = 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + lane * U + u;
      const float l = i < to && i != r.without ? (float)r.row[i] : __int_as_float(0xFF800000);
      v[u] = r.q_row != nullptr ? r.template term<true>(l, i < to ? r.q_row[i] : 0.f) : r.template term<false>(l, 0.f);
      own += v[u];
    }
    double scan = own;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const double o = __shfl_up_sync(0xffffffffu, scan, s);
      if (lane >= s) scan += o;
    }
    // the first lane that passes the target, or the last one with anything so far
    const unsigned hit = __ballot_sync(0xffffffffu, own > 0.0 && run + scan > target);
    const unsigned some = __ballot_sync(0xffffffffu, own > 0.0);
    if (some != 0) {
      int mine = -1;
      double s = run + scan - own;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v[u] > 0.0 && (mine < 0 || !(s > target))) mine = i0 + lane * U + u;
        s += v[u];
      }
      at = __shfl_sync(0xffffffffu, mine, hit != 0 ? __ffs(hit) - 1 : 31 - __clz(some));
    }
    if (hit != 0) break;
    run += __shfl_sync(0xffffffffu, scan, 31);
  }
  if (lane == 0 && from < to) *token = at;
}

static cudaError_t launch_next(void (*kernel)(const VerifyParams), dim3 grid, int threads, const VerifyParams& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  memset(&attr, 0, sizeof attr);
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename X>
static cudaError_t launch_typed(const VerifyParams& p, cudaStream_t stream) {
  draft_rows<X><<<dim3((unsigned)(p.n_drafts + p.B), (unsigned)p.chunks), kRowThreads, 0, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) e = launch_next(draft_merge<X>, dim3((unsigned)p.B), kMergeThreads, p, stream);
  if (p.temperatures == nullptr && p.temperature == 0.f) return e;  // greedy: done
  const unsigned chunks = (unsigned)((p.V + kSumIds - 1) / kSumIds);
  // (a grid's second dimension holds 65535: requests beyond that in further launches)
  for (int b0 = 0; b0 < p.B && e == cudaSuccess; b0 += 65535) {
    VerifyParams q = p;
    q.first_request = b0;
    const dim3 grid(chunks, (unsigned)(p.B - b0 < 65535 ? p.B - b0 : 65535));
    if (p.probs != nullptr) e = launch_next(draft_sums<X, false>, grid, kSumThreads, q, stream);
    if (e == cudaSuccess) e = launch_next(draft_sums<X, true>, grid, kSumThreads, q, stream);
  }
  if (e == cudaSuccess) e = launch_next(draft_pick<X>, dim3((unsigned)p.B), kSumThreads, p, stream);
  return e;
}

cudaError_t launch_verify_drafts(const VerifyParams& p, int dtype, cudaStream_t stream) {
  return dtype == kBf16 ? launch_typed<__nv_bfloat16>(p, stream)
                        : dtype == kF16 ? launch_typed<__half>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace difr
