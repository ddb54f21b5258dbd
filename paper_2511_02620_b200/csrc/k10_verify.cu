// Verification of drafted tokens against the target's logits, from given random words.  Per request, with n drafted tokens
// x_j, target rows l_j (j = 0 .. n), p_j = softmax(l_j / Temp), draft probabilities q_j (1 at x_j where none are given):
//
//   x_j is accepted iff mu_j q_j(x_j) < p_j(x_j);  m = the first refused one (n: none)
//   the next token is the first id i with sum over k <= i of r(k) > nu sum of r,
//   r = max(p_m - q_m, 0) (p_m itself where that is zero everywhere), or p_n where nothing was refused
//
// Two kernels.  `draft_rows` reads every row once, a CTA a chunk of it, and leaves (largest logit, its first id, sum of
// exponentials) per chunk in fp32: bound by the logits' bytes.  `draft_decide`, a cluster of CTAs per request, joins the
// records, walks the drafts, and samples the row it ends at: ids are split into contiguous ranges of CTAs and warps, sums
// are taken in fp64 and the warp whose range holds the target sum walks it once more.  Whole numbers hang on these
// comparisons, so what decides is in fp64: exponentials of the sampled row, and the row sum of a draft whose acceptance lies
// within fp32's error of the border, which the cluster then takes again.
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <string.h>

#include "mx_device.cuh"
#include "step_kernels.h"

namespace cg = cooperative_groups;

namespace difr {

constexpr int kRowThreads = 256, kRowVecs = kVerifyChunkVecs / kRowThreads;
constexpr int kDecideThreads = 512, kDecideWarps = kDecideThreads / 32;
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

template <typename X>
struct LogitVec {
  static constexpr int n = 16 / (int)sizeof(X);
  X e[n];
};

template <typename X>
__global__ void __launch_bounds__(kRowThreads) draft_rows(const VerifyParams p) {
  using V16 = LogitVec<X>;
  constexpr int N = V16::n;
  __shared__ float2 part[kRowThreads / 32];
  __shared__ int part_id[kRowThreads / 32];
  const int64_t row = blockIdx.x;
  const int chunk = blockIdx.y;
  const X* l = static_cast<const X*>(p.logits) + row * p.ld;
  // vectors lie on 16-byte boundaries of memory: the first one of a row may begin before it
  const int before = (int)((reinterpret_cast<uintptr_t>(l) & 15u) / sizeof(X));
  float v[kRowVecs][N];
  const float none = __int_as_float(0xFF800000);
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k) {
    const int64_t at = ((int64_t)chunk * kRowVecs + k) * kRowThreads + threadIdx.x;
    const int64_t e0 = at * N - before;
    if (e0 >= 0 && e0 + N <= p.V) {
      const uint4 raw = __ldg(reinterpret_cast<const uint4*>(l + e0));
      const V16 vec = *reinterpret_cast<const V16*>(&raw);
#pragma unroll
      for (int i = 0; i < N; ++i) v[k][i] = (float)vec.e[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[k][i] = e0 + i >= 0 && e0 + i < p.V ? (float)l[e0 + i] : none;
    }
  }
  float temperature = p.temperature;
  if (p.temperatures != nullptr) temperature = p.temperatures[request_of_row(p.offsets, p.B, row)];
  float m = none;
#pragma unroll
  for (int k = 0; k < kRowVecs; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) m = max_nan(m, v[k][i]);
#pragma unroll
  for (int s = 16; s >= 1; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
  float sum = 0.f;
  int id = 0x7fffffff;
  if (temperature > 0.f) {
    const float c = fminf((float)kLog2e / temperature, 3.4e38f);
    if (m > none) {  // (also false for NaN, which decides by itself)
#pragma unroll
      for (int k = 0; k < kRowVecs; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) sum += ex2_approx((v[k][i] - m) * c);
    }
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
  } else {
#pragma unroll
    for (int k = kRowVecs - 1; k >= 0; --k)
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (v[k][i] == m)
          id = (int)((((int64_t)chunk * kRowVecs + k) * kRowThreads + threadIdx.x) * N - before + i);
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
    const float c = temperature > 0.f ? fminf((float)kLog2e / temperature, 3.4e38f) : 0.f;
    sum = mine.x > none ? mine.y * ex2_approx((mine.x - m) * c) : 0.f;
#pragma unroll
    for (int s = 4; s >= 1; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (mine.x != m) id = 0x7fffffff;
    id = __reduce_min_sync(0xffffffffu, id);
    if (lane == 0) p.records[row * p.chunks + chunk] = make_float4(m, sum, __int_as_float(id), 0.f);
  }
}

// 2^y for y <= 0 in fp64 (0 below 2^-1000): 2^(n / 64) from the table, the rest by the series of exp, |f| <= ln 2 / 128, to
// its fifth power: off by a few 2^-53.
__device__ __forceinline__ double exp2_neg(double y, const double* table) {
  const double magic = 6755399441055744.0 / 64.0;  // 1.5 * 2^52 / 64: rounds to whole 64ths
  const double t = y + magic;
  const int n = __double2loint(t);
  const double f = (y - (t - magic)) * kLn2;
  double s = fma(f, 1.0 / 120.0, 1.0 / 24.0);
  s = fma(f, s, 1.0 / 6.0);
  s = fma(f, s, 0.5);
  s = fma(f, s, 1.0);
  s = fma(f, s, 1.0);
  s *= table[n & 63];
  s = __hiloint2double(__double2hiint(s) + ((n >> 6) << 20), __double2loint(s));
  return y < -1000.0 ? 0.0 : s;
}

enum DraftState : int { kRefused = 0, kAccepted = 1, kNear = 2, kBroken = 3 };

template <typename X>
__global__ void __launch_bounds__(kDecideThreads) draft_decide(const VerifyParams p) {
  __shared__ double table[64];
  __shared__ double warp_sums[kDecideWarps];
  __shared__ double cta_sums[2];
  __shared__ float row_max[kVerifyMaxDrafts + 1];
  __shared__ int row_id[kVerifyMaxDrafts + 1];
  __shared__ int state[kVerifyMaxDrafts + 1];
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b = blockIdx.x / ranks;
  const float none = __int_as_float(0xFF800000);
  if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
  grid_wait();

  const int o0 = p.offsets[b], o1 = p.offsets[b + 1];
  const float temperature = p.temperatures != nullptr ? p.temperatures[b] : p.temperature;
  uint32_t status = 0;
  if (o0 < 0 || o1 < o0 || o1 > p.n_drafts || o1 - o0 > p.max_drafts) status |= kDraftBadOffsets;
  if (!(temperature >= 0.f) || temperature > 3.4e38f) status |= kDraftBadTemperature;
  int32_t* tokens = p.tokens + (int64_t)b * (p.max_drafts + 1);
  if (status != 0) {  // the same in the whole cluster
    if (rank == 0) {
      for (int j = threadIdx.x; j <= p.max_drafts; j += kDecideThreads) tokens[j] = -1;
      if (threadIdx.x == 0) {
        p.n_accepted[b] = 0;
        if (p.status != nullptr) p.status[b] = status;
      }
    }
    return;
  }
  const int n = o1 - o0;
  const int64_t row0 = (int64_t)o0 + b;
  const bool greedy = temperature == 0.f;
  const double c = greedy ? 0.0 : kLog2e / (double)temperature;
  const X* logits = static_cast<const X*>(p.logits);
  __syncthreads();

  auto uniform = [](uint32_t word) { return ((double)word + 0.5) * (1.0 / 4294967296.0); };
  auto draft_q = [&](int j, int x) {
    if (p.probs == nullptr) return 1.0;
    return x >= 0 && x < p.V ? (double)p.probs[(int64_t)(o0 + j) * p.ld_probs + x] : 0.0;
  };
  // Every CTA of the cluster joins the records of all rows for itself, a warp a row.
  int broken_ids = 0;
  for (int j = warp; j <= n; j += kDecideWarps) {
    const float4* rec = p.records + (row0 + j) * p.chunks;
    float m = none;
    for (int k = lane; k < p.chunks; k += 32) m = max_nan(m, rec[k].x);
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
    const bool fine = m > none && m < -none;
    double sum = 0.0;
    int id = 0x7fffffff;
    for (int k = lane; k < p.chunks; k += 32) {
      const float4 r = rec[k];
      if (r.x > none) sum += (double)r.y * exp2_neg(((double)r.x - (double)m) * c, table);
      if (r.x == m) id = min(id, __float_as_int(r.z));
    }
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) sum += shfl_xor_double(sum, s);
    id = __reduce_min_sync(0xffffffffu, id);
    int st = kBroken;
    double pd = __longlong_as_double(0x7FF8000000000000LL);
    if (j < n) {
      const int x = p.drafted[o0 + j];
      const bool known = x >= 0 && x < p.V;
      if (!known) broken_ids = 1;
      if (fine) {
        if (!known)
          pd = 0.0;
        else if (greedy)
          pd = x == id ? 1.0 : 0.0;
        else
          pd = exp2_neg(((double)(float)logits[(row0 + j) * p.ld + x] - (double)m) * c, table) / sum;
        const double bound = uniform(p.accept_words[o0 + j]) * draft_q(j, x);
        st = bound < pd ? kAccepted : kRefused;
        if (!greedy && known && fabs(bound - pd) <= kNearBorder * pd) st = kNear;
      }
      if (rank == 0 && lane == 0 && p.p_draft != nullptr) p.p_draft[o0 + j] = (float)pd;
    } else if (fine) {
      st = kRefused;
    }
    if (lane == 0) {
      row_max[j] = m;
      row_id[j] = id;
      state[j] = st;
    }
  }
  broken_ids = __syncthreads_or(broken_ids);
  if (broken_ids) status |= kDraftBadToken;

  // contiguous ranges of ids: of the CTAs, inside them of the warps
  const int per_cta = (p.V + ranks - 1) / ranks, first = min(p.V, rank * per_cta), last = min(p.V, first + per_cta);
  const int per_warp = (last - first + kDecideWarps - 1) / kDecideWarps;
  const int w_first = min(last, first + warp * per_warp), w_last = min(last, w_first + per_warp);
  // what is summed: exponentials of a row, or what the draft leaves of its probabilities
  const X* row = nullptr;
  const float* q_row = nullptr;
  double m64 = 0.0, inv_z = 1.0;
  int without = -1;
  auto term = [&](float l, float q) {
    const double e = exp2_neg(((double)l - m64) * c, table);
    return q_row != nullptr ? fmax(fma(e, inv_z, -(double)q), 0.0) : e;
  };
  int turn = 0;
  double total = 0.0, before = 0.0;  // of the cluster; of the CTAs before this one
  auto take_sums = [&]() {
    constexpr int U = 8;
    double acc = 0.0;
    for (int i0 = w_first + lane; i0 < w_last; i0 += 32 * U) {
      float l[U], q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + 32 * u;
        l[u] = i < w_last && i != without ? (float)row[i] : none;
        q[u] = q_row != nullptr && i < w_last ? q_row[i] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + 32 * u < w_last) acc += term(l[u], q[u]);
    }
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) acc += shfl_xor_double(acc, s);
    if (lane == 0) warp_sums[warp] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
      double s = 0.0;
      for (int w = 0; w < kDecideWarps; ++w) s += warp_sums[w];
      cta_sums[turn] = s;
    }
    cluster.sync();
    total = before = 0.0;
    for (int r = 0; r < ranks; ++r) {
      const double s = *cluster.map_shared_rank(&cta_sums[turn], r);
      if (r < rank) before += s;
      total += s;
    }
    turn ^= 1;
  };
  auto set_row = [&](int j) {
    row = logits + (row0 + j) * p.ld;
    m64 = (double)row_max[j];
    q_row = nullptr;
    without = -1;
  };

  int m = 0;
  bool broken = false;
  for (; m < n; ++m) {
    int st = state[m];
    if (st == kNear) {
      set_row(m);
      take_sums();
      const int x = p.drafted[o0 + m];
      st = uniform(p.accept_words[o0 + m]) * draft_q(m, x) < exp2_neg(((double)(float)row[x] - m64) * c, table) / total
               ? kAccepted : kRefused;
    }
    if (st == kAccepted) continue;
    broken = st == kBroken;
    break;
  }
  if (m == n) broken = state[n] == kBroken;
  if (broken) status |= kDraftBadRow;
  if (rank == 0) {
    for (int j = threadIdx.x; j <= p.max_drafts; j += kDecideThreads)
      if (j != m || broken) tokens[j] = j < m ? p.drafted[o0 + j] : -1;
    if (threadIdx.x == 0) {
      if (greedy && !broken) tokens[m] = row_id[m];
      p.n_accepted[b] = m;
      if (p.status != nullptr) p.status[b] = status;
    }
  }
  if (!greedy && !broken) {
    set_row(m);
    if (m < n) {
      const int x = p.drafted[o0 + m];
      if (p.probs == nullptr) {
        without = x >= 0 && x < p.V ? x : -1;
      } else {
        take_sums();
        inv_z = 1.0 / total;
        q_row = p.probs + (int64_t)(o0 + m) * p.ld_probs;
      }
    }
    take_sums();
    if (!(total > 0.0)) {  // the draft leaves nothing: the target's own probabilities
      q_row = nullptr;
      without = -1;
      take_sums();
    }
    const double target = uniform(p.sample_words[b]) * total;
    // the CTA whose range holds the target sum; the last one with a sum at all where rounding has it beyond every range
    double mine = 0.0, after = 0.0;
    for (int r = 0; r < ranks; ++r) {
      const double s = *cluster.map_shared_rank(&cta_sums[turn ^ 1], r);
      if (r == rank) mine = s;
      if (r > rank) after += s;
    }
    if (mine > 0.0 && before <= target && (target < before + mine || after == 0.0)) {
      double w_before = before, w_after = 0.0;
      for (int w = 0; w < warp; ++w) w_before += warp_sums[w];
      for (int w = warp + 1; w < kDecideWarps; ++w) w_after += warp_sums[w];
      const double own = warp_sums[warp];
      if (own > 0.0 && w_before <= target && (target < w_before + own || w_after == 0.0)) {
        // this warp's range once more, 32 ids at a time
        double run = w_before;
        int found = -1, last_id = -1;
        for (int i0 = w_first; i0 < w_last && found < 0; i0 += 32) {
          const int i = i0 + lane;
          const bool in = i < w_last;
          const double v = in ? term(i != without ? (float)row[i] : none, q_row != nullptr ? q_row[i] : 0.f) : 0.0;
          double scan = v;
#pragma unroll
          for (int s = 1; s < 32; s <<= 1) {
            const double o = __shfl_up_sync(0xffffffffu, scan, s);
            if (lane >= s) scan += o;
          }
          const unsigned hit = __ballot_sync(0xffffffffu, in && v > 0.0 && run + scan > target);
          const unsigned some = __ballot_sync(0xffffffffu, v > 0.0);
          if (hit != 0) found = i0 + __ffs(hit) - 1;
          if (some != 0) last_id = i0 + 31 - __clz(some);
          run += __shfl_sync(0xffffffffu, scan, 31);
        }
        if (lane == 0) tokens[m] = found >= 0 ? found : last_id;
      }
    }
  }
  cluster.sync();  // (the sums of this CTA may still be read)
}

template <typename X>
static cudaError_t launch_typed(const VerifyParams& p, cudaStream_t stream) {
  draft_rows<X><<<dim3((unsigned)(p.n_drafts + p.B), (unsigned)p.chunks), kRowThreads, 0, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  constexpr int ranks = 8;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)(p.B * ranks), 1, 1);
  cfg.blockDim = dim3(kDecideThreads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  memset(attr, 0, sizeof attr);
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, draft_decide<X>, p);
}

cudaError_t launch_verify_drafts(const VerifyParams& p, int dtype, cudaStream_t stream) {
  return dtype == kBf16 ? launch_typed<__nv_bfloat16>(p, stream)
                        : dtype == kF16 ? launch_typed<__half>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace difr
