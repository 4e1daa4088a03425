// logprob.cu -- log probabilities of logits rows: for each row of z / T the
// log-normaliser, the log probability and the rank of a given column, the
// entropy, and the n best columns.
//
// With M = max z, d_x = (z_x - M) log2(e) / T, S = sum 2^d_x, E = sum 2^d_x d_x:
// lse = M / T + ln S, log p_t = (z_t - M) / T - ln S, and the entropy
// -sum p ln p = ln S - ln 2 E / S. The difference z_x - M is taken first: in the
// product z_x log2(e) / T the rounding of a large z would be an error of the
// whole row. A column of -inf adds nothing (d is held at -256, 2^d is 0).
#include <cstdint>

#include "tt_device.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"

namespace tt {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kLn2 = 0.693147180559945f;

// Order of a logit as an unsigned number (-0 as 0); above 0 for every logit.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// The row's columns c0 .. c1 - 1 in steps of one per thread.
template <int DT, typename F>
__device__ __forceinline__ void each_logit(const char* row, int V, F&& f) {
  for (int x = threadIdx.x; x < V; x += kThreads) f(load_logit<DT>(row, x), x);
}

__device__ __forceinline__ float block_max(float v, float* red) {
  v = warp_max_f(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < kWarps; ++w) v = fmaxf(v, red[w]);
  return v;
}

template <typename T>
__device__ __forceinline__ T block_sum(T v, T* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < kWarps; ++w) v += red[w];
  return v;
}

// The n best of the row's columns above -inf, in order, into best (keys: order
// of the logit above the complement of the column; 0 where there are fewer): a
// radix search for the n-th largest logit, the columns above it, and the first
// of those equal to it.
template <int DT>
__device__ void select_best(const char* row, int V, int n, unsigned long long* best) {
  __shared__ unsigned int hist[256];
  __shared__ unsigned int s_prefix, s_want, s_count;
  __shared__ unsigned int s_warp[kWarps];
  __shared__ unsigned long long found[TT_MAX_TOP_K];
  const int t = threadIdx.x;
  const uint32_t empty = order_key(-INFINITY);
  if (t == 0) {
    s_prefix = 0;
    s_want = n;
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[t] = 0;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    each_logit<DT>(row, V, [&](float z, int) {
      const uint32_t k = order_key(z);
      if (k > empty && (shift == 24 || (k >> (shift + 8)) == prefix >> (shift + 8)))
        atomicAdd(&hist[(k >> shift) & 255], 1u);
    });
    __syncthreads();
    if (t == 0) {
      unsigned int want = s_want;
      int b = 255;
      while (b > 0 && hist[b] < want) want -= hist[b--];
      // (b = 0 with too few left: every column above -inf is taken)
      s_want = min(want, hist[b]);
      s_prefix = prefix | uint32_t(b) << shift;
    }
    __syncthreads();
  }
  const uint32_t tau = s_prefix;      // the n-th largest, or no more than the smallest
  const unsigned int equal = s_want;  // how many of its equals are taken, in column order
  if (t == 0) s_count = 0;
  __syncthreads();
  each_logit<DT>(row, V, [&](float z, int x) {
    const uint32_t k = order_key(z);
    if (k > tau && k > empty) {
      const unsigned int p = atomicAdd(&s_count, 1u);
      if (p < TT_MAX_TOP_K) found[p] = uint64_t(k) << 32 | uint32_t(~x);
    }
  });
  __syncthreads();
  const unsigned int above = min(s_count, unsigned(n));
  unsigned int taken = 0;
  for (int x0 = 0; x0 < V && taken < equal; x0 += kThreads) {
    const int x = x0 + t;
    const uint32_t k = x < V ? order_key(load_logit<DT>(row, x)) : 0u;
    const bool eq = k == tau && k > empty;
    const unsigned int bits = __ballot_sync(0xffffffffu, eq);
    __syncthreads();
    if ((t & 31) == 0) s_warp[t >> 5] = __popc(bits);
    __syncthreads();
    unsigned int p = taken + __popc(bits & ((1u << (t & 31)) - 1));
    unsigned int all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < (t >> 5)) p += s_warp[w];
      all += s_warp[w];
    }
    if (eq && p < equal && above + p < unsigned(n))
      found[above + p] = uint64_t(k) << 32 | uint32_t(~x);
    taken += all;
  }
  __syncthreads();
  const unsigned int have = min(above + min(taken, equal), unsigned(n));
  if (t < n) best[t] = 0;
  __syncthreads();
  if (t < int(have)) {
    int r = 0;
    for (unsigned int j = 0; j < have; ++j) r += found[j] > found[t];
    best[r] = found[t];
  }
  __syncthreads();
}

template <int DT>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const __grid_constant__ LogprobArgs a) {
  __shared__ float red[kWarps];
  __shared__ int redi[kWarps];
  __shared__ unsigned long long best[TT_MAX_TOP_K];
  const int64_t r = blockIdx.x;
  const char* row = a.data + r * a.stride_bytes;
  const int id = a.ids ? a.ids[r] : -1;
  const bool given = id >= 0 && id < a.V;
  const float zt = given ? load_logit<DT>(row, id) : 0.f;
  float m = -INFINITY;
  each_logit<DT>(row, a.V, [&](float z, int) { m = fmaxf(m, z); });
  m = block_max(m, red);
  float S = 0.f, E = 0.f;
  int before = 0;
  each_logit<DT>(row, a.V, [&](float z, int x) {
    const float d = (z - m) * a.scale, e = ex2_approx(d);
    S += e;
    E = fmaf(e, fmaxf(d, -256.f), E);
    before += z > zt || (z == zt && x < id);
  });
  S = block_sum(S, red);
  E = block_sum(E, red);
  before = block_sum(before, redi);
  const bool ok = S > 0.f && S < INFINITY;  // neither empty nor NaN or +inf
  if (a.top_n > 0 && ok) select_best<DT>(row, a.V, a.top_n, best);
  const float nan = __int_as_float(0x7fffffff), ln_s = logf(S), lse = m / a.temp + ln_s;
  if (threadIdx.x == 0) {
    a.out.status[r] = (ok ? 0 : TT_REQ_NOT_FINITE) |
                      (given || id == -1 ? 0 : TT_REQ_ID_OUT_OF_RANGE);
    if (a.out.lse) a.out.lse[r] = ok ? lse : nan;
    if (a.out.entropy) a.out.entropy[r] = ok ? ln_s - kLn2 * (E / S) : nan;
    if (a.out.logprob)
      a.out.logprob[r] = !ok || (!given && id != -1) ? nan : given ? (zt - m) / a.temp - ln_s : 0.f;
    if (a.out.rank) a.out.rank[r] = ok && given ? before : -1;
  }
  if (threadIdx.x < a.top_n) {
    const unsigned long long k = ok ? best[threadIdx.x] : 0;
    const int64_t at = r * a.top_n + threadIdx.x;
    if (a.out.top_ids) a.out.top_ids[at] = k ? int32_t(~uint32_t(k)) : -1;
    if (a.out.top_logprobs)
      a.out.top_logprobs[at] = !ok ? nan
                               : k ? (key_value(uint32_t(k >> 32)) - m) / a.temp - ln_s
                                   : -INFINITY;
  }
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& a, int dt, cudaStream_t stream, int) {
  const dim3 grid{unsigned(a.rows)};
  if (dt == TT_F32)
    logprob_kernel<TT_F32><<<grid, kThreads, 0, stream>>>(a);
  else
    logprob_kernel<TT_BF16><<<grid, kThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t preload_logprobs() {
  cudaFuncAttributes attr;
  cudaError_t e = cudaFuncGetAttributes(&attr, logprob_kernel<TT_F32>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&attr, logprob_kernel<TT_BF16>);
  return e;
}

}  // namespace tt
