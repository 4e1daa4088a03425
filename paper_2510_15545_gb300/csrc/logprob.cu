// logprob.cu -- log probabilities of logits rows: for each row of z / T the
// log-normaliser, the log probability and the rank of a given column, the
// entropy, and the n best columns.
//
// With M = max z, d_x = (z_x - M) log2(e) / T, S = sum 2^d_x, E = sum 2^d_x d_x:
// lse = M / T + ln S, log p_t = (z_t - M) / T - ln S, and the entropy
// -sum p ln p = ln S - ln 2 E / S. The difference z_x - M is taken first: in the
// product z_x log2(e) / T the rounding of a large z would be an error of the
// whole row. A column of -inf adds nothing: it counts as one so low that its 2^d
// is 0, with a finite d.
//
// One pass over the logits: each thread keeps its own M (sums are scaled when it
// rises), S, E and the columns that come before the given one. The best columns
// need a bar that the n best of the row reach: each warp posts the k-th largest
// of its lanes' maxima, k = ceil(n / warps), and since those are k different
// columns of each warp, at least n columns reach the least of the posts. What
// reaches the bar as it stands is gathered; a few hundred of 200,000 columns do.
// Rows for which more than the buffer holds do (long runs of equal logits at the
// bar) are searched digit by digit, reading them again. When there are few rows, a
// cluster of CTAs shares each and joins its parts through distributed shared
// memory.
//
// Measured: 4096 rows of 201,088 bf16 columns with ids and 20 best 314 us, 5.2 TB/s
// (without either 254 us, 6.5 TB/s); 608 rows of 151,936 fp32 columns 62 us, 5.9
// TB/s; one row 7 us. The logits are the bound for the plain sums; the
// ends of rows, where the best columns are gathered and nothing is loaded, take most
// of the rest (45 us), the count of the columns before the given ones 10.
#include <algorithm>
#include <cooperative_groups.h>
#include <cstdint>

#include "tt_device.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"
#include "tt_x2.cuh"

namespace tt {

namespace {

// Vectors of a thread between two looks at the bar, all loaded before the first is
// used: 4096 rows of 201,088 bf16 columns 349 us with 4, 319 with 6, 314 with 8 (3000
// rows of 4096 16, 18 and 20).
constexpr int kBatch = 8;
constexpr int kVectors = 2048;      // room for vectors that reach the bar
constexpr int kCandidates = 1024;   // and for columns that reach the last one
constexpr int kMaxSplit = 16;
// CTAs have 256 threads while those of all rows fit the SMs at once, 4 to an SM, and
// 128, 8 to an SM, for more rows: the end of a row, which has no loads of its own,
// holds up fewer threads, and the last rows leave less idle. Narrow / wide, us: 4096
// rows of 201,088 bf16 columns 312 / 328, 1000 of 32,000 fp32 26.9 / 30.2, 3000 of 4096
// bf16 20.2 / 34.7; but 608 of 151,936 fp32 76 / 62, 310 of 128,256 bf16 44 / 31.
constexpr int kWidePerSm = 4;
constexpr float kLeast = -3.402823466e38f;  // -inf never reaches a bar
constexpr float kLn2 = 0.693147180559945f;

namespace cg = cooperative_groups;

// Order of a logit as an unsigned number (-0 as 0); above 0 for every logit.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

// The columns c0 .. c1 - 1 in steps of one per thread.
template <int DT, int kThreads, typename F>
__device__ __forceinline__ void each_logit(const char* row, int c0, int c1, F&& f) {
  for (int x = c0 + threadIdx.x; x < c1; x += kThreads) f(load_logit<DT>(row, x), x);
}

// The n best of the columns c0 .. c1 - 1 above -inf, in order, into best (keys:
// order of the logit above the complement of the column; 0 where there are
// fewer): a radix search for the n-th largest logit, the columns above it, and
// the first of those equal to it.
template <int DT, int kThreads>
__device__ __noinline__ void select_best(const char* row, int c0, int c1, int n,
                                         unsigned long long* best) {
  constexpr int kWarps = kThreads / 32;
  __shared__ unsigned int hist[256];
  __shared__ unsigned int s_prefix, s_want, s_count;
  __shared__ unsigned int s_warp[kWarps];
  __shared__ unsigned long long found[TT_MAX_TOP_K];
  const int t = threadIdx.x;
  const uint32_t empty = order_key(-INFINITY);
  __syncthreads();
  if (t == 0) {
    s_prefix = 0;
    s_want = n;
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = t; i < 256; i += kThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    each_logit<DT, kThreads>(row, c0, c1, [&](float z, int) {
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
  each_logit<DT, kThreads>(row, c0, c1, [&](float z, int x) {
    const uint32_t k = order_key(z);
    if (k > tau && k > empty) {
      const unsigned int p = atomicAdd(&s_count, 1u);
      if (p < TT_MAX_TOP_K) found[p] = uint64_t(k) << 32 | uint32_t(~x);
    }
  });
  __syncthreads();
  const unsigned int above = min(s_count, unsigned(n));
  unsigned int taken = 0;
  for (int x0 = c0; x0 < c1 && taken < equal; x0 += kThreads) {
    const int x = x0 + t;
    const uint32_t k = x < c1 ? order_key(load_logit<DT>(row, x)) : 0u;
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

// The sums of some columns: their maximum z, sum of 2^d over all but one column
// of that maximum and of 2^d d over all, with d = (z - max) log2(e) / T, and how
// many come before the given column. (The maximum's own 1 is kept apart: next to
// it, the rest of a row that one column dominates would be rounded away, and that
// is all of the column's log probability.)
struct Sums {
  float m, s, e;
  int before;
};
__device__ __forceinline__ void join(Sums& a, const Sums& b, float scale) {
  const bool swap = b.m > a.m;
  const float m = swap ? b.m : a.m, low = swap ? a.m : b.m;
  const float ls = swap ? a.s : b.s, le = swap ? a.e : b.e;
  // (d of -inf, or of the type's whole range: the factor is 0)
  const float d = low == m ? 0.f : fmaxf((low - m) * scale, -256.f), f = ex2_approx(d);
  const float sum = (low > -INFINITY ? 1.f : 0.f) + ls;
  a.s = fmaf(f, sum, swap ? b.s : a.s);
  a.e = fmaf(f, fmaf(sum, d, le), swap ? b.e : a.e);
  a.m = m;
  a.before += b.before;
}

template <int DT>
struct Logit;
template <>
struct Logit<TT_F32> {
  static constexpr uint32_t kMinusInf = 0xff800000u;
};
template <>
struct Logit<TT_BF16> {
  static constexpr uint32_t kMinusInf = 0xff80ff80u;
};

// A logit so far below `top` that its 2^d is 0, but whose d is finite, which the
// d of -inf would not be: taken in place of everything below it. Rounded down to
// a bf16; below the type's lowest value that is -inf (see number).
template <int DT>
__device__ __forceinline__ uint32_t lowest(float top, float reach) {
  float z = top - reach;
  if (!(z < top)) z = fmaf(fabsf(top), -1.2e-7f, top);
  const uint32_t u = __float_as_uint(z);
  if constexpr (DT == TT_F32) return u;
  const uint32_t h = (z < 0.f ? u + 0xffffu : u) >> 16;
  return h << 16 | h;
}

// A thread's E, 0 in place of NaN: it is NaN where a d was -inf, which next to a
// maximum at the end of the type's range is every column but its equals, whose d
// is 0. (A logit that is NaN makes S NaN too.)
__device__ __forceinline__ f32x2 number(f32x2 e) {
  float lo, hi;
  split(e, lo, hi);
  return pair(lo == lo ? lo : 0.f, hi == hi ? hi : 0.f);
}

// How many of a vector's logits are at or above a threshold, added to `n` (two
// counts of up to 256 in bf16, or one in fp32, as a number of the logits' type).
template <int DT>
__device__ __forceinline__ void count_at_least(const uint4& w, uint32_t threshold, uint32_t& n) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t one;
    if constexpr (DT == TT_F32) {
      asm("set.ge.f32.f32 %0, %1, %2;" : "=r"(one) : "r"(x[q]), "r"(threshold));
      asm("add.f32 %0, %0, %1;" : "+r"(n) : "r"(one));
    } else {
      asm("set.ge.bf16x2.bf16x2 %0, %1, %2;" : "=r"(one) : "r"(x[q]), "r"(threshold));
      asm("add.bf16x2 %0, %0, %1;" : "+r"(n) : "r"(one));
    }
  }
}
template <int DT>
__device__ __forceinline__ int count_of(uint32_t n) {
  if constexpr (DT == TT_F32) return int(__uint_as_float(n));
  return int(__uint_as_float(n << 16)) + int(__uint_as_float(n & 0xffff0000u));
}
// The thresholds of the columns before the given one (its equals come first) and
// behind it (they do not: the next logit of the type).
template <int DT>
__device__ __forceinline__ uint32_t logit_bits(float z) {
  const uint32_t u = __float_as_uint(z);
  return DT == TT_F32 ? u : (u & 0xffff0000u) | u >> 16;
}
template <int DT>
__device__ __forceinline__ float logit_above(float z) {
  constexpr int step = DT == TT_F32 ? 1 : 1 << 16;
  const int u = __float_as_int(z + 0.f);
  return __int_as_float(z == 0.f ? step : u > 0 ? u + step : u - step);
}

template <int kWarps>
struct Shared {
  Sums sums[kWarps];
  Sums mine;  // the CTA's share
  float post[kWarps];
  unsigned int count;  // vectors that reached the bar
  unsigned int kept;   // columns that reach the last one
  int holder;          // the thread of the maximum
  float rest[kWarps];
  unsigned long long best[TT_MAX_TOP_K];
  int vecs[kVectors];
  unsigned long long found[kCandidates];
};

// The n best of `count` keys (n <= TT_MAX_TOP_K; 0 where there are fewer), by
// counting those above each one: keys are distinct.
template <int kThreads>
__device__ __forceinline__ void rank_keys(const unsigned long long* key, int count, int n,
                                          unsigned long long* best) {
  if (threadIdx.x < n) best[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const unsigned long long k = key[i];
    int r = 0;
    for (int j = 0; j < count; ++j) r += key[j] > k;
    if (r < n) best[r] = k;
  }
  __syncthreads();
}

template <int DT, int kThreads>
__global__ void __launch_bounds__(kThreads, 256 * kWidePerSm / kThreads)
    logprob_kernel(const __grid_constant__ LogprobArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  constexpr int kWarps = kThreads / 32;
  __shared__ Shared<kWarps> s;
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = a.split, rank = S > 1 ? int(cluster.block_rank()) : 0;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int64_t r = blockIdx.x / S;
  const char* row = a.data + r * a.stride_bytes;
  const int c0 = min(a.V, rank * a.share), c1 = min(a.V, c0 + a.share);
  const int id = a.ids ? a.ids[r] : -1;
  const bool given = id >= 0 && id < a.V;
  const float zt = given ? load_logit<DT>(row, id) : 0.f;
  const int n = a.top_n, k = (n + kWarps - 1) / kWarps;
  const char* base = row + int64_t(c0) * ESZ;
  const int whole = (c1 - c0) / VEC, nvec = (c1 - c0 + VEC - 1) / VEC;

  constexpr uint32_t kNone = Logit<DT>::kMinusInf;
  const uint4 none = make_uint4(kNone, kNone, kNone, kNone);
  uint4 tail = none;  // the row's last columns
  if (nvec > whole && t == whole % kThreads) {
    const int c = c0 + whole * VEC;
    uint32_t bits[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q)
      bits[q] = __float_as_uint(c + q < c1 ? load_logit<DT>(row, c + q) : -INFINITY);
    if constexpr (DT == TT_F32)
      tail = make_uint4(bits[0], bits[1], bits[2], bits[3]);
    else
      tail = make_uint4(bits[0] >> 16 | bits[1], bits[2] >> 16 | bits[3], bits[4] >> 16 | bits[5],
                        bits[6] >> 16 | bits[7]);
  }
  // this thread's vectors of the batch at v0
  auto load = [&](uint4 (&w)[kBatch], int v0) {
    const char* p = base + (uint32_t(v0 + t) << 4);
    if (v0 + kBatch * kThreads <= whole) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) w[u] = ld_stream_v4(p + u * kThreads * 16);
    } else {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int v = v0 + u * kThreads + t;
        w[u] = v == whole ? tail : none;
        if (v < whole) w[u] = ld_stream_v4(p + u * kThreads * 16);
      }
    }
  };

  Sums x{-INFINITY, 0.f, 0.f, 0};
  // (pairs of sums, even and odd columns; of a thread that has seen nothing but
  // -inf: sums of 0 relative to 0)
  f32x2 s2 = 0, e2 = 0, minus = 0;
  const f32x2 scale2 = pair(a.scale, a.scale);
  uint32_t low = lowest<DT>(0.f, a.reach);
  // the vector that holds the given column, and the thresholds around it
  const int v_id = id >= c0 ? (id - c0) / VEC : -1;
  const uint32_t from = logit_bits<DT>(zt), above = logit_bits<DT>(logit_above<DT>(zt));
  float bar = kLeast;
  if (t == 0) s.count = s.kept = 0;
  int it = 0;
  for (int v0 = 0; v0 < nvec; v0 += kBatch * kThreads, ++it) {
    uint4 w[kBatch];
    load(w, v0);
    float vm[kBatch], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      vm[u] = vec_max<DT>(w[u]);
      top = fmaxf(top, vm[u]);
    }
    if (top > x.m) {
      const float d = fmaxf((x.m - top) * a.scale, -256.f), f = ex2_approx(d);
      const f32x2 d2 = pair(d, d), f2 = pair(f, f);
      e2 = mul2(f2, fma2(s2, d2, number(e2)));
      s2 = mul2(s2, f2);
      x.m = top;
      minus = pair(-top, -top);
      low = lowest<DT>(top, a.reach);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const uint4 y = at_least<DT>(w[u], low);
#pragma unroll
      for (int q = 0; q < VEC / 2; ++q) {
        const f32x2 d = mul2(add2(logit_pair<DT>(y, q), minus), scale2), e = exp2_pair(d);
        s2 = add2(s2, e);
        e2 = fma2(e, d, e2);
      }
    }
    if (given && top >= zt) {
      uint32_t n_before = 0;
      if (v0 + kBatch * kThreads <= whole && uint32_t(v_id - v0) >= kBatch * kThreads) {
        // (all of the batch on one side of the given column)
        const uint32_t threshold = v0 < v_id ? from : above;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) count_at_least<DT>(w[u], threshold, n_before);
      } else {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int v = v0 + u * kThreads + t;
          if (vm[u] >= zt && v != v_id && v < nvec)
            count_at_least<DT>(w[u], v < v_id ? from : above, n_before);
        }
      }
      x.before += count_of<DT>(n_before);
    }
    if (n > 0) {
      if (it < 4 || (it & 3) == 0) {
        // the k-th largest of the lanes' maxima, for all warps to see
        uint32_t key = order_key(x.m), kth = 0;
        for (int j = 0; j < k; ++j) {
          kth = __reduce_max_sync(0xffffffffu, key);
          const unsigned int who = __ballot_sync(0xffffffffu, key == kth);
          if (lane == __ffs(who) - 1) key = 0;
        }
        volatile float* post = s.post;
        if (lane == 0) post[warp] = kth ? key_value(kth) : -INFINITY;
        if (it == 0)
          __syncthreads();
        else
          __syncwarp();
        bar = post[0];
#pragma unroll
        for (int j = 1; j < kWarps; ++j) bar = fminf(bar, post[j]);
        bar = fmaxf(bar, kLeast);
      }
      if (top >= bar) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (vm[u] >= bar) {
            const unsigned int p = atomicAdd(&s.count, 1u);
            if (p < kVectors) s.vecs[p] = v0 + u * kThreads + t;
          }
        }
      }
    }
  }

  // (the columns around the given one within its vector)
  int close = 0;
  if (warp == 0 && given && v_id >= 0 && v_id < nvec && lane < VEC) {
    const int col = c0 + v_id * VEC + lane;
    if (col < c1) {
      const float z = load_logit<DT>(row, col);
      close = z > zt || (z == zt && col < id);
    }
  }
  close = __popc(__ballot_sync(0xffffffffu, close));
  // the CTA's sums
  x.s = sum_pair(s2) - (x.m > -INFINITY ? 1.f : 0.f);
  x.e = sum_pair(number(e2));
  for (int turn = 0; turn < 2; ++turn) {
    Sums y = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Sums other;
      other.m = __shfl_xor_sync(0xffffffffu, y.m, o);
      other.s = __shfl_xor_sync(0xffffffffu, y.s, o);
      other.e = __shfl_xor_sync(0xffffffffu, y.e, o);
      other.before = __shfl_xor_sync(0xffffffffu, y.before, o);
      join(y, other, a.scale);
    }
    if (lane == 0) s.sums[warp] = y;
    __syncthreads();
    if (t == 0) {
      y = s.sums[0];
      y.before += close;
      for (int j = 1; j < kWarps; ++j) join(y, s.sums[j], a.scale);
      s.mine = y;
    }
    __syncthreads();
    const float m = s.mine.m;
    if (turn == 1 || !(m > -INFINITY && s.mine.s < 0.5f)) break;
    // One column dominates, and its thread has summed beside its 1: the thread's
    // columns once more, by all threads, without it.
    if (x.m == m) s.holder = t;
    __syncthreads();
    float rest = 0.f;
    for (int v = s.holder + t * kThreads; v < nvec; v += kThreads * kThreads) {
#pragma unroll
      for (int q = 0; q < VEC; ++q) {
        const int col = c0 + v * VEC + q;
        const float z = col < c1 ? load_logit<DT>(row, col) : -INFINITY;
        if (z != m) rest += ex2_approx((z - m) * a.scale);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
    if (lane == 0) s.rest[warp] = rest;
    __syncthreads();
    if (x.m == m) {
      x.s = s.rest[0];
      for (int j = 1; j < kWarps; ++j) x.s += s.rest[j];
    }
  }
  // and its best columns: the last bar leaves little more than them
  if (n > 0) {
    const int count = int(s.count);
    if (count <= kVectors && nvec > 0) {
      bar = s.post[0];
      for (int j = 1; j < kWarps; ++j) bar = fminf(bar, s.post[j]);
      bar = fmaxf(bar, kLeast);
      for (int i = t; i < count * VEC; i += kThreads) {
        const int col = c0 + s.vecs[i / VEC] * VEC + i % VEC;
        const float z = col < c1 ? load_logit<DT>(row, col) : -INFINITY;
        if (z >= bar) {
          const unsigned int p = atomicAdd(&s.kept, 1u);
          if (p < kCandidates) s.found[p] = uint64_t(order_key(z)) << 32 | uint32_t(~col);
        }
      }
    }
    __syncthreads();
    const int kept = int(s.kept);
    if (count > kVectors || kept > kCandidates)
      select_best<DT, kThreads>(row, c0, c1, n, s.best);
    else
      rank_keys<kThreads>(s.found, kept, n, s.best);
  }
  // the row's, by its first CTA
  if (S > 1) {
    cluster.sync();
    if (rank > 0) {
      cluster.sync();  // (its shared memory is read until here)
      return;
    }
    if (n > 0) {
      for (int i = t; i < S * n; i += kThreads) s.found[i] = cluster.map_shared_rank(s.best, i / n)[i % n];
    }
    if (t == 0) {
      Sums y = s.mine;
      for (int j = 1; j < S; ++j) join(y, *cluster.map_shared_rank(&s.mine, j), a.scale);
      s.sums[0] = y;
      s.kept = 0;
    }
    cluster.sync();
    if (n > 0) rank_keys<kThreads>(s.found, S * n, n, s.best);
    if (t == 0) s.mine = s.sums[0];
  }
  __syncthreads();
  const Sums y = s.mine;
  const bool ok = y.m > -INFINITY && y.s < INFINITY;  // neither empty nor NaN or +inf
  const float nan = __int_as_float(0x7fffffff), ln_s = log1pf(y.s);
  if (t == 0) {
    a.out.status[r] = (ok ? 0 : TT_REQ_NOT_FINITE) |
                      (given || id == -1 ? 0 : TT_REQ_ID_OUT_OF_RANGE);
    if (a.out.lse) a.out.lse[r] = ok ? y.m / a.temp + ln_s : nan;
    if (a.out.entropy) a.out.entropy[r] = ok ? ln_s - kLn2 * (y.e / (1.f + y.s)) : nan;
    if (a.out.logprob)
      a.out.logprob[r] =
          !ok || (!given && id != -1) ? nan : given ? (zt - y.m) / a.temp - ln_s : 0.f;
    if (a.out.rank) a.out.rank[r] = ok && given ? y.before : -1;
  }
  if (t < n) {
    const unsigned long long key = ok ? s.best[t] : 0;
    const int64_t at = r * n + t;
    if (a.out.top_ids) a.out.top_ids[at] = key ? int32_t(~uint32_t(key)) : -1;
    if (a.out.top_logprobs)
      a.out.top_logprobs[at] =
          !ok ? nan : key ? (key_value(uint32_t(key >> 32)) - y.m) / a.temp - ln_s : -INFINITY;
  }
}

template <int DT, int kThreads>
cudaError_t launch(LogprobArgs a, cudaStream_t stream, int sm_count) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  // CTAs of a row: enough to fill the SMs, each with a batch of vectors at least
  int S = 1;
  while (S < kMaxSplit && a.rows * S < 2 * sm_count &&
         a.V / (2 * S) >= kBatch * kThreads * VEC)
    S *= 2;
  a.split = S;
  a.share = ((a.V + S - 1) / S + VEC - 1) / VEC * VEC;
  a.reach = 300.f / a.scale;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(a.rows * S));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = S > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, logprob_kernel<DT, kThreads>, a);
}

template <int DT>
cudaError_t choose(const LogprobArgs& a, cudaStream_t stream, int sm_count) {
  return a.rows > kWidePerSm * sm_count ? launch<DT, 128>(a, stream, sm_count)
                                          : launch<DT, 256>(a, stream, sm_count);
}

// (narrow CTAs are never in clusters)
template <int DT>
cudaError_t preload() {
  cudaFuncAttributes attr;
  const cudaError_t e = cudaFuncGetAttributes(&attr, logprob_kernel<DT, 128>);
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(logprob_kernel<DT, 256>,
                                                 cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs& a, int dt, cudaStream_t stream, int sm_count) {
  return dt == TT_F32 ? choose<TT_F32>(a, stream, sm_count) : choose<TT_BF16>(a, stream, sm_count);
}

cudaError_t preload_logprobs() {
  const cudaError_t e = preload<TT_F32>();
  return e == cudaSuccess ? preload<TT_BF16>() : e;
}

}  // namespace tt
