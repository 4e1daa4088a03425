// distill.cu -- the loss of student logits rows against a teacher's top log
// probabilities, and its gradient.
//
// With q = softmax(z / T), the teacher's list (x_i, p_i), P = sum p_i, and in
// tail mode the rest of the teacher's mass r = 1 - P on the columns outside the
// list (r = 0 without it), the loss is
//   sum p_i (ln p_i - ln q_i) + r (ln r - ln t),  t = sum of q outside the list,
// and with W = P + r its derivative to z_j is (W q_j - p_j) / T on the list and
// (W - r / t) q_j / T elsewhere. t is summed from its own terms: 1 - (q on the
// list) would lose all digits of a student that has learned its teacher.
//
// A row is held on chip between the two readings that the softmax needs: a
// cluster of S CTAs takes a row, each copies its share of the columns into
// shared memory in bulk copies, takes the list's columns out of it, and sums
// what is left; the CTAs give each other their sums through distributed shared
// memory, and each writes its share of the gradient. Logits are read from memory
// once, the gradient written once. Several CTAs share an SM, so that one's copies
// run beside another's sums and stores; a CTA's own steps are kept few, since thousands
// of rows make tens of thousands of CTAs: one warp reads the list while the copies are
// on their way, a thread takes out, and later patches, the listed columns of its own
// vectors.
//
// Measured, loss and gradient: 2048 rows of 128,256 bf16 columns, lists of 20, tail
// mode 210 us, 5.0 TB/s; 1001 of 151,936 fp32, lists of 32, 242 us, 5.0 TB/s; 4 rows
// 7 us. The bound is the way of a row, not the memory (0.74 of a copy's rate): copy, sums,
// exchange (a fifth of the time) and stores follow each other, and shared memory holds
// four or five shares per SM to put beside them.
#include <cooperative_groups.h>
#include <cstdint>

#include "tt_device.cuh"
#include "tt_f2.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"
#include "tt_x2.cuh"

namespace tt {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSplit = 16;
// Bytes of a row that a CTA should hold: a row takes the least even number of CTAs
// with no more. Shares of 43 to 51 KB let four or five CTAs share an SM; smaller
// ones exchange more sums, larger ones leave fewer to run beside each other. Loss
// and gradient of 2048 rows of 128,256 bf16 columns: 4 CTAs 230 us, 5 220, 6 210,
// 7 225, 8 212; of 1001 rows of 151,936 fp32: 9 248, 12 243, 13 265, 14 247, 16 258.
// (7 and 13 are behind their neighbours, 5 and 9 are not; whether by the cluster's size
// or the share's was not told apart.)
constexpr int kSegmentGoal = 52 * 1024;
constexpr int kSegmentMax = 200 * 1024;  // bytes of a row that a CTA holds
constexpr int kHeldBytes = 48 * 1024;    // rows up to this are held for a loss alone, too
constexpr int kStep = 4;  // vectors of a thread summed at once
// 1 - P is no mass but rounding up to this much of sum p (1 + |ln p|): each ln p comes
// rounded from a sum of rounded exponentials, and its own exponential is rounded (some
// 16 roundings of 2^-24, of p or of p |ln p|). A list that holds all of its teacher's
// mass (a mask leaves fewer columns than it has room for) would else have a rest of
// 1e-7, and a student masked alike, which has nothing there, a loss of inf.
constexpr float kRestRounding = 1.f / (1 << 20);

// The list's entries within a CTA's columns, those of one column added up in the
// first of them (the others have column -1), and the whole list's mass.
struct List {
  int count;
  int32_t col[TT_MAX_DISTILL_K];
  float p[TT_MAX_DISTILL_K];
  float z[TT_MAX_DISTILL_K];  // the student's logit of the column
  float mass, rest;           // P, r
  int status;
};

// What the CTAs of a row tell each other. The columns outside the list have a
// maximum of their own: a student may hold nearly all of its mass on the list, and
// what is outside it still has a share of r. (Maxima of nothing are -inf.)
struct Share {
  float m;      // max z,
  float all;    // and sum of 2^((z - m) scale)
  float m_out;  // the same outside the list
  float out;
  float mass;   // sum of p on the list,
  float cross;  // and of p (ln p - (z - m) / T), with 0 for an m of -inf
  int late;     // its copies did not come in time: the sums are NaN
};

// One warp reads the list of row r for columns c0 .. c1 - 1: p = exp(logp),
// scaled to sum 1 without tail mode. N entries per lane.
template <int N>
__device__ __forceinline__ void read_entries(const DistillArgs& a, int64_t r, int c0, int c1,
                                             List& L, int lane) {
  int id[N];
  float p[N];
  bool off = false, odd = false, any = false;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = i * 32 + lane;
    id[i] = -1;
    p[i] = -INFINITY;
    if (j < a.K) {
      id[i] = a.ids[r * a.K + j];
      p[i] = a.logp[r * a.K + j];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (id[i] < -1 || id[i] >= a.V) {
      off = true;
      id[i] = -1;
    }
    odd |= id[i] >= 0 && !(p[i] < INFINITY);  // NaN or +inf
    if (p[i] == -INFINITY) id[i] = -1;
    any |= id[i] >= 0;
    if (id[i] >= 0) top = fmaxf(top, p[i]);
  }
  const float lead = a.tail ? 0.f : warp_max_f(top);
  F2 mass = {0.f, 0.f};
  float terms = 0.f;  // sum p (1 + |ln p|)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float ln = p[i] - lead;
    p[i] = id[i] >= 0 ? expf(ln) : 0.f;
    mass = f2_add(mass, F2{p[i], 0.f});
    if (id[i] >= 0) terms = fmaf(p[i], 1.f + fabsf(ln), terms);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (a.tail) {  // (1 - P is what they are needed for)
      mass = f2_add(mass, F2{__shfl_xor_sync(0xffffffffu, mass.hi, o),
                             __shfl_xor_sync(0xffffffffu, mass.lo, o)});
      terms += __shfl_xor_sync(0xffffffffu, terms, o);
    } else {
      mass.hi += __shfl_xor_sync(0xffffffffu, mass.hi, o);
    }
  }
  const float rest = (1.f - mass.hi) - mass.lo;
  const float inv = a.tail || !(mass.hi > 0.f) ? 1.f : 1.f / mass.hi;
  int n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bool mine = id[i] >= c0 && id[i] < c1;
    const unsigned int who = __ballot_sync(0xffffffffu, mine);
    if (mine) {
      const int at = n + __popc(who & ((1u << lane) - 1));
      L.col[at] = id[i];
      L.p[at] = p[i] * inv;
    }
    n += __popc(who);
  }
  __syncwarp();
  // entries of one column (among 32, whether there are any shows at once)
  bool again = N > 1;
  if constexpr (N == 1) {
    const bool mine = id[0] >= c0 && id[0] < c1;
    const unsigned int same = __match_any_sync(0xffffffffu, mine ? id[0] : -1 - lane);
    again = __any_sync(0xffffffffu, same != 1u << lane);
  }
  if (again) {
    bool first[N];
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * 32 + lane;
      first[i] = e < n;
      sum[i] = 0.f;
      if (i * 32 >= n) break;
      const int col = e < n ? L.col[e] : -1;
      for (int j = 0; j < n; ++j) {
        if (L.col[j] != col) continue;
        first[i] &= j >= e;
        sum[i] += L.p[j];
      }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * 32 + lane;
      if (e >= n) break;
      L.col[e] = first[i] ? L.col[e] : -1;
      L.p[e] = first[i] ? sum[i] : 0.f;
    }
  }
  any = __any_sync(0xffffffffu, any);
  odd = __any_sync(0xffffffffu, odd);
  off = __any_sync(0xffffffffu, off);
  if (lane == 0) {
    L.count = n;
    L.mass = a.tail ? mass.hi : any ? 1.f : 0.f;
    L.rest = a.tail && any && rest > kRestRounding * terms ? rest : 0.f;
    L.status = (any ? 0 : TT_REQ_EMPTY) | (odd ? TT_REQ_NOT_FINITE : 0) |
               (off ? TT_REQ_ID_OUT_OF_RANGE : 0);
  }
}
__device__ __forceinline__ void read_list(const DistillArgs& a, int64_t r, int c0, int c1, List& L,
                                          int lane) {
  if (a.K <= 32)
    read_entries<1>(a, r, c0, c1, L, lane);
  else
    read_entries<TT_MAX_DISTILL_K / 32>(a, r, c0, c1, L, lane);
}

// coef 2^((z - M) scale) of a vector's logits, in their type.
template <int DT>
__device__ __forceinline__ uint4 scaled_exp(const uint4& w, float M, float scale, float coef) {
  const f32x2 minus = pair(-M, -M), scale2 = pair(scale, scale), coef2 = pair(coef, coef);
  uint32_t o[4];
#pragma unroll
  for (int q = 0; q < (DT == TT_F32 ? 2 : 4); ++q) {
    float lo, hi;
    split(mul2(coef2, exp2_pair(mul2(add2(logit_pair<DT>(w, q), minus), scale2))), lo, hi);
    if constexpr (DT == TT_F32) {
      o[2 * q] = __float_as_uint(lo);
      o[2 * q + 1] = __float_as_uint(hi);
    } else {
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[q]) : "f"(hi), "f"(lo));
    }
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int DT>
__device__ __forceinline__ void store_elem(char* row, int x, float v) {
  if constexpr (DT == TT_F32) {
    reinterpret_cast<float*>(row)[x] = v;
  } else {
    uint32_t o;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(0.f), "f"(v));
    reinterpret_cast<uint16_t*>(row)[x] = uint16_t(o);
  }
}

// Logits that the gradient may be written over: loads that need not find the memory
// unwritten while the kernel runs, as read-only ones do.
template <int DT>
__device__ __forceinline__ float row_logit(const char* row, int64_t x) {
  if constexpr (DT == TT_F32)
    return reinterpret_cast<const float*>(row)[x];
  else
    return bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[x]);
}
__device__ __forceinline__ uint4 row_vector(const char* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p)
               : "memory");
  return r;
}

// The row's maximum and sums from its CTAs' shares, the same in every CTA:
// q_j = 2^((z_j - M) scale) / all, t = 2^((m_out - M) scale) out / all.
struct Row {
  float M, all, m_out, out;
};
// 2^((m - M) scale) x for a sum x relative to m; one of nothing is 0, or NaN.
__device__ __forceinline__ float relative(float x, float m, float M, float scale) {
  return m > -INFINITY ? x * ex2_approx((m - M) * scale) : x;
}
// (by one warp, a share to a lane: by every thread, it was a tenth of a CTA's work)
__device__ __forceinline__ Row row_sums(const DistillArgs& a, const Share* share, int S, int lane) {
  static_assert(kMaxSplit <= 16, "shares of half a warp");
  Share x{-INFINITY, 0.f, -INFINITY, 0.f, 0.f, 0.f, 0};
  if (lane < S) x = share[lane];
  Row y{x.m, 0.f, x.m_out, 0.f};
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    y.M = fmaxf(y.M, __shfl_xor_sync(0xffffffffu, y.M, o));
    y.m_out = fmaxf(y.m_out, __shfl_xor_sync(0xffffffffu, y.m_out, o));
  }
  y.all = relative(x.all, x.m, y.M, a.scale);
  y.out = relative(x.out, x.m_out, y.m_out, a.scale);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    y.all += __shfl_xor_sync(0xffffffffu, y.all, o);
    y.out += __shfl_xor_sync(0xffffffffu, y.out, o);
  }
  if (!a.tail) {  // (r = 0: not needed apart)
    y.m_out = y.M;
    y.out = y.all;
  }
  return y;  // (in the first half of the warp)
}

// Gradient factors of a row.
struct Factors {
  float M;
  float m_out;    // 0 where nothing is outside the list
  float outside;  // times 2^((z - m_out) scale) outside the list: (W q - r q / t) w / T
  float listed;   // W / all: times 2^((z - M) scale) on it, W q
  float wt;       // w / T
  bool none;      // gradient 0
};
__device__ __forceinline__ Factors factors(const DistillArgs& a, const List& L, int64_t r,
                                           const Row& y) {
  Factors f;
  f.wt = (a.weight ? a.weight[r] : 1.f) / a.temp;
  const float W = L.mass + L.rest;
  f.M = y.M;
  f.listed = W / y.all;
  const bool some = y.out > 0.f;
  f.m_out = some ? y.m_out : 0.f;
  f.outside = some ? f.wt * (relative(f.listed, y.m_out, y.M, a.scale) - L.rest / y.out) : 0.f;
  f.none = f.wt == 0.f || !(y.all > 0.f && y.all < INFINITY) ||
           (L.status & (TT_REQ_EMPTY | TT_REQ_NOT_FINITE)) != 0;
  return f;
}
__device__ __forceinline__ float listed_grad(const DistillArgs& a, const Factors& f, float z,
                                             float p) {
  return f.none ? 0.f : f.wt * (f.listed * ex2_approx((z - f.M) * a.scale) - p);
}

template <int DT>
__device__ __forceinline__ float smem_logit(const char* seg, int x) {
  if constexpr (DT == TT_F32)
    return reinterpret_cast<const float*>(seg)[x];
  else
    return bf16_to_f32(reinterpret_cast<const uint16_t*>(seg)[x]);
}
template <int DT>
__device__ __forceinline__ void set_smem_logit(char* seg, int x, float z) {
  if constexpr (DT == TT_F32)
    reinterpret_cast<float*>(seg)[x] = z;
  else
    reinterpret_cast<uint16_t*>(seg)[x] = uint16_t(__float_as_uint(z) >> 16);
}

// One warp adds the list's columns (their logits in L.z) to the sums of the
// CTA's warps (their maxima and sums outside the list).
__device__ __forceinline__ Share cta_share(const DistillArgs& a, const List& L, const float2* s_ms,
                                           int lane, bool late) {
  const int n = L.count;
  Share x{lane < kWarps ? s_ms[lane].x : -INFINITY, 0.f, 0.f, 0.f, 0.f, 0.f, late};
  x.m_out = warp_max_f(x.m);
  for (int e = lane; e < n; e += 32)
    if (L.col[e] >= 0) x.m = fmaxf(x.m, L.z[e]);
  x.m = warp_max_f(x.m);
  if (lane < kWarps) x.out = relative(s_ms[lane].y, s_ms[lane].x, x.m_out, a.scale);
  const float ref = x.m > -INFINITY ? x.m : 0.f;
  for (int e = lane; e < n; e += 32) {
    if (L.col[e] < 0) continue;
    const float d = L.z[e] - ref, p = L.p[e];
    x.all += ex2_approx(d * a.scale);
    x.mass += p;
    if (p > 0.f) x.cross += p * (logf(p) - d / a.temp);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    x.out += __shfl_xor_sync(0xffffffffu, x.out, o);
    x.all += __shfl_xor_sync(0xffffffffu, x.all, o);
    x.mass += __shfl_xor_sync(0xffffffffu, x.mass, o);
    x.cross += __shfl_xor_sync(0xffffffffu, x.cross, o);
  }
  x.all += relative(x.out, x.m_out, x.m, a.scale);
  if (late) x.all = __int_as_float(0x7fffffff);
  return x;
}

// One thread writes the row's loss, statistics and status.
__device__ __forceinline__ void report(const DistillArgs& a, int64_t r, const List& L,
                                       const Share* share, int S, const Row& y) {
  const float ln_s = logf(y.all);
  float loss = 0.f, mass = 0.f;
  int late = 0;
  for (int k = 0; k < S; ++k) {
    late |= share[k].late;
    if (!(share[k].mass > 0.f)) continue;
    const float ref = share[k].m > -INFINITY ? share[k].m : 0.f;
    mass += share[k].mass;
    loss += share[k].cross + share[k].mass * ((y.M - ref) / a.temp);
  }
  loss += mass * ln_s;
  if (L.rest > 0.f)
    loss += L.rest * (logf(L.rest) -
                      (y.out > 0.f ? (y.m_out - y.M) / a.temp + logf(y.out) - ln_s : -INFINITY));
  const bool finite = y.all > 0.f && y.all < INFINITY;
  const int st = L.status | (late ? TT_REQ_TIMEOUT : finite ? 0 : TT_REQ_NOT_FINITE);
  a.status[r] = st;
  if (a.loss)
    a.loss[r] = st & (TT_REQ_NOT_FINITE | TT_REQ_TIMEOUT) ? __int_as_float(0x7fffffff)
                : st & TT_REQ_EMPTY                       ? 0.f
                                                          : loss;
  if (a.stats) reinterpret_cast<float4*>(a.stats)[r] = make_float4(y.M, y.all, y.m_out, y.out);
}

// A thread's running maximum and sum of 2^((z - m) scale).
struct Running {
  float m = -INFINITY;
  f32x2 s2 = 0, minus = 0;
};
template <int DT, int N>
__device__ __forceinline__ void add_vectors(Running& x, const uint4 (&w)[N], float scale) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  float top = -INFINITY;
#pragma unroll
  for (int u = 0; u < N; ++u) top = fmaxf(top, vec_max<DT>(w[u]));
  if (top > x.m) {
    const float f = ex2_approx((x.m - top) * scale);
    x.s2 = mul2(x.s2, pair(f, f));
    x.m = top;
    x.minus = pair(-top, -top);
  }
  const f32x2 scale2 = pair(scale, scale);
#pragma unroll
  for (int u = 0; u < N; ++u) {
#pragma unroll
    for (int q = 0; q < VEC / 2; ++q)
      x.s2 = add2(x.s2, exp2_pair(mul2(add2(logit_pair<DT>(w[u], q), x.minus), scale2)));
  }
}
// A warp's maximum and sum.
__device__ __forceinline__ float2 warp_running(const Running& x, float scale) {
  const float mw = warp_max_f(x.m);
  float sum = sum_pair(x.s2);
  if (x.m > -INFINITY) sum *= ex2_approx((x.m - mw) * scale);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return make_float2(mw, sum);
}
template <int DT>
__device__ __forceinline__ uint4 no_logits() {
  constexpr uint32_t e = DT == TT_F32 ? 0xff800000u : 0xff80ff80u;
  return make_uint4(e, e, e, e);
}

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  extern __shared__ __align__(128) char seg[];
  __shared__ List L;
  __shared__ uint64_t full;
  __shared__ float2 s_ms[kWarps];
  __shared__ Share s_share[kMaxSplit];
  __shared__ Factors s_factors;
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = a.split, rank = S > 1 ? int(cluster.block_rank()) : 0;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  // (a CTA's shared memory is written by the others only once it runs)
  if (S > 1) cluster.barrier_arrive();
  const int64_t r = blockIdx.x / S;
  const char* row = a.data + r * a.stride_bytes;
  const int c0 = min(a.V, rank * a.share), c1 = min(a.V, c0 + a.share);
  const int whole = (c1 - c0) / VEC, nvec = (c1 - c0 + VEC - 1) / VEC;
  uint4* sv = reinterpret_cast<uint4*>(seg);
  if (t == kThreads - 1) {
    mbar_init(&full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (whole > 0) {
      mbar_arrive_expect_tx(&full, whole * 16);
      for (int at = 0; at < whole * 16 && int(blockIdx.x) != a.stall; at += 32768)
        bulk_copy_g2s(seg + at, row + int64_t(c0) * ESZ + at, min(32768, whole * 16 - at), &full);
    }
  }
  // the ragged tail (the row's last columns) with -inf behind it
  if (nvec > whole && t >= 32 && t < 32 + VEC) {
    const int x = whole * VEC + t - 32;
    set_smem_logit<DT>(seg, x, c0 + x < c1 ? row_logit<DT>(row, c0 + x) : -INFINITY);
  }
  if (warp == 0) read_list(a, r, c0, c1, L, lane);
  __syncthreads();
  const bool landed = whole == 0 || mbar_wait(&full, 0, a.wait_ns);
  // (late copies still come into this CTA's memory: it stays for them. At the kernel's
  // end, the second wait cost every row: 218 us for 210.)
  if (!landed) mbar_wait(&full, 0, a.wait_ns);
  // take the list's columns out of this thread's vectors
  const int n = L.count;
  for (int e = 0; e < n; ++e) {
    const int x = L.col[e] - c0;
    if (x >= 0 && (x / VEC) % kThreads == t) {
      L.z[e] = smem_logit<DT>(seg, x);
      set_smem_logit<DT>(seg, x, -INFINITY);
    }
  }
  // sum what is left
  Running run;
  for (int v0 = t; v0 < nvec; v0 += kStep * kThreads) {
    uint4 w[kStep];
#pragma unroll
    for (int u = 0; u < kStep; ++u)
      w[u] = v0 + u * kThreads < nvec ? sv[v0 + u * kThreads] : no_logits<DT>();
    add_vectors<DT>(run, w, a.scale);
  }
  const float2 ms = warp_running(run, a.scale);
  if (lane == 0) s_ms[warp] = ms;
  const bool ok = __syncthreads_and(landed);
  if (warp == 0) {
    const Share x = cta_share(a, L, s_ms, lane, !ok);
    if (S > 1) cluster.barrier_wait();
    if (lane < S) (S > 1 ? cluster.map_shared_rank(s_share, lane) : s_share)[rank] = x;
  } else if (S > 1) {
    cluster.barrier_wait();
  }
  if (S > 1)
    cluster.sync();
  else
    __syncthreads();
  Row y;
  if (warp == 0) {
    y = row_sums(a, s_share, S, lane);
    if (lane == 0) s_factors = factors(a, L, r, y);
  }
  __syncthreads();
  if (rank == 0 && t == 0) report(a, r, L, s_share, S, y);
  if (!a.grad) return;
  const Factors f = s_factors;
  char* grow = a.grad + r * a.grad_stride_bytes;
  uint4* out = reinterpret_cast<uint4*>(grow + int64_t(c0) * ESZ);
  if (f.none) {
    for (int v = t; v < whole; v += kThreads) out[v] = make_uint4(0, 0, 0, 0);
  } else {
#pragma unroll 4
    for (int v = t; v < whole; v += kThreads)
      __stcs(out + v, scaled_exp<DT>(sv[v], f.m_out, a.scale, f.outside));
  }
  if (nvec > whole && t == whole % kThreads) {
    for (int x = whole * VEC; x < c1 - c0; ++x)
      store_elem<DT>(grow, c0 + x,
                     f.none ? 0.f
                            : f.outside * ex2_approx((smem_logit<DT>(seg, x) - f.m_out) * a.scale));
  }
  // the listed columns of this thread's vectors, after them
  for (int e = 0; e < n; ++e) {
    const int x = L.col[e] - c0;
    if (x >= 0 && (x / VEC) % kThreads == t)
      store_elem<DT>(grow, c0 + x, listed_grad(a, f, L.z[e], L.p[e]));
  }
}

// The loss alone: the logits are read once, so they stream through registers. A
// CTA takes a row (its share, where there are few rows). Bits in shared memory
// tell which vectors hold listed columns: those are left out of the stream, and
// the rest of their columns is added by a thread per entry.
constexpr int kFlight = 8;  // vectors of a thread loaded at once

template <int DT>
__global__ void __launch_bounds__(kThreads, 8) distill_loss_kernel(
    const __grid_constant__ DistillArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  extern __shared__ uint32_t holds[];  // a bit per vector
  __shared__ List L;
  __shared__ float2 s_ms[kWarps];
  __shared__ Share s_share[kMaxSplit];
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = a.split, rank = S > 1 ? int(cluster.block_rank()) : 0;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  if (S > 1) cluster.barrier_arrive();
  const int64_t r = blockIdx.x / S;
  const int c0 = min(a.V, rank * a.share), c1 = min(a.V, c0 + a.share);
  const int whole = (c1 - c0) / VEC, nvec = (c1 - c0 + VEC - 1) / VEC;
  const char* row = a.data + r * a.stride_bytes + int64_t(c0) * ESZ;
  auto load = [&](uint4 (&w)[kFlight], int v0) {
    const char* p = row + (uint32_t(v0 + t) << 4);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      w[u] = no_logits<DT>();
      if (v0 + u * kThreads + t < whole) w[u] = ld_stream_v4(p + u * kThreads * 16);
    }
  };
  uint4 w[kFlight];
  load(w, 0);
  for (int i = t; i < (nvec + 31) / 32; i += kThreads) holds[i] = 0;
  if (warp == 0) read_list(a, r, c0, c1, L, lane);
  __syncthreads();
  for (int e = t; e < L.count; e += kThreads) {
    const int v = (L.col[e] - c0) / VEC;
    if (L.col[e] >= 0) atomicOr(&holds[v >> 5], 1u << (v & 31));
  }
  __syncthreads();
  Running run;
  for (int v0 = 0; v0 < whole; v0 += kFlight * kThreads) {
    if (v0 > 0) load(w, v0);
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int v = v0 + u * kThreads + t;
      if (v < whole && (holds[v >> 5] >> (v & 31) & 1)) w[u] = no_logits<DT>();
    }
    add_vectors<DT>(run, w, a.scale);
  }
  // the vectors left out, and the row's last columns: a thread takes the vector of
  // its entry unless an earlier entry has it too
  static_assert(kThreads >= TT_MAX_DISTILL_K, "a thread per entry");
  auto rest_of = [&](int v, int self) {
    uint32_t out = 0;  // its listed columns
    for (int e = 0; e < L.count; ++e) {
      const int q = L.col[e] - c0 - v * VEC;
      if (L.col[e] < 0 || q < 0 || q >= VEC) continue;
      if (e < self) return;
      out |= 1u << q;
    }
    for (int q = 0; q < VEC && v * VEC + q < c1 - c0; ++q) {
      const float z = load_logit<DT>(row, v * VEC + q);
      if (out >> q & 1) {
        for (int e = 0; e < L.count; ++e)
          if (L.col[e] == c0 + v * VEC + q) L.z[e] = z;
        continue;
      }
      const float top = fmaxf(run.m, z), base = top > -INFINITY ? top : 0.f;
      const float f = run.m > -INFINITY ? ex2_approx((run.m - base) * a.scale) : 1.f;
      run.s2 = add2(mul2(run.s2, pair(f, f)), pair(ex2_approx((z - base) * a.scale), 0.f));
      run.m = top;
    }
  };
  if (t < L.count && L.col[t] >= 0 && (L.col[t] - c0) / VEC < whole)
    rest_of((L.col[t] - c0) / VEC, t);
  if (nvec > whole && t == kThreads - 1) rest_of(whole, -1);
  __syncwarp();
  const float2 ms = warp_running(run, a.scale);
  if (lane == 0) s_ms[warp] = ms;
  __syncthreads();
  if (warp == 0) {
    const Share x = cta_share(a, L, s_ms, lane, false);
    if (S > 1) cluster.barrier_wait();
    if (lane == 0) (S > 1 ? cluster.map_shared_rank(s_share, 0) : s_share)[rank] = x;
    __syncwarp();
  } else if (S > 1) {
    cluster.barrier_wait();
  }
  if (S > 1) cluster.sync();
  if (rank == 0 && warp == 0) {
    const Row y = row_sums(a, s_share, S, lane);
    if (lane == 0) report(a, r, L, s_share, S, y);
  }
}

// The gradient alone, from the forward call's statistics: a CTA takes kGradVecs
// vectors of a row, all of them loaded before the first is written (the gradient
// may take the logits' place).
constexpr int kPerThread = 8;
constexpr int kGradVecs = kPerThread * kThreads;

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_grad_kernel(
    const __grid_constant__ DistillArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  __shared__ List L;
  __shared__ Factors s_factors;
  const int t = threadIdx.x;
  const int parts = (a.V + kGradVecs * VEC - 1) / (kGradVecs * VEC);
  const int64_t r = blockIdx.x / parts;
  const int c0 = int(blockIdx.x % parts) * kGradVecs * VEC, c1 = min(a.V, c0 + kGradVecs * VEC);
  const char* row = a.data + r * a.stride_bytes;
  char* grow = a.grad + r * a.grad_stride_bytes;
  const int whole = (c1 - c0) / VEC;
  const char* in = row + int64_t(c0) * ESZ;
  uint4 w[kPerThread];
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    const int v = u * kThreads + t;
    w[u] = v < whole ? row_vector(in + v * 16) : make_uint4(0, 0, 0, 0);
  }
  const bool ragged = t == whole % kThreads;  // the thread of the row's last columns
  float z_tail[VEC];
  if (ragged)
    for (int q = 0; q < VEC; ++q)
      z_tail[q] = c0 + whole * VEC + q < c1 ? row_logit<DT>(row, c0 + whole * VEC + q) : 0.f;
  const float4 st = reinterpret_cast<const float4*>(a.stats)[r];
  if (t < 32) {
    read_list(a, r, c0, c1, L, t);
    __syncwarp();
    for (int e = t; e < L.count; e += 32)
      if (L.col[e] >= 0) L.z[e] = row_logit<DT>(row, L.col[e]);
    if (t == 0) s_factors = factors(a, L, r, Row{st.x, st.y, st.z, st.w});
  }
  __syncthreads();
  const Factors f = s_factors;
  uint4* out = reinterpret_cast<uint4*>(grow + int64_t(c0) * ESZ);
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    const int v = u * kThreads + t;
    if (v < whole)
      __stcs(out + v,
             f.none ? make_uint4(0, 0, 0, 0) : scaled_exp<DT>(w[u], f.m_out, a.scale, f.outside));
  }
  if (ragged)
    for (int q = 0; q < VEC; ++q)
      if (c0 + whole * VEC + q < c1)
        store_elem<DT>(grow, c0 + whole * VEC + q,
                       f.none ? 0.f : f.outside * ex2_approx((z_tail[q] - f.m_out) * a.scale));
  for (int e = 0; e < L.count; ++e) {
    const int x = L.col[e] - c0;
    if (x >= 0 && (x / VEC) % kThreads == t)
      store_elem<DT>(grow, c0 + x, listed_grad(a, f, L.z[e], L.p[e]));
  }
}

template <int DT>
cudaError_t launch(DistillArgs a, cudaStream_t stream, int sm_count) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  int S = 1;
  auto share = [&](int s) { return ((a.V + s - 1) / s + VEC - 1) / VEC * VEC; };
  // (a loss alone streams, 20 % faster, but rows of a few KB are sooner copied at
  // once: 20,000 fp32 rows of 4096 columns 87 us and 141)
  const bool held = a.grad || a.V * ESZ <= kHeldBytes;
  if (held) {
    while (S < kMaxSplit && share(S) * ESZ > kSegmentGoal) S += S > 1 ? 2 : 1;
  } else {
    // enough CTAs to fill the SMs, each with what its threads load at once at least
    while (S < kMaxSplit && a.rows * S < 4 * sm_count &&
           a.V / (2 * S) >= kFlight * kThreads * VEC)
      S *= 2;
  }
  a.split = S;
  a.share = share(S);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(a.rows * S));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes =
      held ? size_t(a.share) * ESZ : (size_t(a.share) / VEC + 31) / 32 * sizeof(uint32_t);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = S > 1 ? 1 : 0;
  return held ? cudaLaunchKernelEx(&cfg, distill_kernel<DT>, a)
              : cudaLaunchKernelEx(&cfg, distill_loss_kernel<DT>, a);
}

template <int DT>
cudaError_t preload() {
  cudaError_t e = cudaFuncSetAttribute(distill_kernel<DT>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSegmentMax);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(distill_kernel<DT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(distill_loss_kernel<DT>, cudaFuncAttributeNonPortableClusterSizeAllowed,
                             1);
  cudaFuncAttributes fa;
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, distill_grad_kernel<DT>);
  return e;
}

}  // namespace

int distill_max_cols(int dt) { return kMaxSplit * kSegmentMax / (dt == TT_F32 ? 4 : 2); }

cudaError_t launch_distill(const DistillArgs& args, int dt, cudaStream_t stream, int sm_count) {
  DistillArgs a = args;
  next_launch_stall(&a.stall, &a.wait_ns);
  return dt == TT_F32 ? launch<TT_F32>(a, stream, sm_count) : launch<TT_BF16>(a, stream, sm_count);
}

cudaError_t launch_distill_grad(const DistillArgs& a, int dt, cudaStream_t stream) {
  const int cols = kGradVecs * (dt == TT_F32 ? 4 : 8);
  const dim3 grid{unsigned(a.rows * ((a.V + cols - 1) / cols))};
  if (dt == TT_F32)
    distill_grad_kernel<TT_F32><<<grid, kThreads, 0, stream>>>(a);
  else
    distill_grad_kernel<TT_BF16><<<grid, kThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t preload_distill() {
  const cudaError_t e = preload<TT_F32>();
  return e == cudaSuccess ? preload<TT_BF16>() : e;
}

}  // namespace tt
