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
// shared memory in one bulk copy, takes the list's columns out of it, and sums
// what is left; the CTAs give each other their sums and the list's logits
// through distributed shared memory, and each writes its share of the gradient.
// Logits are read from memory once, the gradient written once.
#include <cooperative_groups.h>
#include <cstdint>

#include "tt_device.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"

namespace tt {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSplit = 16;
constexpr int kSegmentMax = 200 * 1024;  // bytes of a row that a CTA holds

// The teacher's list of a row as every CTA of the row sees it: entries of one
// column added up in the first of them, unusable ones dropped (col -1).
struct List {
  int32_t col[TT_MAX_DISTILL_K];
  float p[TT_MAX_DISTILL_K];
  float z[TT_MAX_DISTILL_K];  // the student's logit of the column
  float raw[TT_MAX_DISTILL_K];
  float red[kWarps];
  double redd[kWarps];
  double mass;  // P
  float rest;   // r
  int status;
};

template <typename T, typename Op>
__device__ __forceinline__ T block_reduce(T v, T* red, Op op) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) v = op(v, red[w]);
  return v;
}
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
  template <typename T>
  __device__ T operator()(T a, T b) const { return a + b; }
};

// Reads the list of row r: p_i = exp(logp_i), scaled to sum 1 without tail mode.
__device__ void read_list(const DistillArgs& a, int64_t r, List& L) {
  const int t = threadIdx.x;
  int id = -1;
  float lp = -INFINITY;
  bool off = false, odd = false;
  if (t < a.K) {
    id = a.ids[r * a.K + t];
    lp = a.logp[r * a.K + t];
    off = id < -1 || id >= a.V;
    if (off) id = -1;
    odd = id >= 0 && !(lp < INFINITY);  // NaN or +inf
    if (id >= 0 && lp == -INFINITY) id = -1;
  }
  const float top = block_reduce(id >= 0 ? lp : -INFINITY, L.red, Max());
  const float lead = a.tail || !(top > -INFINITY) ? 0.f : top;
  float p = id >= 0 ? expf(lp - lead) : 0.f;
  if (t < a.K) {
    L.col[t] = id;
    L.raw[t] = p;
  }
  double mass = block_reduce(double(p), L.redd, Sum());
  if (!a.tail && mass > 0.0) {
    p = float(double(p) / mass);
    mass = 1.0;
  }
  const int any = __syncthreads_or(id >= 0);
  const int bad = __syncthreads_or(odd), wrong = __syncthreads_or(off);
  const float scale = float(p > 0.f && t < a.K ? p / L.raw[t] : 0.f);
  bool first = id >= 0;
  float sum = 0.f;
  if (id >= 0) {
    for (int j = 0; j < a.K; ++j) {
      if (L.col[j] != id) continue;
      if (j < t) first = false;
      sum += L.raw[j];
    }
  }
  __syncthreads();
  if (t < a.K) {
    L.col[t] = first ? id : -1;
    L.p[t] = first ? sum * scale : 0.f;
  }
  if (t == 0) {
    L.mass = mass;
    L.rest = a.tail && any ? float(fmax(0.0, 1.0 - mass)) : 0.f;
    L.status = (any ? 0 : TT_REQ_EMPTY) | (bad ? TT_REQ_NOT_FINITE : 0) |
               (wrong ? TT_REQ_ID_OUT_OF_RANGE : 0);
  }
  __syncthreads();
}

template <int DT>
__device__ __forceinline__ uint4 scaled_exp(const uint4& w, float M, float scale, float coef) {
  if constexpr (DT == TT_F32) {
    uint4 o;
    o.x = __float_as_uint(coef * ex2_approx((__uint_as_float(w.x) - M) * scale));
    o.y = __float_as_uint(coef * ex2_approx((__uint_as_float(w.y) - M) * scale));
    o.z = __float_as_uint(coef * ex2_approx((__uint_as_float(w.z) - M) * scale));
    o.w = __float_as_uint(coef * ex2_approx((__uint_as_float(w.w) - M) * scale));
    return o;
  } else {
    uint32_t o[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const float lo = coef * ex2_approx((lane_elem<DT>(w, 2 * h) - M) * scale);
      const float hi = coef * ex2_approx((lane_elem<DT>(w, 2 * h + 1) - M) * scale);
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[h]) : "f"(hi), "f"(lo));
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
  }
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

// Gradient factors of a row: q_j = 2^((z_j - M) scale) / S.
struct Factors {
  float M;
  float outside;  // (W - r / t) w / (T S): times 2^((z - M) scale), outside the list
  float listed;   // W / S
  float wt;       // w / T
};
__device__ __forceinline__ Factors factors(const DistillArgs& a, const List& L, int64_t r, float M,
                                           float S, float S_out) {
  Factors f;
  f.wt = (a.weight ? a.weight[r] : 1.f) / a.temp;
  const float W = float(L.mass + double(L.rest));
  f.M = M;
  f.listed = W / S;
  // (no mass outside the list: nothing there has a gradient)
  f.outside = f.wt * (S_out > 0.f ? W / S - L.rest / S_out : 0.f);
  if (!(S > 0.f && S < INFINITY) || (L.status & (TT_REQ_EMPTY | TT_REQ_NOT_FINITE))) {
    f.outside = f.listed = f.wt = 0.f;
    f.M = INFINITY;  // (2^-inf for whatever the row holds)
  }
  return f;
}

// The gradient of the listed columns of [c0, c1), whose logits are in L.z.
template <int DT>
__device__ __forceinline__ void store_listed(const DistillArgs& a, const List& L, const Factors& f,
                                             char* grow, int c0, int c1) {
  const int t = threadIdx.x;
  if (t < a.K && L.col[t] >= c0 && L.col[t] < c1)
    store_elem<DT>(grow, L.col[t],
                   f.wt == 0.f ? 0.f
                               : f.wt * (f.listed * ex2_approx((L.z[t] - f.M) * a.scale) - L.p[t]));
}

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ DistillArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  extern __shared__ __align__(128) char seg[];
  __shared__ List L;
  __shared__ uint64_t full;
  __shared__ float s_max[kMaxSplit], s_sum[kMaxSplit];
  const cg::cluster_group cluster = cg::this_cluster();
  const int S = a.split, rank = S > 1 ? int(cluster.block_rank()) : 0, t = threadIdx.x;
  // (a CTA's shared memory is written by the others only once it runs)
  if (S > 1) cluster.barrier_arrive();
  const int64_t r = blockIdx.x / S;
  const char* row = a.data + r * a.stride_bytes;
  const int c0 = min(a.V, rank * a.share), c1 = min(a.V, c0 + a.share);
  const int whole = (c1 - c0) / VEC, nvec = (c1 - c0 + VEC - 1) / VEC;
  uint4* sv = reinterpret_cast<uint4*>(seg);
  if (t == 0) {
    mbar_init(&full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (whole > 0) {
      mbar_arrive_expect_tx(&full, whole * 16);
      for (int at = 0; at < whole * 16; at += 32768)
        bulk_copy_g2s(seg + at, row + int64_t(c0) * ESZ + at, min(32768, whole * 16 - at), &full);
    }
  }
  // the ragged tail (the row's last columns) with -inf behind it
  if (nvec > whole && t >= 32 && t < 32 + VEC) {
    const int x = whole * VEC + t - 32;
    const float z = c0 + x < c1 ? load_logit<DT>(row, c0 + x) : -INFINITY;
    if constexpr (DT == TT_F32)
      reinterpret_cast<float*>(seg)[x] = z;
    else
      reinterpret_cast<uint16_t*>(seg)[x] = uint16_t(__float_as_uint(z) >> 16);
  }
  read_list(a, r, L);
  const uint64_t limit = kWaitLimitNs;
  bool ok = whole == 0 || mbar_wait(&full, 0, limit);
  ok = !__syncthreads_or(!ok);
  if (S > 1) cluster.barrier_wait();
  // take the list's columns out
  float zi = -INFINITY;
  if (t < a.K && L.col[t] >= c0 && L.col[t] < c1) {
    const int x = L.col[t] - c0;
    if constexpr (DT == TT_F32) {
      float* p = reinterpret_cast<float*>(seg) + x;
      zi = *p;
      *p = -INFINITY;
    } else {
      uint16_t* p = reinterpret_cast<uint16_t*>(seg) + x;
      zi = bf16_to_f32(*p);
      *p = 0xff80u;
    }
    for (int k = 0; k < S; ++k)
      (S > 1 ? cluster.map_shared_rank(L.z, k) : L.z)[t] = zi;
  }
  __syncthreads();
  float m = -INFINITY;
  for (int v = t; v < nvec; v += kThreads) m = fmaxf(m, vec_max<DT>(sv[v]));
  m = block_reduce(m, L.red, Max());
  const float base = m > -INFINITY ? m : 0.f;
  float sum = 0.f;
  for (int v = t; v < nvec; v += kThreads) {
    const uint4 w = sv[v];
#pragma unroll
    for (int q = 0; q < VEC; ++q) sum += ex2_approx((lane_elem<DT>(w, q) - base) * a.scale);
  }
  sum = block_reduce(sum, L.red, Sum());
  if (!ok) sum = __int_as_float(0x7fffffff);
  if (t < S) {
    (S > 1 ? cluster.map_shared_rank(s_max, t) : s_max)[rank] = m;
    (S > 1 ? cluster.map_shared_rank(s_sum, t) : s_sum)[rank] = sum;
  }
  if (S > 1)
    cluster.sync();
  else
    __syncthreads();
  // the row's maximum and sums, the same in every CTA
  const float zl = t < a.K && L.col[t] >= 0 ? L.z[t] : -INFINITY;
  float M = zl;
  if (t < S) M = fmaxf(M, s_max[t]);
  M = block_reduce(M, L.red, Max());
  float S_out = 0.f;
  for (int k = 0; k < S; ++k)
    S_out += s_max[k] > -INFINITY ? s_sum[k] * ex2_approx((s_max[k] - M) * a.scale) : s_sum[k];
  const float S_all =
      S_out + block_reduce(zl > -INFINITY || zl != zl ? ex2_approx((zl - M) * a.scale) : 0.f, L.red,
                           Sum());
  const bool finite = S_all > 0.f && S_all < INFINITY;
  if (rank == 0) {
    const float ln_s = logf(S_all);
    float term = 0.f;
    if (t < a.K && L.p[t] > 0.f) term = L.p[t] * (logf(L.p[t]) - ((zl - M) / a.temp - ln_s));
    float loss = block_reduce(term, L.red, Sum());
    if (L.rest > 0.f) loss += L.rest * (logf(L.rest) - (logf(S_out) - ln_s));
    if (t == 0) {
      const int st = L.status | (finite ? 0 : TT_REQ_NOT_FINITE) | (ok ? 0 : TT_REQ_TIMEOUT);
      a.status[r] = st;
      if (a.loss)
        a.loss[r] = st & (TT_REQ_NOT_FINITE | TT_REQ_TIMEOUT) ? __int_as_float(0x7fffffff)
                    : st & TT_REQ_EMPTY                       ? 0.f
                                                              : loss;
      if (a.stats) reinterpret_cast<float4*>(a.stats)[r] = make_float4(M, S_all, S_out, 0.f);
    }
  }
  if (!a.grad) return;
  const Factors f = factors(a, L, r, M, S_all, S_out);
  char* grow = a.grad + r * a.grad_stride_bytes;
  uint4* out = reinterpret_cast<uint4*>(grow + int64_t(c0) * ESZ);
  for (int v = t; v < whole; v += kThreads)
    out[v] = f.wt == 0.f ? make_uint4(0, 0, 0, 0) : scaled_exp<DT>(sv[v], f.M, a.scale, f.outside);
  if (nvec > whole && t < c1 - c0 - whole * VEC) {
    const int x = whole * VEC + t;
    const float z = DT == TT_F32 ? reinterpret_cast<float*>(seg)[x]
                                 : bf16_to_f32(reinterpret_cast<uint16_t*>(seg)[x]);
    store_elem<DT>(grow, c0 + x, f.wt == 0.f ? 0.f : f.outside * ex2_approx((z - f.M) * a.scale));
  }
  __syncthreads();  // the listed columns' stores come last
  store_listed<DT>(a, L, f, grow, c0, c1);
}

// The gradient alone, from the forward call's statistics: a CTA takes kGradVecs
// vectors of a row, reads the listed logits among them first (the gradient may
// take the logits' place), and streams the rest.
constexpr int kGradVecs = 8 * kThreads;

template <int DT>
__global__ void __launch_bounds__(kThreads) distill_grad_kernel(
    const __grid_constant__ DistillArgs a) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  __shared__ List L;
  const int t = threadIdx.x;
  const int parts = (a.V + kGradVecs * VEC - 1) / (kGradVecs * VEC);
  const int64_t r = blockIdx.x / parts;
  const int c0 = int(blockIdx.x % parts) * kGradVecs * VEC, c1 = min(a.V, c0 + kGradVecs * VEC);
  const char* row = a.data + r * a.stride_bytes;
  char* grow = a.grad + r * a.grad_stride_bytes;
  read_list(a, r, L);
  const float4 st = reinterpret_cast<const float4*>(a.stats)[r];
  if (t < a.K && L.col[t] >= c0 && L.col[t] < c1) L.z[t] = load_logit<DT>(row, L.col[t]);
  const int whole = (c1 - c0) / VEC;
  const int x = whole * VEC + t;
  const float z = c0 + x < c1 ? load_logit<DT>(row, c0 + x) : 0.f;  // (t < VEC: the tail)
  __syncthreads();
  const Factors f = factors(a, L, r, st.x, st.y, st.z);
  const uint4* in = reinterpret_cast<const uint4*>(row + int64_t(c0) * ESZ);
  uint4* out = reinterpret_cast<uint4*>(grow + int64_t(c0) * ESZ);
  for (int v = t; v < whole; v += kThreads)
    out[v] = f.wt == 0.f ? make_uint4(0, 0, 0, 0) : scaled_exp<DT>(in[v], f.M, a.scale, f.outside);
  if (t < VEC && c0 + x < c1)
    store_elem<DT>(grow, c0 + x, f.wt == 0.f ? 0.f : f.outside * ex2_approx((z - f.M) * a.scale));
  __syncthreads();
  store_listed<DT>(a, L, f, grow, c0, c1);
}

template <int DT>
cudaError_t launch(DistillArgs a, cudaStream_t stream) {
  constexpr int VEC = DT == TT_F32 ? 4 : 8;
  constexpr int ESZ = 16 / VEC;
  // the fewest CTAs whose shares fit
  int S = 1;
  auto share = [&](int s) { return ((a.V + s - 1) / s + VEC - 1) / VEC * VEC; };
  while (S < kMaxSplit && share(S) * ESZ > kSegmentMax) S *= 2;
  a.split = S;
  a.share = share(S);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(a.rows * S));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = size_t(a.share) * ESZ;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = S;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = S > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, distill_kernel<DT>, a);
}

template <int DT>
cudaError_t preload() {
  cudaError_t e = cudaFuncSetAttribute(distill_kernel<DT>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kSegmentMax);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(distill_kernel<DT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  cudaFuncAttributes fa;
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, distill_grad_kernel<DT>);
  return e;
}

}  // namespace

int distill_max_cols(int dt) { return kMaxSplit * kSegmentMax / (dt == TT_F32 ? 4 : 2); }

cudaError_t launch_distill(const DistillArgs& a, int dt, cudaStream_t stream) {
  return dt == TT_F32 ? launch<TT_F32>(a, stream) : launch<TT_BF16>(a, stream);
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
