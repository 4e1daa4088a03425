// tree.cu -- attention of the drafted tokens of every request over its paged
// cache and, within its tree of drafted tokens, over each token's ancestors.
//
// Token i of request b sees the L_b keys of the request's cache, its ancestors
// i, parent(i), parent(parent(i)), ... and nothing else; its output in a head is
// sum_x softmax_x(scale q.k_x) v_x over them, held in the running form: with
// m = max s_x and l = sum 2^(s_x - m), a larger m scales what was summed before.
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tt_device.cuh"
#include "tt_ops.h"

namespace tt {

namespace {

constexpr int kThreads = 256;

// A request's usable range: its nodes and cache length, or why it has none.
struct Request {
  int first, nodes, len, status;
};
__device__ __forceinline__ Request request(const TreeArgs& a, int b) {
  Request r{a.tree_off[b], 0, a.cache_len[b], 0};
  const int end = a.tree_off[b + 1];
  if (r.first < 0 || end < r.first || end > a.n_nodes) {
    r.status = TT_REQ_BAD_OFFSETS;
    return r;
  }
  r.nodes = end - r.first;
  if (r.nodes > a.max_nodes || r.len < 0 || r.len > a.max_len) {
    r.status = TT_REQ_TOO_LONG;
    r.nodes = 0;
  }
  return r;
}

// Whether every parent and page of the request is in range.
__device__ int check_request(const TreeArgs& a, int b, const Request& r) {
  bool bad = false;
  if (a.parents)
    for (int i = threadIdx.x; i < r.nodes; i += blockDim.x) {
      const int p = a.parents[r.first + i];
      bad |= p < -1 || p >= i;
    }
  for (int x = threadIdx.x; int64_t(x) * a.page_size < r.len; x += blockDim.x) {
    const int p = a.page_table[b * a.table_stride + x];
    bad |= p < 0 || p >= a.n_pages;
  }
  return __syncthreads_or(bad) ? TT_REQ_ID_OUT_OF_RANGE : 0;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) tree_kernel(const __grid_constant__ TreeArgs a) {
  __shared__ uint32_t seen[TT_MAX_TREE / 32];
  const int i = blockIdx.x, b = blockIdx.y, t = threadIdx.x, lane = t & 31;
  const Request r = request(a, b);
  if (i == 0) {
    const int bad = r.status ? r.status : check_request(a, b, r);
    if (t == 0) a.status[b] = bad;
  }
  if (i >= r.nodes) return;
  if (t < TT_MAX_TREE / 32) seen[t] = 0;
  __syncthreads();
  if (t == 0) {
    for (int j = i;;) {
      seen[j >> 5] |= 1u << (j & 31);
      const int p = a.parents ? a.parents[r.first + j] : j - 1;
      if (p < 0 || p >= j) break;
      j = p;
    }
  }
  __syncthreads();
  const int G = a.Hq / a.Hkv;
  const float scale = a.scale * 1.4426950408889634f;
  const int64_t node = int64_t(r.first) + i;
  for (int h = t >> 5; h < a.Hq; h += kThreads / 32) {
    const int hk = h / G;
    const T* q = reinterpret_cast<const T*>(a.q) + node * a.q_token + h * a.q_head;
    float qf[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < 4; ++c) qf[c] = c * 32 < a.D ? float(q[c * 32 + lane]) * scale : 0.f;
    float m = -INFINITY, l = 0.f;
    auto take = [&](const T* k, const T* v) {
      float s = 0.f;
      for (int c = 0; c * 32 < a.D; ++c) s = fmaf(qf[c], float(k[c * 32 + lane]), s);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      const float top = fmaxf(m, s);
      if (top == -INFINITY && s == s) return;
      const float f = ex2_approx(m - top), e = ex2_approx(s - top);
      m = top;
      l = fmaf(l, f, e);
      for (int c = 0; c * 32 < a.D; ++c) acc[c] = fmaf(acc[c], f, e * float(v[c * 32 + lane]));
    };
    for (int x0 = 0; x0 < r.len; x0 += a.page_size) {
      const int page = a.page_table[b * a.table_stride + x0 / a.page_size];
      if (page < 0 || page >= a.n_pages) continue;
      const T* k = reinterpret_cast<const T*>(a.kc) + page * a.kc_page + hk * a.kc_head;
      const T* v = reinterpret_cast<const T*>(a.vc) + page * a.vc_page + hk * a.vc_head;
      for (int x = 0; x < a.page_size && x0 + x < r.len; ++x)
        take(k + x * a.kc_slot, v + x * a.vc_slot);
    }
    for (int j = 0; j <= i; ++j) {
      if (!(seen[j >> 5] >> (j & 31) & 1)) continue;
      const int64_t n = int64_t(r.first) + j;
      take(reinterpret_cast<const T*>(a.k) + n * a.k_token + hk * a.k_head,
           reinterpret_cast<const T*>(a.v) + n * a.v_token + hk * a.v_head);
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    T* out = reinterpret_cast<T*>(a.out) + (node * a.Hq + h) * a.D;
    for (int c = 0; c * 32 < a.D; ++c) out[c * 32 + lane] = T(acc[c] * inv);
    if (a.lse && lane == 0)
      a.lse[node * a.Hq + h] = l > 0.f || l != l ? 0.693147180559945f * m + logf(l) : -INFINITY;
  }
}

}  // namespace

size_t tree_workspace_bytes(const TreeArgs&, int) { return 0; }

cudaError_t launch_tree(const TreeArgs& a, int dt, cudaStream_t stream, int) {
  const dim3 grid(unsigned(a.max_nodes), unsigned(a.B));
  if (dt == TT_BF16)
    tree_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(a);
  else
    tree_kernel<__half><<<grid, kThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t preload_tree() {
  cudaFuncAttributes fa;
  cudaError_t e = cudaFuncGetAttributes(&fa, tree_kernel<__nv_bfloat16>);
  return e == cudaSuccess ? cudaFuncGetAttributes(&fa, tree_kernel<__half>) : e;
}

}  // namespace tt
