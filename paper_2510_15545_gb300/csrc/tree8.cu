// tree8.cu -- attention of drafted tokens over a paged cache that is held in 8 bits:
// e4m3 elements times a power of two for each 16 slots of a page and head.
//
// Token i of request b sees the L_b keys of the request's cache, its ancestors
// i, parent(i), parent(parent(i)), ... and nothing else; its output in a head is
// sum_x softmax_x(scale q.k_x) v_x over them, held in the running form.
#include <cstdint>
#include <cstring>

#include "tt_e4m3.cuh"
#include "tt_f2.cuh"
#include "tt_ops.h"
#include "tt_rope.cuh"

namespace tt {

namespace {

constexpr int kWarps = 4;

// One warp per row (token, head): lane l holds elements l D / 32 .. of the head.
template <int D, int DT>
__global__ void __launch_bounds__(kWarps * 32) tree8_kernel(const TreeArgs a, const TreeScales sc) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t row = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int h = int(row % a.Hq), hk = h / (a.Hq / a.Hkv);
  const int i = int(row / a.Hq % a.max_nodes), b = int(row / a.Hq / a.max_nodes);
  if (b >= a.B) return;
  int status = 0;
  const int first = a.tree_off[b], end = a.tree_off[b + 1], len = a.cache_len[b];
  if (first < 0 || end < first || end > a.n_nodes)
    status = TT_REQ_BAD_OFFSETS;
  else if (end - first > a.max_nodes || len < 0 || len > a.max_len)
    status = TT_REQ_TOO_LONG;
  const int nodes = status ? 0 : end - first;
  if (i == 0 && h == 0) {
    bool bad = false;
    if (a.parents)
      for (int j = lane; j < nodes; j += 32) {
        const int up = a.parents[first + j];
        bad |= up < -1 || up >= j;
      }
    if (!status)
      for (int x = lane; x < (len + a.page_size - 1) / a.page_size; x += 32) {
        const int page = a.page_table[b * a.table_stride + x];
        bad |= page < 0 || page >= a.n_pages;
      }
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) a.status[b] = status | (bad ? TT_REQ_ID_OUT_OF_RANGE : 0);
  }
  if (i >= nodes) return;
  float q[E];
  double acc[E] = {}, l = 0.0;  // (sums of many terms, one after the other)
  for (int e = 0; e < E; ++e)
    q[e] = load_elem<DT>(a.q + ((first + i) * a.q_token + h * a.q_head + lane * E + e) * 2);
  float m = -INFINITY;
  auto add = [&](float (&k)[E], float (&v)[E]) {
    float s = 0.f;
    for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    s *= a.scale;
    if (s == -INFINITY) return;  // (no weight)
    const float to = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - to);
    const float w = s != s ? s : expf(s - to);
    m = to;
    l = l * f + w;
    for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + double(w) * v[e];
  };
  for (int x = 0; x < len; ++x) {
    const int page = a.page_table[b * a.table_stride + x / a.page_size], slot = x % a.page_size;
    if (page < 0 || page >= a.n_pages) continue;
    auto read = [&](const char* data, int64_t ps, int64_t ss, int64_t hs, const TreeScale& s,
                    float (&y)[E]) {
      const float f = e8m0(s.data[page * s.page + slot / TT_SCALE_SLOTS * s.group + hk * s.head]);
      const char* at = data + page * ps + slot * ss + hk * hs + lane * E;
      for (int e = 0; e < E; e += 2) {
        const uint32_t two = e4m3x2_to_f16x2(*reinterpret_cast<const uint16_t*>(at + e));
        const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&two));
        y[e] = g.x * f;
        y[e + 1] = g.y * f;
      }
    };
    float k[E], v[E];
    read(a.kc, a.kc_page, a.kc_slot, a.kc_head, sc.k, k);
    read(a.vc, a.vc_page, a.vc_slot, a.vc_head, sc.v, v);
    add(k, v);
  }
  for (int j = i, up; j >= 0; j = up) {
    up = a.parents ? a.parents[first + j] : j - 1;
    if (up < -1 || up >= j) up = -1;
    float k[E], v[E];
    for (int e = 0; e < E; ++e) {
      k[e] = load_elem<DT>(a.k + ((first + j) * a.k_token + hk * a.k_head + lane * E + e) * 2);
      v[e] = load_elem<DT>(a.v + ((first + j) * a.v_token + hk * a.v_head + lane * E + e) * 2);
    }
    add(k, v);
  }
  const int64_t to = int64_t(first + i) * a.Hq + h;
  const double inv = l > 0.0 || l != l ? 1.0 / l : 0.0;
  for (int e = 0; e < E; ++e)
    store_elem<DT>(a.out + (to * D + lane * E + e) * 2, float(acc[e] * inv));
  if (a.lse && lane == 0) a.lse[to] = l > 0.0 || l != l ? m + float(log(l)) : -INFINITY;
}

template <int D, int DT>
cudaError_t launch(const TreeArgs& a, const TreeScales& sc, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned((int64_t(a.B) * a.max_nodes * a.Hq + kWarps - 1) / kWarps));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree8_kernel<D, DT>, a, sc);
}

}  // namespace

size_t tree8_workspace_bytes(const TreeArgs&, int) { return 256; }

bool tree8_fits(const TreeArgs& a, int) {
  return double(a.B) * a.max_nodes * double(a.Hq) <= INT32_MAX;
}

cudaError_t launch_tree8(const TreeArgs& a, const TreeScales& sc, int dt, cudaStream_t stream, int) {
  if (a.D == 128)
    return dt == TT_F16 ? launch<128, TT_F16>(a, sc, stream) : launch<128, TT_BF16>(a, sc, stream);
  return dt == TT_F16 ? launch<64, TT_F16>(a, sc, stream) : launch<64, TT_BF16>(a, sc, stream);
}

cudaError_t preload_tree8() {
  cudaFuncAttributes fa;
  cudaError_t e = cudaFuncGetAttributes(&fa, tree8_kernel<128, TT_F16>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, tree8_kernel<128, TT_BF16>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, tree8_kernel<64, TT_F16>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, tree8_kernel<64, TT_BF16>);
  return e;
}

}  // namespace tt
