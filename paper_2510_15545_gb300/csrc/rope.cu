// rope.cu -- rotary positions of query and key heads, and the host's frequencies.
//
// A pair (a, b) of a head at position x becomes m (a cos - b sin, b cos + a sin) of
// the angle x f; the transposed map (sines negated) takes the gradient back. Every
// element is read and written once, so memory bounds it. A thread turns the same
// pairs, one or two 16-byte vectors, in several heads of one token: their eight
// sines and cosines (some 200 instructions) are formed once for all of those, and
// the loads of four heads are under way at a time. 16,384 tokens of 40 heads of 128 in
// bf16 take 55 us, 6.1 TB/s; 4096 tokens in fp32 and their gradients 18.5 us.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "tt_ops.h"
#include "tt_rope.cuh"

namespace tt {

namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 4;   // heads whose loads a thread has under way
constexpr int kMostHeads = 8;  // of a thread

struct RopeKernelArgs {
  RopeArgs a;
  int pairs;    // n
  int units;    // of a head: those that turn first, then those that copy
  int turning;
  int tokens;   // of a CTA
  int chunk;    // heads of a thread
};

template <int DT, bool PAIRS, bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeKernelArgs p) {
  constexpr int E = Elems<DT>::kBytes;
  constexpr int VE = VEC ? Elems<DT>::kCount : 1;  // elements of a vector
  constexpr int P = VEC ? (PAIRS ? VE / 2 : VE) : 1;  // pairs of a unit
  const RopeArgs& a = p.a;
  const int u = threadIdx.x % p.units, in_cta = threadIdx.x / p.units;
  const uint32_t token = blockIdx.x * p.tokens + in_cta;  // (the last CTA's may pass 2^31)
  if (in_cta >= p.tokens || token >= uint32_t(a.n_tokens)) return;
  const int H = a.Hq + a.Hk;
  const int h0 = blockIdx.y * p.chunk, h1 = min(H, h0 + p.chunk);
  const bool turns = u < p.turning;
  // first element of the unit, and of the other half of its pairs
  int at, other = 0;
  if (turns) {
    at = PAIRS ? (VEC ? u * VE : 2 * u) : u * VE;
    other = PAIRS ? at + 1 : at + p.pairs;
  } else {
    at = 2 * p.pairs + (u - p.turning) * VE;
  }
  Turn turn[P];
  if (turns) {
    const int x = a.positions[token], pair0 = PAIRS ? at / 2 : at;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      turn[i] = turn_of(x, a.turns[pair0 + i]);
      turn[i].c *= a.mscale;
      turn[i].s *= a.back ? -a.mscale : a.mscale;
    }
  }
  auto place = [&](int h, bool out) {
    const bool q = h < a.Hq;
    const RopeTensor& x = out ? (q ? a.q_out : a.k_out) : (q ? a.q : a.k);
    return x.data + (int64_t(token) * x.token + int64_t(q ? h : h - a.Hq) * x.head) * E;
  };
  for (int h = h0; h < h1; h += kAtOnce) {
    if constexpr (VEC) {
      uint4 lo[kAtOnce], hi[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (h + i >= h1) break;
        const char* from = place(h + i, false);
        lo[i] = *reinterpret_cast<const uint4*>(from + at * E);
        if (!PAIRS && turns) hi[i] = *reinterpret_cast<const uint4*>(from + other * E);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (h + i >= h1) break;
        char* to = place(h + i, true);
        if (turns) {
          float x[VE], y[VE];
          unpack16<DT>(lo[i], x);
          if constexpr (PAIRS) {
#pragma unroll
            for (int j = 0; j < P; ++j) turn_pair(turn[j], x[2 * j], x[2 * j + 1]);
          } else {
            unpack16<DT>(hi[i], y);
#pragma unroll
            for (int j = 0; j < P; ++j) turn_pair(turn[j], x[j], y[j]);
            *reinterpret_cast<uint4*>(to + other * E) = pack16<DT>(y);
          }
          lo[i] = pack16<DT>(x);
        }
        *reinterpret_cast<uint4*>(to + at * E) = lo[i];
      }
    } else {
      float x[kAtOnce], y[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (h + i >= h1) break;
        const char* from = place(h + i, false);
        x[i] = load_elem<DT>(from + at * E);
        if (turns) y[i] = load_elem<DT>(from + other * E);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (h + i >= h1) break;
        char* to = place(h + i, true);
        if (turns) {
          turn_pair(turn[0], x[i], y[i]);
          store_elem<DT>(to + other * E, y[i]);
        }
        store_elem<DT>(to + at * E, x[i]);
      }
    }
  }
}

template <int DT, bool PAIRS>
cudaError_t launch(const RopeKernelArgs& p, bool vec, dim3 grid, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  return vec ? cudaLaunchKernelEx(&cfg, rope_kernel<DT, PAIRS, true>, p)
             : cudaLaunchKernelEx(&cfg, rope_kernel<DT, PAIRS, false>, p);
}

template <int DT>
cudaError_t preload() {
  cudaFuncAttributes fa;
  cudaError_t e = cudaFuncGetAttributes(&fa, rope_kernel<DT, false, false>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, rope_kernel<DT, false, true>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, rope_kernel<DT, true, false>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, rope_kernel<DT, true, true>);
  return e;
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int dt, cudaStream_t stream, int sm_count) {
  RopeKernelArgs p;
  std::memset(&p, 0, sizeof p);
  p.a = a;
  p.pairs = a.rot_dim / 2;
  // Whole vectors of the type, where the rotated part ends (and, of halves, begins
  // anew) on one; else single elements.
  const int ve = dt == TT_F32 ? 4 : 8;
  const bool vec = (a.interleaved ? a.rot_dim : p.pairs) % ve == 0;
  const int each = vec ? ve : 1;
  p.turning = (a.interleaved && vec ? a.rot_dim : p.pairs) / each;
  // (in place, what is not turned stays)
  const bool copies = a.q.data != a.q_out.data || (a.Hk > 0 && a.k.data != a.k_out.data);
  p.units = p.turning + (copies ? (a.D - a.rot_dim) / each : 0);
  p.tokens = kThreads / p.units;
  const int H = a.Hq + a.Hk;
  const int64_t blocks = (int64_t(a.n_tokens) + p.tokens - 1) / p.tokens;
  p.chunk = kMostHeads;
  while (p.chunk > 1 && blocks * ((H + p.chunk - 1) / p.chunk) < 2 * sm_count) p.chunk /= 2;
  const dim3 grid(unsigned(blocks), unsigned((H + p.chunk - 1) / p.chunk));
  auto go = [&](auto type) {
    constexpr int DT = decltype(type)::value;
    return a.interleaved ? launch<DT, true>(p, vec, grid, stream)
                         : launch<DT, false>(p, vec, grid, stream);
  };
  switch (dt) {
    case TT_F32: return go(std::integral_constant<int, TT_F32>());
    case TT_BF16: return go(std::integral_constant<int, TT_BF16>());
    default: return go(std::integral_constant<int, TT_F16>());
  }
}

cudaError_t preload_rope() {
  cudaError_t e = preload<TT_F32>();
  if (e == cudaSuccess) e = preload<TT_BF16>();
  if (e == cudaSuccess) e = preload<TT_F16>();
  return e;
}

}  // namespace tt
