// append.cu -- keys and values of new tokens into the requests' paged caches, the
// keys rotated on the way if asked for, in the tokens' type or in 8 bits.
//
// Slot len[b] + i of request b takes its i-th kept token. In 8 bits an element is an
// e4m3 value times 2^e, e of the 16 slots of its page and head: the least with which
// the largest element fits. A power of two costs nothing: e4m3 values of all sizes
// have the same four digits, so a finer factor would only shift where they begin to
// lose them, 2^-15 below the largest; and what is raised to a larger e later loses
// nothing above that, where another factor would round all of it anew. 16 slots: a
// byte for 16 heads' worth of elements is 1/2048 of the cache, and what an outlier
// costs its neighbours stays with 16 of them.
//
// Every element is read and written once, so memory bounds it. Work is one group of
// 16 slots of one head: a warp holds its elements in fp32 registers between finding
// the largest and rounding them, keys first, then values. The warps of a CTA take the
// heads of the same group, and share its sines and cosines, formed once, through
// shared memory: formed by each head they took as many instructions as the copies'
// time allows. The groups that the requests touch form one list, which the CTAs share
// evenly: how many a request brings is known on the device alone.
#include <algorithm>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "tt_e4m3.cuh"
#include "tt_ops.h"
#include "tt_rope.cuh"

namespace tt {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kGroup = TT_SCALE_SLOTS;
constexpr int kMostSets = 4;

enum Rotation { kNone = 0, kHalf = 1, kHalfOdd = 2, kPairs = 3 };

struct AppendKernelArgs {
  AppendArgs a;
  int rotation;   // kHalfOdd: a half that does not begin on a vector
  int pairs;      // n
  int columns;    // of the table: ceil(n / 8)
  int set_warps;  // that share a group
  int sets;       // groups that a CTA has in work at once
};

// What a request brings: its tokens in the batch, how many of them are kept, the slots
// in use before.
struct Fresh {
  int first, tokens, n, len, status;
};
__device__ __forceinline__ Fresh fresh(const AppendArgs& a, int b) {
  Fresh r{a.token_off[b], 0, 0, a.cache_len[b], 0};
  const int end = a.token_off[b + 1];
  if (r.first < 0 || end < r.first || end > a.n_tokens) {
    r.status = TT_REQ_BAD_OFFSETS;
    return r;
  }
  r.tokens = end - r.first;
  const int n = a.keep ? a.keep[b] : r.tokens;
  if (n < 0 || n > r.tokens)
    r.status = TT_REQ_BAD_OFFSETS;
  else if (r.len < 0 || r.len > a.max_len || n > a.max_len - r.len || r.tokens > a.max_new)
    r.status = TT_REQ_TOO_LONG;
  else
    r.n = n;
  return r;
}
__device__ __forceinline__ int groups(const Fresh& r) {
  return r.n > 0 ? (r.len + r.n - 1) / kGroup - r.len / kGroup + 1 : 0;
}

// A group of the list.
struct Walk {
  int b, g;  // its request, and which of that one's groups
  Fresh r;
  __device__ __forceinline__ void forward(const AppendArgs& a, int by) {
    g += by;
    for (int n; b < a.B && g >= (n = groups(r));) {
      g -= n;
      if (++b < a.B) r = fresh(a, b);
    }
  }
};

template <int DT, int D, bool HELD8>
__global__ void __launch_bounds__(kThreads, 2)
    append_kernel(const __grid_constant__ AppendKernelArgs p) {
  constexpr int kLanes = D / 8;            // that hold a token's head
  constexpr int kPer = 32 / kLanes;        // tokens of a warp at once
  constexpr int kPasses = kGroup / kPer;
  const AppendArgs& a = p.a;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  extern __shared__ float2 tables[];  // [2][sets][16 slots][8 columns][..] cosines and sines
  __shared__ int s_row[2][kMostSets][kGroup];  // the batch's row of each slot, -1: none
  __shared__ long long s_sum[kWarps];
  __shared__ int s_b, s_g;

  // the list: each thread adds up a run of requests
  const int each = (a.B + kThreads - 1) / kThreads;
  const int b0 = min(a.B, t * each), b1 = min(a.B, b0 + each);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += groups(fresh(a, b));
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += s_sum[w];
    all += s_sum[w];
  }
  const long long share = (all + gridDim.x - 1) / gridDim.x;
  const long long from = share * blockIdx.x;
  const long long todo = max(0ll, min(share, all - from));
  if (todo > 0 && from >= upto - mine && from < upto) {
    long long at = upto - mine;
    for (int b = b0; b < b1; ++b) {
      const int n = groups(fresh(a, b));
      if (from < at + n) {
        s_b = b;
        s_g = int(from - at);
        break;
      }
      at += n;
    }
  }
  __syncthreads();

  const int set = warp / p.set_warps, in_set = warp % p.set_warps;
  const bool busy = set < p.sets;
  const int per_token = 8 * p.columns, per_set = kGroup * per_token;
  Walk x;
  if (todo > 0) {
    x.b = s_b;
    x.g = 0;
    x.r = fresh(a, x.b);
    x.forward(a, s_g + (busy ? set : 0));
  }
  int it = 0;
  for (long long u = 0; u < todo; u += p.sets, ++it) {
    const bool some = busy && u + set < todo;
    const int slot0 = some ? (x.r.len / kGroup + x.g) * kGroup : 0;  // of the group, in the cache
    // new slots of the group: lead .. end - 1; those before are in use
    const int lead = some ? max(0, x.r.len - slot0) : 0;
    const int end = some ? min(kGroup, x.r.len + x.r.n - slot0) : 0;
    float2* const table = tables + ((it & 1) * p.sets + (busy ? set : 0)) * per_set;
    int* const rows = s_row[it & 1][busy ? set : 0];
    auto row_of = [&](int i) {  // of slot i of the group
      if (i < lead || i >= end) return -1;
      const int k = slot0 + i - x.r.len;
      if (!a.path) return x.r.first + k;
      const int at = a.path[x.r.first + k];
      return at >= 0 && at < x.r.tokens ? x.r.first + at : -1;
    };
    if (some) {
      if (in_set == 0 && lane < kGroup) rows[lane] = row_of(lane);
      if (p.rotation != kNone) {
        for (int i = in_set * 32 + lane; i < (end - lead) * p.pairs; i += p.set_warps * 32) {
          const int slot = lead + i / p.pairs, pair = i % p.pairs;
          int position = slot0 + slot;
          if (a.positions) {
            const int row = row_of(slot);
            position = row >= 0 ? a.positions[row] : 0;
          }
          const Turn turn = turn_of(position, a.turns[pair]);
          table[slot * per_token + (pair & 7) * p.columns + (pair >> 3)] =
              make_float2(turn.c * a.mscale, turn.s * a.mscale);
        }
      }
    }
    __syncthreads();
    if (!some) continue;
    const int page = a.page_table[int64_t(x.b) * a.table_stride + slot0 / a.page_size];
    if (page >= 0 && page < a.n_pages) {
      const int in_page = slot0 % a.page_size, e0 = (lane % kLanes) * 8;
      for (int h = in_set; h < a.H; h += p.set_warps) {
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          const RopeTensor& from = kv ? a.v : a.k;
          const AppendCache& to = kv ? a.v_cache : a.k_cache;
          uint4 own[kPasses], other[kPasses];
          const bool turns = kv == 0 && p.rotation != kNone && e0 < 2 * p.pairs;
          const bool first = e0 < p.pairs;  // of a pair
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            const int row = rows[i * kPer + lane / kLanes];
            own[i] = other[i] = make_uint4(0, 0, 0, 0);
            if (row < 0) continue;
            const char* at = from.data + (int64_t(row) * from.token + int64_t(h) * from.head) * 2;
            own[i] = *reinterpret_cast<const uint4*>(at + e0 * 2);
            if (turns && p.rotation == kHalf)
              other[i] = *reinterpret_cast<const uint4*>(
                  at + (first ? e0 + p.pairs : e0 - p.pairs) * 2);
          }
          float v[kPasses][8];
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            unpack16<DT>(own[i], v[i]);
            const int slot = i * kPer + lane / kLanes;
            const int row = turns ? rows[slot] : -1;
            if (row >= 0) {
              const float2* cs = table + slot * per_token;
              auto turn = [&](int pair) {
                const float2 y = cs[(pair & 7) * p.columns + (pair >> 3)];
                return Turn{y.x, y.y};
              };
              if (p.rotation == kPairs) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (e0 / 2 + j < p.pairs) turn_pair(turn(e0 / 2 + j), v[i][2 * j], v[i][2 * j + 1]);
              } else if (p.rotation == kHalf) {
                float y[8];
                unpack16<DT>(other[i], y);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const Turn c = turn(first ? e0 + j : e0 + j - p.pairs);
                  if (first)
                    turn_pair(c, v[i][j], y[j]);
                  else
                    turn_pair(c, y[j], v[i][j]);
                }
              } else {
                const char* at =
                    from.data + (int64_t(row) * from.token + int64_t(h) * from.head) * 2;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const int e = e0 + j;
                  if (e < p.pairs) {
                    float y = load_elem<DT>(at + (e + p.pairs) * 2);
                    turn_pair(turn(e), v[i][j], y);
                  } else if (e < 2 * p.pairs) {
                    float y = load_elem<DT>(at + (e - p.pairs) * 2);
                    turn_pair(turn(e - p.pairs), y, v[i][j]);
                  }
                }
              }
            }
            if constexpr (HELD8) {
              // What is not finite has no e4m3 value but NaN. The largest values are held
              // back to what rounds to a finite number of the tokens' type again.
              constexpr float kMost = DT == TT_F16 ? 61440.f : 0x1.ep127f;
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const float y = fabsf(v[i][j]);
                if (!(y < INFINITY))
                  v[i][j] = __uint_as_float(0x7fc00000u);
                else if (y > kMost)
                  v[i][j] = copysignf(kMost, v[i][j]);
                top = fmaxf(top, fabsf(v[i][j]));
              }
            }
          }
          char* const head = to.data + (int64_t(page) * to.page + int64_t(h) * to.head +
                                        int64_t(in_page) * to.slot) * (HELD8 ? 1 : 2);
          float inverse = 1.f;
          if constexpr (HELD8) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            uint8_t* const scale = to.scale + int64_t(page) * to.scale_page +
                                   int64_t(in_page / kGroup) * to.scale_group +
                                   int64_t(h) * to.scale_head;
            uint32_t code = e8m0_for(top);
            if (lead > 0) {
              const uint32_t old = *scale;
              if (old != 255) code = max(code, old);
              if (code != old) {  // slots in use: rounded again (NaN where they were that)
                const float by = e8m0(old) * e8m0_inverse(code);
                for (int slot = lane / kLanes; slot < lead; slot += kPer) {
                  uint2* at = reinterpret_cast<uint2*>(head + int64_t(slot) * to.slot + e0);
                  uint2 w = *at;
                  uint32_t* half = &w.x;
#pragma unroll
                  for (int q = 0; q < 2; ++q, half = &w.y) {
                    uint32_t two[2] = {e4m3x2_to_f16x2(*half & 0xffff), e4m3x2_to_f16x2(*half >> 16)};
                    uint32_t r[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                      const float2 f = __half22float2(*reinterpret_cast<__half2*>(&two[k]));
                      r[k] = to_e4m3x2(f.x * by, f.y * by);
                    }
                    *half = r[0] | r[1] << 16;
                  }
                  *at = w;
                }
              }
              __syncwarp();  // (all have read the old code)
            }
            if (lane == 0) *scale = uint8_t(code);
            inverse = e8m0_inverse(code);
          }
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            const int slot = i * kPer + lane / kLanes;
            if (rows[slot] < 0) continue;
            if constexpr (HELD8) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                w[j] = to_e4m3x2(v[i][2 * j] * inverse, v[i][2 * j + 1] * inverse);
              *reinterpret_cast<uint2*>(head + int64_t(slot) * to.slot + e0) =
                  make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
            } else {
              *reinterpret_cast<uint4*>(head + (int64_t(slot) * to.slot + e0) * 2) = pack16<DT>(v[i]);
            }
          }
        }
      }
    }
    x.forward(a, p.sets);
  }

  // what became of the requests
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const Fresh r = fresh(a, b);
    bool bad = false;
    if (a.path)
      for (int i = t; i < r.n; i += kThreads) {
        const int at = a.path[r.first + i];
        bad |= at < 0 || at >= r.tokens;
      }
    if (r.n > 0)
      for (int i = r.len / a.page_size + t; i <= (r.len + r.n - 1) / a.page_size; i += kThreads) {
        const int page = a.page_table[int64_t(b) * a.table_stride + i];
        bad |= page < 0 || page >= a.n_pages;
      }
    bad = __syncthreads_or(bad);
    if (t == 0) {
      a.status[b] = r.status | (bad ? TT_REQ_ID_OUT_OF_RANGE : 0);
      if (a.new_len) a.new_len[b] = bad ? r.len : r.len + r.n;
    }
  }
}

template <int DT, int D, bool HELD8>
cudaError_t launch(const AppendKernelArgs& p, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes =
      p.rotation == kNone ? 0 : size_t(2) * p.sets * kGroup * 8 * p.columns * sizeof(float2);
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, append_kernel<DT, D, HELD8>, p);
}

template <int DT, int D>
cudaError_t preload() {
  // (the largest table: four groups of 64 pairs, twice)
  constexpr int kMost = 2 * kMostSets * kGroup * (D / 2) * int(sizeof(float2));
  cudaError_t e = cudaFuncSetAttribute(append_kernel<DT, D, false>,
                                       cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
  return e == cudaSuccess ? cudaFuncSetAttribute(append_kernel<DT, D, true>,
                                                 cudaFuncAttributeMaxDynamicSharedMemorySize, kMost)
                          : e;
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int dt, bool held8, cudaStream_t stream,
                          int sm_count) {
  AppendKernelArgs p;
  std::memset(&p, 0, sizeof p);
  p.a = a;
  p.pairs = a.rot_dim / 2;
  p.columns = (p.pairs + 7) / 8;
  p.rotation = a.rot_dim == 0 ? kNone : a.interleaved ? kPairs : p.pairs % 8 == 0 ? kHalf : kHalfOdd;
  p.set_warps = std::min(a.H, kWarps);
  p.sets = std::min(kMostSets, kWarps / p.set_warps);
  // (at most so many groups: the first and the last of a request are not whole)
  const int64_t most = std::min(int64_t(a.n_tokens) / kGroup + 2 * int64_t(a.B),
                                int64_t(a.B) * ((int64_t(a.max_new) + kGroup - 2) / kGroup + 1));
  const int ctas = int(std::max<int64_t>(1, std::min<int64_t>((most + p.sets - 1) / p.sets,
                                                              3 * int64_t(sm_count))));
  auto go = [&](auto type, auto dim) {
    constexpr int DT = decltype(type)::value, D = decltype(dim)::value;
    return held8 ? launch<DT, D, true>(p, ctas, stream) : launch<DT, D, false>(p, ctas, stream);
  };
  auto of_type = [&](auto type) {
    return a.D == 128 ? go(type, std::integral_constant<int, 128>())
                      : go(type, std::integral_constant<int, 64>());
  };
  return dt == TT_F16 ? of_type(std::integral_constant<int, TT_F16>())
                      : of_type(std::integral_constant<int, TT_BF16>());
}

cudaError_t preload_append() {
  cudaError_t e = preload<TT_BF16, 128>();
  if (e == cudaSuccess) e = preload<TT_BF16, 64>();
  if (e == cudaSuccess) e = preload<TT_F16, 128>();
  if (e == cudaSuccess) e = preload<TT_F16, 64>();
  return e;
}

}  // namespace tt
