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
// 16 slots of one head: a warp holds its elements in registers between finding the
// largest and rounding them, keys first, then values. The warps of a CTA take the
// heads of the same group, and share its sines and cosines, formed once, through
// shared memory: formed by each head they took as many instructions as the copies'
// time allows. The groups that the requests touch form one list, which the CTAs share
// evenly: how many a request brings is known on the device alone.
//
// 8 prompts of 8192 tokens, 8 heads of 128, turned, to 8 bits: 92 us, 4.4 TB/s. A lane has
// both elements of its pairs (with a vector of its own and its partner's, turned by both
// lanes, 309 us); values are fetched into L2 while sines are formed (98 without). Two CTAs of
// 128 registers to an SM: a third's worth of the list waited for a second round. Single
// tokens of 256 requests: 10 us, one dependent read after another.
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

// kHalf, kPairs: whole vectors of pairs; kOdd: any number, of either layout.
enum Rotation { kNone = 0, kHalf = 1, kPairs = 2, kOdd = 3 };

struct AppendKernelArgs {
  AppendArgs a;
  int pairs;      // n
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

// The larger of three sizes; NaN has none.
__device__ __forceinline__ float most(float x, float a, float b) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}

template <int DT, int D, bool HELD8, int ROT>
__global__ void __launch_bounds__(kThreads, 2)
    append_kernel(const __grid_constant__ AppendKernelArgs p) {
  // A lane holds two vectors of 8 elements of a token's head: of halves that turn against
  // each other, one of each; else neighbours. So it has both elements of its pairs, and
  // they are 8 l .. 8 l + 7 for lane l.
  constexpr int kLanes = D / 16;           // that hold a token's head
  constexpr int kPer = 32 / kLanes;        // tokens of a warp at once
  constexpr int kPasses = kGroup / kPer;
  constexpr int kSet = kGroup * D / 4;     // of a table: two pairs to an entry
  using Raw = uint4[kPasses][2];
  const AppendArgs& a = p.a;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  extern __shared__ float4 tables[];  // [2][sets][16 slots][4 twos][lanes] cosines and sines
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
  const int l = lane % kLanes, slot_of = lane / kLanes;  // (of a pass)
  // the first elements of the lane's vectors
  const bool turns = ROT == kOdd || 8 * l < p.pairs;
  int e0 = 16 * l, e1 = 16 * l + 8;
  if (ROT == kHalf) {
    e0 = turns ? 8 * l : 16 * l;  // (2 n + 16 (l - n / 8))
    e1 = turns ? 8 * l + p.pairs : 16 * l + 8;
  }
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
    auto row_of = [&](int i) {  // the batch's row of slot i of the group, -1: none
      if (i < lead || i >= end) return -1;
      const int k = slot0 + i - x.r.len;
      if (!a.path) return x.r.first + k;
      const int at = a.path[x.r.first + k];
      return at >= 0 && at < x.r.tokens ? x.r.first + at : -1;
    };
    int page = -1, rows[kPasses];
    if (some) page = a.page_table[int64_t(x.b) * a.table_stride + slot0 / a.page_size];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) rows[i] = row_of(i * kPer + slot_of);
    auto load = [&](const RopeTensor& from, int h, Raw& raw) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        raw[i][0] = raw[i][1] = make_uint4(0, 0, 0, 0);
        if (rows[i] < 0) continue;
        const char* at = from.data + (int64_t(rows[i]) * from.token + int64_t(h) * from.head) * 2;
        raw[i][0] = *reinterpret_cast<const uint4*>(at + e0 * 2);
        raw[i][1] = *reinterpret_cast<const uint4*>(at + e1 * 2);
      }
    };
    // (the first head's keys are on their way while the sines are formed)
    Raw raw;
    if (some && in_set < a.H) {
      load(a.k, in_set, raw);
      // (and values come nearer)
      if (l % 4 == 0)
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
          if (rows[i] >= 0)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(
                a.v.data + (int64_t(rows[i]) * a.v.token + int64_t(in_set) * a.v.head) * 2 + 32 * l));
    }
    if constexpr (ROT != kNone) {
      float4* const table = tables + ((it & 1) * p.sets + (busy ? set : 0)) * kSet;
      if (some) {
        float2* const to = reinterpret_cast<float2*>(table);
        for (int i = in_set * 32 + lane; i < (end - lead) * (D / 2); i += p.set_warps * 32) {
          const int slot = lead + i / (D / 2), pair = i % (D / 2);
          if (pair >= p.pairs) continue;
          int position = slot0 + slot;
          if (a.positions) {
            const int row = row_of(slot);
            position = row >= 0 ? a.positions[row] : 0;
          }
          const Turn turn = turn_of(position, a.turns[pair]);
          to[((slot * 4 + (pair >> 1 & 3)) * kLanes + (pair >> 3)) * 2 + (pair & 1)] =
              make_float2(turn.c * a.mscale, turn.s * a.mscale);
        }
      }
      __syncthreads();
    }
    if (!some) continue;
    if (page >= 0 && page < a.n_pages) {
      const float4* const table = tables + ((it & 1) * p.sets + set) * kSet;
      const int in_page = slot0 % a.page_size;
      auto head_of = [&](const AppendCache& to, int h) {  // its first slot of the group
        return to.data + (int64_t(page) * to.page + int64_t(h) * to.head + int64_t(in_page) * to.slot) *
                             (HELD8 ? 1 : 2);
      };
      // The scale of the group, with which the largest element `top` (of a lane) fits: what
      // elements are multiplied by. Slots in use are rounded again where it rises.
      auto scale_for = [&](const AppendCache& to, int h, float top) {
        uint8_t* const scale = to.scale + int64_t(page) * to.scale_page +
                               int64_t(in_page / kGroup) * to.scale_group + int64_t(h) * to.scale_head;
        uint32_t code = e8m0_for(top);
        if (lead > 0) {
          const uint32_t old = *scale;
          if (old != 255) code = max(code, old);
          if (code != old) {  // (NaN where they were that)
            const float by = e8m0(old) * e8m0_inverse(code);
            char* const head = head_of(to, h);
#pragma unroll 1
            for (int slot = slot_of; slot < lead; slot += kPer) {
              uint4* at = reinterpret_cast<uint4*>(head + int64_t(slot) * to.slot + 16 * l);
              uint4 w = *at;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                uint32_t& half = q == 0 ? w.x : q == 1 ? w.y : q == 2 ? w.z : w.w;
                uint32_t two[2] = {e4m3x2_to_f16x2(half & 0xffff), e4m3x2_to_f16x2(half >> 16)};
                uint32_t r[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const float2 f = __half22float2(*reinterpret_cast<__half2*>(&two[k]));
                  r[k] = to_e4m3x2(f.x * by, f.y * by);
                }
                half = r[0] | r[1] << 16;
              }
              *at = w;
            }
          }
          __syncwarp();  // (all have read the old code)
        }
        if (lane == 0) *scale = uint8_t(code);
        return e8m0_inverse(code);
      };
      // (sizes are in the order of their bits)
      auto of_warp = [](float top) {
        return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));
      };
      // What is not finite has no e4m3 value but NaN. The largest values are held back to
      // what rounds to a finite number of the tokens' type again, and is one.
      constexpr float kMost = DT == TT_F16 ? 61440.f : 0x1.ep127f;
      auto held = [](float y) {
        return !(fabsf(y) < INFINITY) ? __uint_as_float(0x7fc00000u)
               : fabsf(y) > kMost     ? copysignf(kMost, y)
                                      : y;
      };
      auto e4m3x8 = [](const float (&z)[8], float by) {
        return make_uint2(to_e4m3x2(z[0] * by, z[1] * by) | to_e4m3x2(z[2] * by, z[3] * by) << 16,
                          to_e4m3x2(z[4] * by, z[5] * by) | to_e4m3x2(z[6] * by, z[7] * by) << 16);
      };
      // Vectors as they came.
      auto put = [&](const AppendCache& to, int h) {
        char* const head = head_of(to, h) + int64_t(slot_of) * to.slot * (HELD8 ? 1 : 2);
        if constexpr (!HELD8) {
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            if (rows[i] < 0) continue;
            char* const at = head + int64_t(i * kPer) * to.slot * 2;
            *reinterpret_cast<uint4*>(at + e0 * 2) = raw[i][0];
            *reinterpret_cast<uint4*>(at + e1 * 2) = raw[i][1];
          }
        } else {
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < kPasses * 2; ++i) {
            float z[8];
            unpack16<DT>(raw[i / 2][i % 2], z);
#pragma unroll
            for (int j = 0; j < 8; j += 2) top = most(top, z[j], z[j + 1]);
          }
          top = of_warp(top);
          if (top > kMost) {
            top = 0.f;
#pragma unroll
            for (int i = 0; i < kPasses * 2; ++i) {
              float z[8];
              unpack16<DT>(raw[i / 2][i % 2], z);
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                z[j] = held(z[j]);
                top = most(top, z[j], z[j]);
              }
              raw[i / 2][i % 2] = pack16<DT>(z);
            }
            top = of_warp(top);
          }
          const float by = scale_for(to, h, top);
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            float z[8];
            unpack16<DT>(raw[i][0], z);
            const uint2 w0 = e4m3x8(z, by);
            unpack16<DT>(raw[i][1], z);
            const uint2 w1 = e4m3x8(z, by);
            if (rows[i] < 0) continue;
            char* const at = head + int64_t(i * kPer) * to.slot;
            if constexpr (ROT == kHalf) {
              *reinterpret_cast<uint2*>(at + e0) = w0;
              *reinterpret_cast<uint2*>(at + e1) = w1;
            } else {
              *reinterpret_cast<uint4*>(at + e0) = make_uint4(w0.x, w0.y, w1.x, w1.y);
            }
          }
        }
      };
      // Keys, turned: in 32 bits until they are rounded.
      auto put_turned = [&](int h) {
        const AppendCache& to = a.k_cache;
        float v[kPasses][2][8];
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
          unpack16<DT>(raw[i][0], v[i][0]);
          unpack16<DT>(raw[i][1], v[i][1]);
          const int slot = i * kPer + slot_of;
          if (turns && rows[i] >= 0) {
            if constexpr (ROT == kOdd) {
              const float2* cs = reinterpret_cast<const float2*>(table);
              auto turn = [&](int pair) {
                const float2 y = cs[((slot * 4 + (pair >> 1 & 3)) * kLanes + (pair >> 3)) * 2 + (pair & 1)];
                return Turn{y.x, y.y};
              };
              const char* at =
                  a.k.data + (int64_t(rows[i]) * a.k.token + int64_t(h) * a.k.head) * 2;
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const int e = 16 * l + 8 * c + j;
                  if (e >= 2 * p.pairs) continue;
                  const bool first = a.interleaved ? !(e & 1) : e < p.pairs;
                  const int pair = a.interleaved ? e / 2 : first ? e : e - p.pairs;
                  const int e_other = a.interleaved ? e ^ 1 : first ? e + p.pairs : e - p.pairs;
                  float y = load_elem<DT>(at + e_other * 2);
                  if (first)
                    turn_pair(turn(pair), v[i][c][j], y);
                  else
                    turn_pair(turn(pair), y, v[i][c][j]);
                }
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const float4 y = table[(slot * 4 + q) * kLanes + l];
                if constexpr (ROT == kHalf) {
                  turn_pair(Turn{y.x, y.y}, v[i][0][2 * q], v[i][1][2 * q]);
                  turn_pair(Turn{y.z, y.w}, v[i][0][2 * q + 1], v[i][1][2 * q + 1]);
                } else {
                  float* z = &v[i][q >> 1][4 * (q & 1)];
                  turn_pair(Turn{y.x, y.y}, z[0], z[1]);
                  turn_pair(Turn{y.z, y.w}, z[2], z[3]);
                }
              }
            }
          }
          if constexpr (HELD8) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int j = 0; j < 8; j += 2) top = most(top, v[i][c][j], v[i][c][j + 1]);
          }
        }
        float by = 1.f;
        if constexpr (HELD8) {
          top = of_warp(top);
          if (top > kMost) {
            top = 0.f;
#pragma unroll
            for (int i = 0; i < kPasses * 16; ++i) {
              float& y = v[i / 16][i / 8 % 2][i % 8];
              y = held(y);
              top = most(top, y, y);
            }
            top = of_warp(top);
          }
          by = scale_for(to, h, top);
        }
        char* const head = head_of(to, h) + int64_t(slot_of) * to.slot * (HELD8 ? 1 : 2);
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
          if (rows[i] < 0) continue;
          char* const at = head + int64_t(i * kPer) * to.slot * (HELD8 ? 1 : 2);
          if constexpr (HELD8) {
            *reinterpret_cast<uint2*>(at + e0) = e4m3x8(v[i][0], by);
            *reinterpret_cast<uint2*>(at + e1) = e4m3x8(v[i][1], by);
          } else {
            *reinterpret_cast<uint4*>(at + e0 * 2) = pack16<DT>(v[i][0]);
            *reinterpret_cast<uint4*>(at + e1 * 2) = pack16<DT>(v[i][1]);
          }
        }
      };
#pragma unroll 1
      for (int h = in_set; h < a.H; h += p.set_warps) {
        if (h != in_set) load(a.k, h, raw);
        if constexpr (ROT == kNone)
          put(a.k_cache, h);
        else
          put_turned(h);
        load(a.v, h, raw);
        put(a.v_cache, h);
      }
    }
    x.forward(a, p.sets);
  }

  // What became of the requests: a warp to each, those of the last CTAs first, which have
  // the least to do where there are few tokens.
  const int back = (int(gridDim.x) - 1 - int(blockIdx.x)) * kWarps + warp;
  for (int64_t b = back; b < a.B; b += int64_t(gridDim.x) * kWarps) {
    const Fresh r = fresh(a, int(b));
    bool bad = false;
    if (a.path)
      for (int i = lane; i < r.n; i += 32) {
        const int at = a.path[r.first + i];
        bad |= at < 0 || at >= r.tokens;
      }
    if (r.n > 0)
      for (int i = r.len / a.page_size + lane; i <= (r.len + r.n - 1) / a.page_size; i += 32) {
        const int page = a.page_table[b * a.table_stride + i];
        bad |= page < 0 || page >= a.n_pages;
      }
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) {
      a.status[b] = r.status | (bad ? TT_REQ_ID_OUT_OF_RANGE : 0);
      if (a.new_len) a.new_len[b] = bad ? r.len : r.len + r.n;
    }
  }
}

// Launches a form of the kernel, or without p prepares it.
template <int DT, int D, bool HELD8, int ROT>
cudaError_t run(const AppendKernelArgs* p, int ctas, cudaStream_t stream) {
  constexpr size_t kTable = 2 * (kGroup * D / 4) * sizeof(float4);  // of a set
  if (!p)
    return cudaFuncSetAttribute(append_kernel<DT, D, HELD8, ROT>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMostSets * kTable));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = ROT == kNone ? 0 : p->sets * kTable;
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, append_kernel<DT, D, HELD8, ROT>, *p);
}
template <int DT, int D, bool HELD8>
cudaError_t of_rotation(int rotation, const AppendKernelArgs* p, int ctas, cudaStream_t stream) {
  switch (rotation) {
    case kNone: return run<DT, D, HELD8, kNone>(p, ctas, stream);
    case kHalf: return run<DT, D, HELD8, kHalf>(p, ctas, stream);
    case kPairs: return run<DT, D, HELD8, kPairs>(p, ctas, stream);
    default: return run<DT, D, HELD8, kOdd>(p, ctas, stream);
  }
}
template <int DT>
cudaError_t of_form(int D, bool held8, int rotation, const AppendKernelArgs* p, int ctas,
                    cudaStream_t stream) {
  if (D == 128)
    return held8 ? of_rotation<DT, 128, true>(rotation, p, ctas, stream)
                 : of_rotation<DT, 128, false>(rotation, p, ctas, stream);
  return held8 ? of_rotation<DT, 64, true>(rotation, p, ctas, stream)
               : of_rotation<DT, 64, false>(rotation, p, ctas, stream);
}

}  // namespace

cudaError_t launch_append(const AppendArgs& a, int dt, bool held8, cudaStream_t stream,
                          int sm_count) {
  AppendKernelArgs p;
  std::memset(&p, 0, sizeof p);
  p.a = a;
  p.pairs = a.rot_dim / 2;
  const int rotation = a.rot_dim == 0       ? kNone
                       : p.pairs % 8        ? kOdd
                       : a.interleaved ? kPairs
                                            : kHalf;
  p.set_warps = std::min(a.H, kWarps);
  p.sets = std::min(kMostSets, kWarps / p.set_warps);
  // (at most so many groups: the first and the last of a request are not whole)
  const int64_t most = std::min(int64_t(a.n_tokens) / kGroup + 2 * int64_t(a.B),
                                int64_t(a.B) * ((int64_t(a.max_new) + kGroup - 2) / kGroup + 1));
  // (two CTAs to an SM: as many as are in work at once)
  const int ctas = int(std::max<int64_t>(1, std::min<int64_t>((most + p.sets - 1) / p.sets,
                                                              2 * int64_t(sm_count))));
  return dt == TT_F16 ? of_form<TT_F16>(a.D, held8, rotation, &p, ctas, stream)
                      : of_form<TT_BF16>(a.D, held8, rotation, &p, ctas, stream);
}

cudaError_t preload_append() {
  for (int D : {64, 128})
    for (bool held8 : {false, true})
      for (int rotation : {kNone, kHalf, kPairs, kOdd}) {
        cudaError_t e = of_form<TT_F16>(D, held8, rotation, nullptr, 0, nullptr);
        if (e == cudaSuccess) e = of_form<TT_BF16>(D, held8, rotation, nullptr, 0, nullptr);
        if (e != cudaSuccess) return e;
      }
  return cudaSuccess;
}

}  // namespace tt
