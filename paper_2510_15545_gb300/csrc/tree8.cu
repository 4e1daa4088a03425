// tree8.cu -- attention of drafted tokens over a paged cache that is held in 8 bits:
// e4m3 elements times a power of two for each 16 slots of a page and head.
//
// Token i of request b sees the L_b keys of the request's cache, its ancestors
// i, parent(i), parent(parent(i)), ... and nothing else; its output in a head is
// sum_x softmax_x(scale q.k_x) v_x over them, held in the running form: with
// m = max s_x and l = sum 2^(s_x - m), a larger m scales what was summed before.
//
// The bound is the cache, half of what 16 bits take, so half the time for each of its
// tiles. Their products are matrix products: 128 rows (token, head of the group) against
// tiles of 128 keys. Keys are multiplied as they are, e4m3 by e4m3: a query is the sum of
// two (bf16) or three (fp16) e4m3 pieces of a power of two of its row, its 8 or 11 digits
// exactly for elements down to 2^-10 of the row's largest, and within 2^-19 of that below;
// the products add the pieces up. Values become fp16, which holds every e4m3 value, by four
// warps of their own, in units of the largest scale so far (2^-24 of that unit is the
// finest); when a larger one comes the sums fall. The request's own drafted tokens are
// tiles of keys and values of the inputs' type.
//
// One CTA per SM: two warps copy (a page's slots at a time) keys and values with their
// scales, four convert, two issue the products, eight hold the rows, two threads each.
// While rows turn a tile's scores into weights, the next tile's scores and the last one's
// product with values are under way: tensor memory holds two tiles' scores, two tiles'
// weights and the output. Tiles of all requests, key heads and 128 rows form one list,
// which the CTAs share evenly: lengths are known on the device alone. Items cut by a CTA's
// end leave unnormalised pieces, which a second kernel joins.
//
// Built and taken back: keys as the rows of the products and tokens as their columns, so
// that they cost what the columns cost. A thread then has a key, and a row's factor,
// maximum and sum come from shared memory or go across threads: 12 instructions a score
// for 4 here, and a serving batch took 199 us.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstring>
#include <numeric>
#include <type_traits>

#include "tt_device.cuh"
#include "tt_e4m3.cuh"
#include "tt_f2.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"
#include "tt_rope.cuh"
#include "tt_umma.cuh"
#include "tt_x2.cuh"

namespace tt {

namespace {

constexpr int kTile = 128;                     // keys of a tile
constexpr int kConvWarps = 4, kConvThreads = kConvWarps * 32;  // that convert values
constexpr int kRows = 128;                     // of an item
constexpr int kRowWarps = 8, kRowThreads = kRowWarps * 32;  // two for each 32 rows
constexpr int kThreads = kRowThreads + kConvThreads + 128;
constexpr int kWords = TT_MAX_TREE / 32;
constexpr int kGroups = kTile / TT_SCALE_SLOTS;  // scales of a tile
constexpr int kScaleRing = 16;                   // tiles' scales that are kept
constexpr int kBatch = 4;                        // tiles whose pages are asked for together
constexpr float kLn2 = 0.693147180559945f;
// A row's reference maximum follows its maximum once that is 2^kSlack above it:
// weights stay below 2^(kSlack + offset), and the output is scaled rarely.
constexpr float kSlack = 8.f;
constexpr int kMinShare = 2;  // places of a CTA, where there are few
// What an item costs beyond its tiles (queries, ancestors, output), in tiles: it
// takes as many places in the list before its first tile.
constexpr int kItemCost = 2;

// mbar_wait in few instructions: the roles wait in some thirty places, and what they
// do in between has to stay in the instruction caches.
__device__ __forceinline__ bool wait8(uint64_t* bar, uint32_t parity, const uint64_t& limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
#pragma unroll 1
  do {
    if (mbar_try_wait(bar, parity)) return true;
  } while (global_ns() - t0 <= limit_ns);
  return false;
}

struct Tree8Args {
  CUtensorMap kc, vc;
  TreeArgs a;
  TreeScales sc;
  float scale2;       // scale * log2(e)
  int group;          // G
  int ctas;           // of the launch
  int box;            // slots of one copy: they lie within a page
  int slots_inner;    // the cache maps' second dimension is the slot, the third the head
  // pieces: CTA c leaves that of an item that began before its tiles at 2 c, that
  // of one that begins in them at 2 c + 1
  float* part;        // [2 ctas * kRows * D] outputs, not normalised
  float2* part_ml;    // [2 ctas * kRows] their reference maximum (log2) and sum
  int32_t* first;     // [B + 1] places before each request's, then the places per CTA
  int32_t* stop;      // [ctas] the place from which a CTA gave up, INT32_MAX if it did not
  uint64_t wait_ns;   // limit of a wait
  int stall;          // the CTA whose copies a test withholds from its second tile on, or -1
};

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

// Rows of a request and key head are (token, query head of the group), in order; an
// item is R of them. The tiles that its rows see: the cache's, then those of drafted
// tokens up to its last row's.
__host__ __device__ inline int cache_tiles(int len) { return len / kTile + (len % kTile != 0); }
__host__ __device__ inline int tree_tiles(int end) { return (end + kTile - 1) / kTile; }
__host__ __device__ inline int items(int nodes, int group) {
  return (nodes * group + kRows - 1) / kRows;
}
__device__ __forceinline__ int item_end(const Request& r, int group, int mt) {  // its last token + 1
  return (min(r.nodes * group, (mt + 1) * kRows) - 1) / group + 1;
}
__device__ __forceinline__ int item_tiles(const Request& r, int group, int mt) {
  return cache_tiles(r.len) + tree_tiles(item_end(r, group, mt));
}
// The places that one key head of a request takes in the list.
__device__ __noinline__ int head_places(const Request r, int group) {
  const int n = items(r.nodes, group);
  int sum = n * (kItemCost + cache_tiles(r.len));
#pragma unroll 1
  for (int mt = 0; mt < n; ++mt) sum += tree_tiles(item_end(r, group, mt));
  return sum;
}
// An item of the list, the first of its tiles that is left, and the places before it.
// (Finding it and stepping on are calls: each role does it, and inlined in all of them
// they made 180 KB of code, whose misses cost more than the work; with them and the
// slow side of a wait apart it is TODO.)
struct Place {
  int b, hk, mt, tile, lead;
  Request r;
};
__device__ __noinline__ Place find_place(const TreeArgs& a, int group, int request_b, int offset) {
  Place x;
  x.b = request_b;
  x.r = request(a, request_b);
  const int per_head = head_places(x.r, group);
  x.hk = offset / per_head;
  offset %= per_head;
  x.mt = 0;
#pragma unroll 1
  for (int n; offset >= (n = kItemCost + item_tiles(x.r, group, x.mt)); ++x.mt) offset -= n;
  x.tile = max(0, offset - kItemCost);
  x.lead = max(0, kItemCost - offset);
  return x;
}
__device__ __noinline__ Place next_place(const TreeArgs& a, int group, Place x) {
  x.tile = 0;
  x.lead = kItemCost;
  if (++x.mt * kRows < x.r.nodes * group) return x;
  x.mt = 0;
  if (++x.hk < a.Hkv) return x;
  x.hk = 0;
#pragma unroll 1
  do {
    if (++x.b >= a.B) return x;
    x.r = request(a, x.b);
  } while (x.r.nodes == 0);
  return x;
}
// The part of an item that a CTA takes: tiles of drafted tokens, which have to come from
// further away, first, then the cache's.
struct Item {
  int n_tree, rows, tile0, tile1, end;
  __device__ __forceinline__ Item(const Tree8Args& p, const Place& x, int todo) {
    rows = min(kRows, x.r.nodes * p.group - x.mt * kRows);
    end = item_end(x.r, p.group, x.mt);
    n_tree = tree_tiles(end);
    tile0 = x.tile;
    tile1 = min(n_tree + cache_tiles(x.r.len), x.tile + todo);
  }
};
// Keys in use of tile j of an item.
__device__ __forceinline__ int tile_keys(int j, int n_tree, int end, int len) {
  return min(kTile, j < n_tree ? end - j * kTile : len - (j - n_tree) * kTile);
}
// What the converting warps, which come to an item first, tell the others of it.
struct Facts {
  int n_tree, rows, tile0, tile1, end, len, first, hk, row0, at;  // at: the place of its first tile
};

// Whether every parent and page of the request is in range (the row threads).
__device__ __noinline__ bool out_of_range(const TreeArgs& a, int b, const Request r, int t, int threads) {
  bool bad = false;
  if (a.parents)
#pragma unroll 1
    for (int i = t; i < r.nodes; i += threads) {
      const int p = a.parents[r.first + i];
      bad |= p < -1 || p >= i;
    }
  const int pages = r.len / a.page_size + (r.len % a.page_size != 0);
#pragma unroll 1
  for (int x = t; x < pages; x += threads) {
    const int p = a.page_table[b * a.table_stride + x];
    bad |= p < 0 || p >= a.n_pages;
  }
  return bad;
}

template <int D, bool F16>
struct Smem8 {
  static constexpr int kPieces = F16 ? 3 : 2;  // of queries
  // Tensor memory: scores of two tiles, weights of two (a column holds two keys'), the output.
  static constexpr int kWeights = 2 * kTile, kOut = 3 * kTile, kColumns = 512;
  // what 227 KB hold
  static constexpr int kStagesK = D == 64 ? 5 : F16 ? 2 : 3, kStagesV = D == 64 ? 5 : 2;
  char w[2][kTile * D * 2];           // values of 16 bits; a drafted tile's keys too
  char q16[kRows * D * 2];            // queries for drafted keys,
  char q8[kPieces * kRows * D];       // and in pieces for the cache's
  char k[kStagesK][kTile * D];        // keys and values as they come
  char v[kStagesV][kTile * D];
  uint32_t seen[kRows][kWords];       // a token's ancestors and itself
  // of this item and the next one
  float factor[2][kRows];             // a row's pieces times it and a key's scale: log2 scores
  uint32_t odd[2][kWords];            // drafted tokens with a value that is not finite
  Facts facts[2];
  // of the tiles under way
  alignas(16) float k_scale[kScaleRing][kGroups];
  uint32_t v_scale[kScaleRing][kGroups];  // two fp16 numbers, of the tile's unit
  uint32_t left_out[2][kScaleRing];   // groups whose page is out of range: keys, values
  int unit[kScaleRing];               // largest scale of the item's values so far
  float half[2][2][kRows];            // what the two threads of a row tell each other
  uint64_t k_full[kStagesK], k_empty[kStagesK], v_full[kStagesV], v_empty[kStagesV];
  uint64_t scale_full[kScaleRing], w_full[2], w_empty[2], s_full[2], s_free[2];
  uint64_t p_full[2], o_done[2], item_full[2], o_free[2], seen_free, q_full, q_empty, own_full,
      drained[2];
  long long sums[kThreads / 32];      // places of the requests, by warps
  int start_b, start_offset;          // where this CTA's places begin
  int share;                          // and how many a CTA has
  uint32_t tmem;
  int end, stop;                      // the place behind this CTA's, and where it gave up
};

// D[tmem] (+)= A[smem] B[smem] over 32 of K, both e4m3.
__device__ __forceinline__ void umma8_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(uint32_t(add))
      : "memory");
}
// Operand of e4m3 elements in rows of D bytes along K, swizzled by as many.
template <int D>
__device__ __forceinline__ uint64_t umma8_desc(uint32_t addr) {
  return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(1) << 16 | uint64_t(8 * D >> 4) << 32 | uint64_t(1) << 46 |
         uint64_t(D == 128 ? 2 : 4) << 61;
}
// Byte `at` of row r of such an operand.
template <int D>
__device__ __forceinline__ int swizzled8(int r, int at) {
  return r * D + (at ^ (D == 128 ? (r & 7) << 4 : (r >> 1 & 3) << 4));
}
// 16-byte unit u of row r in 128-byte swizzled rows.
__device__ __forceinline__ int swizzled16(int r, int u) { return r * 128 + ((u ^ (r & 7)) << 4); }
// Instruction descriptor: fp32 accumulators, M = 128, N columns, e4m3 operands.
__device__ __forceinline__ uint32_t idesc_e4m3(int n) {
  return 1u << 4 | uint32_t(n >> 3) << 17 | uint32_t(128 >> 4) << 24;
}
// Whether any of `threads` threads says so; all of them come to the barrier.
__device__ __forceinline__ bool any_of(int barrier, int threads, bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %3, 0;\n\t"
      "bar.red.or.pred p, %1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(barrier), "r"(threads), "r"(uint32_t(x))
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void sync_of(int barrier, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
}
// -inf in place of the scores whose bit is not set.
__device__ __forceinline__ void hide(uint32_t (&v)[32], uint32_t see) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (!(see >> i & 1)) v[i] = 0xff800000u;
}
// A product that may have become too small for a number, which -inf may be multiplied
// by; NaN stays.
__device__ __forceinline__ float not_zero(float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(0x1p-120f));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
// What drafted tokens with a value that is not finite add to elements d .. d + 31 of token
// i's row: it walks up from there.
template <int DT>
__device__ __noinline__ void odd_values(const TreeArgs& a, const uint32_t* odd, int first, int i, int hk,
                                        int d, float (&sum)[32]) {
#pragma unroll 1
  for (int e = 0; e < 32; ++e) sum[e] = 0.f;
#pragma unroll 1
  for (int up; i >= 0; i = up) {
    up = a.parents ? a.parents[first + i] : i - 1;
    if (up < -1 || up >= i) up = -1;
    if (!(odd[i >> 5] >> (i & 31) & 1)) continue;
#pragma unroll 1
    for (int e = 0; e < 32; ++e) {
      const float z = load_elem<DT>(a.v + ((int64_t(first) + i) * a.v_token + hk * a.v_head + d + e) * 2);
      if (!(fabsf(z) < INFINITY)) sum[e] += z;
    }
  }
}
// 2^-k as two fp16 numbers, k >= 0.
__device__ __forceinline__ uint32_t half_power(int k) {
  const uint32_t x = k <= 14 ? uint32_t(15 - k) << 10 : k <= 24 ? 1u << (24 - k) : 0u;
  return x | x << 16;
}
__device__ __forceinline__ uint32_t half_mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// 32 bytes to memory: one store where they are known to start on 32 bytes (pieces), two
// of 16 for the caller's output.
template <bool TWO>
__device__ __forceinline__ void store_sector(char* to, const uint32_t (&o)[8]) {
  if constexpr (TWO) {
    reinterpret_cast<uint4*>(to)[0] = make_uint4(o[0], o[1], o[2], o[3]);
    reinterpret_cast<uint4*>(to)[1] = make_uint4(o[4], o[5], o[6], o[7]);
  } else {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(o[0]),
                 "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                 : "memory");
  }
}

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1) tree8_kernel(const __grid_constant__ Tree8Args p) {
  using S = Smem8<D, F16>;
  constexpr int DT = F16 ? TT_F16 : TT_BF16;
  constexpr int kPieces = S::kPieces;
  // Drafted values have no scale, 2^0, which their weights in the inputs' type take: fp16
  // holds them beside scales of 2^0 or more, bf16 beside any that are not below 2^-60.
  constexpr int kOwnCode = F16 ? 127 : 67;
  constexpr int kBlock = kTile * 128;         // distance of the 64-element blocks of a 16-bit tile
  constexpr float kOffset = 7.f;              // fp16 weights: away from its small end
  extern __shared__ char raw[];
  S& s = *reinterpret_cast<S*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
  const TreeArgs& a = p.a;
  // (a number that is the same in all lanes, and known to be)
  const int t = threadIdx.x, warp = __shfl_sync(0xffffffffu, t >> 5, 0), lane = t & 31;
  const uint64_t& limit = p.wait_ns;
  grid_launch_dependents();

  if (t == kRowThreads) {
    for (int i = 0; i < S::kStagesK; ++i) {
      mbar_init(&s.k_full[i], 1);
      mbar_init(&s.k_empty[i], 1);
    }
    for (int i = 0; i < S::kStagesV; ++i) {
      mbar_init(&s.v_full[i], 1);
      mbar_init(&s.v_empty[i], kConvThreads);
    }
    for (int i = 0; i < kScaleRing; ++i) mbar_init(&s.scale_full[i], 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.w_full[i], kConvThreads);
      mbar_init(&s.w_empty[i], 1);
      mbar_init(&s.s_full[i], 1);
      mbar_init(&s.s_free[i], kRowThreads);
      mbar_init(&s.p_full[i], kRowThreads);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.item_full[i], kConvThreads);
      mbar_init(&s.o_free[i], kRowThreads);
    }
    mbar_init(&s.q_full, kConvThreads);
    mbar_init(&s.q_empty, 1);
    mbar_init(&s.own_full, kConvThreads);
    mbar_init(&s.seen_free, kRowThreads);
    mbar_init(&s.drained[0], 1);
    mbar_init(&s.drained[1], 1);
    s.stop = INT32_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kRowWarps + kConvWarps) tmem_alloc(&s.tmem, S::kColumns);
  // The list: each thread adds up a run of requests, and the one whose run holds
  // this CTA's first place tells the request.
  int todo;
  {
    const int each = (a.B + kThreads - 1) / kThreads, b0 = min(a.B, t * each),
              b1 = min(a.B, b0 + each);
    long long mine = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) mine += (long long)(head_places(request(a, b), p.group)) * a.Hkv;
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) s.sums[warp] = upto;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    long long all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) upto += s.sums[w];
      all += s.sums[w];
    }
    const long long share = max((long long)(kMinShare), (all + p.ctas - 1) / p.ctas);
    const long long from = share * blockIdx.x;
    todo = int(max(0ll, min(share, all - from)));
    if (t == 0) {
      s.share = int(share);
      s.end = int(min(all, from + share));
    }
    long long at = upto - mine;
    if (todo > 0 && from >= at && from < upto) {
#pragma unroll 1
      for (int b = b0; b < b1; ++b) {
        const long long n = (long long)(head_places(request(a, b), p.group)) * a.Hkv;
        if (from < at + n) {
          s.start_b = b;
          s.start_offset = int(from - at);
          break;
        }
        at += n;
      }
    }
    if (blockIdx.x == 0) {  // for the join
      at = upto - mine;
#pragma unroll 1
      for (int b = b0; b < b1; ++b) {
        p.first[b] = int(at);
        at += (long long)(head_places(request(a, b), p.group)) * a.Hkv;
      }
      if (t == 0) p.first[a.B] = int(share);
    }
  }
  __syncthreads();
  const uint32_t tmem = s.tmem;
  bool ok = true;
  Place x;
  x.lead = 0;
  if (todo > 0 && warp >= kRowWarps) x = find_place(p.a, p.group, s.start_b, s.start_offset);

  if (warp > kRowWarps + kConvWarps + 1) {
    // ------------------------------------------------------------ copies
    // One warp for keys, one for values. Pages of four tiles are asked for at once, two
    // batches ahead, and their scales one: lane 8 k + g has to do with the g-th 16 slots of
    // a batch's k-th tile. It reads their scale, and copies the box that begins with them.
    const bool values = warp != kRowWarps + kConvWarps + 2;
    const TreeScale& sc = values ? p.sc.v : p.sc.k;
    char* const dst = values ? &s.v[0][0] : &s.k[0][0];
    uint64_t* const full = values ? s.v_full : s.k_full;
    uint64_t* const empty = values ? s.v_empty : s.k_empty;
    const int stages = values ? S::kStagesV : S::kStagesK;
    const CUtensorMap* const map = values ? &p.vc : &p.kc;
    struct Batch {
      int hk, page, in_page;  // of the lane's slots
      int tiles;              // 0: no more
      int unit;               // of values, where an item begins, else -1
      uint32_t code;
    };
    int j = 0, j1 = 0, used = 0;
    bool open = false;
    auto next = [&]() {
      Batch y{0, -1, 0, 0, -1, 0};
      for (;;) {
        if (!open) {
          if (todo <= x.lead) return y;
          todo -= x.lead;
          const Item it(p, x, todo);
          j = max(0, it.tile0 - it.n_tree);
          j1 = it.tile1 - it.n_tree;
          used = it.tile1 - it.tile0;
          y.unit = it.tile0 < it.n_tree ? kOwnCode : 1;
          open = true;
        }
        if (j < j1) break;
        todo -= used;
        x = next_place(p.a, p.group, x);
        open = false;
      }
      y.tiles = min(kBatch, j1 - j);
      y.hk = x.hk;
      const int slot = j * kTile + lane * TT_SCALE_SLOTS;
      y.in_page = slot % a.page_size;
      if (lane < y.tiles * kGroups && slot < x.r.len)
        y.page = a.page_table[x.b * a.table_stride + slot / a.page_size];
      j += y.tiles;
      return y;
    };
    auto usable = [&](int page) { return page >= 0 && page < a.n_pages; };
    Batch one, two;
    one.tiles = two.tiles = 0;
    int n = 0, st = 0, unit = 1;
    uint32_t parity = 1;
#pragma unroll 1
    for (int k = 0; ok && (k < 2 || one.tiles); ++k) {
      const Batch c = one;
      one = two;
      const bool mine = c.tiles && usable(c.page), then = one.tiles && usable(one.page);
      if (then)
        one.code = sc.data[one.page * sc.page + (one.in_page / TT_SCALE_SLOTS) * sc.group +
                           one.hk * sc.head];
      two = next();
      if (!c.tiles) continue;
      const bool begins = mine && lane % kGroups * TT_SCALE_SLOTS % p.box == 0;
      const unsigned int lost = __ballot_sync(0xffffffffu, !mine);
      const unsigned int boxes = __ballot_sync(0xffffffffu, begins);
      if (c.unit > 0) unit = c.unit;
      int top = c.code != 255 ? int(c.code) : 0;
#pragma unroll
      for (int o = 1; o < kGroups; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int at1 = p.slots_inner ? c.in_page : c.hk, at2 = p.slots_inner ? c.hk : c.in_page;
#pragma unroll 1
      for (int i = 0; i < c.tiles; ++i) {
        ok = __all_sync(0xffffffffu, wait8(&empty[st], parity, limit)) &&
             (n != 1 || int(blockIdx.x) != p.stall);
        if (!ok) break;
        // (The scales in this place are of kScaleRing tiles ago, which is further back than
        // the stages and the tiles on their way behind them reach.)
        const int ring = n % kScaleRing;
        unit = max(unit, __shfl_sync(0xffffffffu, top, kGroups * i));
        if (lane / kGroups == i) {
          if (values)
            s.v_scale[ring][lane % kGroups] = c.code == 255 ? 0x7e007e00u : half_power(unit - int(c.code));
          else
            s.k_scale[ring][lane % kGroups] = e8m0(c.code);
        }
        if (lane == 0) {
          s.left_out[values][ring] = lost >> (kGroups * i) & 0xff;
          if (values) s.unit[ring] = unit;
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_expect_tx(&full[st], __popc(boxes >> (kGroups * i) & 0xff) * p.box * D);
          mbar_arrive(&s.scale_full[ring]);
        }
        __syncwarp();
        if (begins && lane / kGroups == i)
          tma_load_4d(smem_u32(dst) + st * (kTile * D) + lane % kGroups * TT_SCALE_SLOTS * D, map,
                      smem_u32(&full[st]), 0, at1, at2, c.page);
        ++n;
        if (++st == stages) {
          st = 0;
          parity ^= 1;
        }
      }
    }
    // (the CTA's memory stays until its last copies have come)
#pragma unroll 1
    for (int i = 0; i < stages; ++i)
      if (n > i) wait8(&full[i], ((n - 1 - i) / stages) & 1, limit);
  } else if (warp >= kRowWarps + kConvWarps) {
    // ---------------------------------------------------------- products
    // One warp issues those that give scores, one those with values. (Warps go along as a
    // whole, one lane issues: operands then are uniform registers.)
    auto on = [&](uint64_t* bar, uint32_t parity) {
      return __all_sync(0xffffffffu, wait8(bar, parity, limit)) != 0;
    };
    constexpr uint32_t kWStep = kTile * D * 2 / 16, kKStep = kTile * D / 16;
    int n = 0, w = 0;  // tiles, 16-bit operands
    if (warp == kRowWarps + kConvWarps) {
      const uint64_t kd = umma8_desc<D>(smem_u32(s.k)), qd = umma8_desc<D>(smem_u32(s.q8)),
                     od = umma_desc(smem_u32(s.q16), 16), wk = umma_desc(smem_u32(s.w), 16);
      int turn = 0, st = 0, drafted = 0;
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(p, x, todo);
        ok = on(&s.q_full, seg & 1);
#pragma unroll 1
        for (int j = it.tile0; j < it.tile1 && ok; ++j, ++n, ++w) {
          const int buf = n & 1;
          const uint32_t to = tmem + buf * kTile;
          if (j >= it.n_tree) {
            ok = on(&s.k_full[st], turn & 1) && on(&s.s_free[buf], ((n >> 1) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int q = 0; q < kPieces; ++q)
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
                  umma8_ss(to, qd + q * (kRows * D / 16) + 2 * c, kd + st * kKStep + 2 * c,
                           idesc_e4m3(kTile), q > 0 || c > 0);
              umma_commit(&s.s_full[buf]);
              umma_commit(&s.k_empty[st]);
              if (j + 1 == it.tile1) umma_commit(&s.q_empty);
            }
            if (++st == S::kStagesK) {
              st = 0;
              ++turn;
            }
          } else {
            // (a barrier of their own: on w_full's, this warp could be two phases ahead, where
            // a parity says nothing)
            ok = on(&s.own_full, drafted++ & 1) && on(&s.s_free[buf], ((n >> 1) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int c = 0; c < D / 16; ++c)
                umma_ss(to, od + (c / 4) * (kBlock / 16) + (c % 4) * 2,
                        wk + (w & 1) * kWStep + (c / 4) * (kBlock / 16) + (c % 4) * 2,
                        umma_idesc(F16, kTile, false), c > 0);
              umma_commit(&s.s_full[buf]);
              umma_commit(&s.w_empty[w & 1]);
              if (j + 1 == it.tile1) umma_commit(&s.q_empty);
            }
            ++w;  // (behind its keys, its values)
          }
          __syncwarp();
        }
        todo -= it.tile1 - it.tile0;
        x = next_place(p.a, p.group, x);
      }
    } else {
      const uint64_t wv = umma_desc(smem_u32(s.w), kBlock);
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(p, x, todo);
#pragma unroll 1
        for (int j = it.tile0; j < it.tile1 && ok; ++j, ++n, ++w) {
          if (j < it.n_tree) ++w;
          const int keys = tile_keys(j, it.n_tree, it.end, x.r.len), buf = n & 1;
          ok = on(&s.w_full[w & 1], (w >> 1) & 1) && on(&s.p_full[buf], (n >> 1) & 1) &&
               (j > it.tile0 || seg == 0 || on(&s.o_free[(seg - 1) & 1], ((seg - 1) >> 1) & 1));
          if (!ok) break;
          tc_fence_after();
          const uint32_t idesc = umma_idesc(F16 || j >= it.n_tree, D, true);
          const uint32_t weights = tmem + S::kWeights + buf * (kTile / 2);
          const bool more = j > it.tile0;
          if (elect_one()) {
#pragma unroll
            for (int c = 0; c < kTile / 16; ++c)
              if (16 * c < keys)
                umma_ts(tmem + S::kOut, weights + 8 * c, wv + (w & 1) * kWStep + 128 * c, idesc,
                        more || c > 0);
            umma_commit(&s.o_done[buf]);
            umma_commit(&s.w_empty[w & 1]);
          }
          __syncwarp();
        }
        todo -= it.tile1 - it.tile0;
        x = next_place(p.a, p.group, x);
      }
    }
    // (and until their last products and the arrivals for them are done)
    uint64_t* const drained = &s.drained[warp - kRowWarps - kConvWarps];
    if (elect_one()) umma_commit(drained);
    __syncwarp();
    on(drained, 0);
  } else if (warp >= kRowWarps) {
    // -------------------------------------------------- queries and values
    const int ct = t - kRowThreads;
    auto wait_for = [&](uint64_t* bar, uint32_t parity) {
      if (ok) ok = __all_sync(0xffffffffu, wait8(bar, parity, limit));
      return ok;
    };
    int vt = 0, st = 0, w = 0, seg = 0, drafted = 0;
    uint32_t parity = 0;
#pragma unroll 1
    for (; todo > x.lead && ok; ++seg) {
      todo -= x.lead;
      const Item it(p, x, todo);
      const int side = seg & 1, row0 = x.mt * kRows, token0 = row0 / p.group;
      // (the item before the last one is over)
      if (!wait_for(&s.o_free[side], ((seg >> 1) & 1) ^ 1)) break;
      // Its facts, and a token's ancestors: one thread walks up from each token.
      if (ct == 0)
        s.facts[side] = Facts{it.n_tree, it.rows, it.tile0, it.tile1, it.end,
                              x.r.len,   x.r.first, x.hk,   row0,     s.end - todo};
      if (ct < kWords) s.odd[side][ct] = 0;
      if (it.tile0 < it.n_tree) {
        // (the parents in the place of the values to come, the ancestors once rows are done
        // with the last ones)
        if (!wait_for(&s.w_empty[w & 1], ((w >> 1) & 1) ^ 1) ||
            !wait_for(&s.seen_free, (drafted++ & 1) ^ 1))
          break;
        int16_t* const ups = reinterpret_cast<int16_t*>(s.w[w & 1]);
#pragma unroll 1
        for (int i = ct; i < it.end; i += kConvThreads) {
          const int up = a.parents ? a.parents[x.r.first + i] : i - 1;
          ups[i] = int16_t(up < -1 || up >= i ? -1 : up);
        }
        sync_of(6, kConvThreads);
        if (ct < it.end - token0) {
          const int words = it.n_tree * (kTile / 32);
#pragma unroll 1
          for (int k = 0; k < words; ++k) s.seen[ct][k] = 0;
#pragma unroll 1
          for (int i = token0 + ct; i >= 0; i = ups[i]) s.seen[ct][i >> 5] |= 1u << (i & 31);
        }
        sync_of(6, kConvThreads);
      }
      // Queries: a thread to a row.
      {
        const int row = row0 + ct, token = row / p.group, head = x.hk * p.group + row % p.group;
        const bool valid = ct < it.rows;
        const uint4* from = reinterpret_cast<const uint4*>(
            a.q + ((int64_t(x.r.first) + token) * a.q_token + int64_t(head) * a.q_head) * 2);
        float top = 0.f;
#pragma unroll 4
        for (int u = 0; u < D / 8; ++u) {
          float e[8];
          unpack16<DT>(valid ? from[u] : make_uint4(0, 0, 0, 0), e);
#pragma unroll
          for (int k = 0; k < 8; ++k) top = fabsf(e[k]) < INFINITY ? fmaxf(top, fabsf(e[k])) : top;
        }
        const uint32_t code = e8m0_for(top);
        const float inverse = e8m0_inverse(code);
        if (!wait_for(&s.q_empty, (seg & 1) ^ 1)) break;
        s.factor[side][ct] = p.scale2 * e8m0(code);
#pragma unroll 2
        for (int u = 0; u < D / 8; ++u) {  // (read again: from L1 or L2)
          const uint4 q = valid ? from[u] : make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(s.q16 + (u / 8) * kBlock + swizzled16(ct, u % 8)) = q;
          float e[8];
          unpack16<DT>(q, e);
#pragma unroll
          for (int k = 0; k < 8; ++k)  // (what is not finite has no pieces but NaN)
            e[k] = fabsf(e[k]) < INFINITY ? e[k] * inverse : __uint_as_float(0x7fc00000u);
#pragma unroll
          for (int piece = 0; piece < kPieces; ++piece) {
            uint32_t two[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              two[k] = to_e4m3x2(e[2 * k], e[2 * k + 1]);
              const uint32_t half = e4m3x2_to_f16x2(two[k]);
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&half));
              e[2 * k] -= f.x;
              e[2 * k + 1] -= f.y;
            }
            *reinterpret_cast<uint2*>(s.q8 + swizzled8<D>(piece * kRows + ct, u * 8)) =
                make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
          }
        }
        fence_proxy_async();
        mbar_arrive(&s.q_full);
        mbar_arrive(&s.item_full[side]);
      }
      for (int j = it.tile0; j < it.tile1 && ok; ++j) {
        const int keys = tile_keys(j, it.n_tree, it.end, x.r.len);
        const int steps = (keys + 15) / 16;  // (others are not multiplied)
        constexpr int kUnits = D / 8;  // of 8 elements, of a key
        if (j >= it.n_tree) {
          const int ring = vt % kScaleRing;
          if (!wait_for(&s.v_full[st], parity)) break;
          if (!wait_for(&s.w_empty[w & 1], ((w >> 1) & 1) ^ 1)) break;
          // (a thread takes 8 elements of either half of a key: stores of 16 bytes without
          // bank conflicts)
          const uint32_t lost = s.left_out[1][ring];
          constexpr int kPairs = D / 64, kEach = kTile * 8 / kConvThreads;
          const int u = ct % 8, key0 = ct / 8;  // (its keys are 16 apart)
          const char* const from = s.v[st] + key0 * D + u * 8;
          char* const to = s.w[w & 1] + swizzled16(key0, u);
          auto convert = [](const uint2& in, uint32_t scale) {
            return make_uint4(half_mul2(e4m3x2_to_f16x2(in.x & 0xffff), scale),
                              half_mul2(e4m3x2_to_f16x2(in.x >> 16), scale),
                              half_mul2(e4m3x2_to_f16x2(in.y & 0xffff), scale),
                              half_mul2(e4m3x2_to_f16x2(in.y >> 16), scale));
          };
          // (its k-th key is one of the k-th 16 slots)
          const uint32_t* const scales = s.v_scale[ring];
          if (keys == kTile && lost == 0) {
#pragma unroll
            for (int h = 0; h < kPairs; ++h) {
              uint2 in[kEach];
#pragma unroll
              for (int k = 0; k < kEach; ++k)
                in[k] = *reinterpret_cast<const uint2*>(from + k * 16 * D + h * 64);
#pragma unroll
              for (int k = 0; k < kEach; ++k)
                *reinterpret_cast<uint4*>(to + h * kBlock + k * 2048) = convert(in[k], scales[k]);
            }
          } else {
#pragma unroll 1
            for (int k = 0; k < kEach; ++k) {
              const int key = key0 + 16 * k;
              const bool there = key < keys && !(lost >> (key / TT_SCALE_SLOTS) & 1);
#pragma unroll
              for (int h = 0; h < kPairs; ++h) {
                uint2 in = make_uint2(0, 0);
                if (there) in = *reinterpret_cast<const uint2*>(from + k * 16 * D + h * 64);
                *reinterpret_cast<uint4*>(to + h * kBlock + k * 2048) = there ? convert(in, scales[k]) : make_uint4(0, 0, 0, 0);
              }
            }
          }
          mbar_arrive(&s.v_empty[st]);
          ++vt;
          if (++st == S::kStagesV) {
            st = 0;
            parity ^= 1;
          }
        } else {
          // Drafted tokens: keys as they are, then values without what is not finite (a
          // token outside its branch would get NaN from it; its own gets it at the end).
          const int base = j * kTile;
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            if (!wait_for(&s.w_empty[w & 1], ((w >> 1) & 1) ^ 1)) break;
            const char* from = kv ? a.v : a.k;
            const int64_t ts = kv ? a.v_token : a.k_token, hs = kv ? a.v_head : a.k_head;
#pragma unroll 1
            for (int i = ct; i < steps * 16 * kUnits; i += kConvThreads) {
              const int key = i / kUnits, u = i % kUnits;
              uint4 o = make_uint4(0, 0, 0, 0);
              if (key < keys) {
                o = *reinterpret_cast<const uint4*>(
                    from + ((int64_t(x.r.first) + base + key) * ts + x.hk * hs + u * 8) * 2);
                if (kv) {
                  constexpr uint32_t kExp = F16 ? 0x7c00 : 0x7f80;
                  bool odd = false;
#pragma unroll
                  for (int q = 0; q < 4; ++q) {
                    uint32_t y = q == 0 ? o.x : q == 1 ? o.y : q == 2 ? o.z : o.w;
                    if ((y & kExp) == kExp) {
                      y &= 0xffff0000u;
                      odd = true;
                    }
                    if ((y >> 16 & kExp) == kExp) {
                      y &= 0xffffu;
                      odd = true;
                    }
                    (q == 0 ? o.x : q == 1 ? o.y : q == 2 ? o.z : o.w) = y;
                  }
                  if (odd)
                    atomicOr(&s.odd[side][(base + key) >> 5], 1u << ((base + key) & 31));
                }
              }
              *reinterpret_cast<uint4*>(s.w[w & 1] + (u / 8) * kBlock + swizzled16(key, u % 8)) = o;
            }
            if (kv == 0) {
              fence_proxy_async();
              mbar_arrive(&s.w_full[w & 1]);
              mbar_arrive(&s.own_full);
              ++w;
            }
          }
          if (!ok) break;
        }
        fence_proxy_async();
        mbar_arrive(&s.w_full[w & 1]);
        ++w;
      }
      todo -= it.tile1 - it.tile0;
      x = next_place(p.a, p.group, x);
    }
    // (no more)
    if (ok && wait_for(&s.o_free[seg & 1], ((seg >> 1) & 1) ^ 1)) {
      if (ct == 0) s.facts[seg & 1].tile1 = -1;
      mbar_arrive(&s.item_full[seg & 1]);
    }
  } else {
    // -------------------------------------------------------------- rows
    // (while the first copies are on their way: the requests' statuses)
#pragma unroll 1
    for (int b = blockIdx.x; b < a.B; b += p.ctas) {
      const Request r = request(a, b);
      const bool bad = any_of(5, kRowThreads, !r.status && out_of_range(a, b, r, t, kRowThreads));
      if (t == 0) a.status[b] = r.status | (bad ? TT_REQ_ID_OUT_OF_RANGE : 0);
    }
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    const uint32_t mine = tmem + (uint32_t(quarter * 32) << 16);  // this warp's lanes
    const int c0 = 64 * half;                                     // its first key of a tile
    // tells the row's other thread x, and returns what that told (turn: of two)
    auto other = [&](float y, int turn) {
      s.half[turn][half][row] = y;
      sync_of(1 + quarter, 64);
      return s.half[turn][half ^ 1][row];
    };
    // A warp goes on, or gives up, as one. One that gave up passes the barriers between
    // the warps as often as the others until the item's end, where all give up, but waits
    // and arrives no more and writes nothing: so the others give up, too, and all end.
    int at_place = s.end - todo;
    auto wait_for = [&](uint64_t* bar, uint32_t parity) {
      if (!ok) return;
      ok = __all_sync(0xffffffffu, wait8(bar, parity, limit));
      if (!ok && lane == 0) atomicMin(&s.stop, at_place);
    };
    int n = 0, ct = 0;
#pragma unroll 1
    for (int seg = 0; todo > 0; ++seg) {
      const int side = seg & 1;
      wait_for(&s.item_full[side], (seg >> 1) & 1);
      if (any_of(5, kRowThreads, !ok)) break;
      const Facts it = s.facts[side];
      if (it.tile1 < 0) break;
      at_place = it.at;
      const bool valid = row < it.rows;
      const bool some = __any_sync(0xffffffffu, valid);  // (others only keep step)
      const int token = (it.row0 + row) / p.group, local = token - it.row0 / p.group;
      const float factor = s.factor[side][row];
      float m = -INFINITY, l = 0.f;  // the reference maximum (log2) and the sum
      int code = 0;                  // the output is in units of 2^(code - 127)
#pragma unroll 1
      for (int j = it.tile0; j < it.tile1; ++j, ++n) {
        const bool cache = j >= it.n_tree, first = j == it.tile0;
        const int keys = tile_keys(j, it.n_tree, it.end, it.len), e = ct % kScaleRing;
        float f[4];  // what makes a score of each 16 keys its log2
        int unit = kOwnCode;
        uint32_t lost = 0;
        if (cache) {
          wait_for(&s.scale_full[e], (ct / kScaleRing) & 1);
          const float4 scale = *reinterpret_cast<const float4*>(s.k_scale[e] + 4 * half);
          f[0] = not_zero(scale.x * factor);
          f[1] = not_zero(scale.y * factor);
          f[2] = not_zero(scale.z * factor);
          f[3] = not_zero(scale.w * factor);
          unit = s.unit[e];
          lost = s.left_out[0][e] >> (4 * half);
          ++ct;
        } else {
          f[0] = f[1] = f[2] = f[3] = p.scale2;
        }
        wait_for(&s.s_full[n & 1], (n >> 1) & 1);
        tc_fence_after();
        uint32_t v[2][32];
        float high = -INFINITY;
        if (some) {
#pragma unroll
          for (int h = 0; h < 2; ++h) tmem_ld32(mine + (n & 1) * kTile + c0 + 32 * h, v[h]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            tmem_wait_ld(v[h]);
            // which of 32 keys the row sees
            if (!cache || keys < kTile || lost) {
              const int left = keys - c0 - 32 * h;
              uint32_t see = left >= 32 ? 0xffffffffu : (1u << max(0, left)) - 1;
              if (lost >> (2 * h) & 1) see &= 0xffff0000u;
              if (lost >> (2 * h) & 2) see &= 0xffffu;
              if (!cache) see &= valid ? s.seen[local][(j * kTile + c0) / 32 + h] : 0u;
              hide(v[h], see);
              __syncwarp();
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              float top = __uint_as_float(v[h][16 * g]);
#pragma unroll
              for (int i = 1; i < 15; i += 2)
                top = max3(top, __uint_as_float(v[h][16 * g + i]), __uint_as_float(v[h][16 * g + i + 1]));
              top = fmaxf(top, __uint_as_float(v[h][16 * g + 15]));
              high = fmaxf(high, top * f[2 * h + g]);
            }
          }
        }
        tc_fence_before();
        if (ok) mbar_arrive(&s.s_free[n & 1]);
        // (all ancestors are read)
        if (j + 1 == min(it.n_tree, it.tile1) && ok) mbar_arrive(&s.seen_free);
        // what the values' scale makes of the sums, and a larger maximum of the row's
        float fall = 1.f;
        if (unit > code) {
          if (code > 0) fall = e8m0(code) * e8m0_inverse(unit);
          code = unit;
        }
        bool falls = fall != 1.f;
        if (some) {
          high = fmaxf(high, other(high, n & 1));
          if (high - m > kSlack || (m == -INFINITY && high > -INFINITY)) {
            const float to = fmaxf(m, high), less = m == -INFINITY ? 0.f : ex2_approx(m - to);
            m = to;
            l *= less;
            fall *= less;
          }
          falls = __any_sync(0xffffffffu, fall != 1.f);
          const float shift = (m == -INFINITY ? 0.f : -m) + kOffset;
          const f32x2 shift2 = pair(shift, shift);
          f32x2 sum2 = 0;
          auto weigh = [&](auto own) {
            const float value = e8m0_inverse(code);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float g = f[2 * h + i / 8];
                const f32x2 y = exp2_pair(
                    fma2(pair(__uint_as_float(v[h][2 * i]), __uint_as_float(v[h][2 * i + 1])), pair(g, g),
                         shift2));
                sum2 = add2(sum2, y);
                float lo, hi;
                split(y, lo, hi);
                if constexpr (decltype(own)::value)
                  v[h][i] = pack_pair<DT>(lo * value, hi * value);
                else
                  v[h][i] = pack_pair<TT_F16>(lo, hi);
              }
            }
          };
          if (cache)
            weigh(std::false_type());
          else
            weigh(std::true_type());
          l += sum_pair(sum2);
        }
        // (the product of two tiles ago is done with the weights' place)
        wait_for(&s.o_done[n & 1], ((n >> 1) & 1) ^ 1);
        tc_fence_after();
        if (some) {
          const uint32_t to = mine + S::kWeights + (n & 1) * (kTile / 2) + 32 * half;
#pragma unroll
          for (int h = 0; h < 2; ++h) tmem_st16(to + 16 * h, v[h]);
          if (falls && !first) {
            wait_for(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1);
            tc_fence_after();
#pragma unroll 1
            for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
              uint32_t o[32];
              tmem_ld32(mine + S::kOut + c, o);
              tmem_wait_ld(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fall);
              tmem_st32(mine + S::kOut + c, o);
            }
          }
          tmem_wait_st();
        }
        tc_fence_before();
        if (ok) mbar_arrive(&s.p_full[n & 1]);
      }
      bool odd = false;
      if (it.tile0 < it.n_tree) odd = lane < kWords && s.odd[side][lane];
      odd = __any_sync(0xffffffffu, odd);
      wait_for(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1);
      tc_fence_after();
      if (some) {
        l += other(l, n & 1);
        const bool whole = it.tile0 == 0 && it.tile1 == it.n_tree + cache_tiles(it.len);
        // where the row goes: to the output, or to its place in the CTA's piece
        const int64_t to = whole ? (int64_t(it.first) + token) * a.Hq + it.hk * p.group + it.row0 + row -
                                       token * p.group
                                 : (2 * int64_t(blockIdx.x) + (it.tile0 == 0)) * kRows + row;
        const float unit = e8m0(code);
        const float by = whole ? (l > 0.f || l != l ? unit / l : 0.f) : unit;
#pragma unroll 1
        for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
          uint32_t v[32];
          tmem_ld32(mine + S::kOut + c, v);
          tmem_wait_ld(v);
          if (valid && ok) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * by);
            if (odd) {
              float more[32];
              odd_values<DT>(a, s.odd[side], it.first, token, it.hk, c, more);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + more[i]);
            }
            if (whole) {
              char* out = a.out + (to * D + c) * 2;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint32_t o[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                  o[q] = pack_pair<DT>(__uint_as_float(v[16 * i + 2 * q]),
                                       __uint_as_float(v[16 * i + 2 * q + 1]));
                store_sector<true>(out + 32 * i, o);
              }
            } else {
              char* out = reinterpret_cast<char*>(p.part + to * D + c);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t o[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) o[q] = v[8 * i + q];
                store_sector<false>(out + 32 * i, o);
              }
            }
          }
          __syncwarp();
        }
        if (valid && ok && half == 0) {
          const float m2 = m == -INFINITY ? -INFINITY : m - kOffset;
          if (!whole)
            p.part_ml[to] = make_float2(m2, l);
          else if (a.lse)
            a.lse[to] = l > 0.f || l != l ? fmaf(m2, kLn2, logf(l)) : -INFINITY;
        }
      }
      tc_fence_before();
      if (ok) mbar_arrive(&s.o_free[side]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kRowWarps + kConvWarps) tmem_free(tmem, S::kColumns);
  if (t == 0) p.stop[blockIdx.x] = s.stop;  // (the join tells the requests)
}

// Joins the pieces of every row whose item was cut: with M the largest of their
// references, out = sum 2^(m - M) o / sum 2^(m - M) l. A CTA takes a row; its warps take
// the pieces in turn, the loads of eight before the first is added. It also tells the
// requests that lost places to a CTA that gave up.
constexpr int kJoinWarps = 4, kFewPieces = 16;

template <int D, bool F16, bool FEW>
__global__ void __launch_bounds__(kJoinWarps * 32)
    tree8_join_kernel(const __grid_constant__ Tree8Args p) {
  constexpr int DT = F16 ? TT_F16 : TT_BF16;
  constexpr int N = D / 32, W = FEW ? 1 : kJoinWarps;
  constexpr int C = FEW ? 4 : 8;  // pieces at once
  using Vec = typename std::conditional<N == 4, float4, float2>::type;
  __shared__ __align__(16) float s_acc[W][D];
  __shared__ float2 s_ml[W];
  const TreeArgs& a = p.a;
  const int warp = FEW ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned int at = FEW ? blockIdx.x * kJoinWarps + (threadIdx.x >> 5) : blockIdx.x;
  const int h = int(at % a.Hq), hk = h / p.group;
  const int i = int(at / a.Hq % a.max_nodes), b = int(at / a.Hq / a.max_nodes);
  if (b >= a.B) return;
  grid_dependency_wait();
  const int share = p.first[a.B], first = p.first[b];
  const Request r = request(a, b);
  if (i >= r.nodes) return;
  const int per_head = head_places(r, p.group);
  // (one warp of the request)
  if (i == 0 && h == 0 && (FEW || threadIdx.x < 32)) {
    const int end = first + per_head * a.Hkv - 1;  // its last place
    int stop = INT32_MAX;
    for (int c = first / share + lane; c <= end / share; c += 32) stop = min(stop, p.stop[c]);
    if (__any_sync(0xffffffffu, stop <= end) && lane == 0) a.status[b] |= TT_REQ_TIMEOUT;
  }
  const int row = i * p.group + h % p.group, mt = row / kRows;
  int before = hk * per_head + kItemCost;  // its first tile's place
  for (int k = 0; k < mt; ++k) before += kItemCost + item_tiles(r, p.group, k);
  const int last = before + item_tiles(r, p.group, mt) - 1;
  // the CTAs that the item lies in
  const int c0 = (first + before) / share, pieces = (first + last) / share - c0 + 1;
  if (pieces < 2) return;
  auto place = [&](int k) { return (2 * (int64_t(c0) + k) + (k == 0)) * kRows + row % kRows; };
  float M = -INFINITY, l = 0.f, acc[N];
#pragma unroll
  for (int c = 0; c < N; ++c) acc[c] = 0.f;
  auto add = [&](float l_more, const Vec& o, float f) {
    l = fmaf(l_more, f, l);
    acc[0] = fmaf(o.x, f, acc[0]);
    acc[1] = fmaf(o.y, f, acc[1]);
    if constexpr (N == 4) {
      acc[2] = fmaf(o.z, f, acc[2]);
      acc[3] = fmaf(o.w, f, acc[3]);
    }
  };
  for (int k0 = warp; k0 < pieces; k0 += W * C) {
    float2 ml[C];
    Vec o[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int64_t from = place(min(k0 + c * W, pieces - 1));
      ml[c] = p.part_ml[from];
      o[c] = reinterpret_cast<const Vec*>(p.part + from * D)[lane];
    }
    float top = M;
#pragma unroll
    for (int c = 0; c < C; ++c) top = fmaxf(top, ml[c].x);
    const float f = M == -INFINITY ? 0.f : ex2_approx(M - top);
    M = top;
    l *= f;
#pragma unroll
    for (int c = 0; c < N; ++c) acc[c] *= f;
    // (a piece without a reference: of NaN, or of nothing, which adds 0)
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (k0 + c * W < pieces)
        add(ml[c].y, o[c],
            ml[c].x == -INFINITY ? (ml[c].y != ml[c].y ? 1.f : 0.f) : ex2_approx(ml[c].x - top));
  }
  if constexpr (!FEW) {
#pragma unroll
    for (int c = 0; c < N; ++c) s_acc[warp][lane * N + c] = acc[c];
    if (lane == 0) s_ml[warp] = make_float2(M, l);
    __syncthreads();
    if (warp > 0) return;
    for (int w = 1; w < W; ++w) M = fmaxf(M, s_ml[w].x);
    l = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) acc[c] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = s_ml[w].x == -INFINITY ? (s_ml[w].y != s_ml[w].y ? 1.f : 0.f)
                                             : ex2_approx(s_ml[w].x - M);
      add(s_ml[w].y, reinterpret_cast<const Vec*>(s_acc[w])[lane], f);
    }
  }
  const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
  const int64_t to = (int64_t(r.first) + i) * a.Hq + h;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.out + to * D * 2) + lane * (N / 2);
  out[0] = pack_pair<DT>(acc[0] * inv, acc[1] * inv);
  if constexpr (N == 4) out[1] = pack_pair<DT>(acc[2] * inv, acc[3] * inv);
  if (a.lse && lane == 0) a.lse[to] = l > 0.f || l != l ? fmaf(M, kLn2, logf(l)) : -INFINITY;
}

// ------------------------------------------------------------------- host

// How a call is cut: CTAs, and the workspace.
struct Cut8 {
  int ctas;
  int64_t places;  // in the list, were all lengths the longest
  int64_t pieces;  // of one item, about
  size_t part_bytes, ml_bytes, first_bytes, bytes;
};
Cut8 cut8(const TreeArgs& a, int sm_count) {
  Cut8 c;
  const int group = a.Hq / a.Hkv;
  const int64_t rows = int64_t(a.max_nodes) * group;
  const int64_t row_tiles = (rows + kRows - 1) / kRows;
  const int64_t tiles = cache_tiles(a.max_len) + tree_tiles(a.max_nodes);  // of an item
  const int64_t all = c.places = int64_t(std::min(
      1e18, double(a.B) * double(a.Hkv) * double(row_tiles) * double(kItemCost + tiles)));
  c.ctas = int(std::max<int64_t>(
      1, std::min<int64_t>(sm_count, (all + kMinShare - 1) / kMinShare)));
  // (were all lengths the longest; fewer tiles make shares smaller and pieces more)
  const int64_t share = std::max<int64_t>(kMinShare, (all + c.ctas - 1) / c.ctas);
  c.pieces = tiles / share + 2;
  const size_t held = 2 * size_t(c.ctas) * kRows;
  c.part_bytes = align256(held * a.D * sizeof(float));
  c.ml_bytes = align256(held * sizeof(float2));
  c.first_bytes = align256((size_t(a.B) + 1) * sizeof(int32_t));
  c.bytes = c.part_bytes + c.ml_bytes + c.first_bytes + align256(c.ctas * sizeof(int32_t));
  return c;
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static std::atomic<void*> found{nullptr};
  void* f = found.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return nullptr;
    found.store(f, std::memory_order_release);
  }
  return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
}

// A map of a cache's bytes, in boxes of one head's elements of some slots. Dimensions by
// rising stride: heads within slots, or slots within heads.
bool encode(CUtensorMap* map, const TreeArgs& a, const char* data, int64_t page, int64_t slot,
            int64_t head, int box, bool slots_inner, CUtensorMapSwizzle swizzle) {
  const int64_t size[4] = {a.D, slots_inner ? a.page_size : a.Hkv, slots_inner ? a.Hkv : a.page_size,
                           a.n_pages};
  const int64_t stride[4] = {1, slots_inner ? slot : head, slots_inner ? head : slot, page};
  const cuuint32_t boxes[4] = {cuuint32_t(a.D), cuuint32_t(slots_inner ? box : 1),
                               cuuint32_t(slots_inner ? 1 : box), 1},
                   ones[4] = {1, 1, 1, 1};
  cuuint64_t dims[4], strides[3];
  for (int i = 0; i < 4; ++i) {
    dims[i] = cuuint64_t(size[i]);
    // (a dimension of one entry takes any valid stride)
    if (i > 0) strides[i - 1] = cuuint64_t(size[i] > 1 ? stride[i] : size[0]);
  }
  const auto f = encoder();
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<char*>(data), dims, strides, boxes,
                ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool F16>
cudaError_t launch(const Tree8Args& p, int64_t pieces, cudaStream_t stream) {
  const TreeArgs& a = p.a;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(p.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem8<D, F16>) + 1024;
  cfg.stream = stream;
  cudaError_t e = cudaLaunchKernelEx(&cfg, tree8_kernel<D, F16>, p);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  const bool few = pieces <= kFewPieces;
  const int64_t rows = int64_t(a.B) * a.max_nodes * a.Hq;
  cfg.gridDim = dim3(unsigned(few ? (rows + kJoinWarps - 1) / kJoinWarps : rows));
  cfg.blockDim = dim3(kJoinWarps * 32);
  cfg.dynamicSmemBytes = 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return few ? cudaLaunchKernelEx(&cfg, tree8_join_kernel<D, F16, true>, p)
             : cudaLaunchKernelEx(&cfg, tree8_join_kernel<D, F16, false>, p);
}

template <int D, bool F16>
cudaError_t preload() {
  cudaFuncAttributes fa;
  cudaError_t e = cudaFuncGetAttributes(&fa, tree8_join_kernel<D, F16, true>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, tree8_join_kernel<D, F16, false>);
  if (e != cudaSuccess) return e;
  static_assert(sizeof(Smem8<D, F16>) + 1024 <= 227 * 1024, "shared memory of a CTA");
  return cudaFuncSetAttribute(tree8_kernel<D, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(sizeof(Smem8<D, F16>)) + 1024);
}
}  // namespace

size_t tree8_workspace_bytes(const TreeArgs& a, int sm_count) { return cut8(a, sm_count).bytes; }

// (places of the list, and blocks of the join, are 32-bit numbers)
bool tree8_fits(const TreeArgs& a, int sm_count) {
  return cut8(a, sm_count).places <= INT32_MAX &&
         double(a.B) * a.max_nodes * double(a.Hq) <= INT32_MAX;
}

cudaError_t launch_tree8(const TreeArgs& a, const TreeScales& sc, int dt, cudaStream_t stream,
                         int sm_count) {
  const Cut8 c = cut8(a, sm_count);
  Tree8Args p;
  std::memset(&p, 0, sizeof p);
  p.a = a;
  p.sc = sc;
  p.scale2 = float(double(a.scale) * 1.4426950408889634);
  p.group = a.Hq / a.Hkv;
  p.ctas = c.ctas;
  p.box = std::gcd(a.page_size, kTile);
  p.part = reinterpret_cast<float*>(a.ws);
  p.part_ml = reinterpret_cast<float2*>(a.ws + c.part_bytes);
  p.first = reinterpret_cast<int32_t*>(a.ws + c.part_bytes + c.ml_bytes);
  p.stop = p.first + c.first_bytes / sizeof(int32_t);
  next_launch_stall(&p.stall, &p.wait_ns);
  if (a.max_len > 0) {
    // (one order for both, so that a copy's coordinates are the same)
    p.slots_inner = a.kc_slot < a.kc_head && a.page_size > 1 && a.Hkv > 1;
    if (!encode(&p.kc, a, a.kc, a.kc_page, a.kc_slot, a.kc_head, p.box, p.slots_inner,
                a.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode(&p.vc, a, a.vc, a.vc_page, a.vc_slot, a.vc_head, p.box, p.slots_inner,
                CU_TENSOR_MAP_SWIZZLE_NONE))
      return cudaErrorInvalidValue;
  }
  auto go = [&](auto dim, auto f16) {
    constexpr int D = decltype(dim)::value;
    constexpr bool F16 = decltype(f16)::value;
    return launch<D, F16>(p, c.pieces, stream);
  };
  auto of = [&](auto dim) { return dt == TT_F16 ? go(dim, std::true_type()) : go(dim, std::false_type()); };
  return a.D == 128 ? of(std::integral_constant<int, 128>()) : of(std::integral_constant<int, 64>());
}

cudaError_t preload_tree8() {
  cudaError_t e = preload<128, true>();
  if (e == cudaSuccess) e = preload<128, false>();
  if (e == cudaSuccess) e = preload<64, true>();
  if (e == cudaSuccess) e = preload<64, false>();
  return e;
}

}  // namespace tt
