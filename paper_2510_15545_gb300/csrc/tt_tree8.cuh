// tt_tree8.cuh -- what the kernels of tree8.cu and tree8_few.cu share: the list of tiles
// that the CTAs of a call take, and the instructions that both are made of.
#pragma once

#include <cuda.h>

#include <cstdint>

#include "tt_device.cuh"
#include "tt_e4m3.cuh"
#include "tt_f2.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"
#include "tt_rope.cuh"
#include "tt_umma.cuh"
#include "tt_x2.cuh"

namespace tt {

constexpr int kTile = 128;                     // keys of a tile
constexpr int kConvWarps = 4, kConvThreads = kConvWarps * 32;  // that convert values
constexpr int kManyRows = 128;                 // of an item of the kernel for many
constexpr int kWords = TT_MAX_TREE / 32;
constexpr int kOwnTiles = TT_MAX_TREE / kTile;  // of drafted tokens, of an item
constexpr int kGroups = kTile / TT_SCALE_SLOTS;  // scales of a tile
constexpr int kScaleRing = 16;                   // tiles' scales that are kept
constexpr int kBatch = 4;                        // tiles whose pages are asked for together
constexpr float kLn2 = 0.693147180559945f;
// A row's reference maximum follows its maximum once that is 2^kSlack above it:
// weights stay below 2^(kSlack + offset), and the output is scaled rarely.
constexpr float kSlack = 8.f;
constexpr int kMinShare = 2;  // places of a CTA, where there are few
// What an item costs beyond its tiles (queries, ancestors, output), in tiles: it
// takes as many places in the list before its first tile. (8500 cycles beside 1500 of a
// tile of single tokens; with 2 places those took 281 us, a serving batch 200, for 273 and
// 185; with 8 they took 271 and 185, but a single chain 17.7 for 16.6.)
constexpr int kItemCost = 5;

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
  int rows;           // R, of an item
  int ctas;           // of the launch
  int box;            // slots of one copy: they lie within a page
  int slots_inner;    // the cache maps' second dimension is the slot, the third the head
  // pieces: CTA c leaves that of an item that began before its tiles at 2 c, that
  // of one that begins in them at 2 c + 1
  float* part;        // [2 ctas * R * D] outputs, each over its piece's own sum (before that
                      // is taken out, means near the largest number would pass it)
  float2* part_ml;    // [2 ctas * R] their reference maximum (log2) and sum
  int32_t* first;     // [B + 2] a head's places before each request's, the places per CTA,
                      // the places of a head
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
// item is so many of them. The tiles that its rows see: those of drafted tokens up to its
// last row's, which have to come from further away, then the cache's.
__host__ __device__ inline int cache_tiles(int len) { return len / kTile + (len % kTile != 0); }
__host__ __device__ inline int tree_tiles(int end) { return (end + kTile - 1) / kTile; }
// How a call's requests are cut: query heads of a key head, rows of an item.
struct Shape {
  int group, rows;
  __device__ __forceinline__ int items(const Request& r) const {
    return (r.nodes * group + rows - 1) / rows;
  }
  __device__ __forceinline__ int end(const Request& r, int mt) const {  // its last token + 1
    return (min(r.nodes * group, (mt + 1) * rows) - 1) / group + 1;
  }
  __device__ __forceinline__ int tiles(const Request& r, int mt) const {
    return cache_tiles(r.len) + tree_tiles(end(r, mt));
  }
};
// The places that one key head of a request takes in the list.
static __device__ __noinline__ int head_places(const Request r, const Shape c) {
  const int n = c.items(r);
  int sum = n * (kItemCost + cache_tiles(r.len));
#pragma unroll 1
  for (int mt = 0; mt < n; ++mt) sum += tree_tiles(c.end(r, mt));
  return sum;
}
// The list has all requests' items of one key head, then those of the next one. The heads of
// a slot lie side by side in memory, mostly, and so CTAs that are at the same place of
// different heads read what is side by side at about the same time: with the heads of a
// request one after another memory gave 1.46 times what was needed, and single tokens of 256
// requests took 314 us for 273.
// An item of the list, the first of its tiles that is left, and the places before it.
// (Finding it and stepping on are calls: each role does it, and code beyond the instruction
// caches costs more than they do.)
struct Place {
  int b, hk, mt, tile, lead;
  Request r;
};
static __device__ __noinline__ Place find_place(const TreeArgs& a, const Shape c, int request_b, int hk,
                                                int offset) {
  Place x;
  x.b = request_b;
  x.hk = hk;
  x.r = request(a, request_b);
  x.mt = 0;
#pragma unroll 1
  for (int n; offset >= (n = kItemCost + c.tiles(x.r, x.mt)); ++x.mt) offset -= n;
  x.tile = max(0, offset - kItemCost);
  x.lead = max(0, kItemCost - offset);
  return x;
}
static __device__ __noinline__ Place next_place(const TreeArgs& a, const Shape c, Place x) {
  x.tile = 0;
  x.lead = kItemCost;
  if (++x.mt * c.rows < x.r.nodes * c.group) return x;
  x.mt = 0;
#pragma unroll 1
  do {
    if (++x.b >= a.B) {
      x.b = 0;
      if (++x.hk >= a.Hkv) return x;
    }
    x.r = request(a, x.b);
  } while (x.r.nodes == 0);
  return x;
}
// The part of an item that a CTA takes.
struct Item {
  int n_tree, rows, tile0, tile1, end;
  __device__ __forceinline__ Item(const Shape& c, const Place& x, int todo) {
    rows = min(c.rows, x.r.nodes * c.group - x.mt * c.rows);
    end = c.end(x.r, x.mt);
    n_tree = tree_tiles(end);
    tile0 = x.tile;
    tile1 = min(n_tree + cache_tiles(x.r.len), x.tile + todo);
  }
};
// Keys in use of tile j of an item.
__device__ __forceinline__ int tile_keys(int j, int n_tree, int end, int len) {
  return min(kTile, j < n_tree ? end - j * kTile : len - (j - n_tree) * kTile);
}

// Whether every parent and page of the request is in range (the row threads).
static __device__ __noinline__ bool out_of_range(const TreeArgs& a, int b, const Request r, int t, int threads) {
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
// The size of the largest of 8 elements that is finite, or `top`.
template <int DT>
__device__ __forceinline__ float largest(const uint4& q, float top) {
  float e[8];
  unpack16<DT>(q, e);
#pragma unroll
  for (int k = 0; k < 8; ++k) top = fabsf(e[k]) < INFINITY ? fmaxf(top, fabsf(e[k])) : top;
  return top;
}
// Values of the cache are fp16 numbers in units of 2^-kFiner of the largest scale so far: its
// own are up to 448 2^7 = 57344 then, and of scales down to 2^-31 of it every digit stays that
// is 2^-32 of it or more (in units of itself, values of scales from 2^-25 of it on, up to
// 448 2^-25, came to nothing).
constexpr int kFiner = 7;
constexpr int kLeastUnit = 67;  // (its byte) of sums that drafted values and the cache's share
// The unit (as a scale's byte) of sums that hold drafted values. Their weights have the
// inputs' type, and take it: fp16 holds them in units of 2^0, and the sums go to the cache's
// unit when its tiles begin; bf16 in any that are not below 2^-60. In that unit weights of up to 2^15 for 2^9 drafted tokens stay within
// fp32 with values below 2^43; larger ones need a unit of 2^-102 times their power of two. So
// the converting warps look at a drafted tile's values beside its keys: rows know the unit with
// the scores (single tokens 272 us for 266, a serving batch 185 for 180; with the rows waiting
// for the values that are fetched behind the keys, 295 and 195).
__host__ __device__ constexpr int own_code(bool f16) { return f16 ? 127 : kLeastUnit; }
// (of the bits of the largest, a bf16 number)
__device__ __forceinline__ int own_code_for(uint32_t top) { return int(top >> 7) - 102; }
// Where a tile of drafted tokens has larger ones: the unit that the finite ones of a
// converting thread's vectors of 8 need.
template <int D>
static __device__ __noinline__ void large_values(const TreeArgs& a, int first, int hk, int thread, int keys,
                                                 int* code) {
  constexpr int kUnits = D / 8;
  uint32_t top = 0;
#pragma unroll 1
  for (int i = thread; i < keys * kUnits; i += kConvThreads) {
    const uint16_t* y = reinterpret_cast<const uint16_t*>(a.v) + (int64_t(first) + i / kUnits) * a.v_token +
                        hk * a.v_head + i % kUnits * 8;
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
      const uint32_t size = y[e] & 0x7fffu;
      if (size < 0x7f80u) top = max(top, size);
    }
  }
  atomicMax(code, own_code_for(top));
}
// 8 elements times `by` as sums of e4m3 pieces, each what the ones before leave (of what is
// not finite NaN): put(piece, its 8 bytes).
template <int DT, int PIECES, class Put>
__device__ __forceinline__ void in_pieces(const uint4& q, float by, Put put) {
  float e[8];
  unpack16<DT>(q, e);
#pragma unroll
  for (int k = 0; k < 8; ++k)
    e[k] = fabsf(e[k]) < INFINITY ? e[k] * by : __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int piece = 0; piece < PIECES; ++piece) {
    uint32_t two[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      two[k] = to_e4m3x2(e[2 * k], e[2 * k + 1]);
      const uint32_t half = e4m3x2_to_f16x2(two[k]);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&half));
      e[2 * k] -= f.x;
      e[2 * k + 1] -= f.y;
    }
    put(piece, make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16));
  }
}
// 2^-k as two fp16 numbers, k >= -15; 0 where there is none, from k = 25 on.
__device__ __forceinline__ uint32_t half_power(int k) {
  const uint32_t x = k <= 14 ? uint32_t(15 - k) << 10 : k <= 24 ? 1u << (24 - k) : 0u;
  return x | x << 16;
}
__device__ __forceinline__ uint32_t half_mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// What a CTA finds of the list: it adds up the requests' places of one head, each thread those
// of a run of them, and the one whose run holds the CTA's first place tells the request.
// Returns the CTA's places. (Every thread comes; a barrier behind it makes s.start_* known.)
// (Places are numbers of 32 bits: calls of more are refused.)
template <int THREADS, class S>
__device__ __forceinline__ int begin_list(const Tree8Args& p, const Shape shape, S& s, int t, int warp, int lane) {
  const TreeArgs& a = p.a;
  const int each = (a.B + THREADS - 1) / THREADS, b0 = min(a.B, t * each),
            b1 = min(a.B, b0 + each);
  int mine = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) mine += head_places(request(a, b), shape);
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) s.sums[warp] = upto;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  int head = 0;  // the places of one
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) upto += s.sums[w];
    head += s.sums[w];
  }
  const int all = head * a.Hkv;
  const int share = max(kMinShare, all / p.ctas + (all % p.ctas != 0));
  const long long from = (long long)(share) * blockIdx.x;
  const int todo = int(max(0ll, min((long long)(share), all - from)));
  const int hk = todo > 0 ? int(from) / head : 0;
  if (t == 0) {
    s.share = share;
    s.end = int(min((long long)(all), from + share));
    s.start_hk = hk;
  }
  const int in_head = int(from) - hk * head;
  int at = upto - mine;
  if (todo > 0 && in_head >= at && in_head < upto) {
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const int n = head_places(request(a, b), shape);
      if (in_head < at + n) {
        s.start_b = b;
        s.start_offset = in_head - at;
        break;
      }
      at += n;
    }
  }
  if (blockIdx.x == 0) {  // for the join
    at = upto - mine;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      p.first[b] = at;
      at += head_places(request(a, b), shape);
    }
    if (t == 0) {
      p.first[a.B] = share;
      p.first[a.B + 1] = head;
    }
  }
  return todo;
}

cudaError_t launch_tree8_few(const Tree8Args& p, int dt, cudaStream_t stream);
cudaError_t preload_tree8_few();

}  // namespace tt
