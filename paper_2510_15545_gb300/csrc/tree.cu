// tree.cu -- attention of the drafted tokens of every request over its paged
// cache and, within its tree of drafted tokens, over each token's ancestors.
//
// Token i of request b sees the L_b keys of the request's cache, its ancestors
// i, parent(i), parent(parent(i)), ... and nothing else; its output in a head is
// sum_x softmax_x(scale q.k_x) v_x over them, held in the running form: with
// m = max s_x and l = sum 2^(s_x - m), a larger m scales what was summed before.
//
// The bound is the cache: each key and value is read once for all tokens and all
// query heads that share its head, G = Hq / Hkv. Their products are matrix
// products: 128 rows (token, head of the group) against tiles of 128 keys. A CTA
// takes the rows of one request and key head (more than 128: several CTAs read
// the tiles through L2) over a run of tiles, the request's cache first, then its
// own drafted tokens, on which each row's ancestors are a bit mask. One warp
// copies tiles in (a page at a time), one issues the two products per tile, and
// eight hold the rows: scores come from tensor memory, the weights go
// back over them in the inputs' type as the second product's operand. Two CTAs
// share an SM, so that one's softmax runs beside the other's products and copies.
// A tile's way from scores to weights is mostly waiting (for tensor memory, for
// the special function unit): two threads share a row, one for each half of the
// tile's keys, read their scores once, and agree on the maximum through shared
// memory.
//
// The tiles of all requests, key heads and row tiles form one list, which the
// CTAs, two per SM, share evenly: lengths are known on the device alone, and a
// grid over the longest one would leave SMs idle beside ragged batches. A CTA
// finds its part from the requests' sizes, and takes it item by item (an item:
// one request, key head and row tile); the copies of an item begin while the one
// before it is finished. Items cut by a CTA's end leave unnormalised pieces, which
// a second kernel joins. The row tiles of a head read the same keys, and a CTA goes
// round its own so that all are at the same ones at a time: they come from memory
// once (two documents of up to 131,072 keys under two row tiles 76 us without, 69
// with).
//
// Measured: 64 requests of 9 tokens, 32 heads on 8, up to 8192 keys 175 us, 6.3 TB/s:
// the cache is the bound. 64-token trees of 64-wide heads over up to 4096 keys, 16
// requests, 47 us: the way of a tile is (scores, maximum, weights, product, one after
// the other; tensor pipe 16 % busy, memory at a quarter of its rate), and 9 us of the join.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstring>
#include <numeric>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tt_device.cuh"
#include "tt_f2.cuh"
#include "tt_ops.h"
#include "tt_ring.cuh"
#include "tt_umma.cuh"
#include "tt_x2.cuh"

namespace tt {

namespace {

constexpr int kTile = 128;               // keys of a tile, rows of a CTA
constexpr int kRowWarps = 8;              // two for each 32 rows
constexpr int kRowThreads = kRowWarps * 32;
constexpr int kThreads = (kRowWarps + 2) * 32;
constexpr int kTmemColumns = 256;        // of tensor memory: two CTAs of an SM fit
constexpr int kWords = TT_MAX_TREE / 32;
constexpr float kLn2 = 0.693147180559945f;
// A row's reference maximum follows its maximum once that is 2^kSlack above it:
// weights stay below 2^(kSlack + offset), and the output is scaled rarely.
constexpr float kSlack = 8.f;
constexpr int kMinShare = 2;  // places of a CTA, where there are few
// What an item costs beyond its tiles (queries, ancestors, output), in tiles: it
// takes as many places in the list before its first tile. Without them the CTAs that
// hold requests with short caches took twice the mean time: 64-token trees over
// ragged caches 65 us, 48 with 3 (49 with 2 or 5); a serving batch 186 and 175.
constexpr int kItemCost = 3;

struct TreeKernelArgs {
  CUtensorMap q, k, v, kc, vc;
  TreeArgs a;
  float scale2;       // scale * log2(e)
  int group;          // G
  int per_tile;       // tokens of a 128-row tile
  int ctas;           // of the launch
  int rows;           // rows of an item, at most
  int box;            // slots of one copy: they lie within a page
  int slots_inner;    // the cache maps' second dimension is the slot, the third the head
  // pieces: CTA c leaves that of an item that began before its tiles at 2 c, that
  // of one that begins in them at 2 c + 1
  float* part;        // [2 ctas * rows * D] outputs, not normalised
  float2* part_ml;    // [2 ctas * rows] their reference maximum (log2) and sum
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

// The tiles that the rows of tokens up to end - 1 see: the cache's, then those of
// drafted tokens.
__host__ __device__ inline int cache_tiles(int len) { return len / kTile + (len % kTile != 0); }
__host__ __device__ inline int tree_tiles(int end) { return (end + kTile - 1) / kTile; }
__device__ __forceinline__ int item_tiles(const TreeKernelArgs& p, const Request& r, int mt) {
  return cache_tiles(r.len) + tree_tiles(min(r.nodes, (mt + 1) * p.per_tile));
}
// The place that one key head of a request takes in the list.
__device__ __forceinline__ int head_places(const TreeKernelArgs& p, const Request& r) {
  int n = 0;
  for (int mt = 0; mt * p.per_tile < r.nodes; ++mt) n += kItemCost + item_tiles(p, r, mt);
  return n;
}
// An item of the list, the first of its tiles that is left, and the places before it.
struct Place {
  int b, hk, mt, tile, lead, start;
  Request r;
  __device__ __forceinline__ void find(const TreeKernelArgs& p, int request_b, int offset) {
    b = request_b;
    r = request(p.a, b);
    const int per_head = head_places(p, r);
    hk = offset / per_head;
    offset %= per_head;
    mt = 0;
    for (int n; offset >= (n = kItemCost + item_tiles(p, r, mt)); ++mt) offset -= n;
    tile = max(0, offset - kItemCost);
    lead = max(0, kItemCost - offset);
  }
  // How far into its n tiles of the item a CTA begins, to go round: row tiles of one
  // head read the same keys, CTAs of the same share take them on, and all are to be
  // at the same ones at a time, as those of the first row tile come to them in order.
  __device__ __forceinline__ int turn(const TreeKernelArgs& p, int share, int n) const {
    int shift = 0;
    for (int k = 0; k < mt; ++k) shift += kItemCost + item_tiles(p, r, k);
    shift %= share;
    return shift < n ? shift : 0;
  }
  __device__ __forceinline__ void next_item(const TreeKernelArgs& p) {
    tile = 0;
    lead = kItemCost;
    if (++mt * p.per_tile < r.nodes) return;
    mt = 0;
    if (++hk < p.a.Hkv) return;
    hk = 0;
    do {
      if (++b >= p.a.B) return;
      r = request(p.a, b);
    } while (r.nodes == 0);
  }
};

// Whether every parent and page of the request is in range (the row threads).
__device__ bool out_of_range(const TreeArgs& a, int b, const Request& r, int t) {
  bool bad = false;
  if (a.parents)
    for (int i = t; i < r.nodes; i += kRowThreads) {
      const int p = a.parents[r.first + i];
      bad |= p < -1 || p >= i;
    }
  const int pages = r.len / a.page_size + (r.len % a.page_size != 0);
  for (int x = t; x < pages; x += kRowThreads) {
    const int p = a.page_table[b * a.table_stride + x];
    bad |= p < 0 || p >= a.n_pages;
  }
  return bad;
}

template <int D>
struct Smem {
  static constexpr int kStages = D == 128 ? 1 : 2;  // two CTAs of an SM fit
  // Tensor memory: scores in columns 0 .. 127, weights, output. Narrow heads leave
  // room for weights of their own, and the next tile's scores are computed while
  // this one's weights are; else the weights take the scores' place.
  static constexpr bool kOwn = D == 64;
  static constexpr int kOut = kOwn ? 192 : 128;
  // the column of the weights of key c, two keys to a column (in the scores' place:
  // each half of the tile where its own scores are)
  static __device__ __forceinline__ int weights(int c) {
    return kOwn ? 128 + c / 2 : (c & 64) + (c & 63) / 2;
  }
  char q[kTile * D * 2];
  char k[kStages][kTile * D * 2];
  char v[kStages][kTile * D * 2];
  uint32_t seen[kTile][kWords];  // a token's ancestors and itself
  int16_t up[TT_MAX_TREE];       // parents, -1 for roots
  float half[2][2][kTile];       // what the two threads of a row tell each other
  uint32_t left_out[4];          // boxes of the last tiles that were not copied
  uint32_t odd[kWords];          // drafted tokens with a value that is not finite
  uint64_t q_full, k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t q_empty, s_full, s_free, p_full, o_done, drained;
  long long sums[kThreads / 32];  // places of the requests, by warps
  int start_b, start_offset;      // where this CTA's places begin
  int share;                      // and how many a CTA has
  Place place[kRowWarps];         // where the row warps are (their registers are dear)
  uint32_t tmem;
  int end, stop;                  // the place behind this CTA's, and where it gave up
};

template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (F16)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool F16>
__device__ __forceinline__ float unpack(uint16_t x) {
  if constexpr (F16)
    return __half2float(__ushort_as_half(x));
  else
    return bf16_to_f32(x);
}

// -inf in place of the scores whose bit is not set.
__device__ __forceinline__ void hide(uint32_t (&v)[32], uint32_t see) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (!(see >> i & 1)) v[i] = 0xff800000u;
}

// 32 bytes to memory: one store where they are known to start on 32 bytes (the
// runs' outputs), two of 16 for the caller's output.
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
__global__ void __launch_bounds__(kThreads, 2)
    tree_kernel(const __grid_constant__ TreeKernelArgs p) {
  using S = Smem<D>;
  constexpr int kHalves = D / 64;              // 128-byte column blocks of a tile
  constexpr int kBlock = kTile * 128;          // their distance in bytes
  constexpr float kOffset = F16 ? 7.f : 0.f;   // fp16 weights: away from its small end
  extern __shared__ char raw[];
  S& s = *reinterpret_cast<S*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
  const TreeArgs& a = p.a;
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const uint64_t& limit = p.wait_ns;
  grid_launch_dependents();

  if (t == kRowThreads) {
    prefetch_map(&p.q);
    prefetch_map(&p.kc);
    prefetch_map(&p.vc);
    mbar_init(&s.q_full, 1);
    mbar_init(&s.q_empty, 1);
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&s.k_full[i], 1);
      mbar_init(&s.k_empty[i], 1);
      mbar_init(&s.v_full[i], 1);
      mbar_init(&s.v_empty[i], 1);
    }
    mbar_init(&s.s_full, 1);
    mbar_init(&s.s_free, kRowThreads);
    mbar_init(&s.p_full, kRowThreads);
    mbar_init(&s.o_done, 1);
    mbar_init(&s.drained, 1);
    s.stop = INT32_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kRowWarps + 1) tmem_alloc(&s.tmem, kTmemColumns);
  // The list: each thread adds up a run of requests, and the one whose run holds
  // this CTA's first tile tells the request.
  int todo;
  {
    const int each = (a.B + kThreads - 1) / kThreads, b0 = min(a.B, t * each),
              b1 = min(a.B, b0 + each);
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += (long long)(head_places(p, request(a, b))) * a.Hkv;
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
      for (int b = b0; b < b1; ++b) {
        const long long n = (long long)(head_places(p, request(a, b))) * a.Hkv;
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
      for (int b = b0; b < b1; ++b) {
        p.first[b] = int(at);
        at += (long long)(head_places(p, request(a, b))) * a.Hkv;
      }
      if (t == 0) p.first[a.B] = int(share);
    }
  }
  __syncthreads();
  const uint32_t tmem = s.tmem;
  bool ok = true;

  if (warp == kRowWarps) {
    // ------------------------------------------------------------ copies
    Place x;
    x.lead = 0;
    if (todo > 0) x.find(p, s.start_b, s.start_offset);
    // lane i copies a tile's i-th box of slots
    const int per = kTile / p.box;
    int it = 0, q_copies = 0, k_copies = 0, v_copies = 0;
    for (int seg = 0; todo > x.lead && ok; ++seg) {
      todo -= x.lead;
      const int n_cache = cache_tiles(x.r.len);
      const int node0 = x.mt * p.per_tile, node1 = min(x.r.nodes, node0 + p.per_tile);
      const int tile1 = min(n_cache + tree_tiles(node1), x.tile + todo);
      auto page_of = [&](int tile) {
        const int slot = tile * kTile + lane * p.box;
        return tile < min(tile1, n_cache) && lane < per && slot < x.r.len
                   ? a.page_table[x.b * a.table_stride + slot / a.page_size]
                   : -1;
      };
      int j = x.tile + x.turn(p, s.share, tile1 - x.tile);
      int page = page_of(j);
      // the queries, once the item before has been done with its own
      ok = __all_sync(0xffffffffu, mbar_wait(&s.q_empty, (seg & 1) ^ 1, limit));
      if (!ok) break;
      if (lane == 0) {
        mbar_arrive_expect_tx(&s.q_full, kHalves * p.per_tile * p.group * 128);
        for (int h = 0; h < kHalves; ++h)
          tma_load_3d(smem_u32(s.q) + h * kBlock, &p.q, smem_u32(&s.q_full), 64 * h,
                      x.hk * p.group, x.r.first + node0);
      }
      __syncwarp();
      ++q_copies;
      for (int i = x.tile; i < tile1; ++i, ++it) {
        const int st = it % S::kStages;
        const uint32_t parity = ((it / S::kStages) & 1) ^ 1;
        const int next_j = j + 1 < tile1 ? j + 1 : x.tile, next = page_of(next_j);
        const bool cache = j < n_cache;
        bool mine;
        int bytes, at;
        if (cache) {
          mine = page >= 0 && page < a.n_pages;
          bytes = p.box * 128;
          at = lane * p.box;
        } else {
          at = lane * 16;
          mine = lane < kTile / 16 && (j - n_cache) * kTile + at < node1;
          bytes = 16 * 128;
        }
        const unsigned int copied = __ballot_sync(0xffffffffu, mine);
        const int boxes = __popc(copied);
        auto copy = [&](char* dst, uint64_t* bar, const CUtensorMap* paged,
                        const CUtensorMap* own) {
          if (lane == 0) mbar_arrive_expect_tx(bar, boxes * bytes * kHalves);
          __syncwarp();
          if (mine) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              const uint32_t to = smem_u32(dst) + h * kBlock + at * 128;
              if (cache) {
                const int slot = (j * kTile + at) % a.page_size;
                tma_load_4d(to, paged, smem_u32(bar), 64 * h, p.slots_inner ? slot : x.hk,
                            p.slots_inner ? x.hk : slot, page);
              } else {
                tma_load_3d(to, own, smem_u32(bar), 64 * h, x.hk,
                            x.r.first + (j - n_cache) * kTile + at);
              }
            }
          }
          __syncwarp();
        };
        ok = __all_sync(0xffffffffu, mbar_wait(&s.k_empty[st], parity, limit)) &&
             (it != 1 || int(blockIdx.x) != p.stall);
        if (!ok) break;
        // boxes of slots in use whose page is out of range (told before the copy is)
        if (lane == 0)
          s.left_out[it & 3] =
              cache ? ~copied & ((1u << (min(kTile, x.r.len - j * kTile) + p.box - 1) / p.box) - 1)
                    : 0u;
        copy(s.k[st], &s.k_full[st], &p.kc, &p.k);
        ++k_copies;
        ok = __all_sync(0xffffffffu, mbar_wait(&s.v_empty[st], parity, limit));
        if (!ok) break;
        copy(s.v[st], &s.v_full[st], &p.vc, &p.v);
        ++v_copies;
        page = next;
        j = next_j;
      }
      todo -= tile1 - x.tile;
      x.next_item(p);
    }
    // (the CTA's memory stays until its last copies have come)
    if (q_copies > 0) mbar_wait(&s.q_full, (q_copies - 1) & 1, limit);
    for (int st = 0; st < S::kStages; ++st) {
      if (k_copies > st) mbar_wait(&s.k_full[st], ((k_copies - 1 - st) / S::kStages) & 1, limit);
      if (v_copies > st) mbar_wait(&s.v_full[st], ((v_copies - 1 - st) / S::kStages) & 1, limit);
    }
  } else if (warp == kRowWarps + 1) {
    // ---------------------------------------------------------- products
    if (lane == 0) {
      Place x;
      x.lead = 0;
      if (todo > 0) x.find(p, s.start_b, s.start_offset);
      const uint32_t idesc_o = umma_idesc(F16, D, true);
      int it = 0;
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const int n_cache = cache_tiles(x.r.len);
        const int node1 = min(x.r.nodes, (x.mt + 1) * p.per_tile);
        const int tile1 = min(n_cache + tree_tiles(node1), x.tile + todo);
        // keys of tile j in use, up to a multiple of 32
        auto keys = [&](int j) {
          const int left = j < n_cache ? x.r.len - j * kTile : node1 - (j - n_cache) * kTile;
          return min(kTile, (left + 31) & ~31);
        };
        auto scores = [&](int j, int i, bool last) {
          const int st = i % S::kStages;
          if (!mbar_wait(&s.k_full[st], (i / S::kStages) & 1, limit)) return false;
          tc_fence_after();
          const uint32_t idesc_s = umma_idesc(F16, keys(j), false);
          const uint32_t qa = smem_u32(s.q), ka = smem_u32(s.k[st]);
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint32_t at = (c / 4) * kBlock + (c % 4) * 32;
            umma_ss(tmem, umma_desc(qa + at, 16), umma_desc(ka + at, 16), idesc_s, c > 0);
          }
          umma_commit(&s.s_full);
          umma_commit(&s.k_empty[st]);
          if (last) umma_commit(&s.q_empty);
          return true;
        };
        ok = mbar_wait(&s.q_full, seg & 1, limit);
        // (scores read by all rows: the next ones may take their place)
        if (ok && S::kOwn && it > 0) ok = mbar_wait(&s.s_free, (it - 1) & 1, limit);
        int j = x.tile + x.turn(p, s.share, tile1 - x.tile);
        ok = ok && scores(j, it, x.tile + 1 == tile1);
        for (int i = x.tile; i < tile1 && ok; ++i, ++it) {
          const int st = it % S::kStages;
          const int next = j + 1 < tile1 ? j + 1 : x.tile;
          if (S::kOwn && i + 1 < tile1) {
            ok = mbar_wait(&s.s_free, it & 1, limit) && scores(next, it + 1, i + 2 == tile1);
            if (!ok) break;
          }
          ok = mbar_wait(&s.v_full[st], (it / S::kStages) & 1, limit) &&
               mbar_wait(&s.p_full, it & 1, limit);
          if (!ok) break;
          tc_fence_after();
          const uint32_t va = smem_u32(s.v[st]);
          const int steps = keys(j) / 16;
          for (int c = 0; c < steps; ++c)
            umma_ts(tmem + S::kOut, tmem + S::weights(16 * c), umma_desc(va + c * 2048, kBlock),
                    idesc_o, i > x.tile || c > 0);
          umma_commit(&s.o_done);
          umma_commit(&s.v_empty[st]);
          if (!S::kOwn && i + 1 < tile1) ok = scores(next, it + 1, i + 2 == tile1);
          j = next;
        }
        todo -= tile1 - x.tile;
        x.next_item(p);
      }
      // (and until its last products and their arrivals are done)
      umma_commit(&s.drained);
      mbar_wait(&s.drained, 0, limit);
    }
  } else {
    // -------------------------------------------------------------- rows
    // (while the first copies are on their way: the requests' statuses)
    for (int b = blockIdx.x; b < a.B; b += p.ctas) {
      const Request r = request(a, b);
      const bool bad = __any_sync(0xffffffffu, !r.status && out_of_range(a, b, r, t));
      if (t == 0) s.up[0] = 0;
      asm volatile("bar.sync 5, 256;" ::: "memory");
      if (bad && lane == 0) s.up[0] = 1;
      asm volatile("bar.sync 5, 256;" ::: "memory");
      if (t == 0) a.status[b] = r.status | (s.up[0] ? TT_REQ_ID_OUT_OF_RANGE : 0);
      asm volatile("bar.sync 5, 256;" ::: "memory");
    }
    const int quarter = warp & 3, half = warp >> 2, row = quarter * 32 + lane;
    const uint32_t mine = tmem + (uint32_t(quarter * 32) << 16);  // this warp's lanes
    const int local = row / p.group;                              // token of the row
    // tells the row's other thread x, and returns what that told (turn: of two)
    auto other = [&](float y, int turn) {
      s.half[turn][half][row] = y;
      asm volatile("bar.sync %0, 64;" ::"r"(1 + quarter) : "memory");
      return s.half[turn][half ^ 1][row];
    };
    // A warp goes on, or gives up, as one. One that gave up passes the barriers between
    // the warps as often as the others, but waits and arrives no more and writes
    // nothing: so the others give up, too, and all end.
    auto wait_for = [&](uint64_t* bar, uint32_t parity) {
      if (!ok) return;
      ok = __all_sync(0xffffffffu, mbar_wait(bar, parity, limit));
      if (!ok && lane == 0) atomicMin(&s.stop, s.end - todo);
    };
    Place& x = s.place[warp];
    if (lane == 0) {
      x.lead = 0;
      if (todo > 0) x.find(p, s.start_b, s.start_offset);
    }
    __syncwarp();
    int it = 0;
    while (todo > x.lead) {
      todo -= x.lead;
      const int n_cache = cache_tiles(x.r.len);
      const int node1 = min(x.r.nodes, (x.mt + 1) * p.per_tile);
      const int tile1 = min(n_cache + tree_tiles(node1), x.tile + todo);
      auto first_node = [&] { return x.mt * p.per_tile; };
      const bool valid = row < (node1 - first_node()) * p.group;
      const bool some = __any_sync(0xffffffffu, valid);  // (others only keep step)
      if (tile1 > n_cache) {
        const int node0 = first_node();
        // a token's ancestors: one thread walks up from each token
        asm volatile("bar.sync 5, 256;" ::: "memory");  // (done with the last ones)
        if (t < kWords) s.odd[t] = 0;
        for (int i = t; i < node1; i += kRowThreads) {
          const int up = a.parents ? a.parents[x.r.first + i] : i - 1;
          s.up[i] = int16_t(up < -1 || up >= i ? -1 : up);
        }
        asm volatile("bar.sync 5, 256;" ::: "memory");
        if (t < node1 - node0) {
          const int w1 = tree_tiles(node1) * (kTile / 32);
          for (int w = 0; w < w1; ++w) s.seen[t][w] = 0;
          for (int i = node0 + t; i >= 0; i = s.up[i]) s.seen[t][i >> 5] |= 1u << (i & 31);
        }
        asm volatile("bar.sync 5, 256;" ::: "memory");
      }
      float m = -INFINITY, l = 0.f;  // the reference maximum (of scores) and the sum
      if (lane == 0) x.start = x.tile + x.turn(p, s.share, tile1 - x.tile);
      __syncwarp();
      int j = x.start;
      do {
        const int st = it % S::kStages;
        const uint32_t parity = (it / S::kStages) & 1;
        const bool cache = j < n_cache;
        const int base = (j - n_cache) * kTile;  // first drafted token of a tree tile
        const int left = cache ? x.r.len - j * kTile : node1 - base;
        const int n = min(kTile, (left + 31) & ~31);
        wait_for(&s.s_full, it & 1);
        tc_fence_after();
        const uint32_t bad_boxes = s.left_out[it & 3];
        // which of 32 keys from c on the row sees; `there`: which hold anything
        auto there = [&](int c) {
          uint32_t w = left - c >= 32 ? 0xffffffffu : (1u << max(0, left - c)) - 1;
          if (bad_boxes)
            for (int i = 0; i < 32; i += 16)
              if (bad_boxes >> ((c + i) / p.box) & 1) w &= ~(0xffffu << i);
          return w;
        };
        auto sees = [&](int c) {
          return cache ? there(c) : valid ? s.seen[local][(base + c) >> 5] : 0u;
        };
        // this thread's half of the row's scores: read once, weights in their registers
        // (all of the 64 columns, whatever the tile holds: the rest is hidden)
        const int c0 = 64 * half;
        uint32_t v[2][32];
        float f = 1.f;
        bool raised = false;
        if (some) {
#pragma unroll
          for (int h = 0; h < 2; ++h) tmem_ld32(mine + c0 + 32 * h, v[h]);
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            tmem_wait_ld(v[h]);
            const uint32_t see = sees(c0 + 32 * h);
            if (see != 0xffffffffu) hide(v[h], see);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 32; ++i) top[i & 3] = fmaxf(top[i & 3], __uint_as_float(v[h][i]));
          }
          float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
          high = fmaxf(high, other(high, it & 1));
          // the reference follows the maximum, and with it the sums
          const bool raise = (high - m) * p.scale2 > kSlack || (m == -INFINITY && high > -INFINITY);
          raised = __any_sync(0xffffffffu, raise);
          if (raised) {
            const float to = fmaxf(m, high);
            f = m == -INFINITY ? 0.f : ex2_approx((m - to) * p.scale2);
            m = to;
            l *= f;
          }
          const float shift = (m == -INFINITY ? 0.f : -m * p.scale2) + kOffset;
          const f32x2 scale2 = pair(p.scale2, p.scale2), shift2 = pair(shift, shift);
          f32x2 sum2 = 0;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const f32x2 e = exp2_pair(fma2(
                  pair(__uint_as_float(v[h][2 * i]), __uint_as_float(v[h][2 * i + 1])), scale2, shift2));
              sum2 = add2(sum2, e);
              float lo, hi;
              split(e, lo, hi);
              v[h][i] = pack2<F16>(lo, hi);
            }
          }
          l += sum_pair(sum2);
          tc_fence_before();
        }
        // Weights of their own: the scores' place is free, and the last tile's product
        // has to be done with the weights' place and in the output. (Every warp waits
        // for that, or one without rows would be a tile ahead on p_full.)
        if (S::kOwn) {
          if (ok) mbar_arrive(&s.s_free);
          if (it > 0) {
            wait_for(&s.o_done, (it - 1) & 1);
            tc_fence_after();
          }
        }
        if (some) {
          const uint32_t to = mine + S::weights(c0);
#pragma unroll
          for (int h = 0; h < 2; ++h) tmem_st16(to + 16 * h, v[h]);
          if (raised && j != x.start) {
#pragma unroll 1
            for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
              uint32_t o[32];
              tmem_ld32(mine + S::kOut + c, o);
              tmem_wait_ld(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tmem_st32(mine + S::kOut + c, o);
            }
          }
          tmem_wait_st();
        }
        // Values that no row may touch: slots past the end (0 times what is there
        // could be NaN), and of drafted tokens, what is not finite: a token outside
        // its branch would get NaN from it. (Its own branch gets it at the end.)
        if (left < n || bad_boxes || !cache) {
          wait_for(&s.v_full[st], parity);
          for (int i = t; i < n * kHalves * 8; i += kRowThreads) {
            const int key = (i >> 3) % n, block = (i >> 3) / n;
            uint4* at = reinterpret_cast<uint4*>(s.v[st] + block * kBlock + key * 128 + (i & 7) * 16);
            if (!(there(key & ~31) >> (key & 31) & 1)) {
              *at = make_uint4(0, 0, 0, 0);
            } else if (!cache) {
              constexpr uint16_t kExp = F16 ? 0x7c00 : 0x7f80;
              uint4 w = *at;
              uint16_t* e = reinterpret_cast<uint16_t*>(&w);
              bool odd = false;
#pragma unroll
              for (int q = 0; q < 8; ++q)
                if ((e[q] & kExp) == kExp) {
                  e[q] = 0;
                  odd = true;
                }
              if (odd) {
                *at = w;
                atomicOr(&s.odd[(base + key) >> 5], 1u << ((base + key) & 31));
              }
            }
          }
          fence_proxy_async();
        }
        tc_fence_before();
        if (ok) mbar_arrive(&s.p_full);
        ++it;
        if (++j == tile1) j = x.tile;
      } while (j != x.start);
      wait_for(&s.o_done, (it - 1) & 1);
      tc_fence_after();
      const bool has_tree = tile1 > n_cache;
      if (has_tree) asm volatile("bar.sync 5, 256;" ::: "memory");  // (s.odd is whole)
      if (some) {
        // (the slot of the last tile's maxima: all have read those, or that tile's product
        // would not be done, and the slot's next maxima lie behind another barrier; the
        // other slot is where the next item's first maxima go, with none between)
        l += other(l, (it - 1) & 1);
        const bool whole = x.tile == 0 && tile1 == n_cache + tree_tiles(node1);
        // where the row goes: to the output, or to its place in the CTA's piece
        const int64_t to =
            whole ? (int64_t(x.r.first) + first_node() + local) * a.Hq + x.hk * p.group + row % p.group
                  : (2 * int64_t(blockIdx.x) + (x.tile == 0)) * p.rows + row;
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll 1
        for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
          uint32_t v[32];
          tmem_ld32(mine + S::kOut + c, v);
          tmem_wait_ld(v);
          if (valid && ok) {
            if (has_tree) {
              for (int w = 0; w * 32 < node1; ++w)
                for (uint32_t odd = s.odd[w] & s.seen[local][w]; odd; odd &= odd - 1) {
                  const int64_t peer = int64_t(x.r.first) + w * 32 + __ffs(odd) - 1;
                  const uint16_t* e = reinterpret_cast<const uint16_t*>(a.v) + peer * a.v_token +
                                      x.hk * a.v_head + c;
#pragma unroll
                  for (int i = 0; i < 32; ++i) {
                    const float y = unpack<F16>(e[i]);
                    if (!(fabsf(y) < INFINITY)) v[i] = __float_as_uint(__uint_as_float(v[i]) + y);
                  }
                }
            }
            if (whole) {
              char* out = a.out + (to * D + c) * 2;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                uint32_t o[8];
#pragma unroll
                for (int q = 0; q < 8; ++q)
                  o[q] = pack2<F16>(__uint_as_float(v[16 * i + 2 * q]) * inv,
                                    __uint_as_float(v[16 * i + 2 * q + 1]) * inv);
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
          const float m2 = m == -INFINITY ? -INFINITY : m * p.scale2 - kOffset;
          if (!whole)
            p.part_ml[to] = make_float2(m2, l);
          else if (a.lse)
            a.lse[to] = l > 0.f || l != l ? fmaf(m2, kLn2, logf(l)) : -INFINITY;
        }
        tc_fence_before();
      }
      todo -= tile1 - x.tile;
      __syncwarp();
      if (lane == 0) x.next_item(p);
      __syncwarp();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kRowWarps + 1) tmem_free(tmem, kTmemColumns);
  if (t == 0) p.stop[blockIdx.x] = s.stop;  // (the join tells the requests)
}

// Joins the pieces of every row whose item was cut: with M the largest of their
// references, out = sum 2^(m - M) o / sum 2^(m - M) l. It has little to read and waits
// for it, so what a row needs is asked for at once: the loads of four pieces before
// the first is added (reading the maximum first cost 2.4 us of a call of 17). A few
// pieces: a warp takes two of a key head's rows. More: the CTA's warps take a row's
// pieces in turn (64-token trees over 65,536 keys with 11 pieces a row: 76 and 79 us;
// 1 request of 8 tokens over 8192 with 30: 27 and 18). It also tells the requests that
// lost places to a CTA that gave up.
constexpr int kJoinWarps = 4, kFewPieces = 16;

template <int D, bool F16, bool FEW>
__global__ void __launch_bounds__(kJoinWarps * 32)
    tree_join_kernel(const __grid_constant__ TreeKernelArgs p) {
  constexpr int N = D / 32, R = FEW ? 2 : 1, W = FEW ? 1 : kJoinWarps;
  constexpr int C = FEW ? 4 : 8;  // pieces at once
  using Vec = typename std::conditional<N == 4, float4, float2>::type;
  __shared__ __align__(16) float s_acc[W][D];
  __shared__ float2 s_ml[W];
  const TreeArgs& a = p.a;
  const int warp = FEW ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  // row g0 (and the next) of key head hk, token i of request b
  const unsigned int x = FEW ? blockIdx.x * kJoinWarps + (threadIdx.x >> 5) : blockIdx.x;
  const unsigned int runs = (p.group + R - 1) / R, per_token = runs * a.Hkv;
  const int g0 = int(x % runs) * R, hk = int(x % per_token / runs);
  const int i = int(x / per_token % a.max_nodes), b = int(x / per_token / a.max_nodes);
  if (b >= a.B) return;
  grid_dependency_wait();
  const int share = p.first[a.B], first = p.first[b];
  const Request r = request(a, b);
  if (i >= r.nodes) return;
  const int per_head = head_places(p, r);
  // (one warp of the request)
  if (i == 0 && hk == 0 && g0 == 0 && (FEW || threadIdx.x < 32)) {
    const int end = first + per_head * a.Hkv - 1;  // its last place
    int stop = INT32_MAX;
    for (int c = first / share + lane; c <= end / share; c += 32) stop = min(stop, p.stop[c]);
    if (__any_sync(0xffffffffu, stop <= end) && lane == 0) a.status[b] |= TT_REQ_TIMEOUT;
  }
  const int mt = i / p.per_tile;
  int before = hk * per_head + kItemCost;  // its first tile's place
  for (int k = 0; k < mt; ++k) before += kItemCost + item_tiles(p, r, k);
  const int last = before + item_tiles(p, r, mt) - 1;
  // the CTAs that the item lies in
  const int c0 = (first + before) / share, pieces = (first + last) / share - c0 + 1;
  if (pieces < 2) return;
  const int in_item = (i - mt * p.per_tile) * p.group + g0;
  auto place = [&](int s, int q) {  // of row q in piece s (past the group: the last)
    return (2 * (int64_t(c0) + s) + (s == 0)) * p.rows + in_item + min(q, p.group - 1 - g0);
  };
  float M[R], l[R], acc[R][N];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    M[q] = -INFINITY;
    l[q] = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) acc[q][c] = 0.f;
  }
  auto add = [&](int q, float l_more, const Vec& o, float f) {
    l[q] = fmaf(l_more, f, l[q]);
    acc[q][0] = fmaf(o.x, f, acc[q][0]);
    acc[q][1] = fmaf(o.y, f, acc[q][1]);
    if constexpr (N == 4) {
      acc[q][2] = fmaf(o.z, f, acc[q][2]);
      acc[q][3] = fmaf(o.w, f, acc[q][3]);
    }
  };
  for (int s0 = warp; s0 < pieces; s0 += W * C) {
    float2 ml[C][R];
    Vec o[C][R];
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const int64_t at = place(min(s0 + c * W, pieces - 1), q);
        ml[c][q] = p.part_ml[at];
        o[c][q] = reinterpret_cast<const Vec*>(p.part + at * D)[lane];
      }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      float top = M[q];
#pragma unroll
      for (int c = 0; c < C; ++c) top = fmaxf(top, ml[c][q].x);
      const float f = M[q] == -INFINITY ? 0.f : ex2_approx(M[q] - top);
      M[q] = top;
      l[q] *= f;
#pragma unroll
      for (int c = 0; c < N; ++c) acc[q][c] *= f;
      // (a piece of nothing but -inf scores: 0, whatever the maximum is)
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (s0 + c * W < pieces)
          add(q, ml[c][q].y, o[c][q], ml[c][q].x == -INFINITY ? 0.f : ex2_approx(ml[c][q].x - top));
    }
  }
  if constexpr (!FEW) {
#pragma unroll
    for (int c = 0; c < N; ++c) s_acc[warp][lane * N + c] = acc[0][c];
    if (lane == 0) s_ml[warp] = make_float2(M[0], l[0]);
    __syncthreads();
    if (warp > 0) return;
    for (int w = 1; w < W; ++w) M[0] = fmaxf(M[0], s_ml[w].x);
    l[0] = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) acc[0][c] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = s_ml[w].x == -INFINITY ? 0.f : ex2_approx(s_ml[w].x - M[0]);
      add(0, s_ml[w].y, reinterpret_cast<const Vec*>(s_acc[w])[lane], f);
    }
  }
#pragma unroll
  for (int q = 0; q < R; ++q) {
    if (g0 + q >= p.group) break;
    const float inv = l[q] > 0.f || l[q] != l[q] ? 1.f / l[q] : 0.f;
    const int64_t row = (int64_t(r.first) + i) * a.Hq + hk * p.group + g0 + q;
    uint32_t* out = reinterpret_cast<uint32_t*>(a.out + row * D * 2) + lane * (N / 2);
    out[0] = pack2<F16>(acc[q][0] * inv, acc[q][1] * inv);
    if constexpr (N == 4) out[1] = pack2<F16>(acc[q][2] * inv, acc[q][3] * inv);
    if (a.lse && lane == 0)
      a.lse[row] = l[q] > 0.f || l[q] != l[q] ? fmaf(M[q], kLn2, logf(l[q])) : -INFINITY;
  }
}

// ------------------------------------------------------------------- host

// How a call is cut: tokens per tile of rows, CTAs, and the workspace.
struct Cut {
  int group, per_tile, ctas, rows;
  int64_t places;  // in the list, were all lengths the longest
  int64_t pieces;  // of one item, about
  size_t part_bytes, ml_bytes, first_bytes, bytes;
};
Cut cut(const TreeArgs& a, int sm_count) {
  Cut c;
  c.group = a.Hq / a.Hkv;
  c.per_tile = kTile / c.group;
  const int64_t row_tiles = (a.max_nodes + c.per_tile - 1) / c.per_tile;
  const int64_t tiles = cache_tiles(a.max_len) + tree_tiles(a.max_nodes);  // of an item
  const int64_t all = c.places = int64_t(std::min(
      1e18, double(a.B) * double(a.Hkv) * double(row_tiles) * double(kItemCost + tiles)));
  c.ctas = int(std::max<int64_t>(1, std::min<int64_t>(2 * int64_t(sm_count),
                                                      (all + kMinShare - 1) / kMinShare)));
  // (were all lengths the longest; fewer tiles make shares smaller and pieces more)
  const int64_t share = std::max<int64_t>(kMinShare, (all + c.ctas - 1) / c.ctas);
  c.pieces = tiles / share + 2;
  c.rows = std::min(a.max_nodes, c.per_tile) * c.group;
  const size_t rows = 2 * size_t(c.ctas) * c.rows;
  c.part_bytes = align256(rows * a.D * sizeof(float));
  c.ml_bytes = align256(rows * sizeof(float2));
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

// A map of 16-bit elements, 128-byte swizzled boxes of 64 innermost ones.
// Strides in elements; a dimension of one entry takes any valid stride.
bool encode(CUtensorMap* map, bool f16, const char* data, int rank, const int64_t* size,
            const int64_t* stride, const int* box) {
  cuuint64_t dims[4], strides[3];
  cuuint32_t boxes[4], ones[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    dims[i] = cuuint64_t(size[i]);
    boxes[i] = cuuint32_t(box[i]);
    if (i > 0) strides[i - 1] = cuuint64_t(size[i] > 1 ? stride[i] : size[0]) * 2;
  }
  const auto f = encoder();
  return f && f(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                cuuint32_t(rank), const_cast<char*>(data), dims, strides, boxes, ones,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool F16>
cudaError_t launch(const TreeKernelArgs& p, int64_t pieces, cudaStream_t stream) {
  const TreeArgs& a = p.a;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(p.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem<D>) + 1024;
  cfg.stream = stream;
  cudaError_t e = cudaLaunchKernelEx(&cfg, tree_kernel<D, F16>, p);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  const bool few = pieces <= kFewPieces;
  const int64_t tokens = int64_t(a.B) * a.max_nodes;
  cfg.gridDim = dim3(unsigned(
      few ? (tokens * a.Hkv * ((p.group + 1) / 2) + kJoinWarps - 1) / kJoinWarps : tokens * a.Hq));
  cfg.blockDim = dim3(kJoinWarps * 32);
  cfg.dynamicSmemBytes = 0;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return few ? cudaLaunchKernelEx(&cfg, tree_join_kernel<D, F16, true>, p)
             : cudaLaunchKernelEx(&cfg, tree_join_kernel<D, F16, false>, p);
}

template <int D, bool F16>
cudaError_t preload() {
  cudaFuncAttributes fa;
  cudaError_t e = cudaFuncGetAttributes(&fa, tree_join_kernel<D, F16, true>);
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, tree_join_kernel<D, F16, false>);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(tree_kernel<D, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(sizeof(Smem<D>)) + 1024);
}

}  // namespace

size_t tree_workspace_bytes(const TreeArgs& a, int sm_count) { return cut(a, sm_count).bytes; }

// (places of the list, and blocks of the join, are 32-bit numbers)
bool tree_fits(const TreeArgs& a, int sm_count) {
  return cut(a, sm_count).places <= INT32_MAX &&
         double(a.B) * a.max_nodes * double(a.Hq) <= INT32_MAX;
}

cudaError_t launch_tree(const TreeArgs& a, int dt, cudaStream_t stream, int sm_count) {
  const Cut c = cut(a, sm_count);
  TreeKernelArgs p;
  std::memset(&p, 0, sizeof p);
  p.a = a;
  p.scale2 = float(double(a.scale) * 1.4426950408889634);
  p.group = c.group;
  p.per_tile = c.per_tile;
  p.ctas = c.ctas;
  p.rows = c.rows;
  p.box = std::gcd(a.page_size, kTile);
  p.part = reinterpret_cast<float*>(a.ws);
  p.part_ml = reinterpret_cast<float2*>(a.ws + c.part_bytes);
  p.first = reinterpret_cast<int32_t*>(a.ws + c.part_bytes + c.ml_bytes);
  p.stop = p.first + c.first_bytes / sizeof(int32_t);
  next_launch_stall(&p.stall, &p.wait_ns);
  const bool f16 = dt == TT_F16;
  bool ok = true;
  if (a.n_nodes > 0) {
    const int64_t nq[3] = {a.D, a.Hq, a.n_nodes}, nk[3] = {a.D, a.Hkv, a.n_nodes};
    const int64_t sq[3] = {1, a.q_head, a.q_token}, sk[3] = {1, a.k_head, a.k_token},
                  sv[3] = {1, a.v_head, a.v_token};
    const int bq[3] = {64, c.group, c.per_tile}, bk[3] = {64, 1, 16};
    ok = encode(&p.q, f16, a.q, 3, nq, sq, bq) && encode(&p.k, f16, a.k, 3, nk, sk, bk) &&
         encode(&p.v, f16, a.v, 3, nk, sv, bk);
  }
  if (a.max_len > 0) {
    // (dimensions by rising stride: heads within slots, or slots within heads)
    p.slots_inner = a.kc_slot < a.kc_head && a.page_size > 1 && a.Hkv > 1;
    const bool si = p.slots_inner;
    const int64_t n[4] = {a.D, si ? a.page_size : a.Hkv, si ? a.Hkv : a.page_size, a.n_pages};
    const int64_t sk[4] = {1, si ? a.kc_slot : a.kc_head, si ? a.kc_head : a.kc_slot, a.kc_page};
    const int64_t sv[4] = {1, si ? a.vc_slot : a.vc_head, si ? a.vc_head : a.vc_slot, a.vc_page};
    const int box[4] = {64, si ? p.box : 1, si ? 1 : p.box, 1};
    ok = ok && encode(&p.kc, f16, a.kc, 4, n, sk, box) && encode(&p.vc, f16, a.vc, 4, n, sv, box);
  }
  if (!ok) return cudaErrorInvalidValue;
  if (a.D == 128) return f16 ? launch<128, true>(p, c.pieces, stream) : launch<128, false>(p, c.pieces, stream);
  return f16 ? launch<64, true>(p, c.pieces, stream) : launch<64, false>(p, c.pieces, stream);
}

cudaError_t preload_tree() {
  cudaError_t e = preload<128, true>();
  if (e == cudaSuccess) e = preload<128, false>();
  if (e == cudaSuccess) e = preload<64, true>();
  if (e == cudaSuccess) e = preload<64, false>();
  return e;
}

}  // namespace tt
