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
// two (bf16) or three (fp16) e4m3 pieces of a power of two of its row, which the products
// add up: its 8 or 11 digits, but for what is below 2^-17 of the row's largest element (the
// distance of the smallest e4m3 numbers). Values become fp16, which holds every e4m3 value,
// by four warps of their own, in units that follow the largest scale so far (2^-32 of it is
// the finest); when a larger one comes the sums fall. The request's own drafted tokens are
// tiles of keys and values of the inputs' type.
//
// One CTA per SM: two warps copy (a page's slots at a time) keys and values with their
// scales, four convert, two issue the products, eight hold the rows, two threads each.
// While rows turn a tile's scores into weights, the next tile's scores and the last one's
// product with values are under way: tensor memory holds two tiles' scores, two tiles'
// weights and the output. Tiles of all requests, key heads and 128 rows form one list,
// which the CTAs share evenly: lengths are known on the device alone. Items cut by a CTA's
// end leave pieces, each with its sum and maximum, which a second kernel joins.
//
// Two documents of 131,072 keys with 32 tokens each, 16 heads on 2: 82 us, 2200 cycles a
// tile and CTA, most of them a row's way from its scores to its weights (780 of exponentials).
// Four threads to a row took 109 us: its barriers cost more than its shares saved.
//
// Requests of few rows go to tree8_few.cu, whose products have them as columns; how both
// compare stands at the rule that chooses.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstring>
#include <numeric>
#include <type_traits>

#include "tt_tree8.cuh"

namespace tt {

namespace {

constexpr int kRows = kManyRows;
constexpr int kRowWarps = 8, kRowThreads = kRowWarps * 32;  // two for each 32 rows
constexpr int kThreads = kRowThreads + kConvThreads + 128;

// What the converting warps, which come to an item first, tell the others of it.
struct Facts {
  int n_tree, rows, tile0, tile1, end, len, first, hk, row0, at;  // at: the place of its first tile
};

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
  int own_code[2][kOwnTiles];         // the unit that a drafted tile's values need
  // of the tiles under way
  alignas(16) float k_scale[kScaleRing][kGroups];
  uint32_t v_scale[kScaleRing][kGroups];  // two fp16 numbers, of the tile's unit
  uint32_t left_out[2][kScaleRing];   // groups whose page is out of range: keys, values
  int unit[kScaleRing];               // of the item's values so far
  float half[2][2][kRows];            // what the two threads of a row tell each other
  uint64_t k_full[kStagesK], k_empty[kStagesK], v_full[kStagesV], v_empty[kStagesV];
  uint64_t scale_full[kScaleRing], w_full[2], w_empty[2], s_full[2], s_free[2];
  uint64_t p_full[2], o_done[2], item_full[2], o_free[2], seen_free, q_full, q_empty, own_full,
      drained[2];
  int sums[kThreads / 32];            // places of the requests, by warps
  int start_b, start_hk, start_offset;  // where this CTA's places begin
  int share;                          // and how many a CTA has
  uint32_t tmem;
  int end, stop;                      // the place behind this CTA's, and where it gave up
};

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
  constexpr int kOwnCode = own_code(F16);
  constexpr int kBlock = kTile * 128;         // distance of the 64-element blocks of a 16-bit tile
  constexpr float kOffset = 7.f;              // fp16 weights: away from its small end
  extern __shared__ char raw[];
  S& s = *reinterpret_cast<S*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
  const TreeArgs& a = p.a;
  const Shape shape{p.group, kRows};
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
      mbar_init(&s.v_empty[i], kConvWarps);
    }
    for (int i = 0; i < kScaleRing; ++i) mbar_init(&s.scale_full[i], 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.w_full[i], kConvWarps);
      mbar_init(&s.w_empty[i], 1);
      mbar_init(&s.s_full[i], 2);
      mbar_init(&s.s_free[i], kRowWarps);
      mbar_init(&s.p_full[i], kRowWarps);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.item_full[i], kConvWarps);
      mbar_init(&s.o_free[i], kRowWarps);
    }
    mbar_init(&s.q_full, kConvWarps);
    mbar_init(&s.q_empty, 1);
    mbar_init(&s.own_full, kConvWarps);
    mbar_init(&s.seen_free, kRowWarps);
    mbar_init(&s.drained[0], 1);
    mbar_init(&s.drained[1], 1);
    s.stop = INT32_MAX;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kRowWarps + kConvWarps) tmem_alloc(&s.tmem, S::kColumns);
  // The list: each thread adds up a run of requests, and the one whose run holds
  // this CTA's first place tells the request.
  int todo = begin_list<kThreads>(p, shape, s, t, warp, lane);
  __syncthreads();
  const uint32_t tmem = s.tmem;
  bool ok = true;
  Place x;
  x.lead = 0;
  if (todo > 0 && warp >= kRowWarps) x = find_place(p.a, shape, s.start_b, s.start_hk, s.start_offset);

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
          const Item it(shape, x, todo);
          j = max(0, it.tile0 - it.n_tree);
          j1 = it.tile1 - it.n_tree;
          used = it.tile1 - it.tile0;
          y.unit = it.tile0 < it.n_tree ? kLeastUnit : 1;
          open = true;
        }
        if (j < j1) break;
        todo -= used;
        x = next_place(p.a, shape, x);
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
        unit = max(unit, __shfl_sync(0xffffffffu, top, kGroups * i) - kFiner);
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
      int turn = 0, st = 0, drafted = 0, ct = 0;
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(shape, x, todo);
        ok = on(&s.q_full, seg & 1);
#pragma unroll 1
        for (int j = it.tile0; j < it.tile1 && ok; ++j, ++n, ++w) {
          const int buf = n & 1;
          const uint32_t to = tmem + buf * kTile;
          if (j >= it.n_tree) {
            ok = on(&s.k_full[st], turn & 1) && on(&s.scale_full[ct % kScaleRing], (ct / kScaleRing) & 1) &&
                 on(&s.s_free[buf], ((n >> 1) & 1) ^ 1) && on(&s.o_done[buf], ((n >> 1) & 1) ^ 1);
            ++ct;
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
              mbar_arrive(&s.s_full[buf]);
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
            ok = on(&s.own_full, drafted++ & 1) && on(&s.s_free[buf], ((n >> 1) & 1) ^ 1) &&
                 on(&s.o_done[buf], ((n >> 1) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int c = 0; c < D / 16; ++c)
                umma_ss(to, od + (c / 4) * (kBlock / 16) + (c % 4) * 2,
                        wk + (w & 1) * kWStep + (c / 4) * (kBlock / 16) + (c % 4) * 2,
                        umma_idesc(F16, kTile, false), c > 0);
              umma_commit(&s.s_full[buf]);
              mbar_arrive(&s.s_full[buf]);
              umma_commit(&s.w_empty[w & 1]);
              if (j + 1 == it.tile1) umma_commit(&s.q_empty);
            }
            ++w;  // (behind its keys, its values)
          }
          __syncwarp();
        }
        todo -= it.tile1 - it.tile0;
        x = next_place(p.a, shape, x);
      }
    } else {
      const uint64_t wv = umma_desc(smem_u32(s.w), kBlock);
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(shape, x, todo);
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
        x = next_place(p.a, shape, x);
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
    auto arrive = [&](uint64_t* bar) {  // of the warp
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    int vt = 0, st = 0, w = 0, seg = 0, drafted = 0;
    uint32_t parity = 0;
#pragma unroll 1
    for (; todo > x.lead; ++seg) {
      todo -= x.lead;
      const Item it(shape, x, todo);
      const int side = seg & 1, row0 = x.mt * kRows, token0 = row0 / p.group;
      // (The item before the last one is over. The four warps meet at barriers: they give up
      // as one, here.)
      wait_for(&s.o_free[side], ((seg >> 1) & 1) ^ 1);
      if (any_of(6, kConvThreads, !ok)) {
        ok = false;
        break;
      }
      // Its facts, and a token's ancestors: one thread walks up from each token.
      if (ct == 0)
        s.facts[side] = Facts{it.n_tree, it.rows, it.tile0, it.tile1, it.end,
                              x.r.len,   x.r.first, x.hk,   row0,     s.end - todo};
      if (ct < kOwnTiles) s.own_code[side][ct] = kOwnCode;
      if (ct < kWords) s.odd[side][ct] = 0;
      if (it.tile0 < it.n_tree) {
        // (the parents in the place of the values to come, the ancestors once rows are done
        // with the last ones)
        wait_for(&s.w_empty[w & 1], ((w >> 1) & 1) ^ 1);
        wait_for(&s.seen_free, (drafted++ & 1) ^ 1);
        if (any_of(6, kConvThreads, !ok)) {
          ok = false;
          break;
        }
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
        auto place = [&](int u) {  // 16-byte unit of the row
          return reinterpret_cast<uint4*>(s.q16 + (u / 8) * kBlock + swizzled16(ct, u % 8));
        };
        // (The last loop is rolled, over what waits in the place for drafted keys: code that is
        // run once an item comes from beyond the instruction caches, line by line.)
        if (wait_for(&s.q_empty, (seg & 1) ^ 1)) {
          float top = 0.f;
#pragma unroll 1
          for (int u = 0; u < D / 8; u += 4) {
            uint4 q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = valid ? from[u + i] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              *place(u + i) = q[i];
              top = largest<DT>(q[i], top);
            }
          }
          const uint32_t code = e8m0_for(top);
          const float inverse = e8m0_inverse(code);
          s.factor[side][ct] = p.scale2 * e8m0(code);
#pragma unroll 1
          for (int u = 0; u < D / 8; ++u)
            in_pieces<DT, kPieces>(*place(u), inverse, [&](int piece, uint2 two) {
              *reinterpret_cast<uint2*>(s.q8 + swizzled8<D>(piece * kRows + ct, u * 8)) = two;
            });
          fence_proxy_async();
          arrive(&s.q_full);
          arrive(&s.item_full[side]);
        }
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
          arrive(&s.v_empty[st]);
          ++vt;
          if (++st == S::kStagesV) {
            st = 0;
            parity ^= 1;
          }
        } else {
          // Drafted tokens: keys as they are, then values without what is not finite (a
          // token outside its branch would get NaN from it; its own gets it at the end).
          const int base = j * kTile;
          uint32_t top = 0;  // of even and odd elements of values, the largest sizes' bits
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
                // (values are looked at beside the keys: with the scores rows know their unit)
                if (!F16 && kv == 0) {
                  const uint4 y = *reinterpret_cast<const uint4*>(
                      a.v + ((int64_t(x.r.first) + base + key) * a.v_token + x.hk * a.v_head + u * 8) * 2);
                  top = __vmaxu2(__vmaxu2(__vmaxu2(top, y.x & 0x7fff7fffu), y.y & 0x7fff7fffu),
                                 __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu));
                }
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
              if (!F16 && own_code_for(max(top & 0xffffu, top >> 16)) > kOwnCode)
                large_values<D>(a, x.r.first + base, x.hk, ct, keys, &s.own_code[side][j]);
              fence_proxy_async();
              arrive(&s.w_full[w & 1]);
              arrive(&s.own_full);
              ++w;
            }
          }
          if (!ok) break;
        }
        fence_proxy_async();
        arrive(&s.w_full[w & 1]);
        ++w;
      }
      todo -= it.tile1 - it.tile0;
      x = next_place(p.a, shape, x);
    }
    // (no more)
    if (ok && wait_for(&s.o_free[seg & 1], ((seg >> 1) & 1) ^ 1)) {
      if (ct == 0) s.facts[seg & 1].tile1 = -1;
      arrive(&s.item_full[seg & 1]);
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
    auto arrive = [&](uint64_t* bar) {  // of the warp
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(bar);
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
        // (with the scores, the scales are there, the ancestors, and the weights' place: the
        // product of two tiles ago is done)
        wait_for(&s.s_full[n & 1], (n >> 1) & 1);
        tc_fence_after();
        float f[4];  // what makes a score of each 16 keys its log2
        int unit = kOwnCode;
        uint32_t lost = 0;
        if (cache) {
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
          if (!F16) unit = s.own_code[side][j];
        }
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
        arrive(&s.s_free[n & 1]);
        // (all ancestors are read)
        if (j + 1 == min(it.n_tree, it.tile1)) arrive(&s.seen_free);
        // what the values' scale makes of the sums, and a larger maximum of the row's
        float fall = 1.f;
        if (F16 ? unit != code : unit > code) {
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
          // (in the unit that large drafted values need)
          if constexpr (!F16)
            if (cache && unit < code) {
              const uint32_t by = half_power(code - unit);
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) v[h][i] = half_mul2(v[h][i], by);
            }
        }
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
        arrive(&s.p_full[n & 1]);
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
        const float by = l > 0.f || l != l ? unit / l : 0.f;
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
      arrive(&s.o_free[side]);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kRowWarps + kConvWarps) tmem_free(tmem, S::kColumns);
  if (t == 0) p.stop[blockIdx.x] = s.stop;  // (the join tells the requests)
}

// Joins the pieces of every row whose item was cut: with M the largest of their
// references, out = sum 2^(m - M) l o / sum 2^(m - M) l. A CTA takes a row; its warps take
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
  const int share = p.first[a.B], head = p.first[a.B + 1], first = p.first[b];
  const Request r = request(a, b);
  if (i >= r.nodes) return;
  const Shape shape{p.group, p.rows};
  // (one warp of the request)
  if (i == 0 && h == 0 && (FEW || threadIdx.x < 32)) {
    const int per_head = head_places(r, shape);
    const int most = per_head / share + 2;  // CTAs that a head of it lies in, at most
    bool lost = false;
    for (int x = lane; x < a.Hkv * most; x += 32) {
      const int k = x / most, from = k * head + first, end = from + per_head - 1;
      const int c = from / share + x % most;
      if (c <= end / share) lost |= p.stop[c] <= end;
    }
    if (__any_sync(0xffffffffu, lost) && lane == 0) a.status[b] |= TT_REQ_TIMEOUT;
  }
  const int row = i * p.group + h % p.group, mt = row / p.rows;
  int before = hk * head + first + kItemCost;  // its first tile's place
  for (int k = 0; k < mt; ++k) before += kItemCost + shape.tiles(r, k);
  const int last = before + shape.tiles(r, mt) - 1;
  // the CTAs that the item lies in
  const int c0 = before / share, pieces = last / share - c0 + 1;
  if (pieces < 2) return;
  auto place = [&](int k) { return (2 * (int64_t(c0) + k) + (k == 0)) * p.rows + row % p.rows; };
  // (outputs are added up times 2^-46 l, which is below 1: sums are weights of up to 2^15
  // for fewer than 2^31 keys)
  constexpr float kBelowOne = 0x1p-46f;
  float M = -INFINITY, l = 0.f, acc[N];
#pragma unroll
  for (int c = 0; c < N; ++c) acc[c] = 0.f;
  auto add = [&](const Vec& o, float f) {
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
      if (k0 + c * W < pieces) {
        const float part = ml[c].x == -INFINITY ? (ml[c].y != ml[c].y ? ml[c].y : 0.f)
                                                : ml[c].y * ex2_approx(ml[c].x - top);
        l += part;
        add(o[c], part * kBelowOne);
      }
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
      l = fmaf(s_ml[w].y, f, l);
      add(reinterpret_cast<const Vec*>(s_acc[w])[lane], f);
    }
  }
  const float inv = l > 0.f || l != l ? 1.f / (l * kBelowOne) : 0.f;
  const int64_t to = (int64_t(r.first) + i) * a.Hq + h;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.out + to * D * 2) + lane * (N / 2);
  out[0] = pack_pair<DT>(acc[0] * inv, acc[1] * inv);
  if constexpr (N == 4) out[1] = pack_pair<DT>(acc[2] * inv, acc[3] * inv);
  if (a.lse && lane == 0) a.lse[to] = l > 0.f || l != l ? fmaf(M, kLn2, logf(l)) : -INFINITY;
}

// ------------------------------------------------------------------- host

// How a call is cut: CTAs, and the workspace.
struct Cut8 {
  int rows;        // of an item
  int ctas;
  int64_t places;  // in the list, were all lengths the longest
  int64_t pieces;  // of one item, about
  size_t part_bytes, ml_bytes, first_bytes, bytes;
};
Cut8 cut8(const TreeArgs& a, int sm_count) {
  Cut8 c;
  const int group = a.Hq / a.Hkv;
  const int64_t rows = int64_t(a.max_nodes) * group;
  // Few rows go to the kernel whose products have them as columns, which costs what they
  // cost: 64 caches of 8192 and 8 heads took, with that one and with this,
  //   heads of 128: 131 and 178 us at 16 rows, 176 and 183 at 32;
  //   heads of 64:  120 and 148 us at 16, 156 and 153 at 32
  // (and with 64 columns, which are no longer there, 218 and 189 at 48).
  c.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : kManyRows;
  const int64_t row_tiles = (rows + c.rows - 1) / c.rows;
  const int64_t tiles = cache_tiles(a.max_len) + tree_tiles(a.max_nodes);  // of an item
  const int64_t all = c.places = int64_t(std::min(
      1e18, double(a.B) * double(a.Hkv) * double(row_tiles) * double(kItemCost + tiles)));
  c.ctas = int(std::max<int64_t>(
      1, std::min<int64_t>(sm_count, (all + kMinShare - 1) / kMinShare)));
  // (were all lengths the longest; fewer tiles make shares smaller and pieces more)
  const int64_t share = std::max<int64_t>(kMinShare, (all + c.ctas - 1) / c.ctas);
  c.pieces = tiles / share + 2;
  const size_t held = 2 * size_t(c.ctas) * c.rows;
  c.part_bytes = align256(held * a.D * sizeof(float));
  c.ml_bytes = align256(held * sizeof(float2));
  c.first_bytes = align256((size_t(a.B) + 2) * sizeof(int32_t));
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
  cfg.stream = stream;
  cudaError_t e;
  if (p.rows < kManyRows) {
    e = launch_tree8_few(p, F16 ? TT_F16 : TT_BF16, stream);
  } else {
    cfg.gridDim = dim3(unsigned(p.ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Smem8<D, F16>) + 1024;
    e = cudaLaunchKernelEx(&cfg, tree8_kernel<D, F16>, p);
  }
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
  p.rows = c.rows;
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
  cudaError_t e = preload_tree8_few();
  if (e == cudaSuccess) e = preload<128, true>();
  if (e == cudaSuccess) e = preload<128, false>();
  if (e == cudaSuccess) e = preload<64, true>();
  if (e == cudaSuccess) e = preload<64, false>();
  return e;
}

}  // namespace tt
