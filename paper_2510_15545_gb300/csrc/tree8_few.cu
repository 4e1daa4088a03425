// tree8_few.cu -- the attention of tree8.cu where a request has few rows (tokens times the
// query heads that share a key head).
//
// Keys take the rows of the matrix products and tokens the columns: scores S^T = K Q^T and
// outputs O^T = V^T P^T, of 128 keys and 16 or 32 columns, cost what the columns cost. A
// thread then holds one key's scores of many tokens: its scale is one number, its mask one
// bit. Only a row's maximum goes across threads, and it is asked for only where a score
// passes the reference by 2^kSlack, which a vote tells; the sums of the weights stay with the
// keys, in tensor memory, until an item ends.
//
// Keys, queries, values and drafted tokens are multiplied as there. (The values' scales
// could go to the weights instead, before those are rounded to fp16: single tokens took 259
// us so for 266. But weights 2^-14 below the largest then come to nothing where the scales
// are 2^-18 below theirs, and thousands of such may be what a row has.)
//
// One CTA per SM: two warps copy, four convert, two issue products, eight turn scores into
// weights: half of them the even tiles and half the odd ones, each with references, sums and
// an output of their own. 1.07 GB of caches for 256 single tokens take 272 us, 4.0 TB/s: a
// fifth of it is items' beginnings and ends. Of 32 rows (64 requests, caches up to 8192, 176
// us) what bounds it is how long a tile takes from its scores to its weights, 12 instructions
// a score.
// The loops over the rows are rolled: unrolled, their code came from beyond the instruction
// caches.
#include <algorithm>
#include <type_traits>

#include "tt_tree8.cuh"

namespace tt {

namespace {

// Eight warps turn scores into weights, 32 keys each: half of them take the even tiles and
// half the odd ones, each with references, sums and an output of their own. What a tile takes
// from its scores to its weights is mostly waiting, and so two are on their way.
constexpr int kSets = 2;
constexpr int kRowWarps = 4 * kSets, kRowThreads = kRowWarps * 32;
constexpr int kThreads = kRowThreads + kConvThreads + 128;
// What the converting warps, which come to an item first, tell the others of it.
struct Facts {
  int n_tree, rows, tile0, tile1, end, len, first, hk, at;  // at: the place of its first tile
};

template <int D, int R, bool F16>
struct Smem8 {
  static constexpr int kPieces = F16 ? 3 : 2;  // of queries
  // Tensor memory: scores of four tiles, of each set its output and the sums of its weights.
  static constexpr int kOut = 4 * R, kSums = kOut + kSets * R, kUsed = kSums + kSets * R;
  static constexpr int kColumns = kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
  // what 227 KB hold
  static constexpr int kStagesK = D == 64 ? 6 : R == 16 ? 4 : 3;
  static constexpr int kStagesV = D == 64 ? 6 : 3;
  char w[2][kTile * D * 2];           // values of 16 bits; a drafted tile's keys too
  char p[2][kTile * 128];             // weights, the rows of a key side by side
  char k[kStagesK][kTile * D];        // keys and values as they come
  char q16[R * D * 2];                // queries for drafted keys,
  char q8[kPieces * R * D];           // and in pieces for the cache's
  char v[kStagesV][kTile * D];
  // of this item and the next one
  uint32_t seen[2][R][kWords];        // a token's ancestors and itself
  alignas(16) float factor[2][R];     // a row's pieces times it and a key's scale: log2 scores
  uint32_t odd[2][kWords];            // drafted tokens with a value that is not finite
  int64_t row_to[2][R];               // row of the output, or of the CTA's pieces
  uint8_t token[2][R];                // of a row, from the item's first
  Facts facts[2];
  int own_code[2][kOwnTiles];         // the unit that a drafted tile's values need
  int16_t up[TT_MAX_TREE];            // parents, -1 for roots
  float k_scale[kScaleRing][kGroups];
  alignas(16) uint32_t v_scale[kScaleRing][kGroups];  // two fp16 numbers, of the tile's unit
  uint32_t left_out[2][kScaleRing];   // groups whose page is out of range: keys, values
  int unit[kScaleRing];               // of the item's values so far
  alignas(16) float own_factor[8];    // the factor of drafted keys
  alignas(16) float shift[kSets][R];  // what is added to log2 scores
  alignas(16) float fall[kSets][R];   // a reference's last change
  alignas(16) float share_of[kSets][R];  // of the output, at an item's end
  float ref[kSets][R];                // reference maximum (log2)
  float part[kSets][4][R];            // what the warps of 32 keys each tell
  int code[kSets];                    // units of the outputs, 0: no tile
  uint64_t k_full[kStagesK], k_empty[kStagesK], v_full[kStagesV], v_empty[kStagesV];
  uint64_t scale_full[kScaleRing], w_full[2], w_empty[2], s_full[4], s_free[4];
  uint64_t p_full[2], o_done[2], item_full[2], o_free[2], q_full, q_empty, own_full, drained[2];
  int sums[kThreads / 32];            // places of the requests, by warps
  int start_b, start_hk, start_offset;  // where this CTA's places begin
  int share;                          // and how many a CTA has
  uint32_t tmem;
  int end, stop;                      // the place behind this CTA's, and where it gave up
};

// Numbers 2 i and 2 i + 1.
__device__ __forceinline__ f32x2 both(const uint32_t (&v)[8], int i) {
  return pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
// (The registers pass through, so that nothing reads them before.)
__device__ __forceinline__ void tmem_wait8(uint32_t (&r)[8]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                 "+r"(r[7])
               :
               : "memory");
}
// Instruction descriptor: 16-bit operands that both lie along M and N.
__device__ __forceinline__ uint32_t idesc_mn(bool f16, int n) {
  return umma_idesc(f16, n, true) | 1u << 15;
}
// The largest of a warp's numbers (NaN: none).
__device__ __forceinline__ float warp_max(float x) {
  const int i = x != x ? int(0xff800000) : __float_as_int(x);  // (-inf)
  const int top = __reduce_max_sync(0xffffffffu, i ^ ((i >> 31) & 0x7fffffff));
  return __int_as_float(top ^ ((top >> 31) & 0x7fffffff));
}
// Sums of N numbers over the lanes: lane i gets that of the i-th (mod N).
template <int N>
__device__ __forceinline__ float warp_sums(float (&x)[N], int lane) {
#pragma unroll
  for (int s = N / 2; s > 0; s /= 2)
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float give = lane & s ? x[i] : x[i + s], keep = lane & s ? x[i + s] : x[i];
      x[i] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
#pragma unroll
  for (int s = N; s < 32; s *= 2) x[0] += __shfl_xor_sync(0xffffffffu, x[0], s);
  return x[0];
}

// What drafted tokens with a value that is not finite add to element d of a row that
// sees them.
template <int DT>
__device__ __noinline__ float odd_values(const TreeArgs& a, const uint32_t* odd, const uint32_t* seen,
                                         int end, int first, int hk, int d) {
  float sum = 0.f;
#pragma unroll 1
  for (int w = 0; w * 32 < end; ++w)
#pragma unroll 1
    for (uint32_t both = odd[w] & seen[w]; both; both &= both - 1) {
      const int64_t peer = int64_t(first) + w * 32 + __ffs(both) - 1;
      const float z = load_elem<DT>(a.v + (peer * a.v_token + hk * a.v_head + d) * 2);
      if (!(fabsf(z) < INFINITY)) sum += z;
    }
  return sum;
}

// Which of 8 rows see the drafted token of bit `lane` of a word.
__device__ __noinline__ uint32_t tree_sees(const uint32_t* seen, const uint8_t* tokens, int word, int lane) {
  uint32_t see = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) see |= (seen[tokens[i] * kWords + word] >> lane & 1) << i;
  return see;
}

template <int D, int R, bool F16>
__global__ void __launch_bounds__(kThreads, 1) tree8_few_kernel(const __grid_constant__ Tree8Args p) {
  using S = Smem8<D, R, F16>;
  constexpr int DT = F16 ? TT_F16 : TT_BF16;
  constexpr int kPieces = S::kPieces;
  constexpr int kOwnCode = own_code(F16);
  constexpr int kBlock = kTile * 128;         // distance of the 64-element blocks of a 16-bit tile
  constexpr float kOffset = 7.f;              // fp16 weights: away from its small end
  extern __shared__ char raw[];
  S& s = *reinterpret_cast<S*>(raw + ((1024 - (smem_u32(raw) & 1023)) & 1023));
  const TreeArgs& a = p.a;
  const Shape shape{p.group, R};
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
      mbar_init(&s.p_full[i], 128);
      mbar_init(&s.o_done[i], 1);
      mbar_init(&s.item_full[i], kConvThreads);
      mbar_init(&s.o_free[i], kRowThreads);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&s.s_full[i], 2);
      mbar_init(&s.s_free[i], 128);
    }
    mbar_init(&s.q_full, kConvThreads);
    mbar_init(&s.q_empty, 1);
    mbar_init(&s.own_full, kConvThreads);
    mbar_init(&s.drained[0], 1);
    mbar_init(&s.drained[1], 1);
    s.stop = INT32_MAX;
    for (int i = 0; i < 8; ++i) s.own_factor[i] = not_zero(p.scale2);
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
        if (lane == 0) mbar_arrive_expect_tx(&full[st], __popc(boxes >> (kGroups * i) & 0xff) * p.box * D);
        __syncwarp();
        if (begins && lane / kGroups == i)
          tma_load_4d(smem_u32(dst) + st * (kTile * D) + lane % kGroups * TT_SCALE_SLOTS * D, map,
                      smem_u32(&full[st]), 0, at1, at2, c.page);
        if (lane == 0) mbar_arrive(&s.scale_full[ring]);
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
    constexpr uint32_t kWStep = kTile * D * 2 / 16, kKStep = kTile * D / 16, kPStep = kTile * 128 / 16;
    int n = 0, w = 0;  // tiles, 16-bit operands
    if (warp == kRowWarps + kConvWarps) {
      const uint64_t kd = umma8_desc<D>(smem_u32(s.k)), qd = umma8_desc<D>(smem_u32(s.q8)),
                     od = umma_desc(smem_u32(s.q16), 16), wk = umma_desc(smem_u32(s.w), 16);
      int turn = 0, st = 0, drafted = 0;
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(shape, x, todo);
        ok = on(&s.q_full, seg & 1);
#pragma unroll 1
        for (int j = it.tile0; j < it.tile1 && ok; ++j, ++n, ++w) {
          const int buf = n & 3;
          const uint32_t to = tmem + buf * R;
          if (j >= it.n_tree) {
            ok = on(&s.k_full[st], turn & 1) && on(&s.s_free[buf], ((n >> 2) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int q = 0; q < kPieces; ++q)
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
                  umma8_ss(to, kd + st * kKStep + 2 * c, qd + q * (R * D / 16) + 2 * c, idesc_e4m3(R),
                           q > 0 || c > 0);
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
            ok = on(&s.own_full, drafted++ & 1) && on(&s.s_free[buf], ((n >> 2) & 1) ^ 1);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int c = 0; c < D / 16; ++c)
                umma_ss(to, wk + (w & 1) * kWStep + (c / 4) * (kBlock / 16) + (c % 4) * 2,
                        od + (c / 4) * (R * 128 / 16) + (c % 4) * 2, umma_idesc(F16, R, false), c > 0);
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
      const uint64_t wv = umma_desc(smem_u32(s.w), kBlock), pd = umma_desc(smem_u32(s.p), 16);
#pragma unroll 1
      for (int seg = 0; todo > x.lead && ok; ++seg) {
        todo -= x.lead;
        const Item it(shape, x, todo);
#pragma unroll 1
        for (int j = it.tile0; j < it.tile1 && ok; ++j, ++n, ++w) {
          if (j < it.n_tree) ++w;
          const int keys = tile_keys(j, it.n_tree, it.end, x.r.len), buf = n & 1;
          ok = on(&s.w_full[w & 1], (w >> 1) & 1) && on(&s.p_full[buf], (n >> 1) & 1) &&
               (j - it.tile0 >= kSets || seg == 0 || on(&s.o_free[(seg - 1) & 1], ((seg - 1) >> 1) & 1));
          if (!ok) break;
          tc_fence_after();
          const uint32_t idesc = idesc_mn(F16 || j >= it.n_tree, R);
          const uint32_t to = tmem + S::kOut + buf * R;
          const bool more = j - it.tile0 >= kSets;
          // (heads of 64: the other half of the 128 rows is of what lies behind the operand,
          // the other one or the weights, and nobody reads it)
          if (elect_one()) {
#pragma unroll
            for (int c = 0; c < kTile / 16; ++c)
              if (16 * c < keys)
                umma_ss(to, wv + (w & 1) * kWStep + 128 * c, pd + buf * kPStep + 128 * c, idesc,
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
    int vt = 0, st = 0, w = 0, seg = 0;
    uint32_t parity = 0;
#pragma unroll 1
    for (; todo > x.lead; ++seg) {
      todo -= x.lead;
      const Item it(shape, x, todo);
      const int side = seg & 1, row0 = x.mt * R, token0 = row0 / p.group;
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
                              x.r.len,   x.r.first, x.hk,   s.end - todo};
      if (ct < kOwnTiles) s.own_code[side][ct] = kOwnCode;
      if (ct < R) {
        const int token = (row0 + ct) / p.group;
        s.token[side][ct] = uint8_t(token - token0);
        s.row_to[side][ct] =
            it.tile0 == 0 && it.tile1 == it.n_tree + cache_tiles(x.r.len)
                ? (int64_t(x.r.first) + token) * a.Hq + x.hk * p.group + row0 + ct - token * p.group
                : (2 * int64_t(blockIdx.x) + (it.tile0 == 0)) * R + ct;
      }
      if (ct < kWords) s.odd[side][ct] = 0;
      if (it.tile0 < it.n_tree) {
        sync_of(6, kConvThreads);  // (done with the last ones)
#pragma unroll 1
        for (int i = ct; i < it.end; i += kConvThreads) {
          const int up = a.parents ? a.parents[x.r.first + i] : i - 1;
          s.up[i] = int16_t(up < -1 || up >= i ? -1 : up);
        }
        sync_of(6, kConvThreads);
        if (ct < it.end - token0) {
          const int words = it.n_tree * (kTile / 32);
#pragma unroll 1
          for (int k = 0; k < words; ++k) s.seen[side][ct][k] = 0;
#pragma unroll 1
          for (int i = token0 + ct; i >= 0; i = s.up[i]) s.seen[side][ct][i >> 5] |= 1u << (i & 31);
        }
      }
      // Queries: kEach threads to a row.
      {
        constexpr int kEach = kConvThreads / R, kVecs = D / 8 / kEach;
        const int r = ct / kEach, sub = ct % kEach;
        const int row = x.mt * R + r, token = row / p.group, head = x.hk * p.group + row % p.group;
        const bool valid = r < it.rows;
        const uint4* from = reinterpret_cast<const uint4*>(
            a.q + ((int64_t(x.r.first) + token) * a.q_token + int64_t(head) * a.q_head) * 2) + sub * kVecs;
        uint4 q[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) q[i] = valid ? from[i] : make_uint4(0, 0, 0, 0);
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) top = largest<DT>(q[i], top);
#pragma unroll
        for (int o = 1; o < kEach; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t code = e8m0_for(top);
        const float inverse = e8m0_inverse(code);
        if (wait_for(&s.q_empty, (seg & 1) ^ 1)) {
          if (sub == 0) s.factor[side][r] = not_zero(p.scale2 * e8m0(code));
#pragma unroll
          for (int i = 0; i < kVecs; ++i) {
            const int u = sub * kVecs + i;  // 16-byte unit of the row
            *reinterpret_cast<uint4*>(s.q16 + (u / 8) * (R * 128) + swizzled16(r, u % 8)) = q[i];
            in_pieces<DT, kPieces>(q[i], inverse, [&](int piece, uint2 two) {
              *reinterpret_cast<uint2*>(s.q8 + swizzled8<D>(piece * R + r, u * 8)) = two;
            });
          }
          fence_proxy_async();
          mbar_arrive(&s.q_full);
          mbar_arrive(&s.item_full[side]);
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
            // Four keys' halves at a time, rolled: single tokens took 301 us with all
            // unrolled, 268 with eight at a time, 266 with four.
            const uint4* const fours = reinterpret_cast<const uint4*>(scales);
#pragma unroll 1
            for (int i = 0; i < 2 * kPairs; ++i) {
              const char* const from4 = from + (i & 1) * 64 * D + (i >> 1) * 64;
              char* const to4 = to + (i & 1) * 8192 + (i >> 1) * kBlock;
              const uint4 f = fours[i & 1];
              const uint32_t by[4] = {f.x, f.y, f.z, f.w};
              uint2 in[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) in[k] = *reinterpret_cast<const uint2*>(from4 + k * 16 * D);
#pragma unroll
              for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(to4 + k * 2048) = convert(in[k], by[k]);
            }
          } else {
#pragma unroll 1
            for (int k = 0; k < kEach; ++k) {
              const int key = key0 + 16 * k;
              const bool there = key < keys && !(lost >> (key / TT_SCALE_SLOTS) & 1);
#pragma unroll
              for (int h = 0; h < kPairs; ++h) {
                uint4 out = make_uint4(0, 0, 0, 0);
                if (there) out = convert(*reinterpret_cast<const uint2*>(from + k * 16 * D + h * 64), scales[k]);
                *reinterpret_cast<uint4*>(to + h * kBlock + k * 2048) = out;
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
      x = next_place(p.a, shape, x);
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
    const int quarter = warp & 3, set = warp >> 2, key = quarter * 32 + lane;
    const uint32_t mine = tmem + (uint32_t(quarter * 32) << 16);  // this warp's lanes
    const uint32_t output = mine + S::kOut + set * R, my_sums = mine + S::kSums + set * R;
    const int barrier = 1 + set;  // of its four warps
    float* const my_shift = s.shift[set];
    float* const my_fall = s.fall[set];
    char* const weights = s.p[set] + key * 128;
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
      const int chunks = (it.rows + 7) / 8;
      const bool whole = it.tile0 == 0 && it.tile1 == it.n_tree + cache_tiles(it.len);
      // sums of the weights, from nothing
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        const uint32_t zero[8] = {};
        tmem_st8(my_sums + 8 * c, zero);
      }
      tmem_wait_st();
      bool unset = true;
      int code = 0;  // the output is in units of 2^(code - 127)
#pragma unroll 1
      for (int j = it.tile0; j < it.tile1; ++j, ++n) {
        const bool cache = j >= it.n_tree;
        if ((n & 1) != set) {
          ct += cache;
          continue;
        }
        const bool first = code == 0;
        bool there = key < tile_keys(j, it.n_tree, it.end, it.len);
        float scale = 1.f;
        int unit = kOwnCode;
        if (cache) {
          const int e = ct % kScaleRing;
          wait_for(&s.scale_full[e], (ct / kScaleRing) & 1);
          scale = s.k_scale[e][key / TT_SCALE_SLOTS];
          unit = s.unit[e];
          there = there && !(s.left_out[0][e] >> (key / TT_SCALE_SLOTS) & 1);
          ++ct;
        }
        wait_for(&s.s_full[n & 3], (n >> 2) & 1);
        // (known before the scores' product was issued)
        if (!F16 && j < it.n_tree) unit = s.own_code[side][j];
        tc_fence_after();
        const uint32_t at = mine + (n & 3) * R;
        const f32x2 scale2 = pair(scale, scale);
        // The scores of this thread's key with the rows of chunk c, two to a number; times
        // the key's scale and its row's factor and with its row's shift they are exponents of
        // weights. (They are read again where they are needed again: the loops over chunks
        // are rolled, as unrolled code of this size came from beyond the instruction caches.)
        const float* const factors = cache ? s.factor[side] : s.own_factor;
        const int factor_step = cache ? 4 : 0;
        const uint32_t mask = there ? 0xff : 0;
        const bool plain = cache && __all_sync(0xffffffffu, there);
        auto scores = [&](int c, const uint32_t (&v)[8], f32x2 (&z)[4]) {
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] = mul2(both(v, i), scale2);
          if (plain) return;
          const uint32_t seen =
              cache ? mask
                    : mask & tree_sees(s.seen[side][0], s.token[side] + 8 * c, (j * kTile + key) >> 5, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float lo, hi;
            split(z[i], lo, hi);
            z[i] = pair(seen >> (2 * i) & 1 ? lo : -INFINITY, seen >> (2 * i + 1) & 1 ? hi : -INFINITY);
          }
        };
        auto factor = [&](int c) { return reinterpret_cast<const f32x2*>(factors) + factor_step * c; };
        auto shift = [&](int c) { return reinterpret_cast<const f32x2*>(my_shift + 8 * c); };
        // New references, where a row's maximum is above its own by more than kSlack (or it
        // has none), and what that makes of the output.
        auto raise = [&] {
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            uint32_t v[8];
            tmem_ld8(at + 8 * c, v);
            tmem_wait8(v);
            f32x2 z[4];
            scores(c, v, z);
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float lo, hi;
              split(mul2(z[i], factor(c)[i]), lo, hi);
              lo = warp_max(lo);
              hi = warp_max(hi);
              if (lane == 2 * i) top = lo;
              if (lane == 2 * i + 1) top = hi;
            }
            if (lane < 8) s.part[set][quarter][8 * c + lane] = top;
          }
          sync_of(barrier, 128);
          // (a thread to each row)
          bool none = false;
          const int row = key;
          if (row < it.rows) {
            const auto& part = s.part[set];
            const float top = fmaxf(fmaxf(part[0][row], part[1][row]), fmaxf(part[2][row], part[3][row]));
            const float old = first ? -INFINITY : s.ref[set][row];
            const float to = top - old > kSlack || old == -INFINITY ? fmaxf(old, top) : old;
            s.ref[set][row] = to;
            my_shift[row] = (to == -INFINITY ? 0.f : -to) + kOffset;
            my_fall[row] = old == -INFINITY ? 0.f : ex2_approx(old - to);
            none = to == -INFINITY;
          } else if (row < R) {  // (rows that a chunk has too many)
            my_shift[row] = -INFINITY;
            my_fall[row] = 0.f;
          }
          unset = any_of(barrier, 128, none);
        };
        // Values are in units that follow the largest scale so far; when that rises the output
        // falls (fp16: it rises where the drafted ones' unit ends).
        // (Where large drafted values need a larger unit, the weights of cached keys take what
        // is between.)
        float output_fall = 1.f;
        if (F16 ? unit != code : unit > code) {
          output_fall = code > 0 ? e8m0(code) * e8m0_inverse(unit) : 0.f;
          code = unit;
        }
        const float value = __uint_as_float(max(0, 127 + (cache ? unit : 127) - code) << 23);
        const f32x2 value2 = pair(value, value);
        const bool early = unset;
        // (the product of two tiles ago is done with the weights' place)
        wait_for(&s.o_done[set], ((n >> 1) & 1) ^ 1);
        // 0: references, then weights; 1: weights. One that is too large, seldom: 2, new
        // references, weights again. (The sums were added to in 32 bits, which hold them, or
        // the old ones are nothing to the new.)
        int pass = early ? 0 : 1;
#pragma unroll 1
        do {
          if (pass != 1) raise();
          if (pass < 2) {
            float over = -INFINITY;
            auto fetch = [&](int c, uint32_t (&v)[8], uint32_t (&l)[8]) {
              tmem_ld8(at + 8 * c, v);
              tmem_ld8(my_sums + 8 * c, l);
            };
            auto weigh = [&](int c, const uint32_t (&v)[8], uint32_t (&l)[8]) {
              f32x2 z[4];
              scores(c, v, z);
              uint32_t out[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x2 y = fma2(z[i], factor(c)[i], shift(c)[i]);
                float lo, hi;
                split(y, lo, hi);
                over = max3(over, lo, hi);
                f32x2 e = exp2_pair(y), sum = both(l, i);
                if (early) sum = mul2(sum, reinterpret_cast<const f32x2*>(my_fall + 8 * c)[i]);
                sum = add2(sum, e);
                split(sum, lo, hi);
                l[2 * i] = __float_as_uint(lo);
                l[2 * i + 1] = __float_as_uint(hi);
                split(mul2(e, value2), lo, hi);
                out[i] = F16 || cache ? pack_pair<TT_F16>(lo, hi) : pack_pair<TT_BF16>(lo, hi);
              }
              tmem_st8(my_sums + 8 * c, l);
              *reinterpret_cast<uint4*>(weights + ((c ^ (key & 7)) << 4)) =
                  make_uint4(out[0], out[1], out[2], out[3]);
            };
            // (a chunk is fetched while the one before it is weighed)
            uint32_t v0[8], l0[8], v1[8], l1[8];
            fetch(0, v0, l0);
#pragma unroll 1
            for (int c = 0; c < chunks; c += 2) {
              tmem_wait8(v0);
              tmem_wait8(l0);
              if (c + 1 < chunks) fetch(c + 1, v1, l1);
              weigh(c, v0, l0);
              if (c + 1 >= chunks) break;
              tmem_wait8(v1);
              tmem_wait8(l1);
              if (c + 2 < chunks) fetch(c + 2, v0, l0);
              weigh(c + 1, v1, l1);
            }
            pass = !early && any_of(barrier, 128, over > kSlack + kOffset) ? 2 : 3;
          } else {
#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
              f32x2 z[4];
              uint32_t v[8], l[8];
              tmem_wait_st();
              tmem_ld8(at + 8 * c, v);
              tmem_ld8(my_sums + 8 * c, l);
              tmem_wait8(v);
              tmem_wait8(l);
              scores(c, v, z);
              uint32_t out[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float e[2], lo, hi;
                split(exp2_pair(fma2(z[i], factor(c)[i], shift(c)[i])), e[0], e[1]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const float fall = my_fall[8 * c + 2 * i + k];
                  const float sum = __uint_as_float(l[2 * i + k]);
                  // (NaN stays: one of the scores so far is)
                  l[2 * i + k] = __float_as_uint(fall > 0x1p-60f || sum != sum ? sum * fall : e[k]);
                }
                split(mul2(pair(e[0], e[1]), value2), lo, hi);
                out[i] = F16 || cache ? pack_pair<TT_F16>(lo, hi) : pack_pair<TT_BF16>(lo, hi);
              }
              tmem_st8(my_sums + 8 * c, l);
              *reinterpret_cast<uint4*>(weights + ((c ^ (key & 7)) << 4)) =
                  make_uint4(out[0], out[1], out[2], out[3]);
            }
            pass = 4;
          }
        } while (pass < 3);
        const bool raised = pass == 4;
        tc_fence_before();
        if (ok) mbar_arrive(&s.s_free[n & 3]);
        if ((raised || early || output_fall != 1.f) && !first) {
          // (its last product is done: that of two tiles ago, for which this warp has waited)
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < chunks; ++c) {
            uint32_t v[8];
            tmem_ld8(output + 8 * c, v);
            tmem_wait8(v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              v[i] = __float_as_uint(__uint_as_float(v[i]) * output_fall *
                                     (raised || early ? my_fall[8 * c + i] : 1.f));
            tmem_st8(output + 8 * c, v);
          }
        }
        tmem_wait_st();
        fence_proxy_async();
        tc_fence_before();
        if (ok) mbar_arrive(&s.p_full[set]);
      }
      // the sums of all keys
      if (code) {
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
          uint32_t l[8];
          tmem_ld8(my_sums + 8 * c, l);
          tmem_wait8(l);
          float sums[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) sums[i] = __uint_as_float(l[i]);
          const float sum = warp_sums(sums, lane);
          if (c == 0) sync_of(barrier, 128);  // (done with s.part)
          if (lane < 8) s.part[set][quarter][8 * c + lane] = sum;
        }
      }
      if (quarter == 0 && lane == 0) s.code[set] = code;
      sync_of(5, kRowThreads);
      if (t < it.rows) {
        // the sets' sums and outputs relative to the larger of their references
        float top = -INFINITY, all = 0.f, f[kSets];
#pragma unroll
        for (int k = 0; k < kSets; ++k)
          if (s.code[k]) top = fmaxf(top, s.ref[k][t]);
#pragma unroll
        for (int k = 0; k < kSets; ++k) {
          f[k] = 0.f;
          if (s.code[k]) {
            const float ref = s.ref[k][t];
            const float l = s.part[k][0][t] + s.part[k][1][t] + (s.part[k][2][t] + s.part[k][3][t]);
            f[k] = ref == -INFINITY ? (l != l ? 1.f : 0.f) : ex2_approx(ref - top);
            all = fmaf(l, f[k], all);
          }
        }
        const float m2 = top == -INFINITY ? -INFINITY : top - kOffset;
        const float inverse = all > 0.f || all != all ? 1.f / all : 0.f;
#pragma unroll
        for (int k = 0; k < kSets; ++k)
          s.share_of[k][t] = f[k] * inverse * (s.code[k] ? e8m0(s.code[k]) : 0.f);
        const int64_t to = s.row_to[side][t];
        if (ok && !whole)
          p.part_ml[to] = make_float2(m2, all);
        else if (ok && a.lse)
          a.lse[to] = all > 0.f || all != all ? fmaf(m2, kLn2, logf(all)) : -INFINITY;
      }
      const bool used[kSets] = {s.code[0] != 0, s.code[1] != 0};
      bool odd = false;
      if (it.tile0 < it.n_tree) odd = lane < kWords && s.odd[side][lane];
      odd = __any_sync(0xffffffffu, odd);
      sync_of(5, kRowThreads);
      wait_for(&s.o_done[(n - 1) & 1], ((n - 1) >> 1) & 1);
      if (n > 1) wait_for(&s.o_done[n & 1], ((n - 2) >> 1) & 1);
      tc_fence_after();
      if (D == 128 || quarter < 2) {
#pragma unroll 1
        for (int c = set; c < chunks; c += kSets) {
          float y[8] = {};
#pragma unroll
          for (int k = 0; k < kSets; ++k) {
            if (!used[k]) continue;
            uint32_t v[8];
            tmem_ld8(mine + S::kOut + k * R + 8 * c, v);
            tmem_wait8(v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              y[i] = fmaf(__uint_as_float(v[i]), s.share_of[k][8 * c + i], y[i]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 8 * c + i;
            if (r < it.rows && ok) {
              if (odd)
                y[i] += odd_values<DT>(a, s.odd[side], s.seen[side][s.token[side][r]], it.end, it.first,
                                       it.hk, key);
              const int64_t to = s.row_to[side][r] * D + key;
              if (whole)
                store_elem<DT>(a.out + to * 2, y[i]);
              else
                p.part[to] = y[i];
            }
          }
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

template <int D, int R, bool F16>
cudaError_t launch(const Tree8Args& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(p.ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem8<D, R, F16>) + 1024;
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, tree8_few_kernel<D, R, F16>, p);
}

template <int D, int R, bool F16>
cudaError_t preload() {
  static_assert(sizeof(Smem8<D, R, F16>) + 1024 <= 227 * 1024, "shared memory of a CTA");
  return cudaFuncSetAttribute(tree8_few_kernel<D, R, F16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              int(sizeof(Smem8<D, R, F16>)) + 1024);
}

// go(D, R, F16) of a call, as types.
template <class Go>
cudaError_t of_call(int D, int rows, bool f16, Go go) {
  auto type = [&](auto dim, auto r) {
    return f16 ? go(dim, r, std::true_type()) : go(dim, r, std::false_type());
  };
  auto row = [&](auto dim) {
    return rows == 16 ? type(dim, std::integral_constant<int, 16>())
                      : type(dim, std::integral_constant<int, 32>());
  };
  return D == 128 ? row(std::integral_constant<int, 128>()) : row(std::integral_constant<int, 64>());
}

}  // namespace

cudaError_t launch_tree8_few(const Tree8Args& p, int dt, cudaStream_t stream) {
  return of_call(p.a.D, p.rows, dt == TT_F16, [&](auto dim, auto rows, auto f16) {
    return launch<decltype(dim)::value, decltype(rows)::value, decltype(f16)::value>(p, stream);
  });
}

cudaError_t preload_tree8_few() {
  for (int D : {64, 128})
    for (int rows : {16, 32})
      for (bool f16 : {false, true}) {
        const cudaError_t e = of_call(D, rows, f16, [](auto dim, auto r, auto f) {
          return preload<decltype(dim)::value, decltype(r)::value, decltype(f)::value>();
        });
        if (e != cudaSuccess) return e;
      }
  return cudaSuccess;
}

}  // namespace tt
