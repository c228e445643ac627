// Attention of groups of rows over the beginning of a paged cache that they share, on the fifth-generation tensor cores: the rows'
// queries of a key head are the M side of the products, so that a key and a value are read once for all of them.  Every part of a
// prefix leaves its sums, its reference and its sum of weights; a second kernel joins them with those of the rows' own keys.
#include "qzo_common.cuh"
#include "launch.cuh"
#include "layers.cuh"
#include "mma.cuh"
#include "paged.cuh"
#include "umma.cuh"

#include <cuda_fp16.h>

#include <algorithm>

namespace qzo {
namespace {

constexpr int kM = kPrefixQueries, kTile = kPrefixTile;
constexpr int kSoftmaxWarps = 4, kLoadWarp = 4, kScoreWarp = 5, kValueWarp = 6, kFirstConvertWarp = 7, kConvertWarps = 4, kTileWarps = 2;       // of the converters, for a tile
constexpr int kTmemCols = 256;                         // two CTAs to an SM
constexpr int kThereRing = 8;                          // tiles whose masks are kept: more than the rings hold
constexpr float kSlack = 8.0f;                         // by which scores may pass the reference before it is raised

// Shared memory: the queries, a ring of operand tiles (64 keys or values, in the order in which the products take them: K0 K1 V0 K2
// V1 ...), for 8-bit pages a ring of the tiles as they are stored, barriers.  Tensor memory: sums, scores, weights.
template <int DH, bool F8>
struct PrefixPlan {
  static constexpr int kThreads = (kFirstConvertWarp + (F8 ? kConvertWarps : 0)) * 32;
  static constexpr int kQueryBytes = kM * DH * 2, kSlotBytes = kTile * DH * 2, kRawBytes = kTile * DH;
  static constexpr int kSlots = (F8 ? 3 : 4) * 128 / DH, kRawSlots = F8 ? 3 * 128 / DH : 0;
  static constexpr int kOffSlots = kQueryBytes, kOffRaw = kOffSlots + kSlots * kSlotBytes, kOffBars = kOffRaw + kRawSlots * kRawBytes;
  static constexpr int kBars = 2 * kSlots + 2 * kRawSlots + 10;
  static constexpr int kOffWalks = kOffBars + 8 * kBars, kOffThere = kOffWalks + kSoftmaxWarps * 64, kOffMisc = kOffThere + 4 * kThereRing;
  static constexpr int kDynamicBytes = kOffMisc + 16 + 1024;         // slack for the 1024-byte alignment
  static_assert(2 * (kDynamicBytes + 1024) <= 228 * 1024, "two CTAs to an SM");
  static constexpr int kColSums = 0, kColScores = DH;  // two tiles' scores
  static_assert(kColScores + 2 * kTile <= kTmemCols, "tensor memory budget");
};

// Two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// 32 bytes, a whole sector
__device__ __forceinline__ void store32(float* to, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" :: "l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
               "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Keys and values: in boxes of a block's tokens (64 of a larger block), and of 16 tokens for the end of a prefix
struct PrefixMaps { CUtensorMap whole[2], step[2]; };

// A walk along the line: where a CTA is in it, at a tile.  The same in all lanes of a warp; every role has its own.
struct Walk {
  PrefixGroup group;
  int index, unit, key_tile;                           // group, unit within it, tile of keys

  __device__ __forceinline__ void next_unit(const PagedParams& p) {
    key_tile = 0;
    if (++unit < group.units(p.Hkv)) return;
    unit = 0;
    while (++index < p.groups.n) {                     // to the next group with units
      group = prefix_group(p, index);
      if (group.units(p.Hkv)) return;
    }
  }
  __device__ __forceinline__ void next(const PagedParams& p) {
    if (++key_tile == group.key_tiles) next_unit(p);
  }
  __device__ __forceinline__ bool at_end() const { return key_tile + 1 == group.key_tiles; }
  __device__ __forceinline__ int head() const { return unit / group.tiles; }
  __device__ __forceinline__ int first_item() const { return unit % group.tiles * kM; }
};

// A CTA's stretch of the line: where it starts and how many tiles there are in it, 0 where there are none or where the groups' bounds
// do not ascend within the rows.  Whole warps.
__device__ __forceinline__ int find_stretch(const PagedParams& p, int cta, bool report, Walk* w) {
  const int lane = threadIdx.x & 31;
  int all = 0;
  bool bad = false;
  PrefixGroup first = {};                              // of the first 32 groups this lane's
  for (int i = lane; i < p.groups.n; i += 32) {
    const PrefixGroup g = prefix_group(p, i, report);
    if (i == lane) first = g;
    bad = bad || g.row0 < 0 || g.rows < 0 || g.row0 + g.rows > p.R;
    all += g.units(p.Hkv) * g.places();
  }
  if (__any_sync(0xffffffffu, bad)) {
    if (report && lane == 0 && p.status) atomicOr(p.status, kStatusBadToken);
    return 0;
  }
  all = __reduce_add_sync(0xffffffffu, all);
  const int stretch = prefix_stretch(p, all), from = min(all, cta * stretch), to = min(all, from + stretch);
  if (from >= to) return 0;
  // the group that `from` is in, and the tiles between `from` and `to`: places less the one at the end of each unit
  int places_before = 0, tiles = 0;
  bool found = false;
  for (int i0 = 0; i0 < p.groups.n && places_before < to; i0 += 32) {
    PrefixGroup g = first;
    if (i0) g = i0 + lane < p.groups.n ? prefix_group(p, i0 + lane) : PrefixGroup{};
    const int units = g.units(p.Hkv), places = units * g.places();
    int sum = places;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += up;
    }
    const int begin = places_before + sum - places;
    if (units) {                                       // tiles in front of place x of the group
      auto tiles_to = [&](int x) { return x / g.places() * g.key_tiles + min(x % g.places(), g.key_tiles); };
      tiles += tiles_to(min(max(to - begin, 0), places)) - tiles_to(min(max(from - begin, 0), places));
    }
    const unsigned past = __ballot_sync(0xffffffffu, places_before + sum > from);
    if (!found && past) {
      found = true;
      const int who = __ffs(past) - 1;
      w->index = i0 + who;
      w->group = {__shfl_sync(0xffffffffu, g.row0, who), __shfl_sync(0xffffffffu, g.rows, who), __shfl_sync(0xffffffffu, g.prefix, who),
                  __shfl_sync(0xffffffffu, g.seq, who), __shfl_sync(0xffffffffu, g.tiles, who), __shfl_sync(0xffffffffu, g.key_tiles, who)};
      const int in_group = from - __shfl_sync(0xffffffffu, begin, who);
      w->unit = in_group / w->group.places();
      w->key_tile = in_group % w->group.places();
    }
    places_before += __shfl_sync(0xffffffffu, sum, 31);
  }
  tiles = __reduce_add_sync(0xffffffffu, tiles);
  if (tiles && w->key_tile == w->group.key_tiles) w->next_unit(p);
  return tiles;
}

// Where the weights of a tile's keys c .. c + 15 are, their first or second terms: in the place of the scores of the 32 that they belong to
__device__ __forceinline__ uint32_t weights_at(uint32_t scores, int j, int c, int part) {
  return scores + kTile * (j & 1) + c / 32 * 32 + 16 * part + c % 32 / 2;
}

// Two CTAs on every SM, each with its stretch of the line of tiles, unit after unit.  S = Q K^T goes to tensor memory, to one of two places
// in turn; a thread of the softmax warps takes a query's 64 scores into registers and writes their weights in their place, as the sum of two
// bf16 (2^-15 of a weight; one alone would leave 2^-8, as much as the output's rounding), from where they enter O += P V as the A
// operand; then the place is free for the scores of the tile after the next.  O stays in tensor memory; it is rescaled only when a maximum passes
// the reference by 2^8.
// Bound by the chain of a tile: 2350 cycles for the two tiles of an SM's CTAs, of which the tensor pipe is busy 1790 (8 x 48 for Q K^T, 8 x 64 for
// P V with its two terms, for each) and the exponentials' pipe 1024; with start (5 us) and end 128 rows of 8 heads to each of 4 key heads on
// 2 prefixes of 16384 take 58 us of the call's 71.  One place for the scores and another for the weights took 0.9 us more, tiles of 128 keys with
// one CTA on an SM 30 us more, eight softmax warps 8 us more.  Over e4m3 pages
// two tiles take 3300 cycles with no pipe above 31 % and issue at 37 %: the conversion's latency, not its instructions, is in the chain there.
// A wait goes by the parity of a phase, so that a barrier must not be two phases ahead of whoever waits: scores j + 2 come after values j,
// those after weights j, those after scores j have been read, and tiles in turn have barriers of their own.
template <int DH, bool F8>
__global__ void __launch_bounds__((PrefixPlan<DH, F8>::kThreads), 2)
prefix_attention_kernel(const __grid_constant__ PrefixMaps maps, const __grid_constant__ PagedParams p, int64_t cache_rows, int box_rows) {
  using Plan = PrefixPlan<DH, F8>;
  constexpr int kSlots = Plan::kSlots, kRawSlots = Plan::kRawSlots, kHalves = DH / 64, kRing = F8 ? kRawSlots : kSlots;
  extern __shared__ uint8_t prefix_smem[];
  const uint32_t base = (smem_u32(prefix_smem) + 1023u) & ~1023u;
  uint8_t* const smem = prefix_smem + (base - smem_u32(prefix_smem));
  const uint32_t slots = base + Plan::kOffSlots, raws = base + Plan::kOffRaw, bar0 = base + Plan::kOffBars;
  auto bar_full = [&](int s) { return bar0 + 8u * s; };                          // an operand tile is there, and its slot free again
  auto bar_empty = [&](int s) { return bar0 + 8u * (kSlots + s); };
  auto bar_raw_full = [&](int s) { return bar0 + 8u * (2 * kSlots + s); };       // the same of the tiles as they are stored
  auto bar_raw_empty = [&](int s) { return bar0 + 8u * (2 * kSlots + kRawSlots + s); };
  constexpr int kRest = 2 * kSlots + 2 * kRawSlots;
  // of a tile, by its place's parity: its scores are there, its weights are there, are in the sums; of a unit: its queries are there, its
  // sums have been read; the end after a failed wait
  auto bar_scores = [&](int j) { return bar0 + 8u * (kRest + (j & 1)); };
  auto bar_weights = [&](int j) { return bar0 + 8u * (kRest + 2 + (j & 1)); };
  auto bar_values = [&](int j) { return bar0 + 8u * (kRest + 4 + (j & 1)); };
  const uint32_t bar_queries = bar0 + 8u * (kRest + 6), bar_read = bar_queries + 8u, bar_drain = bar_queries + 16u;   // (two)
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + Plan::kOffMisc);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + Plan::kOffMisc + 4);
  volatile int* const never_set = reinterpret_cast<volatile int*>(smem + Plan::kOffMisc + 8);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long limit = kWaitLimitCycles;

  if (tid == kLoadWarp * 32) {
    *abort_flag = 0;
    *never_set = 0;
    for (int s = 0; s < kSlots; ++s) { mbar_init(bar_full(s), F8 ? kTileWarps : 1); mbar_init(bar_empty(s), 1); }
    for (int s = 0; s < kRawSlots; ++s) { mbar_init(bar_raw_full(s), 1); mbar_init(bar_raw_empty(s), kTileWarps); }
    for (int j = 0; j < 2; ++j) { mbar_init(bar_scores(j), 2); mbar_init(bar_weights(j), kSoftmaxWarps); mbar_init(bar_values(j), 1); }
    mbar_init(bar_queries, kSoftmaxWarps);
    mbar_init(bar_read, kSoftmaxWarps);
    mbar_init(bar_drain, 1);
    mbar_init(bar_drain + 8u, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (warp == kLoadWarp && lane < 4) prefetch_tmap(lane < 2 ? &maps.whole[lane] : &maps.step[lane - 2]);
  serving_begin();
  serving_next();                                      // for the rows' own keys
  Walk start;
  const int n_tiles = find_stretch(p, blockIdx.x, blockIdx.x == 0 && warp == 0, &start);
  if (n_tiles == 0) return;

  // The load warp: lanes 0 .. boxes - 1 each copy a box of a tile (a block of the cache, or 64 keys of one), keys and values from
  // the same place of either; blocks are looked up two tiles ahead.  In the order of the products: K0, then K1 V0, K2 V1 ... V of the last.
  struct Box { int page, row, left; };                 // its block, the row of its first token in that block's rows, tokens of the prefix from there on
  const int boxes = kTile / box_rows;
  int issued = 0;
  Ring ring;
  Walk seek = start;
  Box box[3];
  auto look_up = [&](int j) {
    Box b = {0, 0, 0};
    if (j >= n_tiles) return b;
    const int at = seek.key_tile * kTile + lane * box_rows;
    b.left = lane < boxes ? seek.group.prefix - at : 0;
    if (b.left > 0) b.page = p.table[(size_t)seek.group.seq * p.width + (at >> p.log2_block)];
    b.row = (seek.head() << p.log2_block) + (at & ((1 << p.log2_block) - 1));
    seek.next(p);
    return b;
  };
  volatile uint32_t* const there_ring = reinterpret_cast<volatile uint32_t*>(smem + Plan::kOffThere);      // bit i: the sixteen keys i of a tile are there
  auto load = [&](const Box& b, const CUtensorMap* whole, const CUtensorMap* step, int key_tile) {
    const uint32_t full = F8 ? bar_raw_full(ring.s) : bar_full(ring.s);
    // the first round of the ring is free
    if (!__all_sync(0xffffffffu, mbar_wait_likely(F8 ? bar_raw_empty(ring.s) : bar_empty(ring.s), ring.ph ^ 1u, abort_flag, limit))) return false;
    if (key_tile >= 0) {
      const int from = kPrefixStep * lane / box_rows & 31, page = __shfl_sync(0xffffffffu, b.page, from), left = __shfl_sync(0xffffffffu, b.left, from);
      const unsigned there = __ballot_sync(0xffffffffu, left > kPrefixStep * lane % box_rows && (unsigned)page < (unsigned)p.n_blocks);
      if (lane == 0) there_ring[key_tile % kThereRing] = there & (1u << kTile / kPrefixStep) - 1;
    }
    if (lane == 0) mbar_arrive_expect_tx(full, F8 ? Plan::kRawBytes : Plan::kSlotBytes);
    __syncwarp();
    if (lane < boxes) {
      // behind the cache's end there are zeros: for what lies behind the prefix and for blocks out of range
      const bool there = b.left > 0 && (unsigned)b.page < (unsigned)p.n_blocks;
      if (b.left > 0 && !there && p.status) atomicOr(p.status, kStatusBadToken);
      const int64_t y = there ? (((int64_t)b.page * p.Hkv) << p.log2_block) + b.row : cache_rows;
      auto copy = [&](const CUtensorMap* map, int row, int64_t y) {
        if (F8) {
          tma_load_2d(raws + ring.s * Plan::kRawBytes + row * DH, map, full, 0, (int)y);
        } else {
#pragma unroll
          for (int h = 0; h < kHalves; ++h) tma_load_2d(slots + ring.s * Plan::kSlotBytes + h * (kTile * 128) + row * 128, map, full, 64 * h, (int)y);
        }
      };
      if (!there || b.left >= box_rows) {
        copy(whole, lane * box_rows, y);
      } else {                                         // what stands behind the prefix in its last block is not for the products: it may be anything
        for (int r = 0; r < box_rows; r += kPrefixStep) copy(step, lane * box_rows + r, r < b.left ? y + r : cache_rows);
      }
    }
    __syncwarp();
    ++issued;
    ring.next(kRing);
    return true;
  };
  bool ok = true;
  int loaded = 0;                                      // tiles whose values have been asked for
  auto load_until = [&](int most) {                    // of loads
    while (ok && loaded < n_tiles && issued + 2 <= most) {
      box[2] = look_up(loaded + 2);
      if (loaded + 1 < n_tiles) ok = load(box[1], &maps.whole[0], &maps.step[0], loaded + 1);
      ok = ok && load(box[0], &maps.whole[1], &maps.step[1], -1);
      box[0] = box[1];
      box[1] = box[2];
      ++loaded;
    }
  };
  if (warp == kLoadWarp) {                             // the first load, ahead of everything else
    box[0] = look_up(0);
    box[1] = look_up(1);
    load(box[0], &maps.whole[0], &maps.step[0], 0);
  }
  const int mine = tid & (kM - 1);                     // a softmax thread's query of a tile
  // Rows that do not see the whole prefix take it with their own keys: -1
  auto row_of = [&](const Walk& u) {
    const int item = u.first_item() + mine;
    if (item >= u.group.rows * p.G) return -1;
    int seq;
    const int t = u.group.row0 + item / p.G;
    return row_keys(p, t, &seq, false) >= u.group.prefix ? t : -1;
  };
  // A unit's queries are copied when the last product with those before them is done, and are handed over a tile's softmax later.
  auto ask_queries = [&](const Walk& u, int t) {
    const __nv_bfloat16* q = p.q + (size_t)max(t, 0) * p.ldq + (size_t)(u.head() * p.G + (u.first_item() + mine) % p.G) * DH;
#pragma unroll
    for (int c = 0; c < DH / 8; ++c)
      copy16_or_zero(base + (c >> 3) * (kM * 128) + mine * 128 + (((c & 7) ^ (mine & 7)) << 4), q + 8 * c, t >= 0 ? 16 : 0);
    copies_commit();
  };
  auto hand_over = [&](uint32_t bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  auto queries_there = [&]() {
    copies_wait<0>();
    fence_proxy_async_smem();
    hand_over(bar_queries);
  };
  int row = -1;
  if (warp < kSoftmaxWarps) {
    row = row_of(start);
    ask_queries(start, row);
  }
  if (warp == kScoreWarp) tmem_alloc(smem_u32(tmem_slot), kTmemCols);
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = *tmem_slot, tmem_s = tmem + Plan::kColScores, tmem_o = tmem + Plan::kColSums;

  if (warp == kLoadWarp) {
    load_until(INT32_MAX);
    if (!ok) *abort_flag = 1;
  } else if (warp == kScoreWarp || warp == kValueWarp) {
    // One warp issues the products for the scores, one those with the values: an issue waits for the tensor cores' queue, and then does
    // not hold up the waits for the other's operands.  The whole warp goes through the loop and one lane issues.
    constexpr uint32_t kIdescS = umma_idesc_bf16(kM, kTile), kIdescO = umma_idesc_bf16(kM, DH) | kIdescBMnMajor;
    auto wait = [&](uint32_t bar, int phase) { return __all_sync(0xffffffffu, mbar_wait_likely(bar, (uint32_t)phase & 1u, abort_flag, limit)); };
    Walk w = start;
    int unit = 0;                                      // units since the start
    bool first = true;                                 // first tile of its unit
    if (warp == kScoreWarp) {
      for (int j = 0; j < n_tiles; ++j) {
        const int load = j < 2 ? j : 2 * j - 1, slot = load % kSlots;            // the tile's place among the loads
        ok = wait(bar_full(slot), load / kSlots) && (j < 2 || wait(bar_values(j), (j - 2) >> 1)) && (!first || wait(bar_queries, unit));
        if (!ok) break;
        tcgen05_fence_after();
        const uint64_t q = umma_desc_k_major_sw128(base), k = umma_desc_k_major_sw128(slots + slot * Plan::kSlotBytes);
        if (elect_one()) {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)                // a descriptor's address counts in 16 bytes
              umma_bf16(tmem_s + kTile * (j & 1), q + h * (kM * 128 / 16) + 2 * e, k + h * (kTile * 128 / 16) + 2 * e, kIdescS, h + e > 0);
          umma_commit(bar_empty(slot));
          umma_commit(bar_scores(j));
          mbar_arrive(bar_scores(j));                     // hands on what the load warp wrote of the tile
        }
        __syncwarp();
        first = w.at_end();
        unit += first;
        w.next(p);
      }
    } else {
      for (int j = 0; j < n_tiles; ++j) {
        const int load = j + 1 < n_tiles ? 2 * j + 2 : 2 * n_tiles - 1, slot = load % kSlots;
        // the weights first: with three slots the load before this one in its slot is this tile's keys, which have been used then
        ok = wait(bar_weights(j), j >> 1) && wait(bar_full(slot), load / kSlots) && (!first || unit == 0 || wait(bar_read, unit - 1));
        if (!ok) break;
        tcgen05_fence_after();
        const uint64_t v = umma_desc_mn_major_sw128(slots + slot * Plan::kSlotBytes, kTile * 128);
        const uint32_t add = !first;
        if (elect_one()) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int e = 0; e < kTile / 16; ++e) umma_bf16_tmem_a(tmem_o, weights_at(tmem_s, j, 16 * e, part), v + e * (2048 / 16), kIdescO, part + e > 0 ? 1 : add);
          umma_commit(bar_empty(slot));
          umma_commit(bar_values(j));
        }
        __syncwarp();
        first = w.at_end();
        unit += first;
        w.next(p);
      }
    }
    if (!ok) {
      *abort_flag = 1;
      // what was issued is given time to end before the tensor memory is freed
      const uint32_t drain = bar_drain + (warp == kValueWarp ? 8u : 0u);
      if (elect_one()) umma_commit(drain);
      __syncwarp();
      mbar_wait(drain, 0, never_set, limit);
    }
  } else if (warp < kSoftmaxWarps) {
    const uint32_t my_lane = (uint32_t)(warp * 32) << 16;
    const float2 factor = make_float2(p.scale_log2e, p.scale_log2e);
    // A zero that the compiler does not know: a packed product without it and the sum behind would become one operation that rounds once.
    const float zero1 = __uint_as_float(__float_as_uint(p.scale_log2e) & 0x80000000u);
    const float2 zero = make_float2(zero1, zero1);
    // The walk of a warp is in shared memory: inside a unit its registers are needed for the scores.
    Walk* const place = reinterpret_cast<Walk*>(smem + Plan::kOffWalks + 64 * warp);
    static_assert(sizeof(Walk) <= 64, "");
    auto unit_after = [&]() {
      Walk u = *place;
      u.next_unit(p);
      return u;
    };
    *place = start;                                    // the same from every lane
    __syncwarp();
    queries_there();
    // After a failed wait a warp goes on through the loops, so that its barriers are met; what it computes means nothing then.
    auto wait = [&](uint32_t bar, int phase) {
      if (!__all_sync(0xffffffffu, mbar_wait_likely(bar, (uint32_t)phase & 1u, abort_flag, limit))) { ok = false; *abort_flag = 1; }
      tcgen05_fence_after();
    };
    for (int j = 0; j < n_tiles;) {
      int count, next_row = -1;                        // tiles of this unit that are this CTA's
      bool active;                                     // any query for this warp
      {
        const Walk w = *place;
        count = min(n_tiles - j, w.group.key_tiles - w.key_tile);
        active = w.first_item() + warp * 32 < w.group.rows * p.G;
      }
      const bool more = j + count < n_tiles;
      if (more) next_row = row_of(unit_after());
      float m = -INFINITY, ref = 0.0f;
      float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
      for (int i = 0; i < count; ++i, ++j) {
        wait(bar_scores(j), j >> 1);
        const bool ask = i + 1 == count && more;
        const uint32_t there = there_ring[j % kThereRing];
        constexpr uint32_t kAll = (1u << kTile / kPrefixStep) - 1;
        // Scores are kept in registers where there are enough, and read again otherwise.
        constexpr bool kKeep = !F8;
        uint32_t s[kKeep ? kTile : kTile / 2];
        auto fetch = [&](int half) {
          uint32_t* const to = s + (kKeep ? 32 * half : 0);
          tmem_ld32(tmem_s + kTile * (j & 1) + my_lane + 32 * half, to);
          if (there != kAll) {                         // keys behind the prefix and of blocks out of range: nothing
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(there >> (2 * half + c / kPrefixStep) & 1)) to[c] = __float_as_uint(-INFINITY);
          }
        };
        if (active) {
          float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            fetch(half);
            const uint32_t* const from = s + (kKeep ? 32 * half : 0);
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              most[0] = max3(most[0], __uint_as_float(from[c]), __uint_as_float(from[c + 1]));
              most[1] = max3(most[1], __uint_as_float(from[c + 2]), __uint_as_float(from[c + 3]));
            }
          }
          if (ask) ask_queries(unit_after(), next_row);
          const float top = fmaxf(most[0], most[1]) * p.scale_log2e;
          const bool raise = m == -INFINITY ? top > -INFINITY : top > ref + kSlack;
          if (__any_sync(0xffffffffu, raise)) {
            float by = 1.0f;
            if (raise) {
              by = m == -INFINITY ? 0.0f : fast_exp2(ref - top);
              m = ref = top;
#pragma unroll
              for (int e = 0; e < 2; ++e) sum[e] = make_float2(sum[e].x * by, sum[e].y * by);
            }
            if (i > 0) {                               // O holds the unit's tiles before this one, once their product is done
              wait(bar_values(j - 1), (j - 1) >> 1);
#pragma unroll 1
              for (int c = 0; c < DH; c += 16) {
                uint32_t o[16];
                tmem_ld16(tmem_o + my_lane + c, o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                tmem_st16(tmem_o + my_lane + c, o);
              }
            }
          }
          const float2 less = make_float2(-ref, -ref), up = make_float2(1.0f + 0x1p-20f, 1.0f + 0x1p-20f);
#pragma unroll
          for (int c0 = 0; c0 < kTile; c0 += 16) {
            if (!kKeep && c0 % 32 == 0) fetch(c0 / 32);
            uint32_t hi[8], lo[8];
#pragma unroll
            for (int c = 0; c < 16; c += 2) {
              const uint32_t* const from = s + (kKeep ? c0 : c0 % 32) + c;
              // Scores are rounded before the reference is taken off, as they are for the rows' own keys: what is equal there is equal here
              const float2 x = add2(fma2(make_float2(__uint_as_float(from[0]), __uint_as_float(from[1])), factor, zero), less);
              const float2 v = make_float2(fast_exp2(x.x), fast_exp2(x.y));
              sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], v);
              // the first term is the weight cut to bf16, the second what is left and 2^-20 of the weight: above zero, as the first is, for a
              // weight above zero, so that an infinite value stays one
              const uint32_t a = __float_as_uint(v.x), b = __float_as_uint(v.y);
              hi[c / 2] = __byte_perm(a, b, 0x7632);
              const float2 rest = fma2(v, up, make_float2(__uint_as_float((a & 0xffff0000u) ^ 0x80000000u), __uint_as_float((b & 0xffff0000u) ^ 0x80000000u)));
              lo[c / 2] = pack_bf16x2(rest.x, rest.y);
            }
            tmem_st8(weights_at(tmem_s + my_lane, j, c0, 0), hi);
            tmem_st8(weights_at(tmem_s + my_lane, j, c0, 1), lo);
          }
          tmem_wait_st();
        } else if (ask) {
          ask_queries(unit_after(), next_row);
        }
        tcgen05_fence_before();
        hand_over(bar_weights(j));
        if (ask) queries_there();
      }
      // the unit's sums leave tensor memory
      wait(bar_values(j - 1), (j - 1) >> 1);
      if (active) {
        const size_t part = prefix_query(p, place->group.row0, place->group.rows, place->head(), place->first_item() + mine) + (size_t)kM * blockIdx.x;
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          uint32_t o[32];
          tmem_ld32(tmem_o + my_lane + c, o);
          if (row >= 0) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) store32(p.prefix_o + part * DH + c + e, o + e);
          }
        }
        if (row >= 0) *reinterpret_cast<float2*>(p.prefix_ml + 2 * part) = make_float2(m == -INFINITY ? -INFINITY : ref, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
      }
      tcgen05_fence_before();
      hand_over(bar_read);
      const Walk after = unit_after();
      __syncwarp();
      *place = after;
      __syncwarp();
      row = next_row;
    }
  } else if (F8 && warp >= kFirstConvertWarp) {
    // Converters: a tile's codes to bf16 (exact), into the swizzled layout of the products.  Two warps have the even loads and two the odd
    // ones: a tile is mostly waiting and latency (128 rows on 16384 tokens, 4 key heads: 104 us when all four had every tile, now 89).  They
    // meet behind every two loads: by then the slots in front of these two have been found free, so that no phase that is waited for
    // next is two ahead, and none behind it can be complete before its load has been converted.  That the load before in a slot has landed
    // follows from its being free.  After a failed wait a warp goes on through the loop, so that the others are not left alone.
    static_assert(!F8 || (kRawSlots == kSlots && kConvertWarps == 2 * kTileWarps), "");
    const int number = warp - kFirstConvertWarp, c0 = number % kTileWarps * 32 + lane;
    for (int i = number / kTileWarps; i < 2 * n_tiles; i += 2) {
      const int slot = i % kSlots;
      const uint32_t phase = (uint32_t)(i / kSlots) & 1u;
      if (i > 1) named_bar_sync(1, kConvertWarps * 32);
      ok = ok && __all_sync(0xffffffffu, mbar_wait_likely(bar_empty(slot), phase ^ 1u, abort_flag, limit) && mbar_wait_likely(bar_raw_full(slot), phase, abort_flag, limit));
      if (!ok) {
        *abort_flag = 1;
        continue;
      }
      const uint32_t src = raws + slot * Plan::kRawBytes;
      uint8_t* const dst = smem + Plan::kOffSlots + slot * Plan::kSlotBytes;
      constexpr int kUnits = kTile * DH / 16, kRowUnits = DH / 16;
#pragma unroll 4
      for (int u = c0; u < kUnits; u += kTileWarps * 32) {
        const int r = u / kRowUnits, c = u % kRowUnits, h = c >> 2;
        const uint4 raw16 = lds16(src + 16 * u);
        const uint32_t codes[4] = {raw16.x, raw16.y, raw16.z, raw16.w};
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t a, b;
          asm("{\n.reg .b16 x, y;\nmov.b32 {x, y}, %2;\ncvt.rn.f16x2.e4m3x2 %0, x;\ncvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(a), "=r"(b) : "r"(codes[e]));
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a)), g = __half22float2(*reinterpret_cast<const __half2*>(&b));
          o[2 * e] = pack_bf16x2(f.x, f.y);
          o[2 * e + 1] = pack_bf16x2(g.x, g.y);
        }
        // the second half's lanes write their two units the other way round: eight lanes then meet eight different banks
        uint8_t* const at = dst + h * (kTile * 128) + r * 128;
        const int first = 2 * (c & 3) + h, second = first ^ 1;
        const uint4 lo = make_uint4(o[0], o[1], o[2], o[3]), hi = make_uint4(o[4], o[5], o[6], o[7]);
        *reinterpret_cast<uint4*>(at + ((first ^ (r & 7)) << 4)) = h ? hi : lo;
        *reinterpret_cast<uint4*>(at + ((second ^ (r & 7)) << 4)) = h ? lo : hi;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar_full(slot));
        mbar_arrive(bar_raw_empty(slot));
      }
    }
  }

  if (!ok && p.status) atomicOr(p.status, kStatusTimeout);
  tcgen05_fence_before();
  __syncthreads();
  if (warp == kLoadWarp && *abort_flag) {              // loads that nobody waited for are given time to land
    for (int i = max(0, issued - kRing); i < issued; ++i)
      mbar_wait(F8 ? bar_raw_full(i % kRing) : bar_full(i % kRing), (uint32_t)(i / kRing) & 1u, never_set, limit);
  }
  __syncthreads();
  if (warp == kScoreWarp) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Joins the parts of a row's head where its own keys are in several: those of the prefix, if the row has them, and its own.  A head takes WARPS warps of the
// CTA, which go over the parts in turn and are added up in their order; a lane has DH / 32 dimensions.
constexpr int kJoinWarps = 8;

template <int DH, int WARPS>
__global__ void __launch_bounds__(kJoinWarps * 32)
prefix_join_kernel(PagedParams p) {
  constexpr int kDims = DH / 32;
  struct Dims { float v[kDims]; };
  __shared__ float part_m[kJoinWarps], part_l[kJoinWarps];
  __shared__ Dims part_o[kJoinWarps][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, in_head = warp % WARPS;
  const int64_t item = (int64_t)blockIdx.x * (kJoinWarps / WARPS) + warp / WARPS;
  serving_begin();
  serving_next();
  const bool there = item < (int64_t)p.R * p.H;        // the same for a head's warps
  const int row = there ? (int)(item / p.H) : 0, head = (int)(item % p.H);
  int seq = 0, prefix = 0, n_first = 0, part_step = 0;
  size_t first_part = 0;
  const RowPrefix shared = row_prefix(p, row);
  const int len = there ? row_keys(p, row, &seq, false) : 0;
  if (shared.prefix > 0 && len >= shared.prefix) {
    prefix = shared.prefix;
    n_first = shared.parts(p, head / p.G, (row - shared.row0) * p.G + head % p.G, &first_part, &part_step);
  }
  const int own = len - prefix, per = split_keys(p, own), n_own = own > 0 ? (own + per - 1) / per : 0;
  const bool work = there && (prefix > 0 || n_own > 1);      // other rows are written already
  const int n = work ? n_first + n_own : 0;
  const size_t own_part = (size_t)(there ? item : 0) * p.splits;
  float m = -INFINITY, l = 0.0f;
  Dims o = {};
  constexpr int kAhead = 4;                            // parts whose loads are in flight
  for (int s0 = in_head; s0 < n; s0 += kAhead * WARPS) {
    float2 ml[kAhead];
    Dims x[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int s = s0 + e * WARPS;
      ml[e] = make_float2(-INFINITY, 0.0f);
      x[e] = {};
      if (s >= n) continue;
      const bool own_keys = s >= n_first;
      const size_t at = own_keys ? own_part + (s - n_first) : first_part + (size_t)s * part_step;
      ml[e] = *reinterpret_cast<const float2*>((own_keys ? p.part_ml : p.prefix_ml) + 2 * at);
      const float* from = (own_keys ? p.part_o : p.prefix_o) + at * DH + kDims * lane;
      if constexpr (kDims == 4) {
        const float4 f = *reinterpret_cast<const float4*>(from);
        x[e].v[0] = f.x; x[e].v[1] = f.y; x[e].v[2] = f.z; x[e].v[3] = f.w;
      } else {
        const float2 f = *reinterpret_cast<const float2*>(from);
        x[e].v[0] = f.x; x[e].v[1] = f.y;
      }
    }
    float top = m;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) top = fmaxf(top, ml[e].x);
    const float ref = finite_max(top), by = fast_exp2(m - ref);
    l *= by;
#pragma unroll
    for (int d = 0; d < kDims; ++d) o.v[d] *= by;
    m = top;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const float w = fast_exp2(ml[e].x - ref);
      l = fmaf(w, ml[e].y, l);
#pragma unroll
      for (int d = 0; d < kDims; ++d) o.v[d] = fmaf(w, x[e].v[d], o.v[d]);
    }
  }
  if (WARPS > 1) {
    if (lane == 0) { part_m[warp] = m; part_l[warp] = l; }
    part_o[warp][lane] = o;
    __syncthreads();
    if (in_head) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, part_m[warp + w]);
    const float ref = finite_max(top);
    l = 0.0f;
    o = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float by = fast_exp2(part_m[warp + w] - ref);
      l = fmaf(by, part_l[warp + w], l);
#pragma unroll
      for (int d = 0; d < kDims; ++d) o.v[d] = fmaf(by, part_o[warp + w][lane].v[d], o.v[d]);
    }
  }
  if (!work) return;
  const float f = inverse_sum(p, l);
  __nv_bfloat16* out = p.out + (size_t)row * p.ldo + (size_t)head * DH + kDims * lane;
#pragma unroll
  for (int d = 0; d < kDims; d += 2) *reinterpret_cast<uint32_t*>(out + d) = pack_bf16x2(o.v[d] * f, o.v[d + 1] * f);
}

template <int DH, bool F8>
int run_prefix(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st) {
  using Plan = PrefixPlan<DH, F8>;
  const int64_t rows = (int64_t)c.n_blocks * c.n_kv_heads * c.block_size;
  const int box_rows = std::min(c.block_size, kTile);
  PrefixMaps maps;
  for (int i = 0; i < 4; ++i)
    QZO_TRY(make_tmap(i < 2 ? &maps.whole[i] : &maps.step[i - 2], i & 1 ? c.v : c.k, F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rows,
                      DH, DH * (F8 ? 1 : 2), F8 ? DH : 64, i < 2 ? box_rows : kPrefixStep, F8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B));
  {
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(prefix_attention_kernel<DH, F8>, Plan::kDynamicBytes, allowed));
  }
  return launch_serving(prefix_attention_kernel<DH, F8>, dim3(p.prefix_ctas), dim3(Plan::kThreads), Plan::kDynamicBytes, 1, st, maps, p, rows, box_rows);
}

template <int DH>
int run_prefix_join(const PagedParams& p, cudaStream_t st) {
  // as many warps to a head as fill the SMs
  const int64_t items = (int64_t)p.R * p.H, fill = kSMs * 32 / items;
  const dim3 block(kJoinWarps * 32);
  if (fill >= 8) return launch_serving(prefix_join_kernel<DH, 8>, dim3((unsigned)items), block, 0, 1, st, p);
  if (fill >= 2) return launch_serving(prefix_join_kernel<DH, 4>, dim3((unsigned)ceil_div64(items, kJoinWarps / 4)), block, 0, 1, st, p);
  return launch_serving(prefix_join_kernel<DH, 1>, dim3((unsigned)ceil_div64(items, kJoinWarps)), block, 0, 1, st, p);
}

}  // namespace

// Every group may leave one unfinished tile of queries.
int64_t prefix_units(int R, int n_groups, int G, int Hkv, int items) {
  const int64_t k = std::min(R, n_groups);
  return (k + ((int64_t)R * G - k) / items) * Hkv;
}

int launch_prefix_attention(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st) {
  const bool f8 = c.dtype == QZO_DTYPE_E4M3;
  if (c.head_dim == 128) return f8 ? run_prefix<128, true>(p, c, st) : run_prefix<128, false>(p, c, st);
  return f8 ? run_prefix<64, true>(p, c, st) : run_prefix<64, false>(p, c, st);
}

int launch_prefix_join(const PagedParams& p, int dh, cudaStream_t st) { return dh == 128 ? run_prefix_join<128>(p, st) : run_prefix_join<64>(p, st); }

}  // namespace qzo
