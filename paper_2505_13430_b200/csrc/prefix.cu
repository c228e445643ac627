// Attention of groups of rows over the beginning of a paged cache that they share, on the fifth-generation tensor cores: the rows'
// queries of a key head are the M side of the products, so that a key and a value are read once for all of them.  Every split
// of a prefix leaves its sums, its reference and its sum of weights for paged_join_kernel, which joins them with those of the rows' own keys.
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

constexpr int kM = 128;                                // queries of a CTA: the rows of a group times the query heads of a key head
constexpr int kSoftmaxWarps = 4, kLoadWarp = 4, kIssueWarp = 5, kFirstConvertWarp = 6, kConvertWarps = 4;
constexpr int kTmemCols = 256;                         // two CTAs to an SM
constexpr float kSlack = 8.0f;                         // by which scores may pass the reference before it is raised

// Shared memory: the queries, a ring of operand tiles (64 keys or values, in the order in which the products take them: K0 K1 V0 K2
// V1 ...), for 8-bit pages a ring of the tiles as they are stored, barriers.
template <int DH, bool F8>
struct PrefixPlan {
  static constexpr int kThreads = (6 + (F8 ? kConvertWarps : 0)) * 32;
  static constexpr int kQBytes = kM * DH * 2, kSlotBytes = kPrefixTile * DH * 2, kRawBytes = kPrefixTile * DH;
  static constexpr int kSlots = F8 ? 3 * 128 / DH : 4 * 128 / DH, kRawSlots = F8 ? 3 * 128 / DH : 0;
  static constexpr int kOffSlots = kQBytes, kOffRaw = kOffSlots + kSlots * kSlotBytes, kOffBars = kOffRaw + kRawSlots * kRawBytes;
  static constexpr int kBars = 2 * kSlots + 2 * kRawSlots + 2 + 2 + 2 + 1 + 1;
  static constexpr int kOffMisc = kOffBars + 8 * kBars;
  static constexpr int kDynamicBytes = kOffMisc + 16 + 1024;         // slack for the 1024-byte alignment
  static_assert(2 * (kDynamicBytes + 1024) <= 228 * 1024, "two CTAs to an SM");
};

// Tiles of kM queries of all groups, at most: every group may leave one unfinished.
int64_t most_tiles(int R, int n_groups, int G) {
  const int64_t k = std::min(R, n_groups);
  return k + ((int64_t)R * G - k) / kM;
}

// The group and the tile within it that a CTA takes, false where there is none.  Whole warps.
__device__ __forceinline__ bool find_tile(const PagedParams& p, int tile, int* group, int* in_group, bool report) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  bool bad = false;
  *group = -1;
  for (int i0 = 0; i0 <= p.groups.n; i0 += 32) {
    const int i = i0 + lane;
    const int here = i <= p.groups.n ? p.groups.rows[i] : INT32_MAX, next = i < p.groups.n ? p.groups.rows[i + 1] : here;
    bad = bad || here > next || (i == 0 && here < 0) || (i == p.groups.n && here > p.R);
    int tiles = i < p.groups.n && next > here && here >= 0 && next <= p.R ? (int)(((long long)(next - here) * p.G + kM - 1) / kM) : 0;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + sum > tile);
    if (*group < 0 && past) {
      const int who = __ffs(past) - 1;
      *group = i0 + who;
      *in_group = tile - before - __shfl_sync(0xffffffffu, sum - tiles, who);
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  bad = __any_sync(0xffffffffu, bad);
  if (bad && report && p.status) atomicOr(p.status, kStatusBadToken);
  return !bad && *group >= 0;
}

// A CTA = 128 queries of a group and a key head, one split of the prefix.  S = Q K^T goes to tensor memory (two buffers, so that the
// next tile's product runs while this one's softmax does); a thread of the softmax warps has one query's 64 scores in registers
// and writes their weights over them, as the sum of two bf16 (2^-15 of a weight; one alone would leave 2^-8, as much as the
// output's rounding), from where they enter O += P V as the A operand.  O stays in tensor memory; it is rescaled only when a
// maximum passes the reference by 2^8.
template <int DH, bool F8>
__global__ void __launch_bounds__((PrefixPlan<DH, F8>::kThreads), 2)
prefix_attention_kernel(const __grid_constant__ CUtensorMap keys_map, const __grid_constant__ CUtensorMap values_map, const __grid_constant__ PagedParams p,
                        int tiles, int total_splits, int64_t cache_rows, int box_rows) {
  using Plan = PrefixPlan<DH, F8>;
  constexpr int kSlots = Plan::kSlots, kRawSlots = Plan::kRawSlots, kHalves = DH / 64;
  extern __shared__ uint8_t prefix_smem[];
  const uint32_t base = (smem_u32(prefix_smem) + 1023u) & ~1023u;
  uint8_t* const smem = prefix_smem + (base - smem_u32(prefix_smem));
  const uint32_t slots = base + Plan::kOffSlots, raws = base + Plan::kOffRaw, bar0 = base + Plan::kOffBars;
  auto bar_full = [&](int s) { return bar0 + 8u * s; };
  auto bar_empty = [&](int s) { return bar0 + 8u * (kSlots + s); };
  auto bar_raw_full = [&](int s) { return bar0 + 8u * (2 * kSlots + s); };
  auto bar_raw_empty = [&](int s) { return bar0 + 8u * (2 * kSlots + kRawSlots + s); };
  auto bar_scores = [&](int b) { return bar0 + 8u * (2 * kSlots + 2 * kRawSlots + b); };
  auto bar_weights = [&](int b) { return bar0 + 8u * (2 * kSlots + 2 * kRawSlots + 2 + b); };
  // O with the values of tile j: two in turn, so that who waits for tile j - 1 is never two phases away
  auto bar_values = [&](int b) { return bar0 + 8u * (2 * kSlots + 2 * kRawSlots + 4 + b); };
  const uint32_t bar_done = bar0 + 8u * (2 * kSlots + 2 * kRawSlots + 6), bar_drain = bar_done + 8u;      // O with all tiles; end after a failed wait
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(smem + Plan::kOffMisc);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + Plan::kOffMisc + 4);
  volatile int* const never_set = reinterpret_cast<volatile int*>(smem + Plan::kOffMisc + 8);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long limit = kWaitLimitCycles;

  // tiles of one group, key head and split stand side by side: they read the same keys
  const int tile = blockIdx.x % tiles, hk = blockIdx.x / tiles % p.Hkv, split = blockIdx.x / tiles / p.Hkv;
  serving_begin();
  int group, in_group;
  if (!find_tile(p, tile, &group, &in_group, blockIdx.x == 0 && tid == 0)) return;
  const int prefix = group_prefix(p, group, hk == 0 && split == 0 && in_group == 0 && tid == 0);
  const int per = prefix_keys(p, prefix), k0 = split * per, k1 = min(prefix, k0 + per);
  if (k0 >= k1) return;
  const int n_tiles = (k1 - k0) / kPrefixTile;
  const int row0 = p.groups.rows[group], item0 = in_group * kM;
  const int items = min(kM, (p.groups.rows[group + 1] - row0) * p.G - item0);
  const int32_t* const pages = p.table + (size_t)p.groups.seq[group] * p.width;
  const int active_warps = (items + 31) / 32;

  if (tid == 0) {
    *abort_flag = 0;
    *never_set = 0;
    for (int s = 0; s < kSlots; ++s) { mbar_init(bar_full(s), F8 ? kConvertWarps : 1); mbar_init(bar_empty(s), 1); }
    for (int s = 0; s < kRawSlots; ++s) { mbar_init(bar_raw_full(s), 1); mbar_init(bar_raw_empty(s), kConvertWarps); }
    for (int b = 0; b < 2; ++b) { mbar_init(bar_scores(b), 1); mbar_init(bar_weights(b), active_warps); mbar_init(bar_values(b), 1); }
    mbar_init(bar_done, 1);
    mbar_init(bar_drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssueWarp) tmem_alloc(smem_u32(tmem_slot), kTmemCols);
  // a thread's query: which row and head, and whether the row sees the whole prefix (rows that do not take it with their own keys)
  int row = -1, head = 0;
  if (warp < kSoftmaxWarps && tid < items) {
    const int t = row0 + (item0 + tid) / p.G;
    int seq;
    head = hk * p.G + (item0 + tid) % p.G;
    if (row_keys(p, t, &seq, false) >= prefix) row = t;
  }
  if (warp < kSoftmaxWarps) {
    const uint4* q = reinterpret_cast<const uint4*>(p.q + (size_t)max(row, 0) * p.ldq + (size_t)head * DH);
    uint4 v[DH / 8];
#pragma unroll
    for (int c = 0; c < DH / 8; ++c) v[c] = row >= 0 ? q[c] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int c = 0; c < DH / 8; ++c)
      *reinterpret_cast<uint4*>(smem + (c >> 3) * (kM * 128) + tid * 128 + (((c & 7) ^ (tid & 7)) << 4)) = v[c];
    fence_proxy_async_smem();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = *tmem_slot, tmem_o = tmem, tmem_s = tmem + DH;      // O, then the two buffers of scores
  bool ok = true;
  int issued = 0;                                      // loads of the load warp
  // key and value tile of the i-th load: K0 K1 V0 K2 V1 ... (K0 V0 for a single tile)
  auto is_key = [&](int i) { return n_tiles == 1 ? i == 0 : i < 2 || (i < 2 * n_tiles - 1 && (i & 1)); };
  auto tile_of = [&](int i) { return n_tiles == 1 ? 0 : i < 2 ? i : i == 2 * n_tiles - 1 ? n_tiles - 1 : (i & 1) ? (i + 1) / 2 : i / 2 - 1; };

  if (warp == kLoadWarp) {
    // lanes 0 .. boxes - 1 each copy a box of a tile (a block of the cache, or 64 keys of one)
    const int boxes = kPrefixTile / box_rows, in_block = (1 << p.log2_block) - 1;
    constexpr int kRing = F8 ? kRawSlots : kSlots;
    auto look_up = [&](int i) { return i < 2 * n_tiles && lane < boxes ? pages[(k0 + tile_of(i) * kPrefixTile + lane * box_rows) >> p.log2_block] : 0; };
    Ring ring;
    int page = look_up(0);
    for (int i = 0; i < 2 * n_tiles; ++i) {
      const int next = look_up(i + 1);
      const uint32_t full = F8 ? bar_raw_full(ring.s) : bar_full(ring.s), empty = F8 ? bar_raw_empty(ring.s) : bar_empty(ring.s);
      if (!__all_sync(0xffffffffu, mbar_wait(empty, ring.ph ^ 1u, abort_flag, limit))) { ok = false; break; }
      if (lane == 0) mbar_arrive_expect_tx(full, F8 ? Plan::kRawBytes : Plan::kSlotBytes);
      __syncwarp();
      if (lane < boxes) {
        const bool key = is_key(i);
        const int at = k0 + tile_of(i) * kPrefixTile + lane * box_rows;
        const bool fine = (unsigned)page < (unsigned)p.n_blocks;
        if (!fine && p.status) atomicOr(p.status, kStatusBadToken);
        // a block out of range is read behind the cache's end, which gives zeros
        const int y = (int)(fine ? (((int64_t)page * p.Hkv + hk) << p.log2_block) + (at & in_block) : cache_rows);
        const CUtensorMap* map = key ? &keys_map : &values_map;
        if (F8) {
          tma_load_2d(raws + ring.s * Plan::kRawBytes + lane * box_rows * DH, map, full, 0, y);
        } else {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_2d(slots + ring.s * Plan::kSlotBytes + h * (kPrefixTile * 128) + lane * box_rows * 128, map, full, 64 * h, y);
        }
      }
      __syncwarp();
      ++issued;
      ring.next(kRing);
      page = next;
    }
    if (!ok) *abort_flag = 1;
  } else if (warp == kIssueWarp) {
    if (lane == 0) {
      constexpr uint32_t kIdescS = umma_idesc_bf16(kM, kPrefixTile), kIdescO = umma_idesc_bf16(kM, DH) | kIdescBMnMajor;
      Ring ring;
      auto scores = [&](int j) {                       // S of tile j
        if (!mbar_wait(bar_full(ring.s), ring.ph, abort_flag, limit)) return false;
        tcgen05_fence_after();
        const uint32_t k = slots + ring.s * Plan::kSlotBytes;
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            umma_bf16(tmem_s + (j & 1) * kPrefixTile, umma_desc_k_major_sw128(base + h * (kM * 128) + 32 * e),
                      umma_desc_k_major_sw128(k + h * (kPrefixTile * 128) + 32 * e), kIdescS, h + e > 0);
        umma_commit(bar_empty(ring.s));
        umma_commit(bar_scores(j & 1));
        ring.next(kSlots);
        return true;
      };
      for (int j = 0; j < 2 && ok && j < n_tiles; ++j) ok = scores(j);
      for (int j = 0; j < n_tiles && ok; ++j) {
        ok = mbar_wait(bar_weights(j & 1), (uint32_t)(j >> 1) & 1u, abort_flag, limit) && mbar_wait(bar_full(ring.s), ring.ph, abort_flag, limit);
        if (!ok) break;
        tcgen05_fence_after();
        const uint32_t v = slots + ring.s * Plan::kSlotBytes, w = tmem_s + (j & 1) * kPrefixTile;
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            umma_bf16_tmem_a(tmem_o, w + 32 * part + 8 * e, umma_desc_mn_major_sw128(v + 2048 * e, kPrefixTile * 128), kIdescO, j + part + e > 0);
        umma_commit(bar_empty(ring.s));
        umma_commit(j + 1 < n_tiles ? bar_values(j & 1) : bar_done);
        ring.next(kSlots);
        if (j + 2 < n_tiles) ok = scores(j + 2);
      }
      if (!ok) {
        *abort_flag = 1;
        umma_commit(bar_drain);                        // what was issued is given time to end before the tensor memory is freed
        mbar_wait(bar_drain, 0, never_set, limit);
      }
    }
  } else if (warp < kSoftmaxWarps) {
    if (warp < active_warps) {
      const float factor = p.scale_log2e;
      const uint32_t my_lane = (uint32_t)(warp * 32) << 16;
      float m = -INFINITY, ref = 0.0f, sum = 0.0f;
      auto look_up = [&](int j) {                      // lanes 0 .. 3: is this sixteenth key's block in the cache?
        return j >= n_tiles || lane >= 4 || (unsigned)pages[(k0 + j * kPrefixTile + 16 * lane) >> p.log2_block] < (unsigned)p.n_blocks;
      };
      bool fine = look_up(0);
      for (int j = 0; j < n_tiles; ++j) {
        const unsigned there = __ballot_sync(0xffffffffu, fine);
        fine = look_up(j + 1);
        const uint32_t at = tmem_s + my_lane + (j & 1) * kPrefixTile;
        if (!__all_sync(0xffffffffu, mbar_wait(bar_scores(j & 1), (uint32_t)(j >> 1) & 1u, abort_flag, limit))) { ok = false; break; }
        tcgen05_fence_after();
        uint32_t s[kPrefixTile];
        tmem_ld32(at, s);
        tmem_ld32(at + 32, s + 32);
        if (there != 0xffffffffu) {                    // keys of blocks out of range: nothing
#pragma unroll
          for (int c = 0; c < kPrefixTile; ++c)
            if (!(there >> (c / 16) & 1)) s[c] = __float_as_uint(-INFINITY);
        }
        float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < kPrefixTile; ++c) most[c & 3] = fmaxf(most[c & 3], __uint_as_float(s[c]));
        const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * factor;
        const bool raise = m == -INFINITY ? top > -INFINITY : top > ref + kSlack;
        if (__any_sync(0xffffffffu, raise)) {
          float by = 1.0f;
          if (raise) {
            by = m == -INFINITY ? 0.0f : fast_exp2(ref - top);
            m = ref = top;
            sum *= by;
          }
          if (j > 0) {                                 // O holds the tiles before this one, once their product is done
            if (!__all_sync(0xffffffffu, mbar_wait(bar_values((j - 1) & 1), (uint32_t)((j - 1) >> 1) & 1u, abort_flag, limit))) { ok = false; break; }
            tcgen05_fence_after();
#pragma unroll 1
            for (int c = 0; c < DH; c += 32) {
              uint32_t o[32];
              tmem_ld32(tmem_o + my_lane + c, o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
              tmem_st32(tmem_o + my_lane + c, o);
            }
          }
        }
        float part[4] = {};
#pragma unroll
        for (int c0 = 0; c0 < kPrefixTile; c0 += 32) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float a = fast_exp2(fmaf(__uint_as_float(s[c0 + c]), factor, -ref)), b = fast_exp2(fmaf(__uint_as_float(s[c0 + c + 1]), factor, -ref));
            part[c & 2] += a;
            part[(c & 2) + 1] += b;
            // both terms above zero for a weight above zero, so that an infinite value stays one
            const uint32_t x = below(a), y = below(b);
            hi[c / 2] = __byte_perm(x, y, 0x7632);
            lo[c / 2] = pack_bf16x2(a - upper_half(x), b - upper_half(y));
          }
          tmem_st16(at + c0 / 2, hi);
          tmem_st16(at + 32 + c0 / 2, lo);
        }
        sum += (part[0] + part[1]) + (part[2] + part[3]);
        tmem_wait_st();
        tcgen05_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_weights(j & 1));
      }
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_done, 0, abort_flag, limit));
      if (ok) {
        tcgen05_fence_after();
        const size_t at = ((size_t)max(row, 0) * p.H + head) * total_splits + split;
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          uint32_t o[32];
          tmem_ld32(tmem_o + my_lane + c, o);
          if (row >= 0) {
            uint4* out = reinterpret_cast<uint4*>(p.part_o + at * DH + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        if (row >= 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(m == -INFINITY ? -INFINITY : ref, sum);
      } else {
        *abort_flag = 1;
      }
    }
  } else if (F8) {
    // converters: a tile's codes to bf16 (exact), into the swizzled layout of the products
    const int c0 = tid - kFirstConvertWarp * 32;
    Ring raw, ring;
    for (int i = 0; i < 2 * n_tiles; ++i) {
      if (!__all_sync(0xffffffffu, mbar_wait(bar_raw_full(raw.s), raw.ph, abort_flag, limit) && mbar_wait(bar_empty(ring.s), ring.ph ^ 1u, abort_flag, limit))) {
        ok = false;
        break;
      }
      const uint32_t src = raws + raw.s * Plan::kRawBytes;
      uint8_t* const dst = smem + Plan::kOffSlots + ring.s * Plan::kSlotBytes;
      constexpr int kUnits = kPrefixTile * DH / 16, kRowUnits = DH / 16;
#pragma unroll
      for (int u0 = 0; u0 < kUnits; u0 += kConvertWarps * 32) {
        const int u = u0 + c0, r = u / kRowUnits, c = u % kRowUnits, h = c >> 2;
        const uint4 raw16 = lds16(src + 16 * u);
        const uint32_t w[4] = {raw16.x, raw16.y, raw16.z, raw16.w};
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t a, b;
          asm("{\n.reg .b16 x, y;\nmov.b32 {x, y}, %2;\ncvt.rn.f16x2.e4m3x2 %0, x;\ncvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(a), "=r"(b) : "r"(w[e]));
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a)), g = __half22float2(*reinterpret_cast<const __half2*>(&b));
          o[2 * e] = pack_bf16x2(f.x, f.y);
          o[2 * e + 1] = pack_bf16x2(g.x, g.y);
        }
        // the second half's lanes write their two units the other way round: eight lanes then meet eight different banks
        uint8_t* const at = dst + h * (kPrefixTile * 128) + r * 128;
        const int first = 2 * (c & 3) + h, second = first ^ 1;
        const uint4 lo = make_uint4(o[0], o[1], o[2], o[3]), hi = make_uint4(o[4], o[5], o[6], o[7]);
        *reinterpret_cast<uint4*>(at + ((first ^ (r & 7)) << 4)) = h ? hi : lo;
        *reinterpret_cast<uint4*>(at + ((second ^ (r & 7)) << 4)) = h ? lo : hi;
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar_full(ring.s));
        mbar_arrive(bar_raw_empty(raw.s));
      }
      raw.next(kRawSlots > 0 ? kRawSlots : 1);
      ring.next(kSlots);
    }
    if (!ok) *abort_flag = 1;
  }

  serving_next();
  if (!ok && p.status) atomicOr(p.status, kStatusTimeout);
  tcgen05_fence_before();
  __syncthreads();
  if (warp == kLoadWarp && *abort_flag) {              // loads that nobody waited for are given time to land
    constexpr int kRing = F8 ? kRawSlots : kSlots;
    for (int i = max(0, issued - kRing); i < issued; ++i)
      mbar_wait(F8 ? bar_raw_full(i % kRing) : bar_full(i % kRing), (uint32_t)(i / kRing) & 1u, never_set, limit);
  }
  __syncthreads();
  if (warp == kIssueWarp) {
    tcgen05_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

template <int DH, bool F8>
int run_prefix(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st) {
  using Plan = PrefixPlan<DH, F8>;
  const int64_t rows = (int64_t)c.n_blocks * c.n_kv_heads * c.block_size;
  const int box_rows = std::min(c.block_size, kPrefixTile);
  CUtensorMap maps[2];
  for (int i = 0; i < 2; ++i)
    QZO_TRY(make_tmap(&maps[i], i ? c.v : c.k, F8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rows, DH, DH * (F8 ? 1 : 2),
                      F8 ? DH : 64, box_rows, F8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B));
  {
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(prefix_attention_kernel<DH, F8>, Plan::kDynamicBytes, allowed));
  }
  const int64_t tiles = most_tiles(p.R, p.groups.n, p.G);
  return launch_serving(prefix_attention_kernel<DH, F8>, dim3((unsigned)(tiles * p.Hkv * p.prefix_splits)), dim3(Plan::kThreads), Plan::kDynamicBytes, 1, st,
                        maps[0], maps[1], p, (int)tiles, p.prefix_splits + p.splits, rows, box_rows);
}

}  // namespace

int64_t prefix_ctas(int R, int n_groups, int G, int Hkv) { return most_tiles(R, n_groups, G) * Hkv; }

int prefix_splits(int R, int n_groups, int G, int Hkv, int max_len) {
  const int64_t fill = 2 * kSMs / prefix_ctas(R, n_groups, G, Hkv);
  return (int)std::max<int64_t>(1, std::min<int64_t>(fill, max_len / kPrefixLeast));
}

int launch_prefix_attention(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st) {
  const bool f8 = c.dtype == QZO_DTYPE_E4M3;
  if (c.head_dim == 128) return f8 ? run_prefix<128, true>(p, c, st) : run_prefix<128, false>(p, c, st);
  return f8 ? run_prefix<64, true>(p, c, st) : run_prefix<64, false>(p, c, st);
}

}  // namespace qzo
