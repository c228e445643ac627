// What the kernels of the paged attention share: the launch's parameters, which keys a row sees, the weights' arithmetic.
#pragma once
#include "qzo_common.cuh"

#include <math.h>

namespace qzo {

constexpr float kLog2e = 1.4426950408889634f;

// Rows rows[i] .. rows[i + 1] - 1 are group i, whose first len[i] keys are those of request seq[i].
struct PrefixGroups {
  const int32_t *rows, *seq, *len;
  int n;
};

struct PagedParams {
  const __nv_bfloat16* q;
  int ldq;
  const void *ck, *cv;
  const int32_t* table;
  int n_seqs, width;
  const int32_t *row_seq, *positions, *slots;          // slots may be null
  float scale_log2e, v_scale;                          // the keys' scale is in the first
  __nv_bfloat16* out;
  int ldo, R, H, Hkv, G, chunks, splits, min_keys, round_keys, n_blocks, log2_block;
  float *part_o, *part_ml;                             // [R][H][splits][DH], [R][H][splits][2]
  int* status;
  PrefixGroups groups;                                 // of the rows that share the beginning of their cache; none: n = 0
  int unit_items;                                      // queries of a unit of work on prefixes
  int prefix_ctas;                                     // units of 128: CTAs of the kernel on the tensor cores' line
  int prefix_splits, prefix_least;                     // smaller units: splits of each (0 where units have 128), keys of one, at least
  float *prefix_o, *prefix_ml;                         // results: [..][DH], [..][2], in the order told below
};

// Keys of split s of a row that sees len keys: [s * per, min(len, (s + 1) * per)), per at least the launch's minimum.
__device__ __forceinline__ int split_keys(const PagedParams& p, int len) {
  return max(p.min_keys, ((len + p.splits - 1) / p.splits + p.round_keys - 1) / p.round_keys * p.round_keys);
}
// Number of keys a row sees, 0 for padding; seq receives its request.  One thread reports what is out of range.
__device__ __forceinline__ int row_keys(const PagedParams& p, int row, int* seq, bool report) {
  const int pos = p.positions[row], s = p.row_seq ? p.row_seq[row] : row;
  if (pos < 0 || (p.slots && p.slots[row] < 0)) return 0;
  *seq = s;
  const int most = p.width << p.log2_block;
  const bool bad_seq = s < 0 || s >= p.n_seqs;
  if ((bad_seq || pos >= most) && report && p.status) atomicOr(p.status, kStatusBadToken);
  return bad_seq ? 0 : min(pos, most - 1) + 1;
}

// A row none of whose keys has a score above -inf (no key at all, or only blocks that are out of range) gives zeros.
__device__ __forceinline__ float inverse_sum(const PagedParams& p, float sum) { return sum == 0.0f ? 0.0f : p.v_scale / sum; }

// 2^x, relative error 2^-22, 0 for -inf
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The fp32 number next below w > 0 (0 for 0), as bits: its upper half is the largest bf16 below w
__device__ __forceinline__ uint32_t below(float w) { return (uint32_t)__viaddmax_s32(__float_as_int(w), -1, 0); }
__device__ __forceinline__ float upper_half(uint32_t bits) { return __uint_as_float(bits & 0xffff0000u); }
// What scores are taken relative to: their maximum, or 0 where there is none (all -inf).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

// ----------------------------------------------------------------------------- shared beginnings
// The work on prefixes: a unit is some queries (the rows of a group times the query heads of a key head, in that order) over the
// whole prefix of their group; units are numbered group by group, key head by key head.
// Many queries to a group: units of 128 for the tensor cores' larger instructions (prefix.cu), in tiles of 64 keys and one place more for
// what a change of units costs.  All units stand in one line, of which every CTA takes an equal stretch.
// Few: units of 8 or 16, which are to paged_attention_kernel what the heads of a row are, in splits of their keys.
// Results are as many as there are queries, whatever the units' number: query q of the line leaves what CTA c finds of it at 128 c + q (from one
// stretch to the next a unit's results move by 128, from one unit to the next by the unit's queries), or what split s does at q * splits + s.
constexpr int kPrefixQueries = 128, kPrefixTile = 64;
constexpr int kPrefixStep = 16;                        // tokens that a prefix counts in: what the rows' own kernel starts at
constexpr int kPrefixLeast = 4;                        // places of a CTA's stretch, at least
constexpr int kMostGroups = 1 << 20;                   // every row goes over all of them

struct PrefixGroup {
  int row0, rows, prefix, seq, tiles, key_tiles;       // tiles of queries of a key head, tiles of keys
  __device__ __forceinline__ int units(int Hkv) const { return key_tiles ? tiles * Hkv : 0; }
  __device__ __forceinline__ int places() const { return key_tiles + 1; }        // of a unit
};

// Place in the line of query `item` of a group's rows `row0 ..` at key head hk
__device__ __forceinline__ size_t prefix_query(const PagedParams& p, int row0, int rows, int hk, int item) {
  return (size_t)row0 * p.H + (size_t)hk * rows * p.G + item;
}
// A group; without keys where its request or its length is out of range
__device__ __forceinline__ PrefixGroup prefix_group(const PagedParams& p, int i, bool report = false) {
  const int row0 = p.groups.rows[i], end = p.groups.rows[i + 1], len = p.groups.len[i], seq = p.groups.seq[i];
  const int rows = end < row0 ? -1 : end - row0;       // negative, as row0 < 0: no bounds (differences may wrap then)
  const bool bad = len < 0 || len > (p.width << p.log2_block) || (unsigned)seq >= (unsigned)p.n_seqs;
  if (bad && report && p.status) atomicOr(p.status, kStatusBadToken);
  const int prefix = bad ? 0 : len / kPrefixStep * kPrefixStep;
  return {row0, rows, prefix, seq, (rows * p.G + p.unit_items - 1) / p.unit_items, rows > 0 ? (prefix + kPrefixTile - 1) / kPrefixTile : 0};
}
// Keys of a split of a small unit
__device__ __forceinline__ int prefix_split_keys(const PagedParams& p, int prefix) {
  return max(p.prefix_least, ((prefix + p.prefix_splits - 1) / p.prefix_splits + p.round_keys - 1) / p.round_keys * p.round_keys);
}
// The unit of this number: its group, and its number within it; false where there is none, or where the groups' bounds do not ascend within the
// rows (which is reported).  Whole warps.
__device__ __forceinline__ bool find_unit(const PagedParams& p, int number, bool report, PrefixGroup* group, int* unit) {
  const int lane = threadIdx.x & 31;
  int before = 0;
  bool bad = false, found = false;
  for (int i0 = 0; i0 < p.groups.n; i0 += 32) {
    PrefixGroup g = {};
    if (i0 + lane < p.groups.n) {
      g = prefix_group(p, i0 + lane, report);
      bad = bad || g.row0 < 0 || g.rows < 0 || g.row0 + g.rows > p.R;
    }
    const int units = g.units(p.Hkv);
    int sum = units;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += up;
    }
    const unsigned past = __ballot_sync(0xffffffffu, before + sum > number);
    if (!found && past) {
      found = true;
      const int who = __ffs(past) - 1;
      *group = {__shfl_sync(0xffffffffu, g.row0, who), __shfl_sync(0xffffffffu, g.rows, who), __shfl_sync(0xffffffffu, g.prefix, who),
                __shfl_sync(0xffffffffu, g.seq, who), __shfl_sync(0xffffffffu, g.tiles, who), __shfl_sync(0xffffffffu, g.key_tiles, who)};
      *unit = number - before - __shfl_sync(0xffffffffu, sum - units, who);
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  bad = __any_sync(0xffffffffu, bad);
  if (bad && report && lane == 0 && p.status) atomicOr(p.status, kStatusBadToken);
  return found && !bad;
}

// Places of a CTA's stretch, of `places` in all
__device__ __forceinline__ int prefix_stretch(const PagedParams& p, int places) { return max(kPrefixLeast, (places + p.prefix_ctas - 1) / p.prefix_ctas); }

// Where the results of a row's prefix are.
struct RowPrefix {
  int prefix;                                          // keys that the row's group shares; 0: no group
  int row0, rows, tiles, key_tiles, places;            // of its group
  int places_before, stretch;

  // The results of query `in_group` of the group (rows times heads of a key head) at key head hk: how many, the first one's place, and from one
  // to the next
  __device__ __forceinline__ int parts(const PagedParams& p, int hk, int in_group, size_t* first, int* step) const {
    const size_t query = prefix_query(p, row0, rows, hk, in_group);
    if (p.prefix_splits) {
      const int per = prefix_split_keys(p, prefix);
      *first = query * p.prefix_splits;
      *step = 1;
      return (prefix + per - 1) / per;
    }
    const int t0 = places_before + (hk * tiles + in_group / kPrefixQueries) * places, c0 = t0 / stretch;
    *first = query + (size_t)kPrefixQueries * c0;
    *step = kPrefixQueries;
    return (t0 + key_tiles - 1) / stretch - c0 + 1;
  }
};

// Whole warps, `row` the same in all lanes.  Bounds that do not ascend within the rows make no groups.
__device__ __forceinline__ RowPrefix row_prefix(const PagedParams& p, int row) {
  int places = 0, before = 0, prefix = 0, row0 = 0, rows = 0, tiles = 0, key_tiles = 0;
  bool bad = false, mine = false;
  for (int i = threadIdx.x & 31; i < p.groups.n; i += 32) {
    const PrefixGroup g = prefix_group(p, i);
    bad = bad || g.row0 < 0 || g.rows < 0 || g.row0 + g.rows > p.R;
    const int all = g.units(p.Hkv) * g.places();
    places += all;
    if (g.row0 + g.rows <= row) {
      before += all;
    } else if (g.row0 <= row) {
      mine = true;
      prefix = g.prefix; row0 = g.row0; rows = g.rows; tiles = g.tiles; key_tiles = g.key_tiles;
    }
  }
  RowPrefix r = {};
  const unsigned who = __ballot_sync(0xffffffffu, mine);
  bad = __any_sync(0xffffffffu, bad);
  places = __reduce_add_sync(0xffffffffu, places);
  r.places_before = __reduce_add_sync(0xffffffffu, before);
  if (bad || !who) return r;
  const int lane = __ffs(who) - 1;
  r.prefix = __shfl_sync(0xffffffffu, prefix, lane);
  r.row0 = __shfl_sync(0xffffffffu, row0, lane);
  r.rows = __shfl_sync(0xffffffffu, rows, lane);
  r.tiles = __shfl_sync(0xffffffffu, tiles, lane);
  r.key_tiles = __shfl_sync(0xffffffffu, key_tiles, lane);
  r.places = r.key_tiles + 1;
  r.stretch = prefix_stretch(p, places);
  return r;
}

// prefix.cu: the results of every group's prefix, for the rows that see all of it, and their join with those of the rows' own keys
int launch_prefix_attention(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st);
int launch_prefix_join(const PagedParams& p, int dh, cudaStream_t st);
int64_t prefix_units(int R, int n_groups, int G, int Hkv, int items);      // at most

}  // namespace qzo
