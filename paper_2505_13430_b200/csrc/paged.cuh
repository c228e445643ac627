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
  int prefix_splits;                                   // of the partial results of a row's head, these come first
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
constexpr int kPrefixTile = 64;                        // keys of a tile of the prefix kernel: a prefix counts in whole ones
constexpr int kPrefixLeast = 256;                      // keys of a split of a prefix, at least

// Keys that a group's rows share; 0 where its request or its length is out of range.
__device__ __forceinline__ int group_prefix(const PagedParams& p, int group, bool report) {
  const int len = p.groups.len[group], seq = p.groups.seq[group];
  const bool bad = len < 0 || len > (p.width << p.log2_block) || (unsigned)seq >= (unsigned)p.n_seqs;
  if (bad && report && p.status) atomicOr(p.status, kStatusBadToken);
  return bad ? 0 : len / kPrefixTile * kPrefixTile;
}
// Keys of a split of a prefix
__device__ __forceinline__ int prefix_keys(const PagedParams& p, int prefix) {
  return max(kPrefixLeast, ((prefix + p.prefix_splits - 1) / p.prefix_splits + kPrefixTile - 1) / kPrefixTile * kPrefixTile);
}
// The group of a row, -1 for none.  Called by whole warps, `row` the same in all lanes.  Bounds that do not ascend within the rows
// make no groups at all.
__device__ __forceinline__ int row_group(const PagedParams& p, int row) {
  const int lane = threadIdx.x & 31;
  int at = 0;
  bool bad = false;
  for (int i0 = 0; i0 <= p.groups.n; i0 += 32) {
    const int i = i0 + lane;
    const int here = i <= p.groups.n ? p.groups.rows[i] : INT32_MAX, next = i < p.groups.n ? p.groups.rows[i + 1] : here;
    bad = bad || here > next || (i == 0 && here < 0) || (i == p.groups.n && here > p.R);
    at += __popc(__ballot_sync(0xffffffffu, here <= row));
  }
  return __any_sync(0xffffffffu, bad) || at == 0 || at > p.groups.n ? -1 : at - 1;
}
// How many of the keys that a row sees (len) the prefix kernel takes: those its group shares, or none where it does not see all of them.
__device__ __forceinline__ int row_prefix(const PagedParams& p, int row, int len) {
  const int group = row_group(p, row);
  if (group < 0) return 0;
  const int prefix = group_prefix(p, group, false);
  return len >= prefix ? prefix : 0;
}

// prefix.cu: the partial results of every group's prefix, for the rows that see all of it
int launch_prefix_attention(const PagedParams& p, const qzo_kv_cache& c, cudaStream_t st);
// CTAs of it for one split, and the splits that fill the SMs
int64_t prefix_ctas(int R, int n_groups, int G, int Hkv);
int prefix_splits(int R, int n_groups, int G, int Hkv, int max_len);

}  // namespace qzo
