// The paged key-value cache of the serving path: head norms, rotation and cache write in one pass over the new rows, and
// the attention of one new token per row over the cache.
#include "qzo_common.cuh"
#include "launch.cuh"
#include "layers.cuh"
#include "mma.cuh"

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>

#include <algorithm>

namespace qzo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// =========================================================================================
// Head norms, rotation, cache write
// =========================================================================================

struct RopeCacheParams {
  const __nv_bfloat16 *q, *k, *v;
  int ldq, ldk, ldv;
  const float *q_gain, *k_gain;
  float norm_eps;
  const float* table;
  int max_pos;
  const int32_t *positions, *slots;
  __nv_bfloat16* q_out;
  int ldqo;
  void *ck, *cv;
  float inv_k_scale, inv_v_scale;
  int n_slots, log2_block, H, Hkv, T;
  int rows, parts, part_groups;     // rows of a CTA, or CTAs of a row; groups of lanes of a row in a CTA
  int* status;
};

__device__ __forceinline__ void unpack4(uint2 r, float v[4]) {
  const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.x));
  const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&r.y));
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ uint2 pack4_bf16(const float v[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ uint4 pack8_bf16(const float v[8]) {
  const uint2 a = pack4_bf16(v), b = pack4_bf16(v + 4);
  return make_uint4(a.x, a.y, b.x, b.y);
}
// Codes of v times the scale's fp32 reciprocal: that product is off from v / scale by 2^-23 of it, which shows only where v / scale is
// as near to the middle between two codes (divisions: 4099 rows with norms 26.2 us instead of 22.5, 4096 rows of 32 + 32 heads
// 45.2 instead of 34.7).
__device__ __forceinline__ uint32_t pack4_e4m3(const float v[4], float inv) {
  const __nv_fp8x2_storage_t a = __nv_cvt_float2_to_fp8x2(make_float2(v[0] * inv, v[1] * inv), __NV_SATFINITE, __NV_E4M3);
  const __nv_fp8x2_storage_t b = __nv_cvt_float2_to_fp8x2(make_float2(v[2] * inv, v[3] * inv), __NV_SATFINITE, __NV_E4M3);
  return (uint32_t)a | ((uint32_t)b << 16);
}
__device__ __forceinline__ uint2 pack8_e4m3(const float v[8], float inv) { return make_uint2(pack4_e4m3(v, inv), pack4_e4m3(v + 4, inv)); }

// Eight consecutive floats, 32-byte aligned, of data that no kernel in flight writes: one load instead of two, which asks the
// L1 for every line once
struct Floats8 { float v[8]; };
__device__ __forceinline__ Floats8 load8(const float* p) {
  Floats8 r;
  asm volatile("ld.global.nc.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r.v[0]), "=f"(r.v[1]), "=f"(r.v[2]), "=f"(r.v[3]), "=f"(r.v[4]), "=f"(r.v[5]), "=f"(r.v[6]), "=f"(r.v[7])
               : "l"(p));
  return r;
}

// DH / 16 lanes per pair of neighbouring heads; a lane holds elements 8 l .. 8 l + 7 of a head's lower half and their
// partners of the upper half (a 16-byte load each), so a pair of elements is turned inside a lane and the norm's sum takes
// log2(DH / 16) shuffles.  Two heads to a lane: they share the angles, and twice the bytes are in flight.  A CTA holds whole
// rows where they are short, part of a row's heads where they are long.
// Measured: 4096 rows of 32 + 32 heads of 128, bf16: 36.4 us, 5.6 TB/s (HBM); 4099 rows of 32 + 8 heads with norms and e4m3 pages
// 22.5 us, 4.2 TB/s (latency: the angles wait for the position, 66 registers leave 27 warps on an SM, a scheduler issues 0.6
// instructions a cycle); with 16-byte loads of angles and gains 23.4 us (every line is then asked for two to four times); one row
// 1.8 us (a launch and two dependent loads).
constexpr int kRopeThreads = 128, kLaneHeads = 2;

template <int DH, bool F8>
__global__ void __launch_bounds__(kRopeThreads)
qk_norm_rope_cache_kernel(RopeCacheParams p) {
  constexpr int LPH = DH / 16;
  const int l = threadIdx.x % LPH, group = threadIdx.x / LPH, heads = p.H + 2 * p.Hkv;
  int t, first;                                        // this lane's row, and its first head among queries, keys and values
  if (p.parts == 1) {
    const int row = group / p.part_groups;
    t = row < p.rows ? blockIdx.x * p.rows + row : p.T;
    first = kLaneHeads * (group - row * p.part_groups);
  } else {
    t = group < p.part_groups ? blockIdx.x / p.parts : p.T;
    first = kLaneHeads * (blockIdx.x % p.parts * p.part_groups + group);
  }
  serving_begin();
  serving_next();
  // the row's elements are on their way before it is known whether it is padding (they are not used then)
  int slot = -1, given = 0;
  uint4 lo_raw[kLaneHeads] = {}, hi_raw[kLaneHeads] = {};
  if (t < p.T) {
    slot = p.slots[t];
    given = p.positions[t];
#pragma unroll
    for (int i = 0; i < kLaneHeads; ++i) {
      const int hh = first + i;
      if (hh >= heads) continue;
      const __nv_bfloat16* src = hh < p.H ? p.q + (size_t)t * p.ldq + hh * DH
                               : hh < p.H + p.Hkv ? p.k + (size_t)t * p.ldk + (hh - p.H) * DH
                                                  : p.v + (size_t)t * p.ldv + (hh - p.H - p.Hkv) * DH;
      lo_raw[i] = *reinterpret_cast<const uint4*>(src + 8 * l);
      hi_raw[i] = *reinterpret_cast<const uint4*>(src + DH / 2 + 8 * l);
    }
  }
  const bool work = slot >= 0 && given >= 0;           // lanes of padding go along for the shuffles only
  Floats8 cs[2];                                       // {cos, sin} of four pairs each
  if (p.table && work && first < p.H + p.Hkv) {
    const int pos = min(given, p.max_pos - 1);
    if (pos != given && l == 0 && p.status) atomicOr(p.status, kStatusBadToken);
    const float* row = p.table + 2 * ((size_t)pos * (DH / 2) + 8 * l);
    cs[0] = load8(row);
    cs[1] = load8(row + 8);
  }
  const bool writes = work && slot < p.n_slots;
  if (work && !writes && l == 0 && first == 0 && p.status) atomicOr(p.status, kStatusBadToken);
  const size_t block_row = (size_t)((unsigned)slot >> p.log2_block) * p.Hkv, in_block = slot & ((1 << p.log2_block) - 1);

  float root[kLaneHeads];                              // 1 / rms of the heads
  if (p.q_gain || p.k_gain) {                          // uniform: the shuffles need every lane
#pragma unroll
    for (int i = 0; i < kLaneHeads; ++i) {
      const uint32_t w[8] = {lo_raw[i].x, lo_raw[i].y, lo_raw[i].z, lo_raw[i].w, hi_raw[i].x, hi_raw[i].y, hi_raw[i].z, hi_raw[i].w};
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]));
        ss += f.x * f.x + f.y * f.y;
      }
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      root[i] = rsqrtf(ss * (1.0f / DH) + p.norm_eps);
    }
  }
#pragma unroll
  for (int i = 0; i < kLaneHeads; ++i) {
    const int hh = first + i;
    const bool is_q = hh < p.H, is_v = hh >= p.H + p.Hkv;
    float lo[8], hi[8];
    unpack4(make_uint2(lo_raw[i].x, lo_raw[i].y), lo); unpack4(make_uint2(lo_raw[i].z, lo_raw[i].w), lo + 4);
    unpack4(make_uint2(hi_raw[i].x, hi_raw[i].y), hi); unpack4(make_uint2(hi_raw[i].z, hi_raw[i].w), hi + 4);
    const float* gain = is_v ? nullptr : is_q ? p.q_gain : p.k_gain;
    if (gain) {
      const Floats8 ga = load8(gain + 8 * l), gb = load8(gain + DH / 2 + 8 * l);
      const float r = root[i];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] *= r * ga.v[e];
        hi[e] *= r * gb.v[e];
      }
    }
    if (!work || hh >= heads) continue;
    if (p.table && !is_v) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* c = cs[e >> 1].v + 4 * (e & 1);
        const float x0 = lo[2 * e], y0 = hi[2 * e], x1 = lo[2 * e + 1], y1 = hi[2 * e + 1];
        lo[2 * e] = x0 * c[0] - y0 * c[1];
        hi[2 * e] = y0 * c[0] + x0 * c[1];
        lo[2 * e + 1] = x1 * c[2] - y1 * c[3];
        hi[2 * e + 1] = y1 * c[2] + x1 * c[3];
      }
    }
    if (is_q) {
      __nv_bfloat16* dst = p.q_out + (size_t)t * p.ldqo + hh * DH + 8 * l;
      *reinterpret_cast<uint4*>(dst) = pack8_bf16(lo);
      *reinterpret_cast<uint4*>(dst + DH / 2) = pack8_bf16(hi);
      continue;
    }
    if (!writes) continue;
    const int h = is_v ? hh - p.H - p.Hkv : hh - p.H;
    const size_t at = (((block_row + h) << p.log2_block) + in_block) * DH + 8 * l;
    if (F8) {
      uint8_t* dst = (uint8_t*)(is_v ? p.cv : p.ck) + at;
      const float inv = is_v ? p.inv_v_scale : p.inv_k_scale;
      *reinterpret_cast<uint2*>(dst) = pack8_e4m3(lo, inv);
      *reinterpret_cast<uint2*>(dst + DH / 2) = pack8_e4m3(hi, inv);
    } else {
      __nv_bfloat16* dst = (__nv_bfloat16*)(is_v ? p.cv : p.ck) + at;
      *reinterpret_cast<uint4*>(dst) = pack8_bf16(lo);
      *reinterpret_cast<uint4*>(dst + DH / 2) = pack8_bf16(hi);
    }
  }
}

// =========================================================================================
// Attention of one new token per row
// =========================================================================================

constexpr int kStageBytes = 8192;                      // of a warp's ring: 4 KB of keys and 4 KB of values
constexpr int kSub = 16;                               // keys of one matrix tile; a block of the cache holds whole ones

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
// four codes as two fp16 pairs (exact)
__device__ __forceinline__ void e4m3x4_to_f16x2(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(four));
}

// What one lane holds of a key row: the row's 16-byte units t, t + 4, ... in order, as words of two elements; of a value row
// the units that belong to lane g.  8-bit codes become fp16 pairs, which hold them exactly.
template <int DH, bool F8>
struct Layout {
  static constexpr int kRowBytes = DH * (F8 ? 1 : 2);
  static constexpr int kKeyLoads = kRowBytes / 64;                       // 16-byte loads a lane of four makes
  static constexpr int kKeyWords = DH / 8;                               // element pairs of a lane: DH / 4 elements
  static constexpr int kKeyStep = F8 ? 16 : 8;                           // elements of a load
  static constexpr int kValWords = DH / 16;                              // element pairs of one of eight lanes
  static constexpr int kSubs = 256 / kRowBytes;                          // matrix tiles a warp takes at a time: 4 KB of keys, 4 KB of values
  static constexpr int kTileKeys = kSub * kSubs;
  static constexpr int kValBytes = kRowBytes == 64 ? 8 : 16;             // bytes of a load of one of eight lanes
};

// Where unit c (16 bytes) of a tile's row stands: c ^ swizzle(row), so that the eight lanes of a phase (two g, four t) that read
// keys (rows g, units t) or values (rows 2t, units g) read eight different 16-byte banks.
template <int UNITS>
__device__ __forceinline__ int key_swizzle(int row) { return UNITS >= 8 ? 4 * (row & 1) : 0; }
template <int UNITS>
__device__ __forceinline__ int val_swizzle(int row) { return UNITS >= 8 ? 2 * ((row >> 1) & 3) : (row >> 1) & 3; }

template <int DH, bool F8>
__device__ __forceinline__ void key_words(const uint4 raw[Layout<DH, F8>::kKeyLoads], uint32_t w[Layout<DH, F8>::kKeyWords]) {
#pragma unroll
  for (int j = 0; j < Layout<DH, F8>::kKeyLoads; ++j) {
    const uint32_t r[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (F8) {
        e4m3x4_to_f16x2(r[i], w[8 * j + 2 * i], w[8 * j + 2 * i + 1]);
      } else {
        w[4 * j + i] = r[i];
      }
    }
  }
}
// Value words of lane g: element e of the list is dimension val_dim(g, e)
template <int DH, bool F8>
__device__ __forceinline__ int val_dim(int g, int e) {
  if (!F8 && DH == 128) return (e & 7) + 8 * g + (e >> 3) * 64;
  return (DH / 8) * g + e;
}
template <int DH, bool F8>
struct ValRaw { uint32_t w[DH * (F8 ? 1 : 2) / 32]; };

// what lane g has of a value row, from the tile at `tile` in shared memory
template <int DH, bool F8>
__device__ __forceinline__ void read_val(uint32_t tile, int row, int g, ValRaw<DH, F8>& raw) {
  constexpr int kUnits = Layout<DH, F8>::kRowBytes / 16;
  if (Layout<DH, F8>::kValBytes == 8) {
    const uint2 v = lds8(tile + 16 * (row * kUnits + ((g >> 1) ^ val_swizzle<kUnits>(row))) + 8 * (g & 1));
    raw.w[0] = v.x; raw.w[1] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < Layout<DH, F8>::kRowBytes / 128; ++j) {
      const uint4 v = lds16(tile + 16 * (row * kUnits + ((g + 8 * j) ^ val_swizzle<kUnits>(row))));
      raw.w[4 * j] = v.x; raw.w[4 * j + 1] = v.y; raw.w[4 * j + 2] = v.z; raw.w[4 * j + 3] = v.w;
    }
  }
}
// Words u, u + 1 of keys a and b (keys 2t, 2t + 1 of a half tile): the fragments of elements 2u .. 2u + 3, each the pair
// (a, b) of one dimension.  8-bit codes are paired first and converted as pairs.
template <int DH, bool F8>
__device__ __forceinline__ void val_pairs(const ValRaw<DH, F8>& a, const ValRaw<DH, F8>& b, int u, uint32_t f[4]) {
  if (F8) {
    const uint32_t x = a.w[u / 2], y = b.w[u / 2];
    e4m3x4_to_f16x2(__byte_perm(x, y, 0x5140), f[0], f[1]);
    e4m3x4_to_f16x2(__byte_perm(x, y, 0x7362), f[2], f[3]);
  } else {
    const uint32_t x0 = a.w[u], x1 = a.w[F8 ? 0 : u + 1], y0 = b.w[u], y1 = b.w[F8 ? 0 : u + 1];
    f[0] = __byte_perm(x0, y0, 0x5410);
    f[1] = __byte_perm(x0, y0, 0x7632);
    f[2] = __byte_perm(x1, y1, 0x5410);
    f[3] = __byte_perm(x1, y1, 0x7632);
  }
}
template <bool F8>
__device__ __forceinline__ void mma_step(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (F8) mma16816_f16(c, a0, a1, a2, a3, b0, b1);
  else mma16816_bf16(c, a0, a1, a2, a3, b0, b1);
}

template <bool F16>
__device__ __forceinline__ uint32_t pack_pair(float a, float b) {
  if (F16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The fp32 number next below w > 0 (0 for 0), as bits: its upper half is the largest bf16 below w
__device__ __forceinline__ uint32_t below(float w) { return (uint32_t)__viaddmax_s32(__float_as_int(w), -1, 0); }
__device__ __forceinline__ float upper_half(uint32_t bits) { return __uint_as_float(bits & 0xffff0000u); }
// What scores are taken relative to: their maximum, or 0 where there is none (all -inf).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

// A weight is 2^(score - reference), the reference being the maximum so far less lift().  The maximum is only raised when a score
// passes it by kSlack: until then a tile needs neither the maximum over its keys nor a rescaling, and weights that reach 2^8
// cost no precision.  Where weights become fp16 they are lifted, and those below 2^-kUnder, where fp16 has no more relative steps,
// are raised by 2^kBoost for a product of their own.
constexpr float kSlack = 8.0f, kUnder = 14.0f, kBoost = 29.0f, kUnboost = 0x1p-29f;
template <bool F8> __host__ __device__ constexpr float lift() { return F8 ? 6.0f : 0.0f; }
template <bool F8> __device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m - lift<F8>(); }

// Stages of a ring and CTAs of four warps on an SM, for NT tiles of eight heads: three CTAs with two stages each where their
// registers allow it, two with three stages otherwise (64 rows to 4096 in e4m3: 55.3 us against 58.3 with two CTAs; 16 rows of
// 8192 keys, 24 heads on one: 14.6 us, with three 17.2 when two took 13.9).
__host__ __device__ constexpr int resident_ctas(int NT) { return NT == 1 ? 3 : 2; }
__host__ __device__ constexpr int ring_stages(int NT) { return NT == 1 ? 2 : 3; }

// A CTA = one row, one key head, up to 8 NT of the query heads that share it, one split of its keys; its warps take the
// split's tiles in turn, each with its own running maximum and sum, and are joined at the end.
// A tile is two products: S^T = K Q^T (keys x heads) and O^T += V^T P^T (dimensions x heads), so up to eight heads
// share one pass and the accumulators hold no padding but the heads that are missing from a tile of eight.  The k order of the
// products is free, so a lane's 16 consecutive bytes of a key feed four k positions, and values are paired across two keys
// by byte permutes.
// Bound by HBM where CTAs run long (1 row of 131071 keys, 32 heads on 8: bf16 82.0 us, 6.5 TB/s; 16 rows of 100 to 2048 keys, 32
// key heads: 44.7 us, 6.3 TB/s; e4m3 1 row of 131071 45.9 us, 5.8 TB/s), by what a CTA needs before its first keys and after
// its last where they run short (1 row of 4096 keys, 32 key heads: 16.5 us, 4.1 TB/s).  The rings (64 KB a CTA) keep
// 190 KB in flight or in use on an SM; with the next tile in registers instead, 8 rows of 2048 keys took 51.5 us, now 42.1.
template <int DH, int NT, bool F8, int W>
__global__ void __launch_bounds__(W * 32, 4 * resident_ctas(NT) / W)
paged_attention_kernel(PagedParams p) {
  using Lay = Layout<DH, F8>;
  constexpr int kStages = ring_stages(NT);
  extern __shared__ __align__(128) float att_smem[];
  float (*sm_o)[8 * NT][DH + 1] = reinterpret_cast<float (*)[8 * NT][DH + 1]>(att_smem);
  __shared__ float sm_m[W][8 * NT], sm_l[W][8 * NT];
  __shared__ int sm_n[W][kStages][Lay::kSubs];         // keys of the tiles in the rings
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int per_row = p.Hkv * p.chunks;
  const int row = blockIdx.x / per_row, hk = blockIdx.x % per_row / p.chunks, chunk = blockIdx.x % p.chunks;
  const int head0 = hk * p.G + chunk * 8 * NT;                       // first query head of the CTA
  const int n_heads = min(8 * NT, p.G - chunk * 8 * NT);
  const int split = blockIdx.y;
  serving_begin();
  // Query fragments: the same chunks of dimensions as a key's lane t.
  uint32_t qf[NT][Lay::kKeyWords];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const bool have = nt * 8 + g < n_heads;
    const __nv_bfloat16* qr = p.q + (size_t)row * p.ldq + (size_t)(head0 + (have ? nt * 8 + g : 0)) * DH;
#pragma unroll
    for (int j = 0; j < Lay::kKeyLoads; ++j)
#pragma unroll
      for (int i = 0; i < Lay::kKeyStep / 8; ++i) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (have) v = *reinterpret_cast<const uint4*>(qr + Lay::kKeyStep * (t + 4 * j) + 8 * i);
        uint32_t* w = qf[nt] + Lay::kKeyStep / 2 * j + 4 * i;
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      }
  }
  int seq = 0;
  const int len = row_keys(p, row, &seq, threadIdx.x == 0 && split == 0 && blockIdx.x % per_row == 0);
  const int per = split_keys(p, len);
  const int k0 = split * per, k1 = min(len, k0 + per);
  if (k0 >= k1) {
    if (len == 0 && split == 0)
      for (int i = threadIdx.x; i < n_heads * DH / 8; i += W * 32)
        *reinterpret_cast<uint4*>(p.out + (size_t)row * p.ldo + (size_t)head0 * DH + 8 * i) = make_uint4(0u, 0u, 0u, 0u);
    return;
  }

  // For 8-bit keys the queries become fp16, scaled by a power of two that brings the head's largest element to [64, 128):
  // exact but for elements below 2^-23 of it, which are off by at most 2^-31 of it.
  float factor[NT][2];                                 // from products to scores in powers of two; finite, so that 0 stays 0
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    factor[nt][0] = factor[nt][1] = p.scale_log2e;
    if (F8) {
      float big = 0.0f;
#pragma unroll
      for (int i = 0; i < Lay::kKeyWords; ++i) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[nt][i]));
        big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // exponent of the largest less 6, within what both 2^e and 2^-e can hold (an infinity stays one)
      const int e = big > 0.0f ? max((int)(__float_as_uint(big) >> 23) - 127 - 6, -120) : 0;
      const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
      for (int i = 0; i < Lay::kKeyWords; ++i) {
        const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&qf[nt][i]));
        qf[nt][i] = pack_pair<true>(f.x * down, f.y * down);
      }
      factor[nt][0] = fminf(p.scale_log2e * __shfl_sync(0xffffffffu, up, 8 * t), FLT_MAX);
      factor[nt][1] = fminf(p.scale_log2e * __shfl_sync(0xffffffffu, up, 8 * t + 4), FLT_MAX);
    }
  }

  float o[NT][DH / 16][4];
  float m[NT][2], l[NT][2], ref[NT][2];                // maximum so far, sum of weights, reference
  bool fresh = true;                                   // no maximum yet for some of the heads
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -INFINITY;
    ref[nt][0] = ref[nt][1] = 0.0f;
    l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
    for (int u = 0; u < DH / 16; ++u) o[nt][u][0] = o[nt][u][1] = o[nt][u][2] = o[nt][u][3] = 0.0f;
  }
  const int32_t* pages = p.table + (size_t)seq * p.width;
  const int in_block = (1 << p.log2_block) - 1;
  // Tiles come through a ring of each warp's own in shared memory, filled by 16-byte asynchronous copies kStages - 1 tiles ahead;
  // rows behind the split's end and blocks out of range are filled with zeros.  Block ids are looked up one tile before that.
  constexpr int S = Lay::kSubs, kTileKeys = Lay::kTileKeys, kStep = W * kTileKeys, kUnits = Lay::kRowBytes / 16;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(att_smem) + warp * kStages * kStageBytes;
  int page[S];
  auto look_up = [&](int key0) {
#pragma unroll
    for (int i = 0; i < S; ++i) page[i] = key0 + kSub * i < k1 ? pages[(key0 + kSub * i) >> p.log2_block] : 0;
  };
  auto fill = [&](int key0, int slot) {
    const uint32_t stage = ring + slot * kStageBytes;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      int n = k1 - key0 - kSub * i;
      if ((unsigned)page[i] >= (unsigned)p.n_blocks) {               // uniform over the warp
        if (lane == 0 && p.status) atomicOr(p.status, kStatusBadToken);
        n = page[i] = 0;
      }
      if (lane == 0) sm_n[warp][slot][i] = n;
      const size_t at = ((((size_t)page[i] * p.Hkv + hk) << p.log2_block) + ((key0 + kSub * i) & in_block)) * Lay::kRowBytes + 16 * lane;
      const uint8_t *kp = (const uint8_t*)p.ck + at, *vp = (const uint8_t*)p.cv + at;
      const uint32_t dst = stage + i * kSub * Lay::kRowBytes;
#pragma unroll
      for (int j = 0; j < Lay::kRowBytes / 32; ++j) {                // a tile's rows lie side by side: 512 bytes at a time
        const int unit = 32 * j + lane, row = unit / kUnits, c = unit % kUnits;
        const int bytes = row < n ? 16 : 0;
        copy16_or_zero(dst + 16 * (row * kUnits + (c ^ key_swizzle<kUnits>(row))), kp + 512 * j, bytes);
        copy16_or_zero(dst + kStageBytes / 2 + 16 * (row * kUnits + (c ^ val_swizzle<kUnits>(row))), vp + 512 * j, bytes);
      }
    }
  };
  int key0 = k0 + warp * kTileKeys;
  look_up(key0);
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    if (key0 + s * kStep < k1) fill(key0 + s * kStep, s);
    copies_commit();
    look_up(key0 + (s + 1) * kStep);
  }
  int use = 0, free_stage = kStages - 1;
  for (; key0 < k1; key0 += kStep) {
    copies_wait<kStages - 2>();
    __syncwarp();                                      // the tile has landed, and every lane is done with the one before it
    if (key0 + (kStages - 1) * kStep < k1) fill(key0 + (kStages - 1) * kStep, free_stage);
    copies_commit();
    look_up(key0 + kStages * kStep);
    const uint32_t stage = ring + use * kStageBytes;
    int n_keys[S];
    bool full = true;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      n_keys[i] = sm_n[warp][use][i];
      full = full && n_keys[i] >= kSub;
    }
    float sc[NT][S][4];
#pragma unroll
    for (int i = 0; i < S; ++i) {
      uint4 raw[2][Lay::kKeyLoads];
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < Lay::kKeyLoads; ++j)
          raw[r][j] = lds16(stage + 16 * (i * kSub * kUnits + (g + 8 * r) * kUnits + ((t + 4 * j) ^ key_swizzle<kUnits>(g))));
      uint32_t ka[Lay::kKeyWords], kb[Lay::kKeyWords];
      key_words<DH, F8>(raw[0], ka);
      key_words<DH, F8>(raw[1], kb);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        sc[nt][i][0] = sc[nt][i][1] = sc[nt][i][2] = sc[nt][i][3] = 0.0f;
#pragma unroll
        for (int w = 0; w < Lay::kKeyWords; w += 2)
          mma_step<F8>(sc[nt][i], ka[w], kb[w], ka[w + 1], kb[w + 1], qf[nt][w], qf[nt][w + 1]);
      }
    }
    bool odd = fresh;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float f0 = factor[nt][0], f1 = factor[nt][1];
      float most0 = -INFINITY, most1 = -INFINITY, least0 = INFINITY, least1 = INFINITY;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float (&s)[4] = sc[nt][i];
        s[0] *= f0; s[1] *= f1; s[2] *= f0; s[3] *= f1;
        most0 = fmaxf(most0, fmaxf(s[0], s[2]));
        most1 = fmaxf(most1, fmaxf(s[1], s[3]));
        least0 = fminf(least0, fminf(s[0], s[2]));
        least1 = fminf(least1, fminf(s[1], s[3]));
        if (!full) {                                   // rows of zeros behind the last key: they may make a tile odd, no more
          if (g >= n_keys[i]) s[0] = s[1] = -INFINITY;
          if (g + 8 >= n_keys[i]) s[2] = s[3] = -INFINITY;
        }
      }
      constexpr float kOver = kSlack + lift<F8>();
      odd = odd || most0 > ref[nt][0] + kOver || most1 > ref[nt][1] + kOver;
      if (F8) odd = odd || least0 < ref[nt][0] - kUnder || least1 < ref[nt][1] - kUnder;
    }
    // the tile's weights, as they enter the product with the values, and that product
    constexpr int kParts = F8 ? 1 : 2;
    uint32_t pb[kParts][NT][S][2];
    auto add_values = [&]() {
#pragma unroll
      for (int i = 0; i < S; ++i) {
        ValRaw<DH, F8> vraw[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          read_val<DH, F8>(stage + kStageBytes / 2 + i * kSub * Lay::kRowBytes, 2 * t + (r & 1) + 8 * (r >> 1), g, vraw[r]);
#pragma unroll
        for (int u = 0; u < Lay::kValWords; u += 2) {
          uint32_t lo[4], hi[4];
          val_pairs<DH, F8>(vraw[0], vraw[1], u, lo);
          val_pairs<DH, F8>(vraw[2], vraw[3], u, hi);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
              mma_step<F8>(o[nt][u], lo[0], lo[1], hi[0], hi[1], pb[part][nt][i][0], pb[part][nt][i][1]);
              mma_step<F8>(o[nt][u + 1], lo[2], lo[3], hi[2], hi[3], pb[part][nt][i][0], pb[part][nt][i][1]);
            }
        }
      }
    };
    if (__any_sync(0xffffffffu, odd)) {
      fresh = false;
      bool low = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int i = 0; i < S; ++i) {
          mx0 = fmaxf(mx0, fmaxf(sc[nt][i][0], sc[nt][i][2]));
          mx1 = fmaxf(mx1, fmaxf(sc[nt][i][1], sc[nt][i][3]));
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
          mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
        }
        mx0 = fmaxf(mx0, m[nt][0]);
        mx1 = fmaxf(mx1, m[nt][1]);
        // from one reference to the next: for the largest scores they are not the maxima less the lift to the bit.  Before the first
        // score above -inf there is nothing to rescale.
        const float to0 = reference<F8>(mx0), to1 = reference<F8>(mx1);
        const float corr0 = m[nt][0] == -INFINITY ? 0.0f : fast_exp2(ref[nt][0] - to0);
        const float corr1 = m[nt][1] == -INFINITY ? 0.0f : fast_exp2(ref[nt][1] - to1);
        m[nt][0] = mx0; m[nt][1] = mx1;
        ref[nt][0] = to0; ref[nt][1] = to1;
        l[nt][0] *= corr0; l[nt][1] *= corr1;
#pragma unroll
        for (int u = 0; u < DH / 16; ++u) { o[nt][u][0] *= corr0; o[nt][u][2] *= corr0; o[nt][u][1] *= corr1; o[nt][u][3] *= corr1; }
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) low = low || (sc[nt][i][e] - ref[nt][e & 1] < -kUnder && sc[nt][i][e] > -INFINITY);
        fresh = fresh || mx0 == -INFINITY || mx1 == -INFINITY;
      }
      // Small weights of 8-bit pages go through the product by themselves: the sums so far are raised by the same power of two as
      // they, and lowered after (exact: they stay under 2^53 2^29).  fp16 holds them to 2^-11 down to 2^-49 of the largest, and
      // 2^-60 of it is as good as nothing.  (64 rows of 1 to 4096 keys: 60.5 us where every tile has some, 51.3 where none has.)
      if (F8 && __any_sync(0xffffffffu, low)) {
        auto scale_sums = [&](float by) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int u = 0; u < DH / 16; ++u)
#pragma unroll
              for (int e = 0; e < 4; ++e) o[nt][u][e] *= by;
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < S; ++i) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float& s = sc[nt][i][e];
              const bool small = s - ref[nt][e & 1] < -kUnder;
              w[e] = small ? fast_exp2(s - ref[nt][e & 1] + kBoost) : 0.0f;
              l[nt][e & 1] += w[e] * kUnboost;
              if (small) s = -INFINITY;                // done with
            }
            pb[0][nt][i][0] = transpose8x8(pack_pair<F8>(w[0], w[1]));
            pb[0][nt][i][1] = transpose8x8(pack_pair<F8>(w[2], w[3]));
          }
        scale_sums(1.0f / kUnboost);
        add_values();
        scale_sums(kUnboost);
      }
    }
    // The weights of a tile in the values' type.  fp16 holds them to 2^-11, an eighth of what the output's own rounding adds (a second
    // fp16 with the rest: 64 rows of 1 to 4096 keys 53.1 us when one took 51.2, 40 rows with heads of 64 25.9 when one took 23.5); bf16 only
    // to 2^-8, as much as that rounding, so there they are the sum of two bf16, both above zero for a weight above zero, so that
    // an infinite value stays one: the first is the largest bf16 below the weight, the second the rest, off by 2^-15 in all.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float (&s)[4] = sc[nt][i];
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = fast_exp2(s[e] - ref[nt][e & 1]);
        l[nt][0] += s[0] + s[2];
        l[nt][1] += s[1] + s[3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (F8) {
            pb[0][nt][i][h] = transpose8x8(pack_pair<F8>(s[2 * h], s[2 * h + 1]));
          } else {
            const uint32_t a = below(s[2 * h]), b = below(s[2 * h + 1]);
            pb[0][nt][i][h] = transpose8x8(__byte_perm(a, b, 0x7632));
            pb[kParts - 1][nt][i][h] = transpose8x8(pack_pair<F8>(s[2 * h] - upper_half(a), s[2 * h + 1] - upper_half(b)));
          }
        }
      }
    add_values();
    use = use + 1 == kStages ? 0 : use + 1;
    free_stage = free_stage + 1 == kStages ? 0 : free_stage + 1;
  }

  serving_next();                      // not earlier: CTAs that wait take room from those that load (83.6 us, 86.1 us if at the start)
  __syncthreads();                     // the rings are free: the warps' results go there
  // join the warps
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l[nt][0] += __shfl_xor_sync(0xffffffffu, l[nt][0], d);
      l[nt][1] += __shfl_xor_sync(0xffffffffu, l[nt][1], d);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int h = nt * 8 + 2 * t + i;
      if (h >= n_heads) continue;
      if (g == 0) { sm_m[warp][h] = m[nt][i] == -INFINITY ? -INFINITY : ref[nt][i]; sm_l[warp][h] = l[nt][i]; }
#pragma unroll
      for (int u = 0; u < DH / 16; ++u) {
        sm_o[warp][h][val_dim<DH, F8>(g, 2 * u)] = o[nt][u][i];
        sm_o[warp][h][val_dim<DH, F8>(g, 2 * u + 1)] = o[nt][u][2 + i];
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_heads * (DH / 4); i += W * 32) {
    const int h = i / (DH / 4), d = i % (DH / 4) * 4;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) mx = fmaxf(mx, sm_m[w][h]);
    const float ref = finite_max(mx);
    float sum = 0.0f, val[4] = {};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float c = fast_exp2(sm_m[w][h] - ref);
      sum = fmaf(c, sm_l[w][h], sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) val[e] = fmaf(c, sm_o[w][h][d + e], val[e]);
    }
    if (len <= per) {                                  // one split: nothing to join
      const float f = inverse_sum(p, sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) val[e] *= f;
      *reinterpret_cast<uint2*>(p.out + (size_t)row * p.ldo + (size_t)(head0 + h) * DH + d) = pack4_bf16(val);
    } else {
      const size_t at = ((size_t)row * p.H + head0 + h) * p.splits + split;
      *reinterpret_cast<float4*>(p.part_o + at * DH + d) = make_float4(val[0], val[1], val[2], val[3]);
      if (d == 0) *reinterpret_cast<float2*>(p.part_ml + 2 * at) = make_float2(mx, sum);
    }
  }
}

// Joins the splits of a row's head: a CTA's COLS columns of threads take four dimensions each, its ROWS rows of threads
// every so many of the splits; the rows are then summed in their order.  COLS * 4 < DH: several CTAs share a head.
template <int DH, int COLS, int ROWS>
__global__ void __launch_bounds__(COLS * ROWS)
paged_join_kernel(PagedParams p) {
  constexpr int kThreads = COLS * ROWS, kParts = DH / 4 / COLS;
  extern __shared__ float weight[];                    // [splits]
  __shared__ float4 part[ROWS][COLS];
  __shared__ float part_sum[ROWS], part_max[kThreads / 32];
  serving_begin();
  serving_next();
  const int64_t item = blockIdx.x / kParts;
  const int row = (int)(item / p.H), h = (int)(item % p.H);
  int seq = 0;
  const int len = row_keys(p, row, &seq, false);
  const int per = split_keys(p, len), n = (len + per - 1) / per;
  if (n <= 1) return;                                  // written already
  const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + item * p.splits;
  float mx = -INFINITY;
  for (int s = threadIdx.x; s < n; s += kThreads) mx = fmaxf(mx, ml[s].x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
  if ((threadIdx.x & 31) == 0) part_max[threadIdx.x >> 5] = mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) mx = fmaxf(mx, part_max[w]);
  const float ref = finite_max(mx);
  for (int s = threadIdx.x; s < n; s += kThreads) weight[s] = fast_exp2(ml[s].x - ref);
  __syncthreads();
  const int c = threadIdx.x % COLS, r = threadIdx.x / COLS, d0 = 4 * (c + COLS * (blockIdx.x % kParts));
  const float4* o = reinterpret_cast<const float4*>(p.part_o + item * p.splits * DH + d0);
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float sum = 0.0f;
#pragma unroll 4
  for (int s = r; s < n; s += ROWS) {
    const float w = weight[s];
    const float4 x = o[(size_t)s * (DH / 4)];
    v.x = fmaf(w, x.x, v.x); v.y = fmaf(w, x.y, v.y); v.z = fmaf(w, x.z, v.z); v.w = fmaf(w, x.w, v.w);
    sum = fmaf(w, ml[s].y, sum);
  }
  part[r][c] = v;
  if (c == 0) part_sum[r] = sum;
  __syncthreads();
  if (r > 0) return;
#pragma unroll
  for (int i = 1; i < ROWS; ++i) {
    const float4 x = part[i][c];
    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    sum += part_sum[i];
  }
  const float f = inverse_sum(p, sum);
  const float out[4] = {v.x * f, v.y * f, v.z * f, v.w * f};
  *reinterpret_cast<uint2*>(p.out + (size_t)row * p.ldo + (size_t)h * DH + d0) = pack4_bf16(out);
}

int log2_of(int v) {
  int n = 0;
  while ((1 << n) < v) ++n;
  return n;
}

int head_chunks(int G) { return G <= 8 ? 1 : (G + 15) / 16; }      // CTAs that share a key head's query heads

// How a launch divides its work.  `subs`: matrix tiles that make up 4 KB of keys (1 for 128 dimensions of bf16).
struct Plan { int splits, wide, min_keys; };

Plan attention_plan(int64_t R, int Hkv, int G, int subs, int64_t max_len) {
  const int chunks = head_chunks(G), head_tiles = G <= 8 ? 1 : 2;
  const int64_t ctas = R * Hkv * chunks;                     // without splits
  // At most one CTA per SM and a short cache: CTAs of eight warps and no split, which saves the join's launch.  Measured
  // (heads of 128, bf16; us): 1 row of 256 keys over 32 key heads 4.9 against 7.0, of 768 8.0 against 8.3, of 1024 9.5 against
  // 8.9; 4 rows of 512 8.4 against 11.0, of 1536 18.3 against 20.5.
  if (ctas <= kSMs && max_len <= (ctas <= kSMs / 2 ? 768 : 2048) * subs) return {1, 1, 0};
  // Few CTAs: as many splits as fill the SMs once, but none shorter than 128 keys (1 row of 4096 keys over 32 key heads: 17.1 us
  // with 13 splits, 18.1 with 9, 20.9 with 18).  More rows: pieces of 2048 keys, so that a long row among short ones does not
  // outlast them, as long as the grid stays within eight times what the SMs hold (16 rows of 100 to 2048 keys, 32 key heads: 44.7
  // us; with pieces of 512 keys 47.5, of 1024 47.3; 8 rows of 2048 41.6, 48.3 and 52.1).  The length follows key heads that are
  // not shared, as in this library's models; shorter pieces suit batches over few key heads better (64 rows of 1 to 4096 over 8:
  // 92.5 us, with 512 keys 88.6, of 1024 89.3).  All of this goes by the table's width, the longest a row may be: the rows' own
  // lengths are known on the device only.
  const int64_t slots = kSMs * resident_ctas(head_tiles);
  const int64_t fill = std::min<int64_t>(slots / ctas, max_len / (128 * subs));
  const int64_t even = R > 1 ? std::min<int64_t>(max_len / (2048 * subs), 8 * slots / ctas) : 1;
  return {(int)std::max<int64_t>(1, std::max(fill, even)), 0, (even > fill ? 2048 : 128) * subs};
}
template <int DH, int NT, bool F8, int W>
int run_attention_w(const PagedParams& p, cudaStream_t st) {
  const dim3 grid((unsigned)((int64_t)p.R * p.Hkv * p.chunks), p.splits);
  constexpr int smem = std::max(W * ring_stages(NT) * kStageBytes, W * 8 * NT * (DH + 1) * (int)sizeof(float));
  {
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(paged_attention_kernel<DH, NT, F8, W>, smem, allowed));
  }
  return launch_serving(paged_attention_kernel<DH, NT, F8, W>, grid, dim3(W * 32), smem, 1, st, p);
}

template <int DH, int COLS, int ROWS>
int run_join(const PagedParams& p, cudaStream_t st) {
  return launch_serving(paged_join_kernel<DH, COLS, ROWS>, dim3((unsigned)((int64_t)p.R * p.H * (DH / 4 / COLS))),
                                     dim3(COLS * ROWS), p.splits * sizeof(float), 1, st, p);
}

template <int DH, bool F8>
int run_attention(const PagedParams& p, bool wide, cudaStream_t st) {
  if (p.G <= 8) QZO_TRY(wide ? (run_attention_w<DH, 1, F8, 8>(p, st)) : (run_attention_w<DH, 1, F8, 4>(p, st)));
  else QZO_TRY(wide ? (run_attention_w<DH, 2, F8, 8>(p, st)) : (run_attention_w<DH, 2, F8, 4>(p, st)));
  if (p.splits <= 1) return QZO_OK;
  // many splits of few heads: a head's dimensions go to several CTAs, so that a thread adds up fewer of them
  return p.splits > 16 ? run_join<DH, 8, 32>(p, st) : run_join<DH, DH / 4, 4>(p, st);
}

}  // namespace

bool cache_ok(const qzo_kv_cache* c) {
  if (!c || !c->k || !c->v || ((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15)) return false;
  if (c->n_blocks <= 0 || c->n_kv_heads <= 0 || !block_size_ok(c->block_size)) return false;
  if ((int64_t)c->n_blocks * c->block_size > INT32_MAX) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->dtype == QZO_DTYPE_BF16) return c->k_scale == 1.0f && c->v_scale == 1.0f;
  // both a scale and its reciprocal are used, and the keys' scale times the scores': far from where fp32 ends
  auto fits = [](float v) { return v >= 0x1p-64f && v <= 0x1p64f; };
  return c->dtype == QZO_DTYPE_E4M3 && fits(c->k_scale) && fits(c->v_scale);
}

int launch_qk_norm_rope_cache(const __nv_bfloat16* q, int ldq, const __nv_bfloat16* k, int ldk, const __nv_bfloat16* v, int ldv,
                              const float* q_gain, const float* k_gain, float norm_eps, const float* table, int max_pos,
                              const int32_t* positions, const int32_t* slots, __nv_bfloat16* q_out, int ldqo,
                              const qzo_kv_cache& c, int T, int H, int* status, cudaStream_t st) {
  RopeCacheParams p{q, k, v, ldq, ldk, ldv, q_gain, k_gain, norm_eps, table, max_pos, positions, slots, q_out, ldqo, c.k, c.v,
                    1.0f / c.k_scale, 1.0f / c.v_scale, c.n_blocks * c.block_size, log2_of(c.block_size), H, c.n_kv_heads,
                    T, 1, 1, 1, status};
  const int lanes = c.head_dim / 16, groups = ceil_div(H + 2 * c.n_kv_heads, kLaneHeads);
  p.rows = std::max(1, kRopeThreads / (groups * lanes));
  p.parts = ceil_div(groups * lanes, kRopeThreads);
  p.part_groups = ceil_div(groups, p.parts);
  const int64_t ctas = p.parts == 1 ? ceil_div(T, p.rows) : (int64_t)T * p.parts;
  if (ctas > INT32_MAX) return QZO_ERR_BAD_ARG;
  const dim3 grid((unsigned)ctas), block(ceil_div(p.rows * p.part_groups * lanes, 32) * 32);
  const bool f8 = c.dtype == QZO_DTYPE_E4M3;
  auto kernel = c.head_dim == 128 ? (f8 ? qk_norm_rope_cache_kernel<128, true> : qk_norm_rope_cache_kernel<128, false>)
                                  : (f8 ? qk_norm_rope_cache_kernel<64, true> : qk_norm_rope_cache_kernel<64, false>);
  return launch_serving(kernel, grid, block, 0, 1, st, p);
}

// Workspace for either type of cache: 8-bit keys are split less.
size_t paged_attention_bytes(int R, int H, int Hkv, int dh, int max_len) {
  const int splits = attention_plan(R, Hkv, H / Hkv, 128 / dh, max_len).splits;
  return splits > 1 ? (size_t)R * H * splits * (dh + 2) * sizeof(float) : 0;
}

int launch_paged_attention(const __nv_bfloat16* q, int ldq, const qzo_kv_cache& c, const int32_t* table, int n_seqs, int width,
                           const int32_t* row_seq, const int32_t* positions, const int32_t* slots, float scale, __nv_bfloat16* out,
                           int ldo, int R, int H, void* ws, size_t ws_bytes, bool fewer_splits, int* status, cudaStream_t st) {
  const int G = H / c.n_kv_heads, chunks = head_chunks(G), max_len = width * c.block_size;
  if ((int64_t)R * c.n_kv_heads * chunks > INT32_MAX) return QZO_ERR_BAD_ARG;
  const int subs = 256 / (c.head_dim * (c.dtype == QZO_DTYPE_E4M3 ? 1 : 2));
  const Plan plan = attention_plan(R, c.n_kv_heads, G, subs, max_len);
  int splits = plan.splits;
  const size_t per_split = (size_t)R * H * (c.head_dim + 2) * sizeof(float);
  if (fewer_splits)
    splits = (int)std::max<size_t>(1, std::min<size_t>(splits, ws_bytes / per_split));
  else if (const size_t need = paged_attention_bytes(R, H, c.n_kv_heads, c.head_dim, max_len); need > 0)
    if (!ws || ws_bytes < need || ((uintptr_t)ws & 255)) return QZO_ERR_WORKSPACE;
  PagedParams p{q, ldq, c.k, c.v, table, n_seqs, width, row_seq, positions, slots, scale * kLog2e * c.k_scale, c.v_scale, out, ldo,
                R, H, c.n_kv_heads, G, chunks, splits, plan.min_keys, 64 * subs, c.n_blocks, log2_of(c.block_size), nullptr, nullptr, status};
  if (splits > 1) {
    p.part_o = (float*)ws;
    p.part_ml = p.part_o + (size_t)R * H * splits * c.head_dim;
  }
  const bool f8 = c.dtype == QZO_DTYPE_E4M3;
  if (c.head_dim == 128) return f8 ? run_attention<128, true>(p, plan.wide, st) : run_attention<128, false>(p, plan.wide, st);
  return f8 ? run_attention<64, true>(p, plan.wide, st) : run_attention<64, false>(p, plan.wide, st);
}

}  // namespace qzo

using namespace qzo;

extern "C" {

int qzo_rope_table(float* d_table, int max_pos, int head_dim, float theta, void* stream) {
  if (!d_table || max_pos <= 0 || (head_dim != 64 && head_dim != 128) || !(theta > 0.0f) || !isfinite(theta)) return QZO_ERR_BAD_ARG;
  if ((int64_t)max_pos * head_dim > (1 << 30) || ((uintptr_t)d_table & 31)) return QZO_ERR_BAD_ARG;   // as its reader asks for
  QZO_TRY(check_device());
  return launch_rope_table(d_table, max_pos, head_dim, theta, (cudaStream_t)stream);
}

int qzo_qk_norm_rope_cache(const void* d_q_bf16, int ldq, const void* d_k_bf16, int ldk, const void* d_v_bf16, int ldv,
                           const float* d_q_gain, const float* d_k_gain, float norm_eps, const float* d_table, int max_pos,
                           const int32_t* d_positions, const int32_t* d_slots, void* d_q_out_bf16, int ldqo,
                           const qzo_kv_cache* cache, int T, int n_heads, int* d_status, void* stream) {
  if (!d_q_bf16 || !d_k_bf16 || !d_v_bf16 || !d_positions || !d_slots || !d_q_out_bf16) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_positions, d_slots, d_status)) return QZO_ERR_BAD_ARG;
  if (!cache_ok(cache) || T <= 0 || n_heads <= 0 || n_heads % cache->n_kv_heads) return QZO_ERR_BAD_ARG;
  if ((d_q_gain || d_k_gain) && !(norm_eps > 0.0f)) return QZO_ERR_BAD_ARG;
  if (d_table && max_pos <= 0) return QZO_ERR_BAD_ARG;
  const int64_t wq = (int64_t)n_heads * cache->head_dim, wk = (int64_t)cache->n_kv_heads * cache->head_dim;
  if (ldq < wq || ldqo < wq || ldk < wk || ldv < wk || (ldq % 8) || (ldk % 8) || (ldv % 8) || (ldqo % 8)) return QZO_ERR_BAD_ARG;
  if (((uintptr_t)d_q_bf16 | (uintptr_t)d_k_bf16 | (uintptr_t)d_v_bf16 | (uintptr_t)d_q_out_bf16) & 15) return QZO_ERR_BAD_ARG;
  if (((uintptr_t)d_q_gain | (uintptr_t)d_k_gain | (uintptr_t)d_table) & 31) return QZO_ERR_BAD_ARG;
  if (d_q_out_bf16 == d_q_bf16 && ldq != ldqo) return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  return launch_qk_norm_rope_cache((const __nv_bfloat16*)d_q_bf16, ldq, (const __nv_bfloat16*)d_k_bf16, ldk,
                                   (const __nv_bfloat16*)d_v_bf16, ldv, d_q_gain, d_k_gain, norm_eps, d_table, max_pos, d_positions,
                                   d_slots, (__nv_bfloat16*)d_q_out_bf16, ldqo, *cache, T, n_heads, d_status, (cudaStream_t)stream);
}

int qzo_paged_attention_workspace_bytes(int R, int n_heads, int n_kv_heads, int head_dim, int max_len, size_t* bytes) {
  if (!bytes || R <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || max_len <= 0 || max_len > kMostKeys) return QZO_ERR_BAD_ARG;
  if (head_dim != 64 && head_dim != 128) return QZO_ERR_BAD_ARG;
  *bytes = paged_attention_bytes(R, n_heads, n_kv_heads, head_dim, max_len);
  return QZO_OK;
}

int qzo_paged_attention(const void* d_q_bf16, int ldq, const qzo_kv_cache* cache, const int32_t* d_block_table, int n_seqs,
                        int table_width, const int32_t* d_row_seq, const int32_t* d_positions, float scale, void* d_out_bf16,
                        int ldo, int R, int n_heads, void* d_workspace, size_t workspace_bytes, int* d_status, void* stream) {
  if (!d_q_bf16 || !d_block_table || !d_positions || !d_out_bf16) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_block_table, d_row_seq, d_positions, d_status)) return QZO_ERR_BAD_ARG;
  if (!cache_ok(cache) || R <= 0 || n_seqs <= 0 || table_width <= 0 || n_heads <= 0 || n_heads % cache->n_kv_heads) return QZO_ERR_BAD_ARG;
  if (!d_row_seq && R > n_seqs) return QZO_ERR_BAD_ARG;
  if ((int64_t)table_width * cache->block_size > kMostKeys || !(scale >= 0x1p-40f && scale <= 0x1p40f)) return QZO_ERR_BAD_ARG;
  const int64_t wq = (int64_t)n_heads * cache->head_dim;
  if (ldq < wq || ldo < wq || (ldq % 8) || (ldo % 8)) return QZO_ERR_BAD_ARG;
  if (((uintptr_t)d_q_bf16 & 15) || ((uintptr_t)d_out_bf16 & 15)) return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  return launch_paged_attention((const __nv_bfloat16*)d_q_bf16, ldq, *cache, d_block_table, n_seqs, table_width, d_row_seq, d_positions,
                                nullptr, scale, (__nv_bfloat16*)d_out_bf16, ldo, R, n_heads, d_workspace, workspace_bytes, false,
                                d_status, (cudaStream_t)stream);
}

}  // extern "C"
