// Selection of a beam search: of every request's beams and their continuations by each token of the vocabulary the W best,
// from the logits of a step.  Two kernels: the first goes over the logits once, the second joins what it found.
#include "qzo_common.cuh"
#include "launch.cuh"

#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

namespace qzo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kScanThreads = 256, kScanWarps = kScanThreads / 32;
constexpr int kLaneValues = 16;                        // logits of a thread at a time
constexpr int kTileValues = kScanThreads * kLaneValues;
constexpr uint32_t kNone = 0x007fffffu;                // order_of(-infinity): nothing below it is a candidate

struct BeamParams {
  const float* logits;
  long long ld;
  int n_rows;
  const int32_t* rows;
  const float* scores;
  const int32_t* last;
  int end_token;
  const int32_t* lengths;
  float power;
  int B, W, V, chunks, per;                            // chunks of a row, tokens of a chunk
  float2* sums;                                        // [B W][chunks]: maximum, sum of 2^((x - maximum) log2 e)
  uint2* best;                                         // [B W][chunks][W]: order_of(logit) and token, best first
  int32_t *parents, *tokens;
  float* scores_out;
  int32_t* lengths_out;
  int* status;
};

// Unsigned numbers in the order of the floats (0 is below that of every float but NaN) and back
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_order(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ unsigned long long order_of(double v) {
  const long long u = __double_as_longlong(v);
  return (unsigned long long)(u ^ ((u >> 63) | (long long)0x8000000000000000ull));
}

enum BeamKind { kBeamGone, kBeamEnded, kBeamGoesOn };
// What becomes of a beam; row receives its row of logits.  One thread reports what is out of range.
__device__ __forceinline__ BeamKind beam_kind(const BeamParams& p, int beam, int* row, bool report) {
  const float score = p.scores[beam];
  const int r = p.rows ? p.rows[beam] : beam;
  const bool ended = p.last && p.last[beam] == p.end_token;
  bool bad = !(score < INFINITY);                      // NaN too
  BeamKind kind = kBeamGone;
  if (score > -INFINITY && !bad) {
    if (ended) kind = kBeamEnded;
    else if (r >= p.n_rows) bad = true;
    else if (r >= 0) kind = kBeamGoesOn;
  }
  *row = r;
  if (bad && report && p.status) atomicOr(p.status, kStatusBadToken);
  return kind;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.0f : m; }

// One step of merging lists that are in order: each lane's head (order, token), order 0 or kNone where there is none.  Returns
// whether there was a head at all; who: the lane whose head is the best, the lowest token among equals.
__device__ __forceinline__ bool best_head(uint32_t order, uint32_t token, uint32_t* top, uint32_t* low, int* who) {
  *top = __reduce_max_sync(0xffffffffu, order);
  if (*top <= kNone) return false;
  *low = __reduce_min_sync(0xffffffffu, order == *top ? token : 0xffffffffu);
  *who = __ffs(__ballot_sync(0xffffffffu, order == *top && token == *low)) - 1;
  return true;
}

// A CTA = a chunk of a row.  One pass: every thread keeps a running maximum and sum of exponentials, every warp the W best logits
// it has met, one to a lane in order.  A logit is a candidate only if it reaches what W others are known to reach: the last of the
// warp's list, or the least, over the eight warps, of the (W / 8)-th largest of a warp's lanes' maxima, which leaves about twenty of
// the first tile's 4096 for W = 8; a candidate is put in its place by the whole warp.
// 512 beams of 50272 logits, a fifth of them ended, go by in 24.3 us (29.4 us with the second kernel), 3.4 TB/s, bound by loads that no work hides:
// warps wait for them most, the issue slots are 55 % busy with 20 instructions to a logit, as most tiles have candidates and take the whole search.  Without
// the search behind the first tile it would be 5.6 us less, without the exponentials 1.8 us.  Copies two tiles ahead into shared
// memory took 2.6 us more (three CTAs to an SM instead of five); chunks of 12, 4, 3, 2 tiles for many rows 0.0, 0.5, 1.6, 3.0 us.
// Exponentials are 2^(x c), c = log2 e in fp32: the sums' logarithm is divided by that c in the end, so that its rounding (2^-26) counts
// for a distribution's entropy only.
template <bool VEC>
__global__ void __launch_bounds__(kScanThreads)
beam_scan_kernel(BeamParams p) {
  __shared__ uint2 lists[kScanWarps][32];
  __shared__ float2 warp_sums[kScanWarps];
  __shared__ float4 values[kScanWarps][kLaneValues / 4][32];         // a tile's logits, where there are candidates among them
  __shared__ uint16_t found[kScanWarps][32 * kLaneValues];           // the candidates: number of the thread's logit, lane
  __shared__ volatile uint32_t reached[kScanWarps];    // order of a logit that ceil(W / 8) of a warp's lanes have reached
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int beam = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  serving_begin();
  int row;
  if (beam_kind(p, beam, &row, tid == 0 && chunk == 0) != kBeamGoesOn) return;
  const float* x = p.logits + (size_t)row * p.ld;
  const int t0 = chunk * p.per, t1 = min(p.V, t0 + p.per);

  uint32_t list_order = kNone, list_token = 0xffffffffu;
  uint32_t least_order = kNone, least_token = 0xffffffffu;           // the list's last entry, the W-th
  float m = -INFINITY, sum = 0.0f;
  bool bad = false;
  float v[kLaneValues];
  auto token_of = [&](int base, int i) { return VEC ? base + ((i >> 2) * kScanThreads + tid) * 4 + (i & 3) : base + i * kScanThreads + tid; };
  auto load = [&](int base, auto whole) {              // whole: the tile does not reach beyond the chunk
    if (VEC) {
#pragma unroll
      for (int i = 0; i < kLaneValues; i += 4) {
        const int t = token_of(base, i);
        if (whole.value || t + 3 < t1) {
          const float4 q = *reinterpret_cast<const float4*>(x + t);
          v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i + e] = t + e < t1 ? x[t + e] : -INFINITY;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLaneValues; ++i) {
        const int t = token_of(base, i);
        v[i] = whole.value || t < t1 ? x[t] : -INFINITY;
      }
    }
  };
  for (int base = t0; base < t1; base += kTileValues) {
    if (base + kTileValues <= t1) load(base, std::true_type{});
    else load(base, std::false_type{});
    float most, part;
    auto add_up = [&]() {
      float a = -INFINITY, b = -INFINITY;
#pragma unroll
      for (int i = 0; i < kLaneValues; i += 4) {
        a = fmaxf(a, fmaxf(v[i], v[i + 1]));
        b = fmaxf(b, fmaxf(v[i + 2], v[i + 3]));
      }
      most = fmaxf(a, b);
      const float ref = finite_max(fmaxf(m, most)), scaled = ref * kLog2e;
      float parts[4] = {};
      if (fabsf(ref) < 0x1p16f) {                      // 2^(x c - scaled); what scaled is off from ref c (2^-8 at most) comes in behind
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) parts[i & 3] += exp2_fast(fmaf(v[i], kLog2e, -scaled));
        part = ((parts[0] + parts[1]) + (parts[2] + parts[3])) * exp2_fast(-fmaf(ref, kLog2e, -scaled));
      } else {                                         // there the difference comes first
#pragma unroll
        for (int i = 0; i < kLaneValues; ++i) parts[i & 3] += exp2_fast((v[i] - ref) * kLog2e);
        part = (parts[0] + parts[1]) + (parts[2] + parts[3]);
      }
    };
    add_up();
    if (!(most < INFINITY) || part != part) {          // NaN and +inf count as a token that is not allowed
      bad = true;
#pragma unroll
      for (int i = 0; i < kLaneValues; ++i)
        if (!(v[i] < INFINITY)) v[i] = -INFINITY;
      add_up();
    }
    const float to = fmaxf(m, most);
    sum = sum * (m == -INFINITY ? 0.0f : exp2_fast((m - to) * kLog2e)) + part;
    m = to;

    uint32_t top = order_of(m + 0.0f);
    for (int r = kScanWarps; r < p.W; r += kScanWarps) {               // without the largest, as often as it takes
      const uint32_t most = __reduce_max_sync(0xffffffffu, top);
      if (lane == __ffs(__ballot_sync(0xffffffffu, top == most)) - 1) top = 0;
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) reached[warp] = top;
    if (base == t0) __syncthreads();                   // later, what another warp has not written yet is lower than it might be, no more
    else __syncwarp();
    const uint32_t floor = max(least_order, __reduce_min_sync(0xffffffffu, reached[lane % kScanWarps]));     // logits of a lower order are no candidates
    const float low = fmaxf(of_order(floor), -FLT_MAX);
    if (!__any_sync(0xffffffffu, most >= low)) continue;
    unsigned hits = 0;                                 // of this lane's logits
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) hits |= v[i] >= low ? 1u << i : 0u;
#pragma unroll
    for (int i = 0; i < kLaneValues; i += 4) values[warp][i / 4][lane] = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    int n = __popc(hits);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, n, d);
      if (lane >= d) n += up;
    }
    const int all = __shfl_sync(0xffffffffu, n, 31);
    for (n -= __popc(hits); hits; hits &= hits - 1, ++n) found[warp][n] = (uint16_t)((__ffs(hits) - 1) * 32 + lane);
    __syncwarp();
    for (int c0 = 0; c0 < all; c0 += 32) {
      uint2 mine = make_uint2(0u, 0u);
      if (c0 + lane < all) {
        const int at = found[warp][c0 + lane], i = at / 32, who = at % 32;
        const float value = reinterpret_cast<const float*>(&values[warp][i / 4][who])[i % 4];
        mine = make_uint2(order_of(value + 0.0f), (uint32_t)(token_of(base, i) + (who - lane) * (VEC ? 4 : 1)));       // -0 and +0 are one value
      }
      auto passes = [&]() { return mine.x > least_order || (mine.x == least_order && mine.y < least_token); };
      for (unsigned left = __ballot_sync(0xffffffffu, passes() && mine.x > kNone); left;) {
        const int who = __ffs(left) - 1;
        const uint32_t o = __shfl_sync(0xffffffffu, mine.x, who), t = __shfl_sync(0xffffffffu, mine.y, who);
        const int place = __popc(__ballot_sync(0xffffffffu, list_order > o || (list_order == o && list_token < t)));
        const uint32_t up_order = __shfl_up_sync(0xffffffffu, list_order, 1), up_token = __shfl_up_sync(0xffffffffu, list_token, 1);
        if (lane > place) { list_order = up_order; list_token = up_token; }
        if (lane == place) { list_order = o; list_token = t; }
        least_order = __shfl_sync(0xffffffffu, list_order, p.W - 1);
        least_token = __shfl_sync(0xffffffffu, list_token, p.W - 1);
        left &= ~(1u << who) & __ballot_sync(0xffffffffu, passes());
      }
    }
    __syncwarp();
  }
  serving_next();
  if (__any_sync(0xffffffffu, bad) && lane == 0 && p.status) atomicOr(p.status, kStatusBadToken);
  float top = m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  sum *= m == -INFINITY ? 0.0f : exp2_fast((m - top) * kLog2e);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  lists[warp][lane] = make_uint2(list_order, list_token);
  if (lane == 0) warp_sums[warp] = make_float2(top, sum);
  __syncthreads();
  if (warp) return;
  const size_t out = (size_t)beam * p.chunks + chunk;
  float wm = lane < kScanWarps ? warp_sums[lane].x : -INFINITY, ws = lane < kScanWarps ? warp_sums[lane].y : 0.0f;
  top = wm;
#pragma unroll
  for (int d = kScanWarps / 2; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  ws *= wm == -INFINITY ? 0.0f : exp2_fast((wm - top) * kLog2e);
#pragma unroll
  for (int d = kScanWarps / 2; d > 0; d >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, d);
  if (lane == 0) p.sums[out] = make_float2(top, ws);
  // the warps' lists, one to a lane
  int next = 0;
  uint2 head = lane < kScanWarps ? lists[lane][0] : make_uint2(0u, 0u), mine = make_uint2(0u, 0xffffffffu);
  for (int i = 0; i < p.W; ++i) {
    uint32_t order, token;
    int who;
    if (!best_head(head.x, head.y, &order, &token, &who)) break;
    if (lane == i) mine = make_uint2(order, token);
    if (lane == who) head = ++next < 32 ? lists[lane][next] : make_uint2(0u, 0u);
  }
  if (lane < p.W) p.best[out * p.W + lane] = mine;
}

struct BeamDynamic {                                   // of the second kernel's shared memory, for W beams
  static size_t bytes(int W, int chunks) { return (size_t)W * W * (2 * sizeof(double) + sizeof(int)) + (size_t)W * chunks * W * sizeof(uint2); }
};

// A CTA = a request, a warp = one of its beams: it joins its chunks' sums and lists, then the first warp joins the beams.  Values
// and ranks are formed in 64 bits.  A beam's list stays in the order of its logits, which is that of the ranks before they were rounded: next to
// a score of -1e9 logits that differ by less than 2^-23 have one rank.  Bound by latency: W steps of joining one after
// the other, twice (about 5 us, whatever the vocabulary).
__global__ void __launch_bounds__(1024)
beam_pick_kernel(BeamParams p) {
  extern __shared__ double pick_smem[];
  const int W = p.W, w = threadIdx.x >> 5, lane = threadIdx.x & 31, beam = blockIdx.x * W + w;
  double* const rank = pick_smem;                      // [W][W]
  double* const value = rank + W * W;
  uint2* const lists = reinterpret_cast<uint2*>(value + W * W);      // [W][chunks][W]
  int* const token = reinterpret_cast<int*>(lists + W * p.chunks * W);
  __shared__ int counts[32], lengths[32];
  serving_begin();
  serving_next();
  // what a beam that goes on has in the workspace is on its way before it is known whether this one does (it is not used otherwise)
  uint2* const mine = lists + w * p.chunks * W;
  const uint2* from = p.best + (size_t)beam * p.chunks * W;
  for (int i = lane; i < p.chunks * W; i += 32) mine[i] = from[i];
  const float2 ms = lane < p.chunks ? p.sums[(size_t)beam * p.chunks + lane] : make_float2(-INFINITY, 0.0f);
  int row, n = 0;
  const BeamKind kind = beam_kind(p, beam, &row, false);
  const int length = p.lengths ? p.lengths[beam] : 0;
  const double score = p.scores[beam];
  const double later = fmax((double)length + (kind == kBeamGoesOn ? 1 : 0), 1.0);
  const double divisor = p.power == 0.0f ? 1.0 : p.power == 1.0f ? later : pow(later, (double)p.power);
  if (kind == kBeamEnded) {
    n = 1;
    if (lane == 0) { value[w * W] = score; rank[w * W] = score / divisor + 0.0; token[w * W] = p.end_token; }
  } else if (kind == kBeamGoesOn) {
    float top = ms.x;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    double sum = ms.x == -INFINITY ? 0.0 : (double)ms.y * exp2_fast((ms.x - top) * kLog2e);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    // log2 of the sum: its exponent, and the fp32 logarithm of the rest in [1, 2), off by 2^-24 of at most 1
    const long long bits = __double_as_longlong(sum);
    const double norm = (double)finite_max(top) + ((double)((int)(bits >> 52) - 1023) +
                        (double)log2f((float)__longlong_as_double((bits & 0xfffffffffffffll) | 0x3ff0000000000000ll))) / kLog2e;
    __syncwarp();
    int next = 0;
    uint2 head = lane < p.chunks ? mine[lane * W] : make_uint2(0u, 0u), best = make_uint2(0u, 0u);
    for (; n < W; ++n) {
      uint32_t order, low;
      int who;
      if (!best_head(head.x, head.y, &order, &low, &who)) break;
      if (lane == n) best = make_uint2(order, low);
      if (lane == who) head = ++next < W ? mine[lane * W + next] : make_uint2(0u, 0u);
    }
    if (lane < n) {
      const double v = score + ((double)of_order(best.x) - norm);
      value[w * W + lane] = v;
      rank[w * W + lane] = v / divisor;
      token[w * W + lane] = (int)best.y;
    }
  }
  if (lane == 0) { counts[w] = n; lengths[w] = kind == kBeamGoesOn ? length + 1 : length; }
  __syncthreads();
  if (w) return;
  // the beams' lists, one to a lane; equal ranks go to the lowest beam
  const int have = lane < W ? counts[lane] : 0;
  int next = 0, parent = -1, take = 0;
  for (int i = 0; i < W; ++i) {
    const bool any = next < have;
    const unsigned long long order = any ? order_of(rank[lane * W + next]) : 0ull;
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(order >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(order >> 32) == hi ? (uint32_t)order : 0u);
    const uint32_t top = __ballot_sync(0xffffffffu, any && (uint32_t)(order >> 32) == hi && (uint32_t)order == lo);
    if (!top) break;
    const int who = __ffs(top) - 1, at = __shfl_sync(0xffffffffu, next, who);
    if (lane == i) { parent = who; take = at; }
    if (lane == who) ++next;
  }
  if (lane >= W) return;
  const size_t out = (size_t)blockIdx.x * W + lane;
  const int pick = max(parent, 0) * W + take;
  p.parents[out] = parent < 0 ? -1 : (int)blockIdx.x * W + parent;
  p.tokens[out] = parent < 0 ? -1 : token[pick];
  p.scores_out[out] = parent < 0 ? -INFINITY : (float)value[pick];
  if (p.lengths_out) p.lengths_out[out] = parent < 0 ? 0 : lengths[parent];
}

// How many chunks a row is cut into: enough CTAs to fill the SMs, of at least a thousand tokens; for many rows of about five tiles, so that
// the last of them end together; no more lists than the second kernel has room and lanes for.
int beam_chunks(int64_t beams, int W, int V) {
  const int64_t fill = (kSMs * 4 + beams - 1) / beams;
  return (int)std::max<int64_t>(1, std::min<int64_t>({std::max<int64_t>(V / (5 * kTileValues), std::min<int64_t>(fill, V / 1024)), 32, 256 / W}));
}

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace
}  // namespace qzo

using namespace qzo;

extern "C" {

int qzo_beam_select_workspace_bytes(int B, int W, int V, size_t* bytes) {
  if (!bytes || B <= 0 || W <= 0 || W > QZO_MAX_BEAMS || V <= 0 || V > (1 << 30) || (int64_t)B * W > INT32_MAX / 32) return QZO_ERR_BAD_ARG;
  const int64_t lists = (int64_t)B * W * beam_chunks((int64_t)B * W, W, V);
  *bytes = align_up(lists * sizeof(float2)) + align_up(lists * W * sizeof(uint2));
  return QZO_OK;
}

int qzo_beam_select(const float* d_logits, int64_t ldl, int n_rows, const int32_t* d_rows, const float* d_scores,
                    const int32_t* d_last_tokens, int end_token, const int32_t* d_lengths, float length_power, int B, int W, int V,
                    int32_t* d_parents, int32_t* d_tokens, float* d_scores_out, int32_t* d_lengths_out, void* d_workspace,
                    size_t workspace_bytes, int* d_status, void* stream) {
  size_t need = 0;
  QZO_TRY(qzo_beam_select_workspace_bytes(B, W, V, &need));
  if (!d_logits || !d_scores || !d_parents || !d_tokens || !d_scores_out || n_rows <= 0 || ldl < V) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_logits, d_rows, d_scores, d_last_tokens, d_lengths, d_parents, d_tokens, d_scores_out, d_lengths_out, d_status)) return QZO_ERR_BAD_ARG;
  if (!d_rows && (int64_t)B * W > n_rows) return QZO_ERR_BAD_ARG;
  if (!(length_power >= 0.0f && length_power <= 8.0f) || (!d_lengths && (length_power != 0.0f || d_lengths_out))) return QZO_ERR_BAD_ARG;
  if (!d_workspace || workspace_bytes < need || ((uintptr_t)d_workspace & 255)) return QZO_ERR_WORKSPACE;
  QZO_TRY(check_device());
  const int64_t beams = (int64_t)B * W;
  BeamParams p{d_logits, ldl, n_rows, d_rows, d_scores, d_last_tokens, end_token, d_lengths, length_power, B, W, V, beam_chunks(beams, W, V), 0,
               nullptr, nullptr, d_parents, d_tokens, d_scores_out, d_lengths_out, d_status};
  p.per = ceil_div(V, p.chunks);
  const int step = p.per > kTileValues ? kTileValues : 4;              // whole tiles, so that none is left nearly empty
  p.per = ceil_div(p.per, step) * step;
  p.chunks = ceil_div(V, p.per);                       // rounding may have left the last one empty
  p.sums = (float2*)d_workspace;
  p.best = (uint2*)((uint8_t*)d_workspace + align_up(beams * p.chunks * sizeof(float2)));
  cudaStream_t st = (cudaStream_t)stream;
  const bool vec = ldl % 4 == 0 && ((uintptr_t)d_logits & 15) == 0;
  QZO_TRY(launch_serving(vec ? beam_scan_kernel<true> : beam_scan_kernel<false>, dim3((unsigned)(beams * p.chunks)), dim3(kScanThreads), 0, 1, st, p));
  {
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(beam_pick_kernel, (int)BeamDynamic::bytes(QZO_MAX_BEAMS, 256 / QZO_MAX_BEAMS), allowed));
  }
  return launch_serving(beam_pick_kernel, dim3(B), dim3(32 * W), BeamDynamic::bytes(W, p.chunks), 1, st, p);
}

}  // extern "C"
