// Matrix-vector products with int4 weights and group scales, for up to 16 rows of activations:
//   Y[t][n] = sum_g s[g][n] (sum_{k in group g} X[t][k] q[k][n]) (+ bias[n]).
// The weights are the bytes that count, and each is used for a few rows only; the contraction runs on warp-level matrix
// instructions (m16n8k16: one for up to eight rows, two above), because the tensor-memory path of the GEMM costs more per
// group in hand-offs than the weights take to read (the same linears at 16 rows: 10.8, 18.2, 18.0 and 24.0 us there, 5.4, 12.0,
// 10.5 and 14.5 us here, for K x N = 4096 x 4096, 4096 x 11008, 11008 x 4096 and 5120 x 13824).
// What bounds it: turning nibbles into bf16 takes three instructions per pair of weights (shift, mask-and-or, subtract), and
// a warp's work around the 2 KB of a turn as many again, so at one row the ALU pipe is 60 % busy at
// 4.4 TB/s (8192 x 18944, 18.2 us; its 592 CTAs take a third more than the 444 that fit at a time: 68 registers a thread leave
// an SM three CTAs of eight warps); the 7B-sized linears are bound by what a launch costs before its first bytes
// arrive and after its last ones (1 x 4096 x 11008: 8.2 us, where a plain read of as many bytes takes 6.2 us); at 16 rows the
// activations are twice the bytes of the weights in shared memory, which leaves twelve warps on an SM.
#include "qzo_common.cuh"
#include "launch.cuh"
#include "layers.cuh"
#include "mma.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace qzo {
namespace {

constexpr int kMaxCluster = 8;
constexpr int kSMem = 228 * 1024;    // shared memory of an SM (a CTA may have 1 KB less)

struct GemvLinear {
  const uint4* wq;
  const __nv_bfloat16* scales;
  const float* bias;
  __nv_bfloat16* out;
  int ldo, N, first_cta;
};
struct GemvParams {
  GemvLinear lin[kMaxGroupedLinears];
  const __nv_bfloat16* x;
  int n_lin, ldx, M, K, KB, G;
};

// Two 4-bit values u (bits 4p.. of each half of w) as the bf16 pair (u - 8) / kLowered: 0x3E00 | u is (128 + u) / 1024, less 136 /
// 1024; both exact.  So lowered, the products of a group of 128 stay finite whatever the activations; the sums are raised at the end.
constexpr float kLowered = 1024.0f;
__device__ __forceinline__ uint32_t weight_pair(uint32_t w, int p) {
  uint32_t u;                           // (shifted & mask) | 0x4300 in one instruction
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w >> (4 * p)), "r"(0x000F000Fu), "r"(0x3E003E00u));
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), __floats2bfloat162_rn(136.0f / kLowered, 136.0f / kLowered));
  return *reinterpret_cast<const uint32_t*>(&r);
}

constexpr int kRT = 2;               // tiles of sixteen output features of a warp, which are also a CTA's
constexpr int kCols = 16 * kRT;
constexpr int kStages = 3;           // of a warp's ring: a group of 128 k of the weights, their scales, and of the activations
constexpr int kWeightBytes = kRT * 1024, kScaleBytes = kRT * 32;

// XR: rows of activations that a stage holds (1, 4, 8 or 16, at least M); W: warps of a CTA, which share its output features and
// take the groups of K in turn.  CTAs begin at different groups, so that they do not all ask the L2 for the same activations
// at once (16 x 5120 x 13824: 14.5 us, 15.6 if all begin at the first; 1 x 5120 x 13824: 9.8 and 10.1).
// The weights are the A operand.  A lane's share of a tile is features 2g and 2g + 1 and the 32 k of its quarter t of the
// group: two neighbouring 16-byte units of the kernel layout; its B fragments are then the 32 consecutive activations
// of that quarter.
// Every warp has a ring of its own in shared memory, filled by 16-byte asynchronous copies: no barrier in the loop, which is
// unrolled over the stages, so that every address in them is a register and a constant (a warp sees 2 KB of weights at a
// time: what it issues around them counts as much as what they cost themselves).
// Places in a stage: the unit of feature f and quarter t at (32 t + f) ^ pad(t), pads {0, 1, 4, 5}, and the
// activations' unit q of a row at q ^ (q >> 3) ^ 2 (row & 1), so that the eight lanes of a phase (two g, four t) read eight
// different 16-byte banks.
template <int XR, int W>
__global__ void __launch_bounds__(W * 32)
gemv_w4_kernel(GemvParams p) {
  constexpr int NT = XR > 8 ? 2 : 1;                   // tiles of eight rows
  constexpr int kStageBytes = kWeightBytes + kScaleBytes + 256 * XR;
  extern __shared__ __align__(128) uint8_t gemv_smem[];
  const int rank = blockIdx.x, block = blockIdx.y;     // CTA of the cluster, output features
  int j = 0;
  while (j + 1 < p.n_lin && block >= p.lin[j + 1].first_cta) ++j;
  const GemvLinear& L = p.lin[j];
  const int n0 = (block - L.first_cta) * kCols, N = L.N;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(gemv_smem) + warp * kStages * kStageBytes;
  const int step = W * (int)gridDim.x, mine = (p.G - 1 - (rank * W + warp) + step) / step;       // groups of this warp
  const int first = rank * W + warp + (mine > 0 ? block % mine * step : 0);

  // what a lane copies of a group: of every quarter the unit of feature `lane`, one unit of scales (columns that do not exist: of
  // ones that do, their outputs are not stored), and unit x_q of every other row of activations
  const uint4* w_src = L.wq + ((size_t)(n0 / kTileN) * p.KB + 2 * (size_t)first) * (kPackedTileBytes / 16) + n0 % kTileN + lane;
  const __nv_bfloat16* s_src = L.scales + (size_t)first * N + min(n0 + 8 * (lane % (2 * kRT)), N - 8);
  const int x_row = lane >> 4, x_q = lane & 15;
  const __nv_bfloat16* x_src = p.x + (size_t)x_row * p.ldx + (size_t)first * kGroup + 8 * x_q;
  const uint32_t w_dst[4] = {ring + 16 * lane, ring + 16 * (32 + (lane ^ 1)), ring + 16 * (64 + (lane ^ 4)), ring + 16 * (96 + (lane ^ 5))};
  const uint32_t s_dst = ring + kWeightBytes + 16 * lane;
  const uint32_t x_dst = ring + kWeightBytes + kScaleBytes + 256 * x_row + 16 * (x_q ^ (x_q >> 3) ^ (x_row << 1));
  int next = first, fetched = 0;                       // the group that is copied next
  auto fetch = [&](int at) {                           // `at`: offset of its stage
    const bool last = next == p.G - 1;
    // a last block of 64 that does not exist is read from the one before it: its activations are zeros
    const int second = last && (p.KB & 1) ? 0 : kPackedTileBytes / 16;
    copy16(w_dst[0] + at, w_src);
    copy16(w_dst[1] + at, w_src + kTileN);
    copy16(w_dst[2] + at, w_src + second);
    copy16(w_dst[3] + at, w_src + second + kTileN);
    if (lane < 2 * kRT) copy16(s_dst + at, s_src);
    const bool live = !last || next * kGroup + 8 * x_q < p.K;          // behind K: zeros, whatever stands there
    const __nv_bfloat16* x = live ? x_src : p.x + (size_t)x_row * p.ldx;
#pragma unroll
    for (int i = 0; i < (XR + 1) / 2; ++i, x += 2 * (size_t)p.ldx)
      if (x_row + 2 * i < (XR == 1 ? 1 : p.M)) copy16_or_zero(x_dst + at + 512 * i, x, live ? 16 : 0);
    ++fetched;
    const int jump = next + step < p.G ? step : step - mine * step;    // on to the next group, behind the last one to the first
    next += jump;
    w_src += (int64_t)jump * (2 * kPackedTileBytes / 16);
    s_src += (int64_t)jump * N;
    x_src += (int64_t)jump * kGroup;
  };
  // what it reads: the units of features 2g, 2g + 1 and quarter t of every tile, the activations of quarter t of its rows
  const uint32_t w_lds = ring + 16 * (32 * t + ((2 * g) ^ ((t & 1) + 4 * (t >> 1))));
  const uint32_t w_lds1 = w_lds ^ 16, s_lds = ring + kWeightBytes + 4 * g;
  uint32_t x_lds[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = XR == 1 ? 0 : min(nt * 8 + g, p.M - 1);            // rows that do not exist: any, their sums are not stored
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x_lds[nt][i] = ring + kWeightBytes + kScaleBytes + 256 * row + 16 * ((4 * t + i) ^ (t >> 1) ^ ((row & 1) << 1));
  }
  float acc[kRT][NT][4] = {};
  auto contract = [&](int at) {
    uint4 x[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[nt][i] = lds16(x_lds[nt][i] + at);
    // the words of both tiles in turn, so that the matrix instructions of one do not wait for one another
    uint4 ua[kRT], ub[kRT];
    float c[kRT][NT][4] = {};
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
      ua[r] = lds16(w_lds + at + 256 * r);
      ub[r] = lds16(w_lds1 + at + 256 * r);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        const uint32_t wa = i == 0 ? ua[r].x : i == 1 ? ua[r].y : i == 2 ? ua[r].z : ua[r].w;
        const uint32_t wb = i == 0 ? ub[r].x : i == 1 ? ub[r].y : i == 2 ? ub[r].z : ub[r].w;
        const uint32_t a0 = weight_pair(wa, 0), a1 = weight_pair(wa, 1), a2 = weight_pair(wa, 2), a3 = weight_pair(wa, 3);
        const uint32_t b0 = weight_pair(wb, 0), b1 = weight_pair(wb, 1), b2 = weight_pair(wb, 2), b3 = weight_pair(wb, 3);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816_bf16(c[r][nt], a0, b0, a1, b1, x[nt][i].x, x[nt][i].y);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816_bf16(c[r][nt], a2, b2, a3, b3, x[nt][i].z, x[nt][i].w);
      }
    }
#pragma unroll
    for (int r = 0; r < kRT; ++r) {
      const uint32_t s2 = lds4(s_lds + at + 32 * r);
      const float2 s = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&s2));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        acc[r][nt][0] = fmaf(s.x, c[r][nt][0], acc[r][nt][0]);
        acc[r][nt][1] = fmaf(s.x, c[r][nt][1], acc[r][nt][1]);
        acc[r][nt][2] = fmaf(s.y, c[r][nt][2], acc[r][nt][2]);
        acc[r][nt][3] = fmaf(s.y, c[r][nt][3], acc[r][nt][3]);
      }
    }
  };
  serving_begin();
  serving_next();
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    if (fetched < mine) fetch(s * kStageBytes);
    copies_commit();
  }
  for (int i = 0; i < mine;) {
#pragma unroll
    for (int u = 0; u < kStages; ++u, ++i) {
      if (i >= mine) break;
      copies_wait<kStages - 2>();
      __syncwarp();                                    // this stage has landed, and every lane is done with the one before it
      if (fetched < mine) fetch((u + kStages - 1) % kStages * kStageBytes);
      copies_commit();
      contract(u * kStageBytes);
    }
  }
  __syncthreads();                                     // the rings are free: the sums go there
  float (*red)[8 * NT][kCols + 1] = reinterpret_cast<float (*)[8 * NT][kCols + 1]>(gemv_smem);

  // the warps' sums in their order, then the cluster's CTAs' in theirs
#pragma unroll
  for (int r = 0; r < kRT; ++r)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (XR > 1 || (t == 0 && (e & 1) == 0)) red[warp][nt * 8 + 2 * t + (e & 1)][16 * r + 2 * g + (e >> 1)] = acc[r][nt][e];
  __syncthreads();
  cg::cluster_group cluster = cg::this_cluster();
  const bool alone = gridDim.x == 1;
  const int outs = kCols * (XR == 1 ? 1 : p.M);
  if (!alone) {
    for (int i = threadIdx.x; i < outs; i += W * 32) {
      const int row = i / kCols, n = i % kCols;
      float y = red[0][row][n];
#pragma unroll
      for (int w = 1; w < W; ++w) y += red[w][row][n];
      red[0][row][n] = y;
    }
    cluster.sync();
  }
  // each CTA of the cluster finishes its share of the outputs
  for (int i = rank * W * 32 + threadIdx.x; i < outs; i += W * 32 * gridDim.x) {
    const int row = i / kCols, n = i % kCols;
    if (n0 + n >= N) continue;
    float y = 0.0f;
    if (alone) {
#pragma unroll
      for (int w = 0; w < W; ++w) y += red[w][row][n];
    } else {
      for (int c = 0; c < (int)gridDim.x; ++c) y += *cluster.map_shared_rank(&red[0][row][n], c);
    }
    y *= kLowered;
    if (L.bias) y += L.bias[n0 + n];
    L.out[(size_t)row * L.ldo + n0 + n] = __float2bfloat16_rn(y);
  }
  if (!alone) cluster.sync();                         // no CTA leaves while another reads its sums
}

template <int XR, int W>
int run_gemv(const GemvParams& p, int blocks, cudaStream_t st) {
  // Few output features: the CTAs of a cluster share the groups of K (measured at K = 11008, N = 256, one row: 7.5 us alone,
  // 3.5 us with clusters of eight; at K = N = 4096, 128 CTAs of 32 features, 4.4 us alone, 5.0 us with clusters of two).
  int cluster = 1;
  while (cluster < kMaxCluster && 2 * cluster * blocks <= kSMs && 2 * cluster * W <= p.G) cluster *= 2;
  constexpr int kRing = W * kStages * (kWeightBytes + kScaleBytes + 256 * XR), kSums = W * (XR > 8 ? 16 : 8) * (kCols + 1) * (int)sizeof(float);
  // The CTAs are spread evenly: each asks for so much shared memory that no SM takes more than its share of them (4096 x
  // 9472, 296 CTAs: 6.5 us at one row and 9.2 at sixteen; 7.7 and 11.4 where some SMs take three of them and some one).  From a
  // share of four on it changes nothing for CTAs of eight warps: their registers let an SM hold three.
  const int share = ceil_div(blocks * cluster, kSMs), even = (kSMem / (share + 1) - 1024) / 16 * 16 + 16;
  const int smem = std::max({kRing, kSums, even});
  static std::atomic<unsigned long long> allowed{0};
  QZO_CUDA_TRY(allow_dynamic_smem(gemv_w4_kernel<XR, W>, kSMem - 1024, allowed));
  return launch_serving(gemv_w4_kernel<XR, W>, dim3(cluster, blocks), dim3(W * 32), smem, cluster, st, p);
}

}  // namespace

int launch_gemv_group(const __nv_bfloat16* d_x, int ldx, int M, int K, const GemmLinear* lins, int n_lin, cudaStream_t st) {
  if (M <= 0 || M > QZO_GEMV_MAX_ROWS || K <= 0 || (K % 8) || n_lin < 1 || n_lin > kMaxGroupedLinears) return QZO_ERR_BAD_ARG;
  GemvParams p{};
  int64_t blocks = 0;
  for (int j = 0; j < n_lin; ++j) {
    if (lins[j].N <= 0 || (lins[j].N % 8)) return QZO_ERR_BAD_ARG;
    p.lin[j] = GemvLinear{(const uint4*)lins[j].wq, lins[j].scales, lins[j].bias, lins[j].out, lins[j].ldo, lins[j].N, (int)blocks};
    blocks += ceil_div(lins[j].N, kCols);
  }
  if (blocks > 65535) return QZO_ERR_BAD_ARG;            // the grid's second dimension: two million output features
  p.x = d_x;
  p.n_lin = n_lin; p.ldx = ldx; p.M = M; p.K = K;
  p.KB = ceil_div(K, kBlockK);
  p.G = ceil_div(K, kGroup);
  if (M == 1) return run_gemv<1, 8>(p, (int)blocks, st);
  if (M <= 4) return run_gemv<4, 8>(p, (int)blocks, st);
  if (M <= 8) return run_gemv<8, 8>(p, (int)blocks, st);
  // Two tiles of rows: the activations take two thirds of a stage, and CTAs of eight warps (149 KB) leave room for one of them
  // on an SM only, which pays where there is no more than one CTA per SM (measured with 16 rows: K = N = 4096 5.4 us against 6.1 us
  // with four warps, K = 5120, N = 13824 17.2 us against 14.5 us).
  return blocks <= kSMs ? run_gemv<16, 8>(p, (int)blocks, st) : run_gemv<16, 4>(p, (int)blocks, st);
}

}  // namespace qzo

using namespace qzo;

extern "C" int qzo_gemv_int4(const void* d_x_bf16, int ldx, const void* d_wq, const void* d_scales_bf16, const float* d_bias,
                             void* d_y_bf16, int ldy, int M, int K, int N, void* stream) {
  if (!d_x_bf16 || !d_wq || !d_scales_bf16 || !d_y_bf16) return QZO_ERR_BAD_ARG;
  if (M <= 0 || M > QZO_GEMV_MAX_ROWS || K <= 0 || N <= 0 || (K % 8) || (N % 8)) return QZO_ERR_BAD_ARG;
  if (ldx < K || (ldx % 8) || ldy < N) return QZO_ERR_BAD_ARG;
  if (((uintptr_t)d_x_bf16 & 15) || ((uintptr_t)d_wq & 15) || ((uintptr_t)d_scales_bf16 & 15) || ((uintptr_t)d_y_bf16 & 1) ||
      ((uintptr_t)d_bias & 3))
    return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  const GemmLinear g{d_wq, (const __nv_bfloat16*)d_scales_bf16, d_bias, (__nv_bfloat16*)d_y_bf16, ldy, N, 0};
  return launch_gemv_group((const __nv_bfloat16*)d_x_bf16, ldx, M, K, &g, 1, (cudaStream_t)stream);
}
