// Matrix-vector products with int4 weights and group scales, for up to 16 rows of activations:
//   Y[t][n] = sum_g s[g][n] (sum_{k in group g} X[t][k] q[k][n]) (+ bias[n]).
// The weights are the bytes that count, and each is used for a few rows only; the contraction runs on warp-level matrix
// instructions (m16n8k16: one for up to eight rows, two above), because the tensor-memory path of the GEMM costs more per
// group in hand-offs than the weights take to read (the same linears at 16 rows: 10.8, 18.2, 18.0 and 24.0 us there, 5.9, 12.4,
// 11.7 and 15.3 us here, for K x N = 4096 x 4096, 4096 x 11008, 11008 x 4096 and 5120 x 13824).
// What bounds it: turning nibbles into bf16 takes three instructions per pair of weights (shift, mask-and-or, subtract), so
// at one row the ALU pipe is 60 % busy at 3.5 TB/s (8192 x 18944, 22.7 us); the 7B-sized linears are bound by what a launch
// costs before its first bytes arrive and after its last ones (1 x 4096 x 11008: 9.6 us, where a plain read of as many bytes
// takes 6.2 us); at 16 rows the activations are twice the bytes of the weights in shared memory.
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
constexpr int kSMs = 148, kSMem = 228 * 1024;   // SMs, and the shared memory of one (a CTA may have 1 KB less)

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
  int n_lin, ldx, M, K, KB, G, cluster;
};

// Two 4-bit values u (bits 4p.. of each half of w) as the bf16 pair u - 8: 0x4300 | u is 128 + u, less 136; both exact.
__device__ __forceinline__ uint32_t weight_pair(uint32_t w, int p) {
  uint32_t u;                           // (shifted & mask) | 0x4300 in one instruction
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w >> (4 * p)), "r"(0x000F000Fu), "r"(0x43004300u));
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), __floats2bfloat162_rn(136.0f, 136.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// NT: tiles of eight activation rows; RT: tiles of sixteen output features of a warp; S: stages of its ring; W: warps of a CTA,
// which share its output features and take the groups of K in turn.
// The weights are the A operand.  A lane's share of a tile is features 2g and 2g + 1 and the 32 k of its quarter t of the
// group: two neighbouring 16-byte units of the kernel layout; its B fragments are then the 32 consecutive activations
// of that quarter.
// Every warp has a ring of its own in shared memory, filled by 16-byte asynchronous copies: no barrier in the loop.
// Places in a stage: the unit of feature f and quarter t at (t RT 16 + f) ^ pad(t), pads {0, 1, 4, 5}, and the
// activations' unit q of a row at q ^ (q >> 3) ^ 2 (row & 1), so that the eight lanes of a phase (two g, four t) read eight
// different 16-byte banks.
template <int NT, int RT, int S, int W>
__global__ void __launch_bounds__(W * 32)
gemv_w4_kernel(GemvParams p) {
  constexpr int kWeightBytes = RT * 1024, kScaleBytes = RT * 32;
  extern __shared__ __align__(128) uint8_t gemv_smem[];
  const int rank = blockIdx.x % p.cluster, block = blockIdx.x / p.cluster;
  int j = 0;
  while (j + 1 < p.n_lin && block >= p.lin[j + 1].first_cta) ++j;
  const GemvLinear L = p.lin[j];
  const int n0 = (block - L.first_cta) * 16 * RT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int stage_bytes = kWeightBytes + kScaleBytes + 256 * p.M;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(gemv_smem) + warp * S * stage_bytes;
  const uint4* panel = L.wq + (size_t)(n0 / kTileN) * p.KB * (kPackedTileBytes / 16) + n0 % kTileN;

  // what a lane copies: of every quarter q units lane, lane + 32, ... of the 16 RT features, two neighbouring rows' units of
  // activations at a time, one unit of scales (columns that do not exist: of ones that do, their outputs are not stored)
  constexpr int kPad[4] = {0, 1, 4, 5};
  const uint4* const w_src = panel + lane % (16 * RT);
  const __nv_bfloat16* const s_src = L.scales + min(n0 + 8 * (lane % (2 * RT)), L.N - 8);
  const int x_row = lane >> 4, x_q = lane & 15;
  const __nv_bfloat16* const x_src = p.x + (size_t)x_row * p.ldx + 8 * x_q;
  const uint32_t x_dst = kWeightBytes + kScaleBytes + 256 * x_row + 16 * (x_q ^ (x_q >> 3) ^ (x_row << 1));
  auto fetch = [&](int grp, uint32_t at) {
    // a last block of 64 that does not exist is read from the one before it: its activations are zeros
    const uint4* src = w_src + (size_t)grp * (2 * kPackedTileBytes / 16);
    const int second = 2 * grp + 1 < p.KB ? kPackedTileBytes / 16 : 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int f = 0; f < 16 * RT; f += 32)
        copy16(at + 16 * (q * 16 * RT + f + (lane ^ kPad[q])), src + (q >> 1) * second + (q & 1) * kTileN + f);
    if (lane < 2 * RT) copy16(at + kWeightBytes + 16 * lane, s_src + (size_t)grp * L.N);
    const bool live = grp * kGroup + 8 * x_q < p.K;    // behind K: zeros, whatever stands there
    const __nv_bfloat16* x = x_src + grp * kGroup;
    uint32_t dst = at + x_dst;
    for (int row = x_row; row < p.M; row += 2, x += 2 * (size_t)p.ldx, dst += 512) {
      if (live) copy16(dst, x);
      else zero16(dst);
    }
  };
  // what it reads: the units of features 2g, 2g + 1 and quarter t of every tile, the activations of quarter t of its rows
  const uint32_t w_lds0 = 16 * (t * 16 * RT + ((2 * g) ^ ((t & 1) + 4 * (t >> 1)))), w_lds1 = w_lds0 ^ 16;
  uint32_t x_lds[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = min(nt * 8 + g, p.M - 1);          // rows that do not exist: any, their sums are not stored
    x_lds[nt] = kWeightBytes + kScaleBytes + 256 * row + 16 * ((4 * t) ^ (t >> 1) ^ ((row & 1) << 1));
  }
  float acc[RT][NT][4] = {};
  auto contract = [&](uint32_t at) {
    uint4 x[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[nt][i] = lds16((at + x_lds[nt]) ^ (16 * i));
    // the words of all tiles in turn, so that the matrix instructions of neighbouring ones do not wait for one another (16 x 5120
    // x 13824 15.3 us, 16.1 us tile by tile)
    uint4 ua[RT], ub[RT];
    float c[RT][NT][4] = {};
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      ua[r] = lds16(at + w_lds0 + 256 * r);
      ub[r] = lds16(at + w_lds1 + 256 * r);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
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
    for (int r = 0; r < RT; ++r) {
      const uint32_t s2 = lds4(at + kWeightBytes + 32 * r + 4 * g);
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
  const int step = W * p.cluster, first = rank * W + warp;
#pragma unroll
  for (int s = 0; s < S - 1; ++s) {
    if (first + s * step < p.G) fetch(first + s * step, ring + s * stage_bytes);
    copies_commit();
  }
  int use = 0, fill = S - 1;
  for (int grp = first; grp < p.G; grp += step) {
    copies_wait<S - 2>();
    __syncwarp();                                      // this stage has landed, and every lane is done with the one before it
    if (grp + (S - 1) * step < p.G) fetch(grp + (S - 1) * step, ring + fill * stage_bytes);
    copies_commit();
    contract(ring + use * stage_bytes);
    use = use + 1 == S ? 0 : use + 1;
    fill = fill + 1 == S ? 0 : fill + 1;
  }
  __syncthreads();                                     // the rings are free: the sums go there
  float (*red)[8 * NT][16 * RT + 1] = reinterpret_cast<float (*)[8 * NT][16 * RT + 1]>(gemv_smem);

  // the warps' sums in their order, then the cluster's CTAs' in theirs
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[warp][nt * 8 + 2 * t + (e & 1)][16 * r + 2 * g + (e >> 1)] = acc[r][nt][e];
  __syncthreads();
  cg::cluster_group cluster = cg::this_cluster();
  constexpr int kOut = 16 * RT * 8 * NT;
  if (p.cluster > 1) {
    for (int i = threadIdx.x; i < kOut; i += W * 32) {
      const int row = i / (16 * RT), n = i % (16 * RT);
      float y = red[0][row][n];
#pragma unroll
      for (int w = 1; w < W; ++w) y += red[w][row][n];
      red[0][row][n] = y;
    }
    cluster.sync();
  }
  // each CTA of the cluster finishes its share of the outputs
  for (int i = rank * W * 32 + threadIdx.x; i < kOut; i += W * 32 * p.cluster) {
    const int row = i / (16 * RT), n = i % (16 * RT);
    if (row >= p.M || n0 + n >= L.N) continue;
    float y = 0.0f;
    if (p.cluster > 1) {
      for (int c = 0; c < p.cluster; ++c) y += *cluster.map_shared_rank(&red[0][row][n], c);
    } else {
#pragma unroll
      for (int w = 0; w < W; ++w) y += red[w][row][n];
    }
    if (L.bias) y += L.bias[n0 + n];
    L.out[(size_t)row * L.ldo + n0 + n] = __float2bfloat16_rn(y);
  }
  if (p.cluster > 1) cluster.sync();                  // no CTA leaves while another reads its sums
}

template <int NT, int RT, int S, int W>
int run_gemv(GemvParams& p, cudaStream_t st) {
  int blocks = 0;
  for (int j = 0; j < p.n_lin; ++j) {
    p.lin[j].first_cta = blocks;
    blocks += ceil_div(p.lin[j].N, 16 * RT);
  }
  // Few output features: the CTAs of a cluster share the groups of K (measured at K = 11008, N = 256, one row: 9.4 us alone,
  // 4.2 us with clusters of eight; at K = N = 4096, 128 CTAs of 32 features, 5.5 us alone, 5.9 us with clusters of two).
  int cluster = 1;
  while (cluster < kMaxCluster && 2 * cluster * blocks <= kSMs && 2 * cluster * W <= p.G) cluster *= 2;
  p.cluster = cluster;
  constexpr int kSums = W * 8 * NT * (16 * RT + 1) * (int)sizeof(float);
  // The CTAs are spread evenly: each asks for so much shared memory that no SM takes more than its share of them (1 x 4096 x
  // 11008, 344 CTAs: 9.7 us, 11.7 us where an SM may take a fourth one; 1 x 5120 x 13824 11.6 us against 14.5).
  const int share = ceil_div(blocks * cluster, kSMs), even = (kSMem / (share + 1) - 1024) / 16 * 16 + 16;
  const int smem = std::max({W * S * (RT * 1056 + 256 * p.M), kSums, even});
  static std::atomic<unsigned long long> allowed{0};
  QZO_CUDA_TRY(allow_dynamic_smem(gemv_w4_kernel<NT, RT, S, W>, kSMem - 1024, allowed));
  return launch_serving<GemvParams>(gemv_w4_kernel<NT, RT, S, W>, dim3(blocks * cluster), dim3(W * 32), smem, cluster, st, p);
}

}  // namespace

int launch_gemv_group(const __nv_bfloat16* d_x, int ldx, int M, int K, const GemmLinear* lins, int n_lin, cudaStream_t st) {
  if (M <= 0 || M > QZO_GEMV_MAX_ROWS || K <= 0 || (K % 8) || n_lin < 1 || n_lin > kMaxGroupedLinears) return QZO_ERR_BAD_ARG;
  GemvParams p{};
  for (int j = 0; j < n_lin; ++j) {
    if (lins[j].N <= 0 || (lins[j].N % 8)) return QZO_ERR_BAD_ARG;
    p.lin[j] = GemvLinear{(const uint4*)lins[j].wq, lins[j].scales, lins[j].bias, lins[j].out, lins[j].ldo, lins[j].N, 0};
  }
  p.x = d_x;
  p.n_lin = n_lin; p.ldx = ldx; p.M = M; p.K = K;
  p.KB = ceil_div(K, kBlockK);
  p.G = ceil_div(K, kGroup);
  if (M <= 8) return run_gemv<1, 2, 3, 8>(p, st);
  // Two tiles of rows: the activations take half of a stage, so CTAs of eight warps leave room for two of them on an SM
  // only, which pays where there is no more than one CTA per SM (measured with 16 rows: K = N = 4096 6.5 us against 8.0 us
  // with four warps, K = 5120, N = 13824 19.0 us against 16.6 us).
  int blocks = 0;
  for (int j = 0; j < n_lin; ++j) blocks += ceil_div(lins[j].N, 32);
  return blocks <= kSMs ? run_gemv<2, 2, 3, 8>(p, st) : run_gemv<2, 2, 3, 4>(p, st);
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
