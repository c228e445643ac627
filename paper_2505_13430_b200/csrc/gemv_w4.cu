// Matrix-vector products with int4 weights and group scales, for up to 16 rows of activations:
//   Y[t][n] = sum_g s[g][n] (sum_{k in group g} X[t][k] q[k][n]) (+ bias[n]).
#include "qzo_common.cuh"
#include "launch.cuh"
#include "layers.cuh"
#include "mma.cuh"

#include <algorithm>

namespace qzo {
namespace {

constexpr int kGemvWarps = 8;        // warps of a CTA: they share its output rows and take the groups of K in turn
constexpr int kGemvThreads = kGemvWarps * 32;

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

// Two 4-bit values u (bits 4p.. of each half of w) as the bf16 pair u - 8: 0x4300 | u is 128 + u, less 136; both exact.
__device__ __forceinline__ uint32_t weight_pair(uint32_t w, int p) {
  const uint32_t u = ((w >> (4 * p)) & 0x000F000Fu) | 0x43004300u;
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), __floats2bfloat162_rn(136.0f, 136.0f));
  return *reinterpret_cast<const uint32_t*>(&r);
}

template <int NT>   // tiles of eight activation rows
__global__ void __launch_bounds__(kGemvThreads)
gemv_w4_kernel(const GemvParams p) {
  __shared__ float red[kGemvWarps][8 * NT][16 + 1];
  int j = 0;
  while (j + 1 < p.n_lin && (int)blockIdx.x >= p.lin[j + 1].first_cta) ++j;
  const GemvLinear L = p.lin[j];
  const int n0 = ((int)blockIdx.x - L.first_cta) * 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint4* panel = L.wq + (size_t)(n0 / kTileN) * p.KB * (kPackedTileBytes / 16) + (t & 1) * kTileN + n0 % kTileN + g;
  const uint4 none = make_uint4(0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u);   // all zero weights
  float acc[NT][4] = {};
  for (int grp = warp; grp < p.G; grp += kGemvWarps) {
    const int kb = 2 * grp + (t >> 1);
    uint4 w0 = none, w1 = none;
    if (kb < p.KB) {
      w0 = load_stream16(panel + (size_t)kb * (kPackedTileBytes / 16));
      w1 = load_stream16(panel + (size_t)kb * (kPackedTileBytes / 16) + 8);
    }
    const __nv_bfloat16* srow = L.scales + (size_t)grp * L.N + n0 + g;
    const float s0 = n0 + g < L.N ? __bfloat162float(srow[0]) : 0.0f;
    const float s1 = n0 + g + 8 < L.N ? __bfloat162float(srow[8]) : 0.0f;
    float c[NT][4] = {};
    const uint32_t wa[4] = {w0.x, w0.y, w0.z, w0.w}, wb[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = grp * kGroup + 32 * t + 8 * i;
      const uint32_t a[4] = {weight_pair(wa[i], 0), weight_pair(wa[i], 1), weight_pair(wa[i], 2), weight_pair(wa[i], 3)};
      const uint32_t b[4] = {weight_pair(wb[i], 0), weight_pair(wb[i], 1), weight_pair(wb[i], 2), weight_pair(wb[i], 3)};
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (k < p.K && nt * 8 + g < p.M) x = *reinterpret_cast<const uint4*>(p.x + (size_t)(nt * 8 + g) * p.ldx + k);
        mma16816_bf16(c[nt], a[0], b[0], a[1], b[1], x.x, x.y);
        mma16816_bf16(c[nt], a[2], b[2], a[3], b[3], x.z, x.w);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      acc[nt][0] = fmaf(s0, c[nt][0], acc[nt][0]);
      acc[nt][1] = fmaf(s0, c[nt][1], acc[nt][1]);
      acc[nt][2] = fmaf(s1, c[nt][2], acc[nt][2]);
      acc[nt][3] = fmaf(s1, c[nt][3], acc[nt][3]);
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    red[warp][nt * 8 + 2 * t][g] = acc[nt][0];
    red[warp][nt * 8 + 2 * t + 1][g] = acc[nt][1];
    red[warp][nt * 8 + 2 * t][g + 8] = acc[nt][2];
    red[warp][nt * 8 + 2 * t + 1][g + 8] = acc[nt][3];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 8 * NT; i += kGemvThreads) {
    const int row = i / 16, n = i % 16;
    if (row >= p.M || n0 + n >= L.N) continue;
    float y = 0.0f;
#pragma unroll
    for (int w = 0; w < kGemvWarps; ++w) y += red[w][row][n];
    if (L.bias) y += L.bias[n0 + n];
    L.out[(size_t)row * L.ldo + n0 + n] = __float2bfloat16_rn(y);
  }
}

}  // namespace

int launch_gemv_group(const __nv_bfloat16* d_x, int ldx, int M, int K, const GemmLinear* lins, int n_lin, cudaStream_t st) {
  if (M <= 0 || M > QZO_GEMV_MAX_ROWS || K <= 0 || (K % 8) || n_lin < 1 || n_lin > kMaxGroupedLinears) return QZO_ERR_BAD_ARG;
  GemvParams p{};
  int ctas = 0;
  for (int j = 0; j < n_lin; ++j) {
    if (lins[j].N <= 0 || (lins[j].N % 8)) return QZO_ERR_BAD_ARG;
    p.lin[j] = GemvLinear{(const uint4*)lins[j].wq, lins[j].scales, lins[j].bias, lins[j].out, lins[j].ldo, lins[j].N, ctas};
    ctas += ceil_div(lins[j].N, 16);
  }
  p.x = d_x;
  p.n_lin = n_lin; p.ldx = ldx; p.M = M; p.K = K;
  p.KB = ceil_div(K, kBlockK);
  p.G = ceil_div(K, kGroup);
  if (M <= 8) QZO_LAUNCH(gemv_w4_kernel<1>, dim3(ctas), dim3(kGemvThreads), 0, st, p);
  else QZO_LAUNCH(gemv_w4_kernel<2>, dim3(ctas), dim3(kGemvThreads), 0, st, p);
  return QZO_OK;
}

}  // namespace qzo

using namespace qzo;

extern "C" int qzo_gemv_int4(const void* d_x_bf16, int ldx, const void* d_wq, const void* d_scales_bf16, const float* d_bias,
                             void* d_y_bf16, int ldy, int M, int K, int N, void* stream) {
  if (!d_x_bf16 || !d_wq || !d_scales_bf16 || !d_y_bf16) return QZO_ERR_BAD_ARG;
  if (M <= 0 || M > QZO_GEMV_MAX_ROWS || K <= 0 || N <= 0 || (K % 8) || (N % 8)) return QZO_ERR_BAD_ARG;
  if (ldx < K || (ldx % 8) || ldy < N) return QZO_ERR_BAD_ARG;
  if (((uintptr_t)d_x_bf16 & 15) || ((uintptr_t)d_wq & 15) || ((uintptr_t)d_scales_bf16 & 1) || ((uintptr_t)d_y_bf16 & 1) ||
      ((uintptr_t)d_bias & 3))
    return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  const GemmLinear g{d_wq, (const __nv_bfloat16*)d_scales_bf16, d_bias, (__nv_bfloat16*)d_y_bf16, ldy, N, 0};
  return launch_gemv_group((const __nv_bfloat16*)d_x_bf16, ldx, M, K, &g, 1, (cudaStream_t)stream);
}
