// Kernel launch wrapper: counts launches (reported by the benchmark) and turns a launch
// error into QZO_ERR_CUDA.
#pragma once
#include "qzo_common.cuh"

namespace qzo {
void count_launch();
void add_launches(long long n);   // kernels run by replaying a recorded step

#define QZO_LAUNCH(kernel, grid, block, smem, stream, ...)                  \
  do {                                                                      \
    kernel<<<(grid), (block), (smem), (stream)>>>(__VA_ARGS__);             \
    ::qzo::count_launch();                                                  \
    cudaError_t _le = cudaGetLastError();                                   \
    if (_le != cudaSuccess) {                                               \
      ::qzo::set_last_cuda_error(_le);                                      \
      return QZO_ERR_CUDA;                                                  \
    }                                                                       \
  } while (0)

constexpr int kSMs = 148;   // of a B200: what the serving kernels' launch rules fill (on another count of SMs they only spread work less evenly)

// Launch of a serving kernel: allowed to start while the kernel before it in the stream ends (a decode step is a chain of
// launches of a few microseconds).  Such a kernel calls serving_begin() before it touches global memory, in every CTA.
// cluster > 1: CTAs of a cluster.
template <typename... Params, typename... Args>
int launch_serving(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attrs[2]{};
  attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attrs[0].val.programmaticStreamSerializationAllowed = 1;
  attrs[1].id = cudaLaunchAttributeClusterDimension;
  attrs[1].val.clusterDim.x = (unsigned)cluster;
  attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
  cfg.attrs = attrs;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  QZO_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...));
  count_launch();
  return QZO_OK;
}

#ifdef __CUDACC__
// Waits for the end of the kernel before this one and sees its writes.  Every CTA calls it, those without work too: the end
// of this kernel stands for the end of all before it.  Returns at once in a kernel launched the ordinary way.  What is loaded
// behind it must not come through a __restrict__ pointer: the compiler may move such a load in front of it.
__device__ __forceinline__ void serving_begin() { cudaGridDependencySynchronize(); }
// From here on the next kernel's CTAs may take their places (once every CTA has come here or ended).
__device__ __forceinline__ void serving_next() { cudaTriggerProgrammaticLaunchCompletion(); }
#endif

// prims.cu
int launch_philox_words(uint64_t seed, uint64_t block_base, int64_t n_blocks, uint32_t* d_words,
                        float* d_uniforms, cudaStream_t st);
int launch_normals(uint64_t seed, uint64_t index_base, int64_t count, float* d_z, cudaStream_t st);
int launch_quantize(const float* d_w, int K, int N, uint32_t* d_packed, __nv_bfloat16* d_scales, cudaStream_t st);
int launch_unpack(const uint32_t* d_packed, int K, int N, int8_t* d_q, cudaStream_t st);
size_t repacked_bytes(int K, int N);
int launch_repack(const uint32_t* d_packed, int K, int N, void* d_out, cudaStream_t st);
int launch_unpack_kernel_layout(const void* d_wq, int K, int N, int8_t* d_q, cudaStream_t st);
int launch_update_scales(__nv_bfloat16* d_s, int64_t count, uint64_t seed, uint64_t index_base,
                         float coef_host, const float* coef_dev, cudaStream_t st);
// joint mode: plain SPSA on the un-quantised tensors
int launch_perturb_dense_bf16(const __nv_bfloat16* src, __nv_bfloat16* dst, int64_t count, uint64_t seed,
                              uint64_t index_base, float sign_eps, cudaStream_t st);
int launch_perturb_vectors(const float* const* src_table, const unsigned long long* base_table, int n_vec, int d,
                           uint64_t seed, float eps, float* plus, float* minus, cudaStream_t st);
int launch_update_dense_bf16(__nv_bfloat16* th, int64_t count, uint64_t seed, uint64_t index_base, const float* coef_dev,
                             cudaStream_t st);
int launch_update_vectors(float* const* table, const unsigned long long* base_table, int n_vec, int d, uint64_t seed,
                          const float* coef_dev, cudaStream_t st);
}  // namespace qzo
