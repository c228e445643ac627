/*
 * qzo.h - C ABI of the QZO hot path on NVIDIA B200 (sm_100a).
 *
 * QZO (Quantized Zeroth-order Optimization) fine-tunes a weight-only int4 LLM by
 * perturbing only its quantisation scales.  One optimisation step (Algorithm 1) is
 *   l+ = L((Delta + eps z) (.) theta_bar; B)          first forward
 *   l- = L((Delta - eps z) (.) theta_bar; B)          second forward
 *   d  = (l+ - l-) / (2 eps),  d' = clip(d, -C, C)    Eq. 5, Eq. 6
 *   Delta_i <- max(Delta_i - eta d' z_i, 0)           seeded update
 * with z ~ N(0, I) regenerated from a seed and never stored (Sec. 3.1).
 *
 * Conventions
 *  - Every pointer named d_* is a DEVICE pointer owned by the caller; h_* is a HOST
 *    pointer.  The library allocates no device memory: model state lives in the
 *    caller's tensors and in one caller-provided workspace.
 *  - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *    Calls are asynchronous on that stream unless stated otherwise.
 *  - Every function returns QZO_OK (0) or a negative qzo_status.  No exceptions cross
 *    the boundary.  A model handle must not be used from two threads at once.
 *  - Only compute-capability 10.x devices are supported; there is no CPU or other
 *    backend (QZO_ERR_UNSUPPORTED_DEVICE).
 *
 * Interchange layouts
 *  - int4 weights, logical q[k][n] in [-8, 7] for Y[t][n] = sum_k X[t][k] W[k][n]:
 *    uint32 [K/8][N] row-major, nibble j (bits 4j..4j+3) of word [kw][n] holds
 *    u = q[8 kw + j][n] + 8.  K must be a multiple of 8, N a multiple of 8.
 *  - scales: bf16 [G][N] row-major, G = ceil(K / 128); group g covers rows
 *    128 g .. 128 g + 127 (Eq. 3, Eq. 4 with the group of 128 the paper uses).
 *  - logical scale index of scale [g][n] of a linear: index_base + g N + n.  It selects
 *    the Gaussian z_i = z(seed, i) (Philox4x32-10, see qzo_normals) and is independent of
 *    any tiling.  index_base must be a multiple of 4.
 *  - kernel layout of the int4 weights: produced by qzo_repack_int4; opaque.
 */
#ifndef QZO_H_
#define QZO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  QZO_OK = 0,
  QZO_ERR_BAD_ARG = -1,            /* null pointer, bad size, sign not in {-1,0,1}, eps <= 0, clip < 0 ... */
  QZO_ERR_UNSUPPORTED_DEVICE = -2, /* current device is not sm_100 */
  QZO_ERR_WORKSPACE = -3,          /* workspace too small or misaligned (256 bytes) */
  QZO_ERR_NONFINITE = -4,          /* a loss or g is NaN/Inf; scales were left untouched */
  QZO_ERR_DEVICE_TIMEOUT = -5,     /* a bounded device-side wait expired (status word); scales untouched by that step */
  QZO_ERR_CUDA = -6,               /* a CUDA call failed; see qzo_last_cuda_error */
  QZO_ERR_MISSING_TENSOR = -7      /* qzo_init_model: a required tensor was not supplied */
} qzo_status;

enum { QZO_ARCH_LLAMA = 0, QZO_ARCH_OPT = 1 };
enum { QZO_DTYPE_BF16 = 0, QZO_DTYPE_F32 = 1, QZO_DTYPE_U32 = 2, QZO_DTYPE_I32 = 3, QZO_DTYPE_E4M3 = 4 };

/* Human-readable text of a status code (static storage). */
const char* qzo_strerror(int status);
/* cudaError_t value of the last failed CUDA call in this process (0 if none). */
int qzo_last_cuda_error(void);

/* ------------------------------------------------------------------------------------
 * Building blocks (each is one step of the path; exported for parity tests and sweeps)
 * ---------------------------------------------------------------------------------- */

/* Philox4x32-10 words of counter blocks block_base .. block_base+n_blocks-1 under key
 * `seed` (Sec. 3.1: only the seed is stored).  d_words: uint32 [n_blocks][4].
 * d_uniforms (may be NULL): float [n_blocks][4], U(x) = ((x >> 9) + 0.5) 2^-23. */
int qzo_philox_words(uint64_t seed, uint64_t block_base, int64_t n_blocks,
                     uint32_t* d_words, float* d_uniforms, void* stream);

/* z_i for i = index_base .. index_base+count-1 (Algorithm 1: "z ~ N(0,1)" after the
 * generator is reset with seed s).  d_z: float [count]. */
int qzo_normals(uint64_t seed, uint64_t index_base, int64_t count, float* d_z, void* stream);

/* Eq. 3 with Delta = absmax / (2^(4-1) - 1) per group of 128 rows and per column:
 * d_w float [K][N] -> d_qpacked uint32 [K/8][N] (interchange), d_scales bf16 [G][N].
 * Scale = bf16(absmax/7); q = clamp(rne(w / scale), -8, 7); zero scale gives q = 0. */
int qzo_quantize_int4(const float* d_w, int K, int N, uint32_t* d_qpacked, void* d_scales_bf16,
                      void* stream);

/* Eq. 4 storage: interchange uint32 [K/8][N] -> int8 q [K][N] (for bit-exact checks). */
int qzo_unpack_int4(const uint32_t* d_qpacked, int K, int N, int8_t* d_q, void* stream);

/* Size in bytes of the kernel-layout copy of a K x N int4 weight. */
int qzo_repacked_bytes(int K, int N, size_t* bytes);
/* interchange -> kernel layout (done once; theta_bar is fixed for the whole run,
 * the integer weights that Algorithm 1 takes as an input).  d_out: `bytes` from qzo_repacked_bytes, 256-aligned. */
int qzo_repack_int4(const uint32_t* d_qpacked, int K, int N, void* d_out, size_t out_bytes,
                    void* stream);
/* kernel layout -> int8 q [K][N]: what the GEMM's prologue sees (bit-exact check). */
int qzo_unpack_kernel_layout(const void* d_wq, int K, int N, int8_t* d_q, void* stream);

/* Workspace the GEMM needs for a problem (0 if none; split-K partial sums otherwise). */
int qzo_gemm_workspace_bytes(int M, int K, int N, size_t* bytes);

/* Perturbed W4A16 linear (Eq. 4 inside Eq. 5):
 *   Y[t][n] = sum_k X[t][k] (s[k/128][n] + sign eps z_i) q[k][n] (+ bias[n]),
 *   i = scale_index_base + (k/128) N + n; the perturbed scale is formed in fp32 inside the
 *   de-quantisation prologue; the stored scales are never modified.
 * d_x bf16 [M][K] row-major; d_wq kernel layout (qzo_repack_int4); d_scales bf16 [G][N];
 * d_bias float [N] or NULL; d_y bf16 [M][N], 16-byte aligned.  sign in {-1, 0, +1} (0 = unperturbed).
 * d_workspace: qzo_gemm_workspace_bytes, 256-aligned (may be NULL when that is 0).
 * d_status: int on the device, set non-zero if a bounded wait expired (may be NULL). */
int qzo_perturbed_gemm(const void* d_x_bf16, const void* d_wq, const void* d_scales_bf16,
                       const float* d_bias, void* d_y_bf16, int M, int K, int N,
                       uint64_t seed, uint64_t scale_index_base, int sign, float eps,
                       void* d_workspace, size_t workspace_bytes, int* d_status, void* stream);

/* The same linear for weights stored as 4-bit codes into a 16-entry table with one scale per block of 64
 * rows (block-scaled codebook storage such as NF4; the paper applies QZO to NF4 weights in its appendix
 * "Results with Stable Diffusion" and to codebook weights with channel-wise scales in Sec. 4.1: what QZO
 * perturbs and updates is the format's continuous scale, Eq. 5, so only the de-quantisation prologue differs):
 *   Y[t][n] = sum_k X[t][k] (s[k/64][n] + sign eps z_i) table[c[k][n]] (+ bias[n]),  i = scale_index_base + (k/64) N + n.
 * d_codes: codes c in [0, 15] in the kernel layout of qzo_repack_int4 (pack them like int4 values, code =
 * stored nibble); d_scales bf16 [ceil(K/64)][N]; h_table16: HOST pointer to the 16 table values (read during
 * the call, rounded to bf16 on the device).  Everything else as qzo_perturbed_gemm; the seeded update of such
 * scales is qzo_update_scales_flat. */
int qzo_perturbed_gemm_table16(const void* d_x_bf16, const void* d_codes, const void* d_scales_bf16,
                               const float* h_table16, const float* d_bias, void* d_y_bf16, int M, int K, int N,
                               uint64_t seed, uint64_t scale_index_base, int sign, float eps,
                               void* d_workspace, size_t workspace_bytes, int* d_status, void* stream);

/* The same table prologue for weights whose only continuous parameter is one scale per OUTPUT CHANNEL (the
 * paper's codebook setting, Sec. 4.1: AQLM-style codebook weights, of which QZO tunes the channel-wise scales;
 * here with a 16-entry scalar table standing in for the codebook):
 *   Y[t][n] = (s[n] + sign eps z_i) sum_k X[t][k] table[c[k][n]] (+ bias[n]),  i = scale_index_base + n.
 * d_scales bf16 [N]; everything else as qzo_perturbed_gemm_table16.  The seeded update of such scales is
 * qzo_update_scales_flat over N entries. */
int qzo_perturbed_gemm_codebook16_channelwise(const void* d_x_bf16, const void* d_codes, const void* d_scales_bf16,
                                              const float* h_table16, const float* d_bias, void* d_y_bf16,
                                              int M, int K, int N, uint64_t seed, uint64_t scale_index_base,
                                              int sign, float eps, void* d_workspace, size_t workspace_bytes,
                                              int* d_status, void* stream);

/* The same linear for callers that must not allocate device memory and have no workspace to
 * lend: for example a serving process that gave all device memory to its own pool when it
 * started, or a latency-critical loop in which the device-wide synchronisation of an allocation
 * is not acceptable.  (The paper has no counterpart; this is a property of the library.)
 * Arguments and result are those of qzo_perturbed_gemm without the workspace.  The split-K
 * partial sums go to a fixed array of QZO_NOALLOC_SCRATCH_BYTES inside the library image: every
 * device that loads the library holds that much until the process exits.  The call allocates
 * nothing: no cudaMalloc, no cudaFree, no allocating library routine.
 *  - A problem whose partial sums (qzo_gemm_workspace_bytes) exceed the array returns
 *    QZO_ERR_WORKSPACE and launches nothing.
 *  - The first call on each device looks the array's device address up (with that device
 *    current).  If no kernel of the library has run on that device yet, this is also the moment the
 *    driver loads the library's device code and reserves the array, which may synchronise the device:
 *    make that first call at start-up, and before any stream capture begins.  Later calls do neither.
 *  - All calls on a device share the one array, which keeps the last call's partial sums (none
 *    of it needs clearing: each call overwrites every element it later reads).  Two calls that
 *    overlap on the GPU (different streams) race on it; keep them on one stream or order them. */
#define QZO_NOALLOC_SCRATCH_BYTES (16u << 20)
int qzo_perturbed_gemm_noalloc(const void* d_x_bf16, const void* d_wq, const void* d_scales_bf16,
                               const float* d_bias, void* d_y_bf16, int M, int K, int N,
                               uint64_t seed, uint64_t scale_index_base, int sign, float eps,
                               int* d_status, void* stream);

/* Seeded update of a flat run of scales (Algorithm 1, last loop, with Eq. 6 applied to g):
 *   s_i <- bf16(max(s_i - (lr clip(g,-C,C)) z_i, 0)), i = index_base .. index_base+count-1.
 * d_scales bf16 [count], in place.  g must be finite, clip >= 0. */
int qzo_update_scales_flat(void* d_scales_bf16, int64_t count, uint64_t seed, uint64_t index_base,
                           float lr, float g, float clip, void* stream);

/* ------------------------------------------------------------------------------------
 * Serving operators: what a tuned model needs to answer.  (The paper tunes by forward passes and evaluates
 * the tuned model on question-answering tasks, Sec. 4.1; how it is served is this library's own design.)
 * All of them can be captured into a CUDA graph: they launch kernels and do nothing else.
 * Words "row", "slot", "position": a row is one token of this step; its position is its place in its
 * request, 0 for the first token; its slot is where its key and value live in the paged cache, block id *
 * block_size + place in the block.  A row with a negative position or slot is padding.
 * All int32 and float arrays lie on 4-byte boundaries.
 * d_status (int on the device, may be NULL): bit 1 is set when an index out of range is met (see each call).
 * ---------------------------------------------------------------------------------- */

/* Matrix-vector products with int4 weights and group scales, for up to QZO_GEMV_MAX_ROWS rows (the linear of
 * qzo_perturbed_gemm at sign 0 for a step of few tokens):
 *   Y[t][n] = sum_k X[t][k] s[k/128][n] q[k][n] (+ bias[n]).
 * The products X q of a group of 128 are summed in fp32 (each is exact; lowered by 2^10 until the end, so that no finite X
 * overflows there), then scaled in fp32.  Y is rounded once.
 * d_x bf16 [M][ldx], 16-byte aligned, ldx a multiple of 8 and >= K; d_wq kernel layout (qzo_repack_int4); d_scales bf16
 * [ceil(K/128)][N], both 16-byte aligned; d_bias float [N] or NULL; d_y bf16 [M][ldy], ldy >= N, must not overlap d_x.  K and N multiples of 8. */
#define QZO_GEMV_MAX_ROWS 16
int qzo_gemv_int4(const void* d_x_bf16, int ldx, const void* d_wq, const void* d_scales_bf16, const float* d_bias,
                  void* d_y_bf16, int ldy, int M, int K, int N, void* stream);

/* A paged key-value cache of one layer, described by the caller (host struct, read during the call): keys and
 * values in blocks [n_blocks][n_kv_heads][block_size][head_dim], 16-byte aligned.  dtype QZO_DTYPE_BF16 (both
 * scales 1) or QZO_DTYPE_E4M3: the stored code times the scale (2^-64 to 2^64) is the value; codes saturate at +-448 and are
 * those of the value times the scale's reciprocal in fp32.
 * block_size is a power of two from 16 to 256, head_dim 64 or 128, n_blocks * block_size < 2^31. */
typedef struct {
  void* k;
  void* v;
  int dtype;
  int n_blocks, block_size, n_kv_heads, head_dim;
  float k_scale, v_scale;
} qzo_kv_cache;

/* Table of the rotation: float [max_pos][head_dim/2][2] = {cos, sin}(pos * theta^(-2i/head_dim)), the angles
 * formed in fp64 (the table the model builds for itself).  32-byte aligned, max_pos * head_dim <= 2^30, head_dim 64 or 128. */
int qzo_rope_table(float* d_table, int max_pos, int head_dim, float theta, void* stream);

/* One pass over the new rows' queries, keys and values in front of the attention:
 *   q'[t][h] = rot(norm(q[t][h]) q_gain),  k'[t][h] = rot(norm(k[t][h]) k_gain),  v'[t][h] = v[t][h],
 * norm(x) = x / sqrt(mean(x^2) + norm_eps) over the head (left out, with its gain, where that gain is NULL), rot the
 * rotation of the pairs (i, i + head_dim/2) by the row's position (left out when d_table is NULL).  q' goes to
 * d_q_out, k' and v' into the cache at the row's slot; each is rounded once, from fp32.
 * d_q bf16 [T][ldq] with head h at h * head_dim, d_k and d_v alike with n_kv_heads heads; 16-byte aligned, strides
 * multiples of 8; d_q_out bf16 [T][ldqo], may be d_q itself (same stride) but not overlap it otherwise, nor d_k, d_v; gains float
 * [head_dim], d_table as qzo_rope_table writes it (gains and table 32-byte aligned).  d_positions, d_slots int32 [T]; the slots of one call are distinct.
 * A row with a negative position or slot is padding: nothing is written for it.  A slot beyond the cache or a position
 * beyond the table sets bit 1 of the status word: the first is not written, the second is turned by the table's last. */
int qzo_qk_norm_rope_cache(const void* d_q_bf16, int ldq, const void* d_k_bf16, int ldk, const void* d_v_bf16, int ldv,
                           const float* d_q_gain, const float* d_k_gain, float norm_eps, const float* d_table,
                           int max_pos, const int32_t* d_positions, const int32_t* d_slots, void* d_q_out_bf16,
                           int ldqo, const qzo_kv_cache* cache, int T, int n_heads, int* d_status, void* stream);

/* Workspace of qzo_paged_attention for R rows over tables of max_len = table_width * block_size <= 2^30 tokens (0 if none: the
 * partial results of rows whose cache is split over several CTAs otherwise). */
int qzo_paged_attention_workspace_bytes(int R, int n_heads, int n_kv_heads, int head_dim, int max_len, size_t* bytes);

/* Attention of one new token per row over the paged cache:
 *   out[t][h] = sum_j softmax_j(scale q[t][h] . k_j) v_j,  j = 0 .. position[t] (the row's own key among them),
 * with keys and values of head h / (n_heads / n_kv_heads) found through the block table: token j of request r lives in
 * block d_block_table[r][j / block_size].  A row with a negative position gives zeros, and so does one none of whose keys
 * scores above -inf.  Infinite and NaN values of keys that a row sees count as the sum says (an infinite value under a weight of
 * less than 2^-100 of the row's largest may give NaN).  Entries of the table behind a row's position, and the rest of its last block, are not looked at.
 * Several rows may belong to one request (a prompt's rows, each of which sees the keys up to its own).
 * d_q bf16 [R][ldq] and d_out bf16 [R][ldo], head h at h * head_dim, 16-byte aligned, strides multiples of 8, not
 * overlapping; d_block_table int32 [n_seqs][table_width], at most 2^30 tokens wide; d_row_seq int32 [R] = the request of each row, NULL: row t is
 * request t (R <= n_seqs); scale from 2^-40 to 2^40 (1 / sqrt(head_dim) as a rule); n_heads a multiple of n_kv_heads.
 * d_workspace: qzo_paged_attention_workspace_bytes, 256-aligned; calls that may run at the same time (two streams, two
 * captured graphs) need one each.  Nothing in it outlives the call.
 * A request outside [0, n_seqs), a position beyond the table or a block id outside the cache sets bit 1 of the status
 * word; such a row sees nothing, only the table's tokens, or nothing of that block. */
int qzo_paged_attention(const void* d_q_bf16, int ldq, const qzo_kv_cache* cache, const int32_t* d_block_table,
                        int n_seqs, int table_width, const int32_t* d_row_seq, const int32_t* d_positions, float scale,
                        void* d_out_bf16, int ldo, int R, int n_heads, void* d_workspace, size_t workspace_bytes,
                        int* d_status, void* stream);

/* Block tables and slot maps of a step, built on the device from the requests' lengths.
 * d_lens int32 [B]: tokens each request holds in the cache; d_new int32 [B]: tokens it adds in this step, 0 for none,
 * negative when it is finished.  d_block_table int32 [B][table_width]: entry j of request r names the block of its tokens
 * j * block_size ...; entries beyond its length mean nothing.  d_free int32 [free_capacity], d_free_count int32 [1]: the
 * stack of free blocks, its top at [count - 1].  In the order of the requests,
 *  - the blocks of finished requests are pushed on the stack (first entry first);
 *  - then each growing request takes the blocks it lacks from the top, one after the other, into its table;
 *  - rows are numbered request by request: d_row_seq, d_positions, d_slots int32 [max_rows], -1 behind the last row;
 *  - d_lens_out int32 [B] = the new lengths (0 for finished requests), d_free_count_out int32 [1] = the new count.
 * d_lens_out may be d_lens and d_free_count_out may be d_free_count; no other arguments overlap.
 * Ids are handed on as they are found; a row whose block id no cache can hold (negative, or 2^31 / block_size and more) gets
 * slot 2^31 - 1, which qzo_qk_norm_rope_cache reports.
 * When the step cannot be served (too few free blocks, a table too narrow, more rows than max_rows, a negative length, a
 * stack beyond its capacity), nothing is changed: lengths and count are handed on as they are, every row is padding, and
 * bit 2 of the status word is set.  B from 1 to QZO_MAX_REQUESTS, max_rows up to 2^30, block_size as in qzo_kv_cache. */
#define QZO_MAX_REQUESTS 4096
int qzo_assign_slots(const int32_t* d_lens, const int32_t* d_new, int B, int32_t* d_block_table, int table_width,
                     int block_size, int32_t* d_free, int free_capacity, const int32_t* d_free_count, int max_rows,
                     int32_t* d_row_seq, int32_t* d_positions, int32_t* d_slots, int32_t* d_lens_out,
                     int32_t* d_free_count_out, int* d_status, void* stream);

/* ------------------------------------------------------------------------------------
 * Model-level entry points
 * ---------------------------------------------------------------------------------- */

typedef struct qzo_model qzo_model; /* opaque handle (host memory owned by the library) */

typedef struct {
  int arch;        /* QZO_ARCH_LLAMA: RMSNorm, RoPE, SiLU-gated MLP, no bias;
                      QZO_ARCH_OPT: LayerNorm, learned positions, ReLU MLP, biases */
  int n_layers, d_model, n_heads, d_ffn, vocab, max_seq;
  int group_size;  /* must be 128 */
  float norm_eps, rope_theta;
} qzo_model_desc;

typedef struct {
  const char* name; /* see qzo_init_model */
  void* dptr;       /* device pointer */
  int dtype;        /* QZO_DTYPE_* */
  int64_t shape[2]; /* rows, cols (cols = 1 for vectors) */
} qzo_tensor;

/* Number of entries of the flat scale buffer (all block linears, layer-major, in the order
 * q,k,v,o,gate,up,down (Llama) / q,k,v,o,fc1,fc2 (OPT), each base rounded up to a multiple
 * of 8) and the number of trainable scales (Table 2: block linear weights / 128). */
int qzo_num_scales(const qzo_model_desc* desc, int64_t* flat_entries, int64_t* trainable);
/* Where linear `linear` (position in the order above) of layer `layer` sits in the flat buffer. */
int qzo_scale_layout(const qzo_model_desc* desc, int layer, int linear,
                     int64_t* index_base, int* G, int* N);

/* Bytes of workspace qzo_init_model needs for batches up to max_tokens = B*S tokens
 * (kernel-layout weights + activations + fp32 logits + split-K partials).  The activation
 * buffers hold 2 * max_tokens rows, because qzo_step runs both passes as one forward. */
int qzo_workspace_bytes(const qzo_model_desc* desc, int max_tokens, size_t* bytes);

/* Binds a model to caller-owned tensors (the inputs of Algorithm 1: scales Delta, integer
 * weights theta_bar).  Tensors, by name:
 *   "embed" bf16 [V][d]; "lm_head" bf16 [V][d]; "pos_embed" bf16 [max_seq][d] (OPT);
 *   "final_norm_w" f32 [d] (+ "final_norm_b", OPT); "scales" bf16 [flat_entries] (trained in place);
 *   "L<i>.norm1_w", "L<i>.norm2_w" f32 [d] (+ "_b", OPT);
 *   "L<i>.<lin>.qweight" u32 [K/8][N] interchange layout (copied into the workspace in kernel
 *   layout during this call; the caller may free it after the stream has drained);
 *   "L<i>.<lin>.bias" f32 [N] (OPT).
 * d_workspace: qzo_workspace_bytes, 256-aligned, must outlive the handle. */
int qzo_init_model(const qzo_model_desc* desc, const qzo_tensor* tensors, int n_tensors,
                   void* d_workspace, size_t workspace_bytes, int max_tokens, void* stream,
                   qzo_model** out);
int qzo_free_model(qzo_model* m);

/* One forward pass, L(Delta' (.) theta_bar; B) with Delta' = Delta + sign eps z(seed)
 * (either forward pass of Algorithm 1; sign 0 = unperturbed).  d_tokens, d_labels:
 * int32 [B][S]; label -100 is ignored; loss = mean next-token cross entropy over kept
 * positions, written to d_loss (float, device). */
int qzo_forward_loss(qzo_model* m, const int32_t* d_tokens, const int32_t* d_labels, int B, int S,
                     uint64_t seed, int sign, float eps, float* d_loss);

/* Seeded update of every scale of the model with a host-side g (clipped here, Eq. 6).
 * Non-finite g: QZO_ERR_NONFINITE and no write. */
int qzo_update_scales(qzo_model* m, uint64_t seed, float lr, float g, float clip);

/* Whole step of Algorithm 1 on device-resident tokens: two forwards (sign +1, -1), d, d' and
 * the update, with d formed on the device.  When B*S is 16, 32, 64, 128 or a multiple of 256 the
 * two forwards run as ONE pass over two copies of the batch (rows of the second copy take
 * -eps z); every kernel works row by row or sequence by sequence, so the losses are the ones two
 * separate passes give, bit for bit.
 * From the second call with the same (B, S) on, the launch sequence of the two forwards is replayed from a CUDA
 * graph recorded once (its GEMMs read seed and eps from device memory, the tokens come from the model's own
 * buffers); results are bit-identical to the direct launches.  See qzo_use_recorded_steps.
 * h_out (may be NULL): {l+, l-, d, d'}; when
 * non-NULL the call synchronises the stream.  The scales are left untouched (the update coefficient is
 * forced to zero on the device) and, when h_out is given, an error is returned if
 *  - either loss is not finite: QZO_ERR_NONFINITE;
 *  - a bounded device-side wait expired in any launch since qzo_init_model: QZO_ERR_DEVICE_TIMEOUT;
 *  - a token id lies outside [0, vocab): QZO_ERR_BAD_ARG.
 * The last two are sticky (status word, see qzo_device_status). */
int qzo_step(qzo_model* m, const int32_t* d_tokens, const int32_t* d_labels, int B, int S,
             uint64_t seed, float eps, float lr, float clip, float* h_out);

/* Recorded steps (CUDA graphs) of qzo_step / qzo_step_host / qzo_step_begin: on != 0 (the default) allows them, 0 makes every
 * step issue its launches directly.  They are bypassed anyway while joint mode, a debug capture or the per-GEMM
 * timing is on, for batch shapes beyond the first 16 a model has seen, and switched off for good if recording
 * ever fails. */
int qzo_use_recorded_steps(qzo_model* m, int on);
/* *h_count = number of batch shapes whose step is recorded at the moment, or -1 when recorded steps are
 * switched off (by qzo_use_recorded_steps, or because recording failed). */
int qzo_recorded_step_count(qzo_model* m, int* h_count);

/* The two halves of qzo_step, for data-parallel replicas (every rank holds the same theta_bar and Delta
 * and its own part of the batch; z depends on (seed, index) only, Sec. 3.1, so ranks exchange losses,
 * never parameters).
 * qzo_step_begin runs the two forward passes of Algorithm 1 on this rank's tokens and writes
 *   d_sums (device, float[4], 16-byte aligned) = {sum of token losses with +eps z, the same with -eps z,
 *   kept tokens of the + pass, kept tokens of the - pass}.
 * Between the calls the caller may add the d_sums of all ranks element by element (one all-reduce of four
 * floats, asynchronously on the same stream).  qzo_step_finish then forms l+- = sum / count, d = (l+ - l-) /
 * (2 eps), d' = clip(d, -C, C) (Eq. 6) and applies the seeded update (Algorithm 1, last loop), all on the
 * device; given equal d_sums and seed every rank ends with bit-identical scales.  h_out and the error
 * behaviour are those of qzo_step.  qzo_step is qzo_step_begin followed by qzo_step_finish. */
int qzo_step_begin(qzo_model* m, const int32_t* d_tokens, const int32_t* d_labels, int B, int S,
                   uint64_t seed, float eps, float* d_sums);
int qzo_step_finish(qzo_model* m, const float* d_sums, uint64_t seed, float eps, float lr, float clip,
                    float* h_out);

/* Joint mode (Sec. 3.2.1, closing remark: Q-SPSA on the scales may be combined with SPSA on the
 * un-quantised parts; Sec. 4.1, implementation details: the experiments with codebook weights train the
 * un-quantised parts that way, with plain SPSA and ZO-SGD).
 * After qzo_enable_joint_spsa every perturbed forward (sign +1 / -1) also perturbs the embedding matrix, the
 * lm_head matrix and every norm gain (and norm bias, OPT) as theta + sign eps z (Def. 3.1), and every step
 * also updates them in place, theta <- theta - lr_dense d' z (Def. 3.2; no clamp, that belongs to the
 * scales), with the same clipped d' as the scales.  z comes from the same (seed, index) stream at indices
 * that follow the scales': each base rounded up to a multiple of 8, in the order embed, lm_head, then per
 * layer norm1 gain (bias), norm2 gain (bias), then the final norm.  Position embeddings and the biases of
 * the linears stay fixed.  The caller's "embed", "lm_head" and norm tensors must be writable.
 * d_workspace: qzo_joint_workspace_bytes (perturbed copies of the vectors and of the lm_head for both
 * signs), 256-aligned, must outlive the handle; NULL switches the mode off.  Synchronises the stream. */
int qzo_joint_workspace_bytes(const qzo_model_desc* desc, size_t* bytes);
int qzo_enable_joint_spsa(qzo_model* m, void* d_workspace, size_t workspace_bytes, float lr_dense);

/* Same step with HOST token / label buffers (int32 [B][S]); copies them in, runs the step and
 * reads {l+, l-, d, d'} back.  Synchronises. */
int qzo_step_host(qzo_model* m, const int32_t* h_tokens, const int32_t* h_labels, int B, int S,
                  uint64_t seed, float eps, float lr, float clip, float* h_out);

/* One step of answering with the tuned model: R rows (new tokens of any requests, prompts' tokens among them) go
 * through the unperturbed model, their keys and values into the paged cache, and d_logits (float [R][vocab], 16-byte
 * aligned) receives the logits of each row.  Every row attends to its request's cached tokens up to itself, so a prompt is
 * a step of its own rows (the keys of all rows of a layer are written before its attention reads them).
 * h_caches: HOST array of n_layers cache descriptions (n_kv_heads = n_heads of the model, one block_size); d_tokens, d_row_seq,
 * d_positions, d_slots int32 [R], as qzo_assign_slots writes the last three; R <= max_tokens; positions < max_seq.
 * Rows of padding (negative position or slot) give logits that mean nothing and touch no cache.  An index out of range
 * (token, position, slot, block) sets bit 1 of what qzo_device_status reads; training steps go on as if it had not been met.
 * Up to QZO_GEMV_MAX_ROWS rows the linears run as qzo_gemv_int4, above as qzo_perturbed_gemm with sign 0.  Asynchronous on the model's
 * stream, and nothing but launches: a model whose stream is not the legacy default one can have its steps captured (they use the
 * model's buffers, so replays belong on that stream, in turn with its other work). */
int qzo_decode(qzo_model* m, const qzo_kv_cache* h_caches, const int32_t* d_tokens, const int32_t* d_row_seq,
               const int32_t* d_positions, const int32_t* d_slots, int R, const int32_t* d_block_table, int n_seqs,
               int table_width, float* d_logits);

/* The same step from the requests' side: qzo_assign_slots on (d_lens, d_new, ...), in place and for R rows, then qzo_decode of the
 * rows it numbers.  d_tokens int32 [R]: the new tokens, request by request, anything behind the last row; d_maps int32 [3][R]
 * receives row_seq, positions and slots.  The block size is the caches', d_block_table int32 [B][table_width], the other
 * arguments are those of the two calls.  d_status (may be NULL): bit 2 = the step could not be served; every row is padding
 * then and nothing else has changed. */
int qzo_decode_requests(qzo_model* m, const qzo_kv_cache* h_caches, const int32_t* d_tokens, int32_t* d_lens, const int32_t* d_new,
                        int B, int32_t* d_block_table, int table_width, int32_t* d_free, int free_capacity,
                        int32_t* d_free_count, int R, int32_t* d_maps, float* d_logits, int* d_status);

/* The trainable state (the inputs of Algorithm 1: the quantisation scales Delta that the caller hands over
 * and gets back).  linear_id = layer * L + position, L = 7 (Llama: q,k,v,o,gate,up,down) or 6 (OPT:
 * q,k,v,o,fc1,fc2): copies that linear's bf16 [G][N] scales out of / into the model's flat buffer;
 * linear_id = -1: the whole flat buffer (qzo_num_scales entries).  d_bf16 is a device pointer; `bytes` must
 * be exactly the size of what is copied (QZO_ERR_BAD_ARG otherwise).  Asynchronous on the model's stream.
 * Because z is a function of (seed, index) only, scales + step counter + base seed resume a run exactly. */
int qzo_get_scales(qzo_model* m, int linear_id, void* d_bf16, size_t bytes);
int qzo_set_scales(qzo_model* m, int linear_id, const void* d_bf16, size_t bytes);

/* Selects the decoder block whose output later forwards keep a copy of (-1 = none). */
int qzo_debug_set_capture(qzo_model* m, int layer);
/* Copies an intermediate of the LAST forward into d_out (bf16 [T][d] for which = 0: output of
 * decoder block `layer`, which must be the block chosen with qzo_debug_set_capture before that
 * forward; float [T][V] for which = 1: logits, layer ignored).  T is the token count of that
 * forward: B*S after qzo_forward_loss, 2*B*S after a qzo_step that ran both signs as one pass
 * (rows of the sign +1 copy first).  bytes below the size needed: QZO_ERR_BAD_ARG. */
int qzo_debug_layer_output(qzo_model* m, int layer, int which, void* d_out, size_t bytes);

/* Test entry for the bounded device-side waits (failure detection without a fault): runs the perturbed GEMM
 * (seed 1, sign +1, eps 1e-3, no bias, a problem without split-K) with the copies of quantisation group
 * `skip_group` of every CTA announced but never issued and with every wait bounded by wait_limit_cycles
 * (capped at the normal limit of about two seconds).  Every role of the kernel then runs out of its wait,
 * the CTA drains the copies it did issue, frees its tensor memory and RETURNS; *d_status becomes non-zero.
 * Nothing traps and nothing spins without bound.  The output is unspecified.  Later calls are unaffected. */
int qzo_debug_gemm_wait_expiry(const void* d_x_bf16, const void* d_wq, const void* d_scales_bf16, void* d_y_bf16,
                               int M, int K, int N, int skip_group, int64_t wait_limit_cycles, int* d_status,
                               void* stream);

/* Reads the device status: bit 0 = a bounded device-side wait expired in some launch since init
 * (returns QZO_ERR_DEVICE_TIMEOUT), bit 1 = a token id outside [0, vocab) was seen, or in qzo_decode another index
 * out of range (QZO_ERR_BAD_ARG); 0 = nothing to report.  What qzo_decode reports of indices stands in a word of its own,
 * which is read here with the training's but keeps no step from updating.  Synchronises. */
int qzo_device_status(qzo_model* m, int* h_status);
/* Overwrites the training's status word from the host and clears qzo_decode's (0 clears both).  For tests of the error path
 * of a step and for clearing the words after the caller has dealt with a report.  Synchronises. */
int qzo_debug_set_status(qzo_model* m, int value);

/* Per-GEMM timing: with max_launches > 0 every later perturbed-GEMM launch of this model (up to
 * max_launches between two reads) is bracketed by a pair of CUDA events on the model's stream;
 * 0 switches it off.  qzo_profile_read synchronises, returns the number of bracketed launches,
 * the sum of their durations in ms and of their algorithmic FLOPs (2 M K N), and rearms. */
int qzo_profile_gemms(qzo_model* m, int max_launches);
int qzo_profile_read(qzo_model* m, int64_t* launches, double* total_ms, double* total_flops);

/* Number of kernels the library launched since the process started, those of replayed recorded steps
 * included (for benchmark accounting). */
int64_t qzo_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* QZO_H_ */
