// Block tables and slot maps of a serving step, from the requests' lengths: prefix sums over the requests, then one
// look-up per row, per block taken and per block given back.  Nothing a row reads is changed before the lengths are
// handed on at the end: blocks taken are named by their place on the stack (free list, then the finished requests'
// blocks), not read back from the table.
#include "qzo_common.cuh"
#include "launch.cuh"

#include <algorithm>

namespace qzo {
namespace {

constexpr int kSlotThreads = 1024;
constexpr int kRowsAndBlocks = 1, kLengths = 2;   // parts of the work a launch does

struct SlotParams {
  const int32_t *lens, *add;
  int B;
  int32_t* table;
  int width, log2_block;
  int32_t* free_list;
  int capacity;
  const int32_t* free_count;
  int max_rows;
  int32_t *row_seq, *positions, *slots, *lens_out, *free_count_out;
  int* status;
  int parts;
};

// Number of entries <= v[i] in the ascending a[0..n), for U values at once: as many steps for each, none waiting for another.
template <int U>
__device__ __forceinline__ void upper_bounds(const int* a, int n, const int v[U], int at[U]) {
#pragma unroll
  for (int i = 0; i < U; ++i) at[i] = 0;
  for (int step = 1 << (31 - __clz(n)); step > 0; step >>= 1) {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (at[i] + step <= n && a[at[i] + step - 1] <= v[i]) at[i] += step;
  }
}
__device__ __forceinline__ int upper_bound(const int* a, int n, int v) {
  int at[1];
  upper_bounds<1>(a, n, &v, at);
  return at[0];
}

struct Sums { long long rows, need, back; };

__device__ __forceinline__ Sums add_sums(Sums a, Sums b) { return {a.rows + b.rows, a.need + b.need, a.back + b.back}; }
__device__ __forceinline__ Sums shfl_up_sums(Sums v, int d) {
  return {__shfl_up_sync(0xffffffffu, v.rows, d), __shfl_up_sync(0xffffffffu, v.need, d), __shfl_up_sync(0xffffffffu, v.back, d)};
}

// Every CTA forms the same prefix sums, the rows and blocks are shared out among all threads.  Lengths and count are handed on
// by the last of the launches that read them (p.parts).  Short steps are bound by latency (loads that wait for one another),
// long ones by the instructions of the searches: 1024 requests, 65536 rows take 9.5 us on 32 SMs, 20 us on 8.
// kRows: rows of a thread at a time, whose searches and loads overlap.
template <int kRows>
__global__ void __launch_bounds__(kSlotThreads)
assign_slots_kernel(SlotParams p) {
  extern __shared__ int starts[];          // of each request: first row, first block taken, first block given back, length
  int* const row_start = starts;
  int* const need_start = starts + p.B;
  int* const back_start = starts + 2 * p.B;
  int* const lens = starts + 3 * p.B;
  __shared__ Sums warp_sums[kSlotThreads / 32];
  __shared__ int bad;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, threads = blockDim.x;
  const int all = threads * gridDim.x, me = blockIdx.x * threads + tid;
  const int mask = (1 << p.log2_block) - 1;
  auto blocks = [&](long long len) { return (len + mask) >> p.log2_block; };
  if (tid == 0) bad = 0;
  __syncthreads();
  serving_begin();
  serving_next();

  // each thread takes consecutive requests
  const int per = (p.B + threads - 1) / threads;
  Sums mine{0, 0, 0};
  bool wrong = false;
  auto sums_of = [&](int r) {
    const long long len = p.lens[r], add = p.add[r];
    if (len < 0 || blocks(len + (add > 0 ? add : 0)) > p.width) { wrong = true; return Sums{0, 0, 0}; }
    return add < 0 ? Sums{0, 0, blocks(len)} : Sums{add, blocks(len + add) - blocks(len), 0};
  };
  const int r0 = tid * per, r1 = min(p.B, r0 + per);
  for (int r = r0; r < r1; ++r) {
    mine = add_sums(mine, sums_of(r));
    lens[r] = p.lens[r];
  }
  const long long held = *p.free_count;
  Sums scan = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums up = shfl_up_sums(scan, d);
    if (lane >= d) scan = add_sums(scan, up);
  }
  if (lane == 31) warp_sums[warp] = scan;
  if (wrong) bad = 1;
  __syncthreads();
  // every warp scans the warps' sums
  Sums warps = lane * 32 < threads ? warp_sums[lane] : Sums{0, 0, 0};
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Sums up = shfl_up_sums(warps, d);
    if (lane >= d) warps = add_sums(warps, up);
  }
  const Sums total{__shfl_sync(0xffffffffu, warps.rows, 31), __shfl_sync(0xffffffffu, warps.need, 31), __shfl_sync(0xffffffffu, warps.back, 31)};
  Sums before{__shfl_sync(0xffffffffu, warps.rows, max(warp - 1, 0)), __shfl_sync(0xffffffffu, warps.need, max(warp - 1, 0)),
              __shfl_sync(0xffffffffu, warps.back, max(warp - 1, 0))};
  if (warp == 0) before = Sums{0, 0, 0};
  const long long top = held + total.back;
  const bool served = !bad && held >= 0 && top <= p.capacity && total.need <= top && total.rows <= p.max_rows;
  if (!served) {                                     // the same in every CTA
    if (p.parts & kRowsAndBlocks)
      for (int t = me; t < p.max_rows; t += all) { p.row_seq[t] = -1; p.positions[t] = -1; p.slots[t] = -1; }
    if (!(p.parts & kLengths)) return;
    for (int r = me; r < p.B; r += all) p.lens_out[r] = lens[r];
    if (me == 0) {
      *p.free_count_out = (int32_t)held;
      if (p.status) atomicOr(p.status, kStatusNotServed);
    }
    return;
  }
  Sums at = add_sums(before, Sums{scan.rows - mine.rows, scan.need - mine.need, scan.back - mine.back});
  for (int r = r0; r < r1; ++r) {
    row_start[r] = (int)at.rows; need_start[r] = (int)at.need; back_start[r] = (int)at.back;
    at = add_sums(at, sums_of(r));
  }
  __syncthreads();

  auto given_back = [&](int i) {                     // block i of those the finished requests give back
    const int r = upper_bound(back_start, p.B, i) - 1;
    return p.table[(size_t)r * p.width + (i - back_start[r])];
  };
  auto taken = [&](int i) {                          // block i of those the growing requests take
    const int s = (int)top - 1 - i;
    return s < held ? p.free_list[s] : given_back(s - (int)held);
  };
  if (p.parts & kRowsAndBlocks) {
    for (int t0 = me; t0 < p.max_rows; t0 += kRows * all) {
      int t[kRows], seq[kRows], id[kRows], pos[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) t[i] = t0 + i * all;
      upper_bounds<kRows>(row_start, p.B, t, seq);
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int r = --seq[i];
        pos[i] = id[i] = -1;
        if (t[i] < total.rows) {
          pos[i] = lens[r] + (t[i] - row_start[r]);
          const int have = (int)blocks(lens[r]), b = pos[i] >> p.log2_block;
          id[i] = b < have ? p.table[(size_t)r * p.width + b] : taken(need_start[r] + b - have);
        }
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        if (t[i] >= p.max_rows) continue;
        p.row_seq[t[i]] = t[i] < total.rows ? seq[i] : -1;
        p.positions[t[i]] = pos[i];
        // an id that no pool can have (a table or stack of the caller's that holds one) must not wrap to a slot of another block
        p.slots[t[i]] = pos[i] < 0 ? -1 : (unsigned)id[i] > (unsigned)(INT32_MAX >> p.log2_block) ? INT32_MAX : (id[i] << p.log2_block) | (pos[i] & mask);
      }
    }
    for (int i = me; i < (int)total.need; i += all) {
      const int r = upper_bound(need_start, p.B, i) - 1;
      p.table[(size_t)r * p.width + blocks(lens[r]) + (i - need_start[r])] = taken(i);
    }
    for (int i = me; i < (int)total.back; i += all) p.free_list[held + i] = given_back(i);
  }
  if (!(p.parts & kLengths)) return;
  __syncthreads();                                   // alone in its launch, or the outputs are not the inputs
  for (int r = me; r < p.B; r += all) {
    const int add = p.add[r];
    p.lens_out[r] = add < 0 ? 0 : lens[r] + add;
  }
  if (me == 0) *p.free_count_out = (int32_t)(top - total.need);
}

}  // namespace
}  // namespace qzo

using namespace qzo;

extern "C" int qzo_assign_slots(const int32_t* d_lens, const int32_t* d_new, int B, int32_t* d_block_table, int table_width,
                                int block_size, int32_t* d_free, int free_capacity, const int32_t* d_free_count, int max_rows,
                                int32_t* d_row_seq, int32_t* d_positions, int32_t* d_slots, int32_t* d_lens_out,
                                int32_t* d_free_count_out, int* d_status, void* stream) {
  if (!d_lens || !d_new || !d_block_table || !d_free || !d_free_count || !d_row_seq || !d_positions || !d_slots ||
      !d_lens_out || !d_free_count_out)
    return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_lens, d_new, d_block_table, d_free, d_free_count, d_row_seq, d_positions, d_slots, d_lens_out, d_free_count_out, d_status))
    return QZO_ERR_BAD_ARG;
  if (B <= 0 || B > QZO_MAX_REQUESTS || table_width <= 0 || free_capacity <= 0 || max_rows <= 0 || max_rows > (1 << 30)) return QZO_ERR_BAD_ARG;
  if (!block_size_ok(block_size)) return QZO_ERR_BAD_ARG;
  // a request's length and the slots of the pool are 32-bit numbers
  if ((int64_t)table_width * block_size > INT32_MAX || (int64_t)free_capacity * block_size > INT32_MAX) return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  int log2_block = 0;
  while ((1 << log2_block) < block_size) ++log2_block;
  SlotParams p{d_lens, d_new, B, d_block_table, table_width, log2_block, d_free, free_capacity, d_free_count, max_rows,
               d_row_seq, d_positions, d_slots, d_lens_out, d_free_count_out, d_status, kRowsAndBlocks | kLengths};
  const int smem = 4 * B * (int)sizeof(int);
  constexpr int kMostSmem = 4 * QZO_MAX_REQUESTS * (int)sizeof(int);
  if (max_rows <= 2 * kSlotThreads) {
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(assign_slots_kernel<1>, kMostSmem, allowed));
    const int threads = std::min(kSlotThreads, ceil_div(std::max(B, max_rows), 32) * 32);
    return launch_serving(assign_slots_kernel<1>, dim3(1), dim3(threads), smem, 1, (cudaStream_t)stream, p);
  }
  // several CTAs for the rows; where lengths or count are replaced in place, a CTA of its own does that behind them
  static std::atomic<unsigned long long> allowed{0};
  QZO_CUDA_TRY(allow_dynamic_smem(assign_slots_kernel<4>, kMostSmem, allowed));
  constexpr int kThreads = 512;
  const bool in_place = d_lens_out == d_lens || d_free_count_out == d_free_count;
  if (in_place) p.parts = kRowsAndBlocks;
  QZO_TRY(launch_serving(assign_slots_kernel<4>, dim3(std::min(64, ceil_div(max_rows, 4 * kThreads))), dim3(kThreads), smem,
                                     1, (cudaStream_t)stream, p));
  if (!in_place) return QZO_OK;
  p.parts = kLengths;
  return launch_serving(assign_slots_kernel<4>, dim3(1), dim3(kThreads), smem, 1, (cudaStream_t)stream, p);
}
