// Block tables and slot maps of a serving step, from the requests' lengths: prefix sums over the requests, then one
// look-up per row, per block taken and per block given back.  Nothing a row reads is changed before the lengths are
// handed on at the end: blocks taken are named by their place on the stack (free list, then the finished requests'
// blocks), not read back from the table.
#include "qzo_common.cuh"
#include "launch.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace qzo {
namespace {

constexpr int kSlotThreads = 1024;
constexpr int kSlotCluster = 8;

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
};

// number of entries <= v in the ascending a[0..n)
__device__ __forceinline__ int upper_bound(const int* a, int n, int v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid + 1; else hi = mid;
  }
  return lo;
}

struct Sums { long long rows, need, back; };

__device__ __forceinline__ Sums add_sums(Sums a, Sums b) { return {a.rows + b.rows, a.need + b.need, a.back + b.back}; }
__device__ __forceinline__ Sums shfl_up_sums(Sums v, int d) {
  return {__shfl_up_sync(0xffffffffu, v.rows, d), __shfl_up_sync(0xffffffffu, v.need, d), __shfl_up_sync(0xffffffffu, v.back, d)};
}

// A cluster of CTAs (one for short steps): every CTA forms the same prefix sums, the rows and blocks are shared out among all
// of their threads.  What bounds it is latency: loads that wait for one another and searches in shared memory.
__global__ void __launch_bounds__(kSlotThreads)
assign_slots_kernel(SlotParams p) {
  extern __shared__ int starts[];          // of each request: first row, first block taken, first block given back, length
  int* const row_start = starts;
  int* const need_start = starts + p.B;
  int* const back_start = starts + 2 * p.B;
  int* const lens = starts + 3 * p.B;
  __shared__ Sums warp_sums[kSlotThreads / 32];
  __shared__ int bad;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, threads = blockDim.x;
  const int all = threads * (int)cluster.num_blocks(), me = (int)cluster.block_rank() * threads + tid;
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
  Sums before{0, 0, 0}, total{0, 0, 0};
  for (int w = 0; w * 32 * per < p.B; ++w) {         // warps that have requests
    if (w == warp) before = total;
    total = add_sums(total, warp_sums[w]);
  }
  const long long top = held + total.back;
  const bool served = !bad && held >= 0 && top <= p.capacity && total.need <= top && total.rows <= p.max_rows;
  if (!served) {                                     // the same in every CTA
    for (int t = me; t < p.max_rows; t += all) { p.row_seq[t] = -1; p.positions[t] = -1; p.slots[t] = -1; }
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
  int seq = 0;                                       // the request of the thread's last row: the next row's is no earlier one
  for (int t = me; t < p.max_rows; t += all) {
    int pos = -1, slot = -1;
    const bool row = t < total.rows;
    if (row) {
      if (seq + 1 < p.B && t >= row_start[seq + 1]) seq += upper_bound(row_start + seq, p.B - seq, t) - 1;
      pos = lens[seq] + (t - row_start[seq]);
      const int have = (int)blocks(lens[seq]), b = pos >> p.log2_block;
      const int id = b < have ? p.table[(size_t)seq * p.width + b] : taken(need_start[seq] + b - have);
      slot = id < 0 ? -1 : (id << p.log2_block) | (pos & mask);
    }
    p.row_seq[t] = row ? seq : -1; p.positions[t] = pos; p.slots[t] = slot;
  }
  for (int i = me; i < (int)total.need; i += all) {
    const int r = upper_bound(need_start, p.B, i) - 1;
    p.table[(size_t)r * p.width + blocks(lens[r]) + (i - need_start[r])] = taken(i);
  }
  for (int i = me; i < (int)total.back; i += all) p.free_list[held + i] = given_back(i);
  cluster.sync();                                    // every CTA has read the lengths and the count
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
  if (B <= 0 || B > QZO_MAX_REQUESTS || table_width <= 0 || free_capacity <= 0 || max_rows <= 0) return QZO_ERR_BAD_ARG;
  if (!block_size_ok(block_size)) return QZO_ERR_BAD_ARG;
  // a request's length and the slots of the pool are 32-bit numbers
  if ((int64_t)table_width * block_size > INT32_MAX || (int64_t)free_capacity * block_size > INT32_MAX) return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  int log2_block = 0;
  while ((1 << log2_block) < block_size) ++log2_block;
  const SlotParams p{d_lens, d_new, B, d_block_table, table_width, log2_block, d_free, free_capacity, d_free_count, max_rows,
                     d_row_seq, d_positions, d_slots, d_lens_out, d_free_count_out, d_status};
  const int smem = 4 * B * (int)sizeof(int);
  if (smem > 40 * 1024) {   // beyond the default limit of 48 KB with the kernel's own arrays
    static std::atomic<unsigned long long> allowed{0};
    QZO_CUDA_TRY(allow_dynamic_smem(assign_slots_kernel, 4 * QZO_MAX_REQUESTS * (int)sizeof(int), allowed));
  }
  const int threads = std::min(kSlotThreads, ceil_div(std::max(B, max_rows), 32) * 32);
  const int cluster = max_rows <= 2 * kSlotThreads ? 1 : kSlotCluster;
  return launch_serving<SlotParams>(assign_slots_kernel, dim3(cluster), dim3(threads), smem, cluster, (cudaStream_t)stream, p);
}
