// Pages of a cache whose requests share blocks: requests that go on as copies of one another, blocks that nobody holds given
// back, the live blocks moved to the front of the pool, and the copies of pages that either asks for.  Who holds a block is
// read from the tables each time; there are no counters to keep.
#include "qzo_common.cuh"
#include "launch.cuh"
#include "layers.cuh"

#include <cooperative_groups.h>

#include <algorithm>

namespace cg = cooperative_groups;

namespace qzo {
namespace {

constexpr int kPageThreads = 1024;
constexpr int kMostCtas = 8;                           // of a cluster
constexpr int kItem = 256;                             // table entries that a warp looks at in one go: eight to a lane

__device__ __forceinline__ int sum_before(int v, int* warp_sums, int* total) {      // exclusive prefix sum over the CTA
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int scan = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = scan;
  __syncthreads();
  int warps = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, warps, d);
    if (lane >= d) warps += up;
  }
  *total = __shfl_sync(0xffffffffu, warps, 31);
  const int before = __shfl_sync(0xffffffffu, warps, max(warp - 1, 0));
  return (warp ? before : 0) + scan - v;
}

struct TableParams {
  const int32_t *lens, *table;
  int B, width, log2_block, n_blocks, words;           // words: 32 blocks each
  int32_t *table_out, *free_list;
  int capacity;
  int32_t* free_count_out;
  int32_t *copies, *copy_count;                        // [most_copies][3]: from, to, tokens
  int most_copies;
  int* status;
};

// The warps of a cluster share out the tables' entries in pieces of kItem entries of one row: this lane's entries of a piece are
// j0 + 32 e.  Its loads are issued together.
struct Pieces {
  int per_row, first, step, all;
  __device__ Pieces(int B, int width, int rank, int ctas) {
    per_row = (width + kItem - 1) / kItem;
    all = B * per_row;
    step = (int)(blockDim.x >> 5) * ctas;
    first = rank * (int)(blockDim.x >> 5) + (int)(threadIdx.x >> 5);
  }
};
__device__ __forceinline__ void load_piece(const int32_t* row, int j0, int n, int id[kItem / 32]) {
#pragma unroll
  for (int e = 0; e < kItem / 32; ++e) id[e] = j0 + 32 * e < n ? row[j0 + 32 * e] : -1;
}
// Marks the blocks of a piece; false where an id is no block of the pool
__device__ __forceinline__ bool mark_piece(const int id[kItem / 32], int j0, int n, int n_blocks, uint32_t* map) {
  bool fine = true;
#pragma unroll
  for (int e = 0; e < kItem / 32; ++e) {
    if (j0 + 32 * e >= n) continue;
    if ((unsigned)id[e] >= (unsigned)n_blocks) fine = false;
    else atomicOr(&map[id[e] >> 5], 1u << (id[e] & 31));
  }
  return fine;
}
// The tables as they are, for a call that cannot be served
__device__ void hand_on_tables(const TableParams& t, int me, int all) {
  if (t.table_out != t.table)
    for (size_t i = me; i < (size_t)t.B * t.width; i += all) t.table_out[i] = t.table[i];
  for (int i = me; i < 3 * t.most_copies; i += all) t.copies[i] = -1;
  if (me) return;
  *t.copy_count = 0;
  if (t.status) atomicOr(t.status, kStatusNotServed);
}

// The word of a map joined over the cluster's CTAs
__device__ __forceinline__ uint32_t joined(cg::cluster_group& cluster, uint32_t* word) {
  uint32_t v = 0;
  for (int c = 0; c < (int)cluster.num_blocks(); ++c) v |= *cluster.map_shared_rank(word, c);
  return v;
}

// ----------------------------------------------------------------------------- fork

struct ForkParams {
  TableParams t;
  const int32_t *parents, *free_count;
  int32_t* lens_out;
};

// Every CTA of the cluster knows all lengths and parents; the tables are shared out among its warps.  A CTA marks the blocks it
// meets in bit maps of its own, held by a request that goes on (kept) or by one that does not (left); the maps are joined over
// the cluster, each CTA taking a range of words.  Left and not kept: the block is free.
// Bound by what has to come one after the other: lengths and parents, tables, maps, numbers before a CTA, the stack, the new tables, with a
// barrier of the cluster at three places (4.8 us for 4 requests by one CTA of 256 threads, 8.1 us for 64 requests, 15.3 us for 1024 of up to
// 250 blocks each, whose tables are read twice and written at 0.2 TB/s).
__global__ void __launch_bounds__(kPageThreads)
fork_requests_kernel(ForkParams p) {
  const TableParams& t = p.t;
  extern __shared__ int smem[];
  int* const lens = smem;                              // [B]
  int* const first = lens + t.B;                       // [B]: the first request that goes on from this one
  int* const order = first + t.B;                      // [B]: how many before this one take a block, -1 where it takes none
  uint32_t* const kept = (uint32_t*)(order + t.B);     // [words]
  uint32_t* const left = kept + t.words;               // [words]
  __shared__ int warp_sums[32];
  __shared__ int given_here, bad;                      // blocks that this CTA's words give back; whether something is wrong
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
  const int me = rank * threads + tid, all = ctas * threads;
  const int mask = (1 << t.log2_block) - 1;
  auto blocks = [&](int len) { return (int)(((unsigned)len + mask) >> t.log2_block); };
  for (int i = tid; i < t.B; i += threads) first[i] = INT32_MAX;
  for (int i = tid; i < 2 * t.words; i += threads) kept[i] = 0u;
  if (tid == 0) bad = 0;
  __syncthreads();
  serving_begin();
  serving_next();
  const int held = *p.free_count;
  for (int r = tid; r < t.B; r += threads) {
    const int len = t.lens[r], parent = p.parents[r];
    const bool fine = len >= 0 && blocks(len) <= t.width && parent < t.B;
    lens[r] = fine ? len : 0;
    if (!fine) bad = 1;
    else if (parent >= 0) atomicMin(&first[parent], r);
  }
  __syncthreads();
  // who takes a block of its own: consecutive requests to a thread
  const int per = (t.B + threads - 1) / threads, r0 = min(t.B, tid * per), r1 = min(t.B, r0 + per);
  auto takes = [&](int r) {
    const int parent = p.parents[r];
    return parent >= 0 && parent < t.B && (lens[parent] & mask) && first[parent] != r;
  };
  int mine = 0, taken;
  for (int r = r0; r < r1; ++r) mine += takes(r);
  int at = sum_before(mine, warp_sums, &taken);
  for (int r = r0; r < r1; ++r) order[r] = takes(r) ? at++ : -1;

  const Pieces pieces(t.B, t.width, rank, ctas);
  for (int i = pieces.first; i < pieces.all; i += pieces.step) {
    const int r = i / pieces.per_row, n = blocks(lens[r]), j0 = i % pieces.per_row * kItem + lane;
    if (j0 - lane >= n) continue;
    int id[kItem / 32];
    load_piece(t.table + (size_t)r * t.width, j0, n, id);
    if (!mark_piece(id, j0, n, t.n_blocks, first[r] == INT32_MAX ? left : kept)) bad = 1;
  }
  cluster.sync();
  // each CTA a range of words, each thread consecutive ones of it
  const int range = (t.words + ctas - 1) / ctas, range0 = min(t.words, rank * range), range1 = min(t.words, range0 + range);
  const int each = (range + threads - 1) / threads, w0 = min(range1, range0 + tid * each), w1 = min(range1, w0 + each);
  mine = 0;
  for (int w = w0; w < w1; ++w) {
    const uint32_t free_now = joined(cluster, left + w) & ~joined(cluster, kept + w);
    left[w] = free_now;                                // no other CTA reads these words of this one
    mine += __popc(free_now);
  }
  int given;
  at = sum_before(mine, warp_sums, &given);
  if (tid == 0) given_here = given;
  cluster.sync();
  int before = 0, total = 0, wrong = 0;
  for (int c = 0; c < ctas; ++c) {
    const int n = *cluster.map_shared_rank(&given_here, c);
    if (c < rank) before += n;
    total += n;
    wrong |= *cluster.map_shared_rank(&bad, c);
  }
  const long long top = (long long)held + total;
  const bool served = !wrong && held >= 0 && top <= t.capacity && taken <= top;      // the same in every CTA
  if (served) {
    at += held + before;
    for (int w = w0; w < w1; ++w)
      for (uint32_t m = left[w]; m; m &= m - 1) t.free_list[at++] = 32 * w + __ffs(m) - 1;
  }
  cluster.sync();                                      // the stack is written, and no CTA looks into another any more
  if (!served) {
    hand_on_tables(t, me, all);
    for (int r = me; r < t.B; r += all) p.lens_out[r] = t.lens[r];
    if (me == 0) *t.free_count_out = held;
    return;
  }
  auto fresh = [&](int r) { return t.free_list[(int)top - 1 - order[r]]; };
  for (int i = pieces.first; i < pieces.all; i += pieces.step) {
    const int r = i / pieces.per_row, parent = p.parents[r], j0 = i % pieces.per_row * kItem + lane;
    const int n = parent < 0 ? 0 : blocks(lens[parent]);
    int id[kItem / 32];
    load_piece(t.table + (size_t)max(parent, 0) * t.width, j0, n, id);
#pragma unroll
    for (int e = 0; e < kItem / 32; ++e) {
      const int j = j0 + 32 * e;
      if (j == n - 1 && order[r] >= 0) {
        int32_t* const copy = t.copies + 3 * order[r];
        copy[0] = id[e];
        copy[1] = id[e] = fresh(r);
        copy[2] = lens[parent] & mask;
      }
      if (j < t.width) t.table_out[(size_t)r * t.width + j] = id[e];
    }
  }
  for (int r = me; r < t.B; r += all) p.lens_out[r] = p.parents[r] < 0 ? 0 : lens[p.parents[r]];
  for (int i = 3 * taken + me; i < 3 * t.most_copies; i += all) t.copies[i] = -1;
  if (me) return;
  *t.copy_count = taken;
  *t.free_count_out = (int32_t)(top - taken);
}

// ----------------------------------------------------------------------------- compaction

struct CompactParams {
  TableParams t;
  int keep;                                            // blocks of the pool afterwards
  int range_log2;                                      // words that a CTA joins
};

// The blocks that are held are marked as above.  With n of them, those from n on move to the holes below n, both in ascending
// order: a block's place among its kind follows from the number of held blocks below it, kept for each word of the map.
// Bound as the kernel above is: 6.9 us for a pool of some dozens of blocks, 11.7 us for one of a thousand.
__global__ void __launch_bounds__(kPageThreads)
compact_blocks_kernel(CompactParams p) {
  const TableParams& t = p.t;
  extern __shared__ int smem[];
  uint32_t* const map = (uint32_t*)smem;               // [words]
  int* const below = smem + t.words;                   // [words]: held blocks in front of the word, within its CTA's range
  __shared__ int warp_sums[32], offsets[kMostCtas];
  __shared__ int held_here, bad;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ctas = cluster.num_blocks(), tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
  const int me = rank * threads + tid, all = ctas * threads;
  const int mask = (1 << t.log2_block) - 1;
  auto blocks = [&](int len) { return (int)(((unsigned)len + mask) >> t.log2_block); };
  for (int i = tid; i < t.words; i += threads) map[i] = 0u;
  if (tid == 0) bad = 0;
  __syncthreads();
  serving_begin();
  serving_next();
  const Pieces pieces(t.B, t.width, rank, ctas);
  for (int i = pieces.first; i < pieces.all; i += pieces.step) {
    const int r = i / pieces.per_row, len = t.lens[r], n = blocks(max(len, 0)), j0 = i % pieces.per_row * kItem + lane;
    if (len < 0 || n > t.width) { bad = 1; continue; }
    if (j0 - lane >= n) continue;
    int id[kItem / 32];
    load_piece(t.table + (size_t)r * t.width, j0, n, id);
    if (!mark_piece(id, j0, n, t.n_blocks, map)) bad = 1;
  }
  cluster.sync();
  const int range = 1 << p.range_log2, range0 = min(t.words, rank * range), range1 = min(t.words, range0 + range);
  const int each = (range + threads - 1) / threads, w0 = min(range1, range0 + tid * each), w1 = min(range1, w0 + each);
  int mine = 0;
  for (int w = w0; w < w1; ++w) {
    map[w] = joined(cluster, map + w);                 // no other CTA reads these words of this one before the next barrier
    mine += __popc(map[w]);
  }
  int total;
  int at = sum_before(mine, warp_sums, &total);
  for (int w = w0; w < w1; ++w) {
    below[w] = at;
    at += __popc(map[w]);
  }
  if (tid == 0) held_here = total;
  cluster.sync();
  // the other ranges' words and counts come here; a CTA's own range stays as it is
  for (int w = tid; w < t.words; w += threads) {
    const int c = w >> p.range_log2;
    if (c == rank) continue;
    map[w] = *cluster.map_shared_rank(map + w, c);
    below[w] = *cluster.map_shared_rank(below + w, c);
  }
  int n_held = 0, wrong = 0;
  for (int c = 0; c < ctas; ++c) {
    if (tid == 0) offsets[c] = n_held;
    n_held += *cluster.map_shared_rank(&held_here, c);
    wrong |= *cluster.map_shared_rank(&bad, c);
  }
  __syncthreads();
  auto held_below = [&](int id) {                      // for id < 32 words
    const int w = id >> 5;
    return offsets[w >> p.range_log2] + below[w] + __popc(map[w] & ((1u << (id & 31)) - 1));
  };
  const int stay = n_held < 32 * t.words ? held_below(n_held) : n_held, moves = n_held - stay;
  const bool served = !wrong && n_held <= p.keep && p.keep - n_held <= t.capacity && moves <= t.most_copies;      // the same in every CTA
  if (served) {
    for (int w = w0; w < w1; ++w) {
      for (int b = 0; b < 32; ++b) {
        const int id = 32 * w + b;
        const bool here = map[w] >> b & 1;
        if (here && id >= n_held) t.copies[3 * (held_below(id) - stay)] = id;
        if (!here && id < n_held) {
          int32_t* const copy = t.copies + 3 * (id - held_below(id));
          copy[1] = id;
          copy[2] = 1 << t.log2_block;
        }
      }
    }
  }
  cluster.sync();                                      // the copies are listed, and no CTA looks into another any more
  if (!served) return hand_on_tables(t, me, all);
  for (int i = pieces.first; i < pieces.all; i += pieces.step) {
    const int r = i / pieces.per_row, n = blocks(t.lens[r]), j0 = i % pieces.per_row * kItem + lane;
    int id[kItem / 32];
    load_piece(t.table + (size_t)r * t.width, j0, n, id);
#pragma unroll
    for (int e = 0; e < kItem / 32; ++e)
      if (id[e] >= n_held) id[e] = t.copies[3 * (held_below(id[e]) - stay) + 1];
#pragma unroll
    for (int e = 0; e < kItem / 32; ++e)
      if (j0 + 32 * e < t.width) t.table_out[(size_t)r * t.width + j0 + 32 * e] = id[e];
  }
  for (int i = me; i < p.keep - n_held; i += all) t.free_list[i] = p.keep - 1 - i;
  for (int i = 3 * moves + me; i < 3 * t.most_copies; i += all) t.copies[i] = -1;
  if (me) return;
  *t.copy_count = moves;
  *t.free_count_out = p.keep - n_held;
}

// ----------------------------------------------------------------------------- copies of pages

constexpr int kCopyThreads = 256, kCopyUnroll = 8, kMostPlanes = 256;      // planes: keys and values of a layer each

struct CopyParams {
  uint8_t* planes[kMostPlanes];
  int n_planes;
  const int32_t *copies, *copy_count;
  int most, n_blocks, heads, block_size, row_units;    // 16-byte units of a head's token
  int parts, part_heads;                               // a block's heads in parts
  int* status;
};

// A turn of a CTA = some heads of one block in one plane: in each head the listed tokens lie side by side.
// Bound by HBM: every byte is read and written once (198 MB each way in 64 us, 6.2 TB/s, the rate of a plain copy).
__global__ void __launch_bounds__(kCopyThreads)
copy_blocks_kernel(const __grid_constant__ CopyParams p) {
  serving_begin();
  serving_next();
  const int count = min(max(*p.copy_count, 0), p.most);
  const long long turns = (long long)count * p.n_planes * p.parts;
  const int head_units = p.block_size * p.row_units;
  for (long long turn = blockIdx.x; turn < turns; turn += gridDim.x) {
    const int part = (int)(turn % p.parts), plane = (int)(turn / p.parts % p.n_planes), k = (int)(turn / p.parts / p.n_planes);
    const int from = p.copies[3 * k], to = p.copies[3 * k + 1], tokens = p.copies[3 * k + 2];
    if ((unsigned)from >= (unsigned)p.n_blocks || (unsigned)to >= (unsigned)p.n_blocks || (unsigned)tokens > (unsigned)p.block_size) {
      if (threadIdx.x == 0 && p.status) atomicOr(p.status, kStatusBadToken);
      continue;
    }
    const int h0 = part * p.part_heads, heads = min(p.heads - h0, p.part_heads), run = tokens * p.row_units, all = heads * run;
    const uint4* src = reinterpret_cast<const uint4*>(p.planes[plane]) + ((size_t)from * p.heads + h0) * head_units;
    uint4* dst = reinterpret_cast<uint4*>(p.planes[plane]) + ((size_t)to * p.heads + h0) * head_units;
    for (int i0 = threadIdx.x; i0 < all; i0 += kCopyThreads * kCopyUnroll) {
      uint4 v[kCopyUnroll];
      int at[kCopyUnroll];
#pragma unroll
      for (int e = 0; e < kCopyUnroll; ++e) {
        const int i = i0 + e * kCopyThreads;
        at[e] = i < all ? i / run * head_units + i % run : -1;
        if (at[e] >= 0) v[e] = src[at[e]];
      }
#pragma unroll
      for (int e = 0; e < kCopyUnroll; ++e)
        if (at[e] >= 0) dst[at[e]] = v[e];
    }
  }
}

int log2_up(int v) {
  int n = 0;
  while ((1 << n) < v) ++n;
  return n;
}

bool tables_ok(const void* lens, const void* table, const void* table_out, const void* free_list, const void* count, const void* copies,
               const void* copy_count, int B, int width, int block_size, int n_blocks, int capacity) {
  if (!lens || !table || !table_out || !free_list || !count || !copies || !copy_count) return false;
  if (B <= 0 || B > QZO_MAX_REQUESTS || width <= 0 || capacity <= 0 || n_blocks <= 0 || n_blocks > QZO_MAX_POOL_BLOCKS) return false;
  return block_size_ok(block_size) && (int64_t)width * block_size <= kMostKeys && (int64_t)n_blocks * block_size <= INT32_MAX;
}

// CTAs of the cluster that goes over B tables and a pool, and their threads: small ones do with fewer, which meet sooner.  A compaction goes over every
// block of the pool and its whole stack, a fork over its bit maps (4 requests of 32 blocks, one CTA against eight, us: compaction in a pool of
// 4096 blocks 9.0 and 10.2, of 16384 12.6 and 9.8, of 524288 102 and 30; fork of 65536 6.1 and 7.7, of 524288 22.0 and 15.5).
constexpr int kCompactPool = 16384, kForkPool = 131072;              // blocks from which on eight take the call
int table_ctas(int B, int width, int n_blocks, int most_blocks) { return (int64_t)B * width > 4096 || n_blocks >= most_blocks ? kMostCtas : 1; }
int table_threads(int B, int width, int words) { return (int64_t)B * width <= 1024 && words <= 1024 ? 256 : kPageThreads; }

}  // namespace
}  // namespace qzo

using namespace qzo;

extern "C" {

int qzo_fork_requests(const int32_t* d_lens, const int32_t* d_parents, int B, const int32_t* d_block_table, int table_width, int block_size,
                      int n_blocks, int32_t* d_free, int free_capacity, const int32_t* d_free_count, int32_t* d_lens_out,
                      int32_t* d_block_table_out, int32_t* d_free_count_out, int32_t* d_copies, int32_t* d_copy_count, int* d_status, void* stream) {
  if (!tables_ok(d_lens, d_block_table, d_block_table_out, d_free, d_free_count, d_copies, d_copy_count, B, table_width, block_size, n_blocks, free_capacity))
    return QZO_ERR_BAD_ARG;
  if (!d_parents || !d_lens_out || !d_free_count_out || d_block_table_out == d_block_table) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_lens, d_parents, d_block_table, d_free, d_free_count, d_lens_out, d_block_table_out, d_free_count_out, d_copies, d_copy_count, d_status))
    return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  const int words = ceil_div(n_blocks, 32);
  ForkParams p{{d_lens, d_block_table, B, table_width, log2_up(block_size), n_blocks, words, d_block_table_out, d_free, free_capacity, d_free_count_out,
                d_copies, d_copy_count, B, d_status}, d_parents, d_free_count, d_lens_out};
  {
    static std::atomic<unsigned long long> allowed{0};
    constexpr int kMost = (3 * QZO_MAX_REQUESTS + 2 * (QZO_MAX_POOL_BLOCKS / 32)) * (int)sizeof(int);
    QZO_CUDA_TRY(allow_dynamic_smem(fork_requests_kernel, kMost, allowed));
  }
  const int ctas = table_ctas(B, table_width, n_blocks, kForkPool);
  return launch_serving(fork_requests_kernel, dim3(ctas), dim3(table_threads(B, table_width, words)), (3 * B + 2 * words) * sizeof(int), ctas, (cudaStream_t)stream, p);
}

int qzo_compact_blocks(const int32_t* d_lens, int B, const int32_t* d_block_table, int table_width, int block_size, int n_blocks, int keep,
                       int32_t* d_block_table_out, int32_t* d_free, int free_capacity, int32_t* d_free_count_out, int32_t* d_copies,
                       int max_copies, int32_t* d_copy_count, int* d_status, void* stream) {
  if (!tables_ok(d_lens, d_block_table, d_block_table_out, d_free, d_free_count_out, d_copies, d_copy_count, B, table_width, block_size, n_blocks, free_capacity))
    return QZO_ERR_BAD_ARG;
  if (keep <= 0 || keep > n_blocks || max_copies <= 0 || max_copies > QZO_MAX_POOL_BLOCKS) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_lens, d_block_table, d_block_table_out, d_free, d_free_count_out, d_copies, d_copy_count, d_status)) return QZO_ERR_BAD_ARG;
  QZO_TRY(check_device());
  const int words = ceil_div(n_blocks, 32), ctas = table_ctas(B, table_width, n_blocks, kCompactPool);
  CompactParams p{{d_lens, d_block_table, B, table_width, log2_up(block_size), n_blocks, words, d_block_table_out, d_free, free_capacity, d_free_count_out,
                   d_copies, d_copy_count, max_copies, d_status}, keep, log2_up(ceil_div(words, ctas))};
  {
    static std::atomic<unsigned long long> allowed{0};
    constexpr int kMost = 2 * (QZO_MAX_POOL_BLOCKS / 32) * (int)sizeof(int);
    QZO_CUDA_TRY(allow_dynamic_smem(compact_blocks_kernel, kMost, allowed));
  }
  return launch_serving(compact_blocks_kernel, dim3(ctas), dim3(table_threads(B, table_width, words)), 2 * words * sizeof(int), ctas, (cudaStream_t)stream, p);
}

int qzo_copy_blocks(const qzo_kv_cache* h_caches, int n_caches, const int32_t* d_copies, const int32_t* d_copy_count, int max_copies,
                    int* d_status, void* stream) {
  if (!h_caches || n_caches <= 0 || !d_copies || !d_copy_count || max_copies <= 0 || max_copies > QZO_MAX_POOL_BLOCKS) return QZO_ERR_BAD_ARG;
  if (!words_aligned(d_copies, d_copy_count, d_status)) return QZO_ERR_BAD_ARG;
  const qzo_kv_cache& c0 = h_caches[0];
  for (int i = 0; i < n_caches; ++i) {
    const qzo_kv_cache& c = h_caches[i];
    if (!cache_ok(&c)) return QZO_ERR_BAD_ARG;
    if (c.dtype != c0.dtype || c.n_blocks != c0.n_blocks || c.block_size != c0.block_size || c.n_kv_heads != c0.n_kv_heads || c.head_dim != c0.head_dim)
      return QZO_ERR_BAD_ARG;
  }
  QZO_TRY(check_device());
  CopyParams p{};
  p.copies = d_copies;
  p.copy_count = d_copy_count;
  p.most = max_copies;
  p.n_blocks = c0.n_blocks;
  p.heads = c0.n_kv_heads;
  p.block_size = c0.block_size;
  p.row_units = c0.head_dim * (c0.dtype == QZO_DTYPE_E4M3 ? 1 : 2) / 16;
  p.part_heads = std::max(1, kCopyThreads * kCopyUnroll / (p.block_size * p.row_units));
  p.parts = ceil_div(p.heads, p.part_heads);
  p.status = d_status;
  for (int first = 0; first < n_caches; first += kMostPlanes / 2) {
    p.n_planes = 2 * std::min(n_caches - first, kMostPlanes / 2);
    for (int i = 0; i < p.n_planes / 2; ++i) {
      p.planes[2 * i] = (uint8_t*)h_caches[first + i].k;
      p.planes[2 * i + 1] = (uint8_t*)h_caches[first + i].v;
    }
    const int64_t turns = (int64_t)max_copies * p.n_planes * p.parts;
    QZO_TRY(launch_serving(copy_blocks_kernel, dim3((unsigned)std::min<int64_t>(turns, kSMs * 8)), dim3(kCopyThreads), 0, 1, (cudaStream_t)stream, p));
  }
  return QZO_OK;
}

}  // extern "C"
