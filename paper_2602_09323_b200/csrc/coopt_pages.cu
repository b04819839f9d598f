// The pages of a cache: blocks copied, reserved, shared by forked sequences, released and compacted, for all layers that
// share a block table.
//
// A pool is a count per physical block of the table entries that hold it (0: free), the block table and the lengths.  There
// is no list of free blocks: whoever needs blocks gets the lowest free ones, in the order of the call's list, which makes
// every result a function of the inputs.  Finding them takes one look through the counts (4 bytes a block, against
// kilobytes that a block's contents have), by a planning kernel of one cluster: each CTA turns its slice of the counts
// into bits in shared memory, the slices' sums are exchanged through distributed shared memory, and ranks follow from
// population counts.  What is then to be moved (contents, rows of the table, counts) is moved by a kernel over the whole
// device that reads the plan from the workspace.
#include "coopt_decode.cuh"

#include <cooperative_groups.h>
#include <limits.h>

namespace coopt {

namespace {

namespace cg = cooperative_groups;

constexpr int kClusterCtas = 8;                     // a cluster
constexpr int kPlanThreads = 1024;
constexpr int kMaxPoolBlocks = 1 << 20;          // bits of a slice: at most 16 KB of shared memory
constexpr int kMaxRows = 8192;
constexpr int kMaxPlanSmem = kMaxPoolBlocks / kClusterCtas / 8 + 2 * kMaxRows * 4;
constexpr int kCopyThreads = 256;
constexpr int kCachesPerLaunch = 64;

struct Pool {
  int* refs;
  int* table;
  int* lens;
  int blocks, rows, width;
};
// The workspace behind the control words that all calls share: [0] blocks in use, [1] pairs to copy; pairs; free blocks, or
// where every block goes.
struct Plan {
  int* status;
  int* header;
  int* src;                // [max(rows, blocks / 2 + 1)]
  int* dst;
  int* list;               // [blocks]: free blocks in order (fork, reserve); new number of every block, -1 if free (compact)
  int* fork_len;           // [rows]: tokens that a fork takes over, -1 if it is refused
  unsigned* used;          // [blocks / 32]: fork: the blocks in use before the call, as bits
};
long long plan_pairs(long long blocks, long long rows) { return blocks / 2 + 1 > rows ? blocks / 2 + 1 : rows; }
Plan plan_of(void* workspace, int blocks, int rows) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Plan p;
  p.status = reinterpret_cast<int*>(ws);
  p.header = reinterpret_cast<int*>(ws + workspace_control_bytes());
  p.src = p.header + 32;
  p.dst = p.src + plan_pairs(blocks, rows);
  p.list = p.dst + plan_pairs(blocks, rows);
  p.fork_len = p.list + blocks;
  p.used = reinterpret_cast<unsigned*>(p.fork_len + rows);
  return p;
}

__device__ __forceinline__ void report(int* status, int code) { atomicCAS(status, 0, code); }

// ---- the pool as bits: used blocks of this CTA's slice ----------------------------------------------------------------
// Exclusive sum over the threads of a CTA; `total` for all.
__device__ __forceinline__ int cta_scan(int x, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  __syncthreads();                       // (the array may still be read from the scan before)
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  const int s = warp_sums[lane];         // kPlanThreads / 32 == 32 warps
  int before = lane < warp ? s : 0;
  before = __reduce_add_sync(0xffffffffu, before);
  total = __reduce_add_sync(0xffffffffu, s);
  return before + inc - x;
}
struct Slice {
  unsigned* bits;          // shared memory: bit set = used; past the end of the pool: clear, and not taken for free (write_free)
  int first, words, per_thread;
  int before;              // used blocks of the slices before, then (thread) of the words before
  int used;                // .. of the whole pool
};
__device__ __forceinline__ int slice_blocks(int blocks) { return ((blocks + kClusterCtas - 1) / kClusterCtas + 31) / 32 * 32; }
// Reads the slice's counts.  (The cluster meets: from here on its CTAs may write to each other's shared memory.)
__device__ __forceinline__ void load_slice(const int* refs, int blocks, unsigned* bits, Slice& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = static_cast<int>(cg::this_cluster().block_rank());
  const int per = slice_blocks(blocks);
  s.bits = bits;
  s.first = rank * per;
  s.words = max(0, min(per, blocks - s.first) + 31) / 32;
  s.per_thread = (s.words + kPlanThreads - 1) / kPlanThreads;
  constexpr int kUnroll = 8;
  for (int w0 = warp * kUnroll; w0 < s.words; w0 += kPlanThreads / 32 * kUnroll) {
    int r[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int id = s.first + (w0 + k) * 32 + lane;
      r[k] = w0 + k < s.words && id < blocks ? refs[id] : 0;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const unsigned b = __ballot_sync(0xffffffffu, r[k] > 0);
      if (lane == 0 && w0 + k < s.words) bits[w0 + k] = b;
    }
  }
  cg::this_cluster().sync();
}
// Ranks: every thread has `per_thread` consecutive words.
__device__ __forceinline__ void rank_slice(Slice& s, int* warp_sums, int* cluster_sums) {
  auto cluster = cg::this_cluster();
  int n = 0, total;
  const int w0 = threadIdx.x * s.per_thread;
  for (int w = w0; w < min(s.words, w0 + s.per_thread); ++w) n += __popc(s.bits[w]);
  s.before = cta_scan(n, warp_sums, total);
  const int rank = static_cast<int>(cluster.block_rank());
  if (threadIdx.x < kClusterCtas) cluster.map_shared_rank(cluster_sums, threadIdx.x)[rank] = total;
  cluster.sync();
  s.used = 0;
#pragma unroll
  for (int r = 0; r < kClusterCtas; ++r) {
    if (r < rank) s.before += cluster_sums[r];
    s.used += cluster_sums[r];
  }
}
// The free blocks of rank < n, in order, to the list.
__device__ __forceinline__ void write_free(const Slice& s, int blocks, int n, int* list) {
  const int w0 = threadIdx.x * s.per_thread;
  int used = s.before;
  for (int w = w0; w < min(s.words, w0 + s.per_thread); ++w) {
    const int id0 = s.first + 32 * w;
    unsigned free_bits = ~s.bits[w];
    if (id0 + 32 > blocks) free_bits &= (1u << (blocks - id0)) - 1u;     // (the pool's last word)
    int rank = id0 - used;                                               // free blocks before this word
    used += __popc(s.bits[w]);
    for (; free_bits != 0 && rank < n; free_bits &= free_bits - 1, ++rank) list[rank] = id0 + __ffs(free_bits) - 1;
  }
}

// The first place in a call's list that names a row, INT_MAX if none does: the same row twice is refused at its second.
__device__ __forceinline__ void first_places(const int* list, int n, int rows, int* owner) {
  for (int r = threadIdx.x; r < rows; r += kPlanThreads) owner[r] = INT_MAX;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int r = list[i];
    if (r >= 0 && r < rows) atomicMin(&owner[r], i);
  }
  __syncthreads();
}

// ---- reserve ----------------------------------------------------------------------------------------------------------
// need[i]: blocks that the i-th row of the list still lacks (-1: refused).  Rows are served in order, as long as the free
// blocks suffice for a row and all before it.
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kPlanThreads, 1)
pages_reserve_kernel(const Pool pool, const Plan plan, const int* row_ids, const int* new_lens, int n) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32], cluster_sums[kClusterCtas];
  wait_previous_kernel();
  auto cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int* owner = reinterpret_cast<int*>(smem);
  int* need = owner + pool.rows;
  unsigned* bits = reinterpret_cast<unsigned*>(need + n);
  Slice s;
  load_slice(pool.refs, pool.blocks, bits, s);
  first_places(row_ids, n, pool.rows, owner);
  // a warp looks at a row's entries (every CTA of the cluster at an eighth of the list, for all)
  for (int i = rank + kClusterCtas * warp; i < n; i += kClusterCtas * (kPlanThreads / 32)) {
    const int row = row_ids[i], to = new_lens[i];
    int lacks = -1;
    if (row >= 0 && row < pool.rows && owner[row] == i) {
      const int len = max(0, min(pool.lens[row], pool.width * kBlockSize));
      if (to >= len && to <= pool.width * kBlockSize) {
        lacks = 0;
        for (int j = (len + kBlockSize - 1) / kBlockSize + lane; j < (to + kBlockSize - 1) / kBlockSize; j += 32)
          lacks += pool.table[static_cast<size_t>(row) * pool.width + j] < 0;
        lacks = __reduce_add_sync(0xffffffffu, lacks);
      }
    }
    if (lane < kClusterCtas) cluster.map_shared_rank(need, lane)[i] = lacks;
    if (lacks < 0 && lane == 0) report(plan.status, COOPT_ERR_INVALID_ARG);
  }
  rank_slice(s, warp_sums, cluster_sums);          // (meets the whole cluster: all needs are there behind it)
  const int free_blocks = pool.blocks - s.used;
  // need[i] becomes the first free block's rank, or -1
  const int per = (n + kPlanThreads - 1) / kPlanThreads, i0 = threadIdx.x * per;
  long long sum = 0;
  for (int i = i0; i < min(n, i0 + per); ++i) sum += max(0, need[i]);
  static_assert(INT_MAX / kPlanThreads > kMaxPoolBlocks, "a sum that is cut short is still more than there is");
  int total, at = cta_scan(static_cast<int>(min(sum, static_cast<long long>(INT_MAX / kPlanThreads))), warp_sums, total);
  for (int i = i0; i < min(n, i0 + per); ++i) {
    const int k = need[i];
    if (k > 0) {
      const bool fits = k <= free_blocks && at <= free_blocks - k;
      if (!fits && rank == 0) report(plan.status, COOPT_ERR_PAGES);
      need[i] = fits ? at : -1;
      at = fits ? at + k : INT_MAX;
    }
  }
  __syncthreads();
  write_free(s, pool.blocks, min(total, free_blocks), plan.list);
  cluster.sync();
  for (int i = rank + kClusterCtas * warp; i < n; i += kClusterCtas * (kPlanThreads / 32)) {
    int from = need[i];
    if (from < 0) continue;
    const int row = row_ids[i], to = new_lens[i];
    const int len = max(0, min(pool.lens[row], pool.width * kBlockSize));
    int* entries = pool.table + static_cast<size_t>(row) * pool.width;
    const int end = (to + kBlockSize - 1) / kBlockSize;
    for (int j0 = (len + kBlockSize - 1) / kBlockSize; j0 < end; j0 += 32) {
      const bool lacks = j0 + lane < end && entries[j0 + lane] < 0;
      const unsigned all = __ballot_sync(0xffffffffu, lacks);
      if (lacks) {
        const int id = plan.list[from + __popc(all & ((1u << lane) - 1u))];
        entries[j0 + lane] = id;
        pool.refs[id] = 1;
      }
      from += __popc(all);
    }
    __syncwarp();
    if (lane == 0) pool.lens[row] = to;
  }
}

// ---- fork -------------------------------------------------------------------------------------------------------------
// Only blocks in use can be shared or copied: an entry that names a free one (a table that its counts do not stand for) must
// not raise a count, since the same call may hand that block out.  "In use" is by the counts as they were before the call: as
// bits, since the counts change on its way.
__device__ __forceinline__ bool is_used(const unsigned* bits, int blocks, int id) { return id >= 0 && id < blocks && ((bits[id >> 5] >> (id & 31)) & 1u) != 0; }

__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kPlanThreads, 1)
pages_fork_plan_kernel(const Pool pool, const Plan plan, const int* parents, const int* children, int n) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32], cluster_sums[kClusterCtas];
  wait_previous_kernel();
  auto cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  int* owner = reinterpret_cast<int*>(smem);
  int* tail = owner + pool.rows;                  // by place in the list: the block to be copied, -1 if none, -2 if the fork is refused
  unsigned* bits = reinterpret_cast<unsigned*>(tail + n);
  Slice s;
  load_slice(pool.refs, pool.blocks, bits, s);
  first_places(children, n, pool.rows, owner);
  const int per = (n + kPlanThreads - 1) / kPlanThreads, i0 = threadIdx.x * per;
  auto length = [&](int row) { return max(0, min(pool.lens[row], pool.width * kBlockSize)); };
  int sum = 0;
  for (int i = i0; i < min(n, i0 + per); ++i) {
    const int p = parents[i], c = children[i];
    int t = -2;
    // a child is an empty row, named once, and no parent of another
    if (p >= 0 && p < pool.rows && c >= 0 && c < pool.rows && owner[c] == i && owner[p] == INT_MAX && pool.lens[c] == 0) {
      const int L = length(p);
      t = -1;
      if (L % kBlockSize != 0) {
        // (the counts themselves: they change behind the cluster's last meeting)
        const int id = pool.table[static_cast<size_t>(p) * pool.width + L / kBlockSize];
        t = id >= 0 && id < pool.blocks && pool.refs[id] > 0 ? id : -2;
      }
    }
    if (t == -2 && rank == 0) report(plan.status, COOPT_ERR_INVALID_ARG);
    tail[i] = t;
    sum += t >= 0;
  }
  for (int w = threadIdx.x; w < s.words; w += kPlanThreads) plan.used[s.first / 32 + w] = s.bits[w];
  rank_slice(s, warp_sums, cluster_sums);
  const int free_blocks = pool.blocks - s.used;
  int total, at = cta_scan(sum, warp_sums, total);
  write_free(s, pool.blocks, min(total, free_blocks), plan.list);
  cluster.sync();                                  // the list is there, and all have read the lengths
  if (rank != 0) return;
  for (int i = i0; i < min(n, i0 + per); ++i) {
    const int t = tail[i];
    int dst = -1, len = t == -2 ? -1 : length(parents[i]);
    if (t >= 0) {
      if (at < free_blocks) {
        dst = plan.list[at];
        pool.refs[dst] = 1;
      } else {
        report(plan.status, COOPT_ERR_PAGES);
        len = -1;
      }
      ++at;
    }
    plan.src[i] = t;
    plan.dst[i] = dst;
    plan.fork_len[i] = len;
    if (len > 0) pool.lens[children[i]] = len;
  }
}

// ---- compact ----------------------------------------------------------------------------------------------------------
// Of U used blocks those numbered U and above move into the holes below, the i-th into the i-th.
__global__ void __cluster_dims__(kClusterCtas, 1, 1) __launch_bounds__(kPlanThreads, 1)
pages_compact_plan_kernel(const Pool pool, const Plan plan, int* used_out) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32], cluster_sums[kClusterCtas], below_sums[kClusterCtas];
  wait_previous_kernel();
  auto cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank());
  Slice s;
  load_slice(pool.refs, pool.blocks, reinterpret_cast<unsigned*>(smem), s);
  rank_slice(s, warp_sums, cluster_sums);
  const int U = s.used, w0 = threadIdx.x * s.per_thread, w1 = min(s.words, w0 + s.per_thread);
  auto below = [&](int id0) { return id0 + 32 <= U ? 0xFFFFFFFFu : id0 >= U ? 0u : (1u << (U - id0)) - 1u; };
  int n = 0, total;
  for (int w = w0; w < w1; ++w) n += __popc(s.bits[w] & below(s.first + 32 * w));
  cta_scan(n, warp_sums, total);
  if (threadIdx.x < kClusterCtas) cluster.map_shared_rank(below_sums, threadIdx.x)[rank] = total;
  cluster.sync();
  int stay = 0;                                    // used blocks below U
#pragma unroll
  for (int r = 0; r < kClusterCtas; ++r) stay += below_sums[r];
  int used = s.before;
  for (int w = w0; w < w1; ++w) {
    const int id0 = s.first + 32 * w;
    const unsigned b = s.bits[w], low = below(id0);
    int hole = id0 - used, mover = used - stay;
    if (low != 0xFFFFFFFFu) mover += __popc(b & low);
    for (unsigned f = ~b & low; f != 0; f &= f - 1, ++hole) plan.dst[hole] = id0 + __ffs(f) - 1;
    for (unsigned m = b & ~low; m != 0; m &= m - 1, ++mover) plan.src[mover] = id0 + __ffs(m) - 1;
    used += __popc(b);
  }
  cluster.sync();
  // where every block goes: movers by the pairs, the others stay
  for (int w = threadIdx.x >> 5; w < s.words; w += kPlanThreads / 32) {
    const int id = s.first + 32 * w + (threadIdx.x & 31);
    const bool is_used = (s.bits[w] >> (threadIdx.x & 31)) & 1u;
    if (id < pool.blocks && !(is_used && id >= U)) plan.list[id] = is_used ? id : -1;
  }
  for (int i = rank * kPlanThreads + threadIdx.x; i < U - stay; i += kClusterCtas * kPlanThreads) plan.list[plan.src[i]] = plan.dst[i];
  if (rank == 0 && threadIdx.x == 0) {
    plan.header[0] = U;
    plan.header[1] = U - stay;
    *used_out = U;
  }
}

// ---- what is moved ----------------------------------------------------------------------------------------------------
struct Copies {
  uint8_t* cache[kCachesPerLaunch];      // one layer each
  const int* src;
  const int* dst;
  const int* count;                      // pairs: on the device, or null: `pairs`
  int pairs;
  int blocks, heads;
  int granule, bytes;                    // of a granule, and those that hold anything (a multiple of 16)
};
enum Tables { kNoTables, kForkTables, kCompactTables };
struct TableWork {
  Pool pool;
  Plan plan;
  const int* parents;
  const int* children;
  int forks;
  int* table_out;
  int* refs_out;
};

// A warp copies a granule at a time, kDepth 16-byte pieces of a lane in flight: HBM bounds it (one read and one write of
// what is copied), and with 32 warps an SM 128 KB are under way, more than the latency needs.
// (Nine: the 258 pieces of a granule at head_dim 128 are on their way at once.  With eight and a second round for two of them
// 700 blocks of 16 layers took 124 us.)
constexpr int kDepth = 9;
__device__ __forceinline__ void copy_granule(const Copies& c, uint8_t* cache, int from, int to, unsigned head, int lane) {
  if (from < 0 || from >= c.blocks || to < 0 || to >= c.blocks) return;
  const uint4* in = reinterpret_cast<const uint4*>(cache + (static_cast<size_t>(from) * c.heads + head) * c.granule);
  uint4* out = reinterpret_cast<uint4*>(cache + (static_cast<size_t>(to) * c.heads + head) * c.granule);
  const int n = c.bytes / 16;
  for (int i0 = lane; i0 < n; i0 += 32 * kDepth) {
    uint4 v[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (i0 + 32 * k < n) v[k] = in[i0 + 32 * k];
#pragma unroll
    for (int k = 0; k < kDepth; ++k)
      if (i0 + 32 * k < n) out[i0 + 32 * k] = v[k];
  }
}
// A warp's place among all: neighbours in a CTA, which copy neighbouring granules, or (few granules) spread over the SMs.
__device__ __forceinline__ unsigned place_of_warp(unsigned items, int warps) {
  const unsigned in_cta = blockDim.x >> 5, warp = threadIdx.x >> 5;
  return items >= static_cast<unsigned>(warps) ? blockIdx.x * in_cta + warp : warp * gridDim.x + blockIdx.x;
}
__device__ __forceinline__ void copy_granules(const Copies& c, int warps, int lane) {
  const int pairs = c.count != nullptr ? *c.count : c.pairs;
  const unsigned items = static_cast<unsigned>(pairs) * c.heads, first_warp = place_of_warp(items, warps);
  for (unsigned t = first_warp; t < items; t += warps) {
    const unsigned pair = t / c.heads;
    copy_granule(c, c.cache[blockIdx.y], c.src[pair], c.dst[pair], t - pair * c.heads, lane);
  }
}
// A row of the table that a fork writes: entry j of a child whose parent holds `len` tokens.  `used`: see is_used.
__device__ __forceinline__ void fork_entry(const Pool& pool, const unsigned* used, int* status, int parent, int child, int len, int tail_dst, int j) {
  int id = -1;
  if (j < len / kBlockSize) {
    id = pool.table[static_cast<size_t>(parent) * pool.width + j];
    if (id >= 0) {
      if (is_used(used, pool.blocks, id)) {
        atomicAdd(&pool.refs[id], 1);
      } else {
        report(status, COOPT_ERR_INVALID_ARG);
        id = -1;
      }
    } else {
      id = -1;
    }
  } else if (j * kBlockSize < len) {
    id = tail_dst;
  }
  pool.table[static_cast<size_t>(child) * pool.width + j] = id;
}

template <Tables kTables>
__global__ void __launch_bounds__(kCopyThreads) pages_move_kernel(const __grid_constant__ Copies c, const __grid_constant__ TableWork w) {
  wait_previous_kernel();
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) * gridDim.x + blockIdx.x, warps = gridDim.x * (kCopyThreads / 32);
  if (kTables != kNoTables && blockIdx.y == 0) {
    const Pool& pool = w.pool;
    const int thread = blockIdx.x * kCopyThreads + threadIdx.x, threads = gridDim.x * kCopyThreads;
    if (kTables == kForkTables) {
      // rows: a warp takes 32 entries of a child
      const int per_row = (pool.width + 31) / 32;
      for (long long t = warp; t < static_cast<long long>(w.forks) * per_row; t += warps) {
        const int i = static_cast<int>(t / per_row), j = static_cast<int>(t - static_cast<long long>(i) * per_row) * 32 + lane;
        const int len = w.plan.fork_len[i];
        if (len >= 0 && j < pool.width) fork_entry(pool, w.plan.used, w.plan.status, w.parents[i], w.children[i], len, w.plan.dst[i], j);
      }
    } else {
      const int U = w.plan.header[0];
      for (int id = thread; id < pool.blocks; id += threads) {
        const int to = w.plan.list[id];
        if (to >= 0) w.refs_out[to] = pool.refs[id];
        if (id >= U) w.refs_out[id] = 0;            // (a hole below U gets its mover's count)
      }
      const long long entries = static_cast<long long>(pool.rows) * pool.width;
      for (long long e = thread; e < entries; e += threads) {
        int id = pool.table[e];
        if (id >= 0) {
          id = id < pool.blocks ? w.plan.list[id] : -1;
          if (id < 0) report(w.plan.status, COOPT_ERR_INVALID_ARG);
        }
        w.table_out[e] = id;
      }
    }
  }
  copy_granules(c, warps, lane);
}

// ---- fork and compaction of smaller pools, in one launch ---------------------------------------------------------------------
// Every CTA looks through the counts and makes the whole plan for itself, in shared memory, then does its part of the work: what a
// second launch and the way of the plan through memory would take is saved.  Nothing that a CTA writes on its way changes
// another one's plan: only counts of blocks in use are raised (is_used), which stay so, parents are no children.  What would (the new blocks' counts and the
// children's lengths; in place, the moved counts) is written by the CTA that has counted itself last, when all have made
// their plans.
// (us with a planning launch / so; release and fork of 8 rows over four layers, pool of 700 / 8000 / 30000 blocks 10.0 / 7.2, 9.9 /
// 7.4, 10.3 / 9.5; compaction of two layers, 900 / 8000 / 30000 8.4 / 5.7, 11.0 / 9.1, 25.0 / 25.4; reserve by a cluster / by one
// CTA, 700 / 16000 / 30000 6.5 / 4.4, 6.8 / 5.2, 6.5 / 6.6.)
constexpr int kOneThreads = 1024;
constexpr int kOneBlocks = 1 << 15;
constexpr int kOneReserve = 1 << 14;
constexpr int kOneForks = 1024;              // forks, or rows, of a call
constexpr int kMaxOneSmem = 180 * 1024;
static_assert((kMaxRows + kOneForks) * 4 + kOneBlocks / 8 <= kMaxOneSmem && kMaxRows * 4 + kOneBlocks / 8 + kOneBlocks * 4 <= kMaxOneSmem && (2 * (kOneBlocks / 32) + 2 * (kOneBlocks / 2 + 1)) * 4 <= kMaxOneSmem, "shared memory");
int* one_counter(void* workspace) { return reinterpret_cast<int*>(static_cast<uint8_t*>(workspace) + kWsHeaderBytes); }

struct OneSlice {
  unsigned* bits;          // [blocks / 32]: used
  int words, per_thread;
  int before, used;        // as in Slice
};
__device__ __forceinline__ void load_pool(const Pool& pool, unsigned* bits, int* warp_sums, OneSlice& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  s.bits = bits;
  s.words = (pool.blocks + 31) / 32;
  s.per_thread = (s.words + kOneThreads - 1) / kOneThreads;
  constexpr int kUnroll = 8, kWarps = kOneThreads / 32;
  for (int w0 = warp; w0 < s.words; w0 += kWarps * kUnroll) {
    int r[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int id = (w0 + k * kWarps) * 32 + lane;
      r[k] = id < pool.blocks ? __ldcg(pool.refs + id) : 0;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      if (w0 + k * kWarps >= s.words) break;
      const unsigned b = __ballot_sync(0xffffffffu, r[k] > 0);
      if (lane == 0) bits[w0 + k * kWarps] = b;
    }
  }
  __syncthreads();
  int n = 0;
  for (int w = threadIdx.x * s.per_thread; w < min(s.words, (static_cast<int>(threadIdx.x) + 1) * s.per_thread); ++w) n += __popc(bits[w]);
  s.before = cta_scan(n, warp_sums, s.used);
}
// By all threads, behind the last read that a plan is made of: whether this CTA is the last to get here.
__device__ __forceinline__ bool last_to_plan(int* counter, int* flag) {
  __syncthreads();
  if (threadIdx.x == 0) {
    int old;
    asm volatile("atom.add.acq_rel.gpu.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
    *flag = old == static_cast<int>(gridDim.x) - 1;
    if (*flag) *counter = 0;             // ready for the next call
  }
  __syncthreads();
  return *flag != 0;
}

__global__ void __launch_bounds__(kOneThreads, 1) pages_fork_one_kernel(const __grid_constant__ Copies c, int layers, const Pool pool, int* status, int* counter,
                                                                        const int* parents, const int* children, int n) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32], flag;
  __shared__ int src[kOneForks], dst[kOneForks], lens[kOneForks];
  wait_previous_kernel();
  int* owner = reinterpret_cast<int*>(smem);
  int* list = owner + pool.rows;
  unsigned* bits = reinterpret_cast<unsigned*>(list + n);
  const int i = threadIdx.x, lane = threadIdx.x & 31;
  static_assert(kOneThreads == kOneForks, "a fork to a thread");
  const int p = i < n ? parents[i] : -1, child = i < n ? children[i] : -1;
  const bool rows_ok = p >= 0 && p < pool.rows && child >= 0 && child < pool.rows;
  const int L = rows_ok ? max(0, min(__ldcg(pool.lens + p), pool.width * kBlockSize)) : 0, old_len = rows_ok ? __ldcg(pool.lens + child) : 1;
  for (int r = threadIdx.x; r < pool.rows; r += kOneThreads) owner[r] = INT_MAX;
  int tail = L % kBlockSize != 0 ? pool.table[static_cast<size_t>(p) * pool.width + L / kBlockSize] : -1;
  OneSlice s;
  load_pool(pool, bits, warp_sums, s);
  if (i < n && child >= 0 && child < pool.rows) atomicMin(&owner[child], i);
  __syncthreads();
  // a child is an empty row, named once, and no parent of another
  const bool ok = rows_ok && owner[child] == i && owner[p] == INT_MAX && old_len == 0 && (L % kBlockSize == 0 || is_used(bits, pool.blocks, tail));
  if (i < n && !ok && blockIdx.x == 0) report(status, COOPT_ERR_INVALID_ARG);
  const bool copy = ok && tail >= 0;
  int total;
  const int rank = cta_scan(copy ? 1 : 0, warp_sums, total), free_blocks = pool.blocks - s.used;
  {
    int used = s.before;
    for (int w = threadIdx.x * s.per_thread; w < min(s.words, (static_cast<int>(threadIdx.x) + 1) * s.per_thread); ++w) {
      unsigned free_bits = ~bits[w];
      if (32 * w + 32 > pool.blocks) free_bits &= (1u << (pool.blocks - 32 * w)) - 1u;
      int k = 32 * w - used;
      used += __popc(bits[w]);
      for (; free_bits != 0 && k < total; free_bits &= free_bits - 1, ++k) list[k] = 32 * w + __ffs(free_bits) - 1;
    }
  }
  const bool last = last_to_plan(counter, &flag);
  const bool refused = !ok || (copy && rank >= free_blocks);
  if (i < n) {
    src[i] = refused ? -1 : tail;
    dst[i] = copy && !refused ? list[rank] : -1;
    lens[i] = refused ? -1 : L;
    if (ok && refused && blockIdx.x == 0) report(status, COOPT_ERR_PAGES);
    if (last && !refused) {
      if (copy) pool.refs[dst[i]] = 1;
      if (L > 0) pool.lens[child] = L;
    }
  }
  __syncthreads();
  const int warp = (threadIdx.x >> 5) * gridDim.x + blockIdx.x, warps = gridDim.x * (kOneThreads / 32);     // (few granules: on all SMs)
  const int per_row = (pool.width + 31) / 32;
  for (int t = warp; t < n * per_row; t += warps) {
    const int f = t / per_row, j = (t - f * per_row) * 32 + lane;
    if (lens[f] >= 0 && j < pool.width) fork_entry(pool, bits, status, parents[f], children[f], lens[f], dst[f], j);
  }
  const unsigned granules = static_cast<unsigned>(n) * c.heads, items = granules * layers;
  for (unsigned t = place_of_warp(items, warps); t < items; t += warps) {
    const unsigned y = t / granules, at = t - y * granules, f = at / c.heads;
    copy_granule(c, c.cache[y], src[f], dst[f], at - f * c.heads, lane);
  }
}

__global__ void __launch_bounds__(kOneThreads, 1) pages_compact_one_kernel(const __grid_constant__ Copies c, int layers, const Pool pool, int* status, int* counter,
                                                                           int* table_out, int* refs_out, int* used_out, int* new_ids) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32], flag;
  wait_previous_kernel();
  unsigned* bits = reinterpret_cast<unsigned*>(smem);
  OneSlice s;
  load_pool(pool, bits, warp_sums, s);
  int* before = reinterpret_cast<int*>(bits + s.words);      // used blocks ahead of every word
  int* holes = before + s.words;                             // [blocks / 2 + 1] each
  int* movers = holes + pool.blocks / 2 + 1;
  const int U = s.used, lane = threadIdx.x & 31;
  const int w0 = threadIdx.x * s.per_thread, w1 = min(s.words, w0 + s.per_thread);
  auto below = [&](int id0) { return id0 + 32 <= U ? 0xFFFFFFFFu : id0 >= U ? 0u : (1u << (U - id0)) - 1u; };
  int n = 0, stay;                                           // used blocks below U
  for (int w = w0; w < w1; ++w) n += __popc(bits[w] & below(32 * w));
  cta_scan(n, warp_sums, stay);
  int used = s.before;
  for (int w = w0; w < w1; ++w) {
    const int id0 = 32 * w;
    const unsigned b = bits[w], low = below(id0);
    before[w] = used;
    int hole = id0 - used, mover = used - stay;
    if (low != 0xFFFFFFFFu) mover += __popc(b & low);
    for (unsigned f = ~b & low; f != 0; f &= f - 1, ++hole) holes[hole] = id0 + __ffs(f) - 1;
    for (unsigned m = b & ~low; m != 0; m &= m - 1, ++mover) movers[mover] = id0 + __ffs(m) - 1;
    used += __popc(b);
  }
  const int moves = U - stay;
  const bool in_place = refs_out == pool.refs;
  if (last_to_plan(counter, &flag)) {
    if (in_place)
      for (int i = threadIdx.x; i < moves; i += kOneThreads) {
        refs_out[holes[i]] = __ldcg(pool.refs + movers[i]);
        refs_out[movers[i]] = 0;
      }
    if (threadIdx.x == 0) *used_out = U;
  }
  // the number of a block from now on, -1 if it is free
  auto goes = [&](int id) {
    const unsigned b = bits[id >> 5], bit = 1u << (id & 31);
    if ((b & bit) == 0) return -1;
    return id < U ? id : holes[before[id >> 5] + __popc(b & (bit - 1u)) - stay];
  };
  const int thread = blockIdx.x * kOneThreads + threadIdx.x, threads = gridDim.x * kOneThreads;
  if (!in_place) {
    for (int id = thread; id < pool.blocks; id += threads) {
      const int to = goes(id);
      if (to >= 0) refs_out[to] = pool.refs[id];
      if (id >= U) refs_out[id] = 0;                         // (a hole below U gets its mover's count)
    }
  }
  if (new_ids != nullptr)
    for (int id = thread; id < pool.blocks; id += threads) new_ids[id] = goes(id);
  const long long entries = static_cast<long long>(pool.rows) * pool.width;
  for (long long e = thread; e < entries; e += threads) {
    int id = pool.table[e];
    if (id >= 0) {
      id = id < pool.blocks ? goes(id) : -1;
      if (id < 0) report(status, COOPT_ERR_INVALID_ARG);
    }
    table_out[e] = id;
  }
  const unsigned granules = static_cast<unsigned>(moves) * c.heads, items = granules * layers;
  for (unsigned t = place_of_warp(items, threads >> 5); t < items; t += threads >> 5) {
    const unsigned y = t / granules, at = t - y * granules, i = at / c.heads;
    copy_granule(c, c.cache[y], movers[i], holes[i], at - i * c.heads, lane);
  }
}

// Reserve, by one CTA: all that it does after the look through the counts is a trip to memory or two for every 128 rows.
__global__ void __launch_bounds__(kOneThreads, 1) pages_reserve_one_kernel(const Pool pool, int* status, const int* row_ids, const int* new_lens, int n) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int warp_sums[32];
  __shared__ int rows[kOneForks], begin[kOneForks], end[kOneForks], need[kOneForks];
  __shared__ unsigned first[kOneForks];            // which of a row's first 32 entries lack a block
  wait_previous_kernel();
  int* owner = reinterpret_cast<int*>(smem);
  unsigned* bits = reinterpret_cast<unsigned*>(owner + pool.rows);
  int* list = reinterpret_cast<int*>(bits + (pool.blocks + 31) / 32);
  const int i = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = i < n ? row_ids[i] : -1, to = i < n ? new_lens[i] : 0;
  const bool row_ok = row >= 0 && row < pool.rows;
  const int len = row_ok ? max(0, min(pool.lens[row], pool.width * kBlockSize)) : 0;
  for (int r = threadIdx.x; r < pool.rows; r += kOneThreads) owner[r] = INT_MAX;
  OneSlice s;
  load_pool(pool, bits, warp_sums, s);
  if (row_ok) atomicMin(&owner[row], i);
  __syncthreads();
  const bool ok = row_ok && owner[row] == i && to >= len && to <= pool.width * kBlockSize;
  if (i < n) {
    if (!ok) report(status, COOPT_ERR_INVALID_ARG);
    rows[i] = row;
    begin[i] = ok ? (len + kBlockSize - 1) / kBlockSize : 0;
    end[i] = ok ? (to + kBlockSize - 1) / kBlockSize : 0;
  }
  __syncthreads();
  // entries without a block: a warp to a row, four rows on their way at a time
  constexpr int kRowsAt = 4, kWarps = kOneThreads / 32;
  for (int f0 = warp; f0 < n; f0 += kRowsAt * kWarps) {
    bool lacks[kRowsAt];
#pragma unroll
    for (int k = 0; k < kRowsAt; ++k) {
      const int f = f0 + k * kWarps, j = f < n ? begin[f] + lane : 0;
      lacks[k] = f < n && j < end[f] && pool.table[static_cast<size_t>(rows[f]) * pool.width + j] < 0;
    }
#pragma unroll
    for (int k = 0; k < kRowsAt; ++k) {
      const int f = f0 + k * kWarps;
      if (f >= n) break;
      const unsigned mask = __ballot_sync(0xffffffffu, lacks[k]);
      int more = 0;
      for (int j = begin[f] + 32 + lane; j < end[f]; j += 32) more += pool.table[static_cast<size_t>(rows[f]) * pool.width + j] < 0;
      more = __reduce_add_sync(0xffffffffu, more);
      if (lane == 0) { first[f] = mask; need[f] = more + __popc(mask); }
    }
  }
  __syncthreads();
  const int wants = i < n && ok ? need[i] : 0;
  int total;
  static_assert(INT_MAX / kOneThreads > kOneBlocks, "a sum that is cut short is still more than there is");
  const int from = cta_scan(min(wants, INT_MAX / kOneThreads), warp_sums, total), free_blocks = pool.blocks - s.used;
  const bool fits = wants == 0 || (wants <= free_blocks && from <= free_blocks - wants);
  if (i < n) {
    if (ok && !fits) report(status, COOPT_ERR_PAGES);
    need[i] = ok && fits ? from : -1;
  }
  {
    const int most = min(total, free_blocks);
    int used = s.before;
    for (int w = threadIdx.x * s.per_thread; w < min(s.words, (static_cast<int>(threadIdx.x) + 1) * s.per_thread); ++w) {
      unsigned free_bits = ~bits[w];
      if (32 * w + 32 > pool.blocks) free_bits &= (1u << (pool.blocks - 32 * w)) - 1u;
      int k = 32 * w - used;
      used += __popc(bits[w]);
      for (; free_bits != 0 && k < most; free_bits &= free_bits - 1, ++k) list[k] = 32 * w + __ffs(free_bits) - 1;
    }
  }
  __syncthreads();
  if (ok && fits) pool.lens[row] = to;
  for (int f = warp; f < n; f += kWarps) {
    int at = need[f];
    if (at < 0) continue;
    int* entries = pool.table + static_cast<size_t>(rows[f]) * pool.width;
    for (int j0 = begin[f]; j0 < end[f]; j0 += 32) {
      const unsigned all = j0 == begin[f] ? first[f] : __ballot_sync(0xffffffffu, j0 + lane < end[f] && entries[j0 + lane] < 0);
      if ((all >> lane) & 1u) {
        const int id = list[at + __popc(all & ((1u << lane) - 1u))];
        entries[j0 + lane] = id;
        pool.refs[id] = 1;
      }
      at += __popc(all);
    }
  }
}

// ---- release ----------------------------------------------------------------------------------------------------------
// A warp takes 32 entries of a row at a time.  An entry is taken by an exchange, so a row that is named twice is released
// once.
__global__ void __launch_bounds__(kCopyThreads) pages_release_kernel(const Pool pool, int* status, const int* row_ids, int n, int window, int sinks) {
  wait_previous_kernel();
  const int lane = threadIdx.x & 31, warp = (blockIdx.x * kCopyThreads + threadIdx.x) >> 5, warps = gridDim.x * (kCopyThreads / 32);
  const int per_row = (pool.width + 31) / 32;
  for (long long t = warp; t < static_cast<long long>(n) * per_row; t += warps) {
    const int i = static_cast<int>(t / per_row), piece = static_cast<int>(t - static_cast<long long>(i) * per_row), j = piece * 32 + lane;
    const int row = row_ids[i];
    if (row < 0 || row >= pool.rows) {
      if (lane == 0) report(status, COOPT_ERR_INVALID_ARG);
      continue;
    }
    int first = 0, end = pool.width;
    if (window > 0) {
      first = sink_blocks(sinks);
      end = max(0, min(pool.lens[row], pool.width * kBlockSize) - window) / kBlockSize;
    } else if (piece == 0 && lane == 0) {
      pool.lens[row] = 0;
    }
    if (j < first || j >= end) continue;
    const int id = atomicExch(&pool.table[static_cast<size_t>(row) * pool.width + j], -1);
    if (id < 0) continue;
    if (id >= pool.blocks) {
      report(status, COOPT_ERR_INVALID_ARG);
    } else if (atomicSub(&pool.refs[id], 1) <= 0) {       // nobody held it
      atomicAdd(&pool.refs[id], 1);
      report(status, COOPT_ERR_INVALID_ARG);
    }
  }
}

// ---- host side ----------------------------------------------------------------------------------------------------------
int check_caches(const coopt_cache* caches, int32_t n, int32_t num_blocks) {
  if (n < 0 || (n > 0 && caches == nullptr)) return COOPT_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const coopt_cache& c = caches[i];
    if (c.data == nullptr || c.num_blocks <= 0 || c.num_kv_heads <= 0) return COOPT_ERR_INVALID_ARG;
    if ((c.head_dim != 64 && c.head_dim != 128) || c.block_size != kBlockSize || !(is_fp8(c.dtype) || c.dtype == COOPT_KV_BF16)) return COOPT_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(c.data) % 32 != 0) return COOPT_ERR_INVALID_ARG;
    if (c.num_blocks != caches[0].num_blocks || c.num_kv_heads != caches[0].num_kv_heads || c.head_dim != caches[0].head_dim || c.dtype != caches[0].dtype)
      return COOPT_ERR_INVALID_ARG;
  }
  if (n > 0 && num_blocks > 0 && caches[0].num_blocks != num_blocks) return COOPT_ERR_INVALID_ARG;
  if (n > 0 && static_cast<long long>(caches[0].num_blocks) * caches[0].num_kv_heads >= (1ll << 31)) return COOPT_ERR_UNSUPPORTED;
  return COOPT_OK;
}
int check_pool(const coopt_pages* p, const void* workspace, size_t workspace_bytes) {
  if (p == nullptr || p->refs == nullptr || p->block_table == nullptr || p->context_lens == nullptr) return COOPT_ERR_INVALID_ARG;
  if (p->num_blocks <= 0 || p->rows <= 0 || p->max_blocks_per_seq <= 0) return COOPT_ERR_INVALID_ARG;
  if (p->num_blocks > kMaxPoolBlocks || p->rows > kMaxRows || p->max_blocks_per_seq > (1 << 29) / kBlockSize) return COOPT_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < coopt_pages_workspace_bytes(p->num_blocks, p->rows)) return COOPT_ERR_WORKSPACE;
  return COOPT_OK;
}
Pool pool_of(const coopt_pages* p) {
  return {p->refs, p->block_table, p->context_lens, p->num_blocks, p->rows, p->max_blocks_per_seq};
}
int plan_smem(const coopt_pages* p, int listed) {
  const int slice = ((p->num_blocks + kClusterCtas - 1) / kClusterCtas + 31) / 32;
  return (listed > 0 ? (p->rows + listed) * 4 : 0) + slice * 4;
}
template <class Kernel, class... Args>
int launch_plan(Kernel* kernel, int smem, cudaStream_t stream, const Args&... args) {
  if (!configure_kernel_smem(reinterpret_cast<const void*>(kernel), kMaxPlanSmem)) return COOPT_ERR_CUDA;
  return launch_dependent(kernel, kClusterCtas, kPlanThreads, smem, stream, args...) ? COOPT_OK : COOPT_ERR_CUDA;
}
void describe(const coopt_cache* caches, int layers, Copies& c) {
  const coopt_cache& k = caches[0];
  c.blocks = k.num_blocks;
  c.heads = k.num_kv_heads;
  c.granule = granule_bytes(k.head_dim, is_fp8(k.dtype));
  c.bytes = is_fp8(k.dtype) ? header_offset(k.head_dim) + kFp8Header : c.granule;
  for (int y = 0; y < layers; ++y) c.cache[y] = static_cast<uint8_t*>(caches[y].data);
}
// CTAs of a launch that plans in every one: a warp to eight granules, or entries of tables, and no more than there are SMs.
int one_grid(long long granules, long long entries, int num_sms) {
  const long long work = (granules > entries / 32 ? granules : entries / 32) / 8 + 1;
  return static_cast<int>(work < num_sms ? work : num_sms);
}
// `most`: pairs there can be at most; `entries`: of tables and counts, for the first launch.
template <Tables kTables>
int launch_move(const coopt_cache* caches, int num_caches, Copies c, const TableWork& w, long long most, long long entries, cudaStream_t stream) {
  const DeviceInfo* di = device_info();
  if (di == nullptr) return COOPT_ERR_CUDA;
  int done = 0;
  do {
    const int layers = num_caches - done < kCachesPerLaunch ? num_caches - done : kCachesPerLaunch;
    if (layers > 0) {
      describe(caches + done, layers, c);
    } else {
      c.pairs = 0;
      c.count = nullptr;
      c.heads = 1;
    }
    const long long warps = most * c.heads, tables = done == 0 ? (entries + 31) / 32 : 0;
    long long ctas = ((warps > tables ? warps : tables) + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
    const long long full = (static_cast<long long>(di->num_sms) * 8 + layers - 1) / (layers > 0 ? layers : 1);
    ctas = ctas < 1 ? 1 : ctas > full ? full : ctas;
    const dim3 grid(static_cast<unsigned>(ctas), static_cast<unsigned>(layers > 0 ? layers : 1));
    const bool ok = done == 0 ? launch_dependent(pages_move_kernel<kTables>, grid, kCopyThreads, 0, stream, c, w)
                              : launch_dependent(pages_move_kernel<kNoTables>, grid, kCopyThreads, 0, stream, c, w);
    if (!ok) return COOPT_ERR_CUDA;
    done += layers;
  } while (done < num_caches);
  return COOPT_OK;
}

}  // namespace

}  // namespace coopt

using namespace coopt;

extern "C" {

size_t coopt_pages_workspace_bytes(int32_t num_blocks, int32_t rows) {
  if (num_blocks <= 0 || rows <= 0) return 0;
  const size_t ints = 32 + 2 * static_cast<size_t>(plan_pairs(num_blocks, rows)) + num_blocks + rows + (num_blocks + 31) / 32;
  return (workspace_control_bytes() + ints * 4 + 255) / 256 * 256;
}

int coopt_pages_copy(const coopt_cache* caches, int32_t num_caches, const int32_t* src, const int32_t* dst, int32_t num_pairs, void* stream) {
  if (num_caches <= 0) return COOPT_ERR_INVALID_ARG;
  const int rc = check_caches(caches, num_caches, 0);
  if (rc != COOPT_OK) return rc;
  if (num_pairs < 0) return COOPT_ERR_INVALID_ARG;
  if (num_pairs == 0) return COOPT_OK;
  if (!src || !dst) return COOPT_ERR_INVALID_ARG;
  if (static_cast<long long>(num_pairs) * caches[0].num_kv_heads >= (1ll << 31)) return COOPT_ERR_UNSUPPORTED;
  Copies c = {};
  c.src = src;
  c.dst = dst;
  c.pairs = num_pairs;
  return launch_move<kNoTables>(caches, num_caches, c, TableWork{}, num_pairs, 0, static_cast<cudaStream_t>(stream));
}

int coopt_pages_reserve(const coopt_pages* pages, const int32_t* row_ids, const int32_t* new_lens, int32_t num_rows, void* workspace,
                        size_t workspace_bytes, void* stream) {
  const int rc = check_pool(pages, workspace, workspace_bytes);
  if (rc != COOPT_OK) return rc;
  if (num_rows < 0 || num_rows > pages->rows) return COOPT_ERR_INVALID_ARG;
  if (num_rows == 0) return COOPT_OK;
  if (!row_ids || !new_lens) return COOPT_ERR_INVALID_ARG;
  if (pages->num_blocks <= kOneReserve && num_rows <= kOneForks) {
    if (!configure_kernel_smem(reinterpret_cast<const void*>(&pages_reserve_one_kernel), kMaxOneSmem)) return COOPT_ERR_CUDA;
    const int smem = pages->rows * 4 + (pages->num_blocks + 31) / 32 * 4 + pages->num_blocks * 4;
    return launch_dependent(pages_reserve_one_kernel, 1, kOneThreads, smem, static_cast<cudaStream_t>(stream), pool_of(pages), static_cast<int*>(workspace), row_ids,
                            new_lens, static_cast<int>(num_rows))
               ? COOPT_OK
               : COOPT_ERR_CUDA;
  }
  return launch_plan(&pages_reserve_kernel, plan_smem(pages, num_rows), static_cast<cudaStream_t>(stream), pool_of(pages),
                     plan_of(workspace, pages->num_blocks, pages->rows), row_ids, new_lens, static_cast<int>(num_rows));
}

int coopt_pages_fork(const coopt_cache* caches, int32_t num_caches, const coopt_pages* pages, const int32_t* parents, const int32_t* children,
                     int32_t num_forks, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_pool(pages, workspace, workspace_bytes);
  if (rc != COOPT_OK) return rc;
  rc = check_caches(caches, num_caches, pages->num_blocks);
  if (rc != COOPT_OK) return rc;
  if (num_forks < 0 || num_forks > pages->rows) return COOPT_ERR_INVALID_ARG;
  if (num_forks == 0) return COOPT_OK;
  if (!parents || !children) return COOPT_ERR_INVALID_ARG;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const DeviceInfo* di = device_info();
  if (di == nullptr) return COOPT_ERR_CUDA;
  Copies c = {};
  const long long row_entries = static_cast<long long>(num_forks) * pages->max_blocks_per_seq;
  if (pages->num_blocks <= kOneBlocks && num_forks <= kOneForks && num_caches <= kCachesPerLaunch && row_entries < (1ll << 30) &&
      static_cast<long long>(num_forks) * num_caches * (num_caches > 0 ? caches[0].num_kv_heads : 1) < (1ll << 31)) {
    if (num_caches > 0) describe(caches, num_caches, c); else c.heads = 1;
    const int smem = (pages->rows + num_forks) * 4 + (pages->num_blocks + 31) / 32 * 4;
    if (!configure_kernel_smem(reinterpret_cast<const void*>(&pages_fork_one_kernel), kMaxOneSmem)) return COOPT_ERR_CUDA;
    const int grid = one_grid(static_cast<long long>(num_forks) * num_caches * c.heads, row_entries, di->num_sms);
    return launch_dependent(pages_fork_one_kernel, grid, kOneThreads, smem, st, c, static_cast<int>(num_caches), pool_of(pages), static_cast<int*>(workspace),
                            one_counter(workspace), parents, children, static_cast<int>(num_forks))
               ? COOPT_OK
               : COOPT_ERR_CUDA;
  }
  const Plan plan = plan_of(workspace, pages->num_blocks, pages->rows);
  rc = launch_plan(&pages_fork_plan_kernel, plan_smem(pages, num_forks), st, pool_of(pages), plan, parents, children, static_cast<int>(num_forks));
  if (rc != COOPT_OK) return rc;
  c = {};
  c.src = plan.src;
  c.dst = plan.dst;
  c.pairs = num_forks;
  const TableWork w = {pool_of(pages), plan, parents, children, num_forks, nullptr, nullptr};
  return launch_move<kForkTables>(caches, num_caches, c, w, num_forks, static_cast<long long>(num_forks) * ((pages->max_blocks_per_seq + 31) / 32) * 32, st);
}

int coopt_pages_release(const coopt_pages* pages, const int32_t* row_ids, int32_t num_rows, int32_t window, int32_t sinks, void* workspace,
                        size_t workspace_bytes, void* stream) {
  const int rc = check_pool(pages, workspace, workspace_bytes);
  if (rc != COOPT_OK) return rc;
  if (num_rows < 0 || window < 0 || sinks < 0) return COOPT_ERR_INVALID_ARG;
  if (num_rows == 0) return COOPT_OK;
  if (!row_ids) return COOPT_ERR_INVALID_ARG;
  const long long warps = static_cast<long long>(num_rows) * ((pages->max_blocks_per_seq + 31) / 32), ctas = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  const int limit = 1 << 29;
  return launch_dependent(pages_release_kernel, static_cast<unsigned>(ctas < 2048 ? ctas : 2048), kCopyThreads, 0, static_cast<cudaStream_t>(stream), pool_of(pages),
                          static_cast<int*>(workspace), row_ids, static_cast<int>(num_rows), static_cast<int>(window < limit ? window : limit),
                          static_cast<int>(sinks < limit ? sinks : limit))
             ? COOPT_OK
             : COOPT_ERR_CUDA;
}

int coopt_pages_compact(const coopt_cache* caches, int32_t num_caches, const coopt_pages* pages, int32_t* table_out, int32_t* refs_out, int32_t* used_out,
                        int32_t* new_ids, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_pool(pages, workspace, workspace_bytes);
  if (rc != COOPT_OK) return rc;
  rc = check_caches(caches, num_caches, pages->num_blocks);
  if (rc != COOPT_OK) return rc;
  if (!table_out || !refs_out || !used_out) return COOPT_ERR_INVALID_ARG;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const long long entries = static_cast<long long>(pages->rows) * pages->max_blocks_per_seq;
  const DeviceInfo* di = device_info();
  if (di == nullptr) return COOPT_ERR_CUDA;
  Copies c = {};
  if (pages->num_blocks <= kOneBlocks && num_caches <= kCachesPerLaunch &&
      static_cast<long long>(pages->num_blocks) * num_caches * (num_caches > 0 ? caches[0].num_kv_heads : 1) < (1ll << 31)) {
    if (num_caches > 0) describe(caches, num_caches, c); else c.heads = 1;
    const int words = (pages->num_blocks + 31) / 32, smem = (2 * words + 2 * (pages->num_blocks / 2 + 1)) * 4;
    if (!configure_kernel_smem(reinterpret_cast<const void*>(&pages_compact_one_kernel), kMaxOneSmem)) return COOPT_ERR_CUDA;
    const int grid = one_grid(static_cast<long long>(pages->num_blocks / 2) * num_caches * c.heads, entries, di->num_sms);
    return launch_dependent(pages_compact_one_kernel, grid, kOneThreads, smem, st, c, static_cast<int>(num_caches), pool_of(pages), static_cast<int*>(workspace),
                            one_counter(workspace), static_cast<int*>(table_out), static_cast<int*>(refs_out), static_cast<int*>(used_out),
                            static_cast<int*>(new_ids))
               ? COOPT_OK
               : COOPT_ERR_CUDA;
  }
  Plan plan = plan_of(workspace, pages->num_blocks, pages->rows);
  if (new_ids != nullptr) plan.list = new_ids;
  rc = launch_plan(&pages_compact_plan_kernel, plan_smem(pages, 0), st, pool_of(pages), plan, static_cast<int*>(used_out));
  if (rc != COOPT_OK) return rc;
  c = {};
  c.src = plan.src;
  c.dst = plan.dst;
  c.count = plan.header + 1;
  const TableWork w = {pool_of(pages), plan, nullptr, nullptr, 0, table_out, refs_out};
  return launch_move<kCompactTables>(caches, num_caches, c, w, pages->num_blocks / 2 + 1, entries > pages->num_blocks ? entries : pages->num_blocks, st);
}

}  // extern "C"
