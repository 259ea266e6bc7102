// Blocks of a step's new tokens: block tables, cache slots and the free list,
// built on the device from the requests' lengths.
//
// Request r holds owned_r blocks and L_r tokens; n_r new tokens need
//     need_r = max(0, ceil((L_r + n_r) / 16) - owned_r)
// more.  Requests are served in order: with U_r the inclusive prefix sum of
// the needs and F free ids, r is granted iff need_r = 0 or U_r <= F, and its
// k-th new block is the free list's entry F - 1 - (U_r - need_r) - k (the list
// is a stack whose top is its last entry).  As U does not fall, the granted
// requests that need blocks are a prefix of those that do.  Trimming is the
// inverse: the blocks past ceil(keep_r / 16) are pushed in request order.
//
// Both are a prefix sum over at most 8192 requests followed by independent
// work per block or per token, bound by latency: a few launches' worth of
// dependent loads (lengths, scan, search, id, store).  Every workgroup scans
// the whole batch into LDS by itself (a few reads of at most 32 KiB arrays
// from L2) rather than waiting for another launch's scan, then takes its share
// of the tokens and blocks, each found by a binary search over the prefix in
// LDS.  The new counters may be written over the old ones, which other
// workgroups may still be reading: one workgroup writes them after its own
// scan, and several leave aliased ones to a second launch.
//
// Measured: 256 requests of one token 4.8 us (of which a launch is about 3); 4096 requests of
// 53 k tokens 8.5 us in 52 workgroups (12.8 where a thread's requests followed each other in
// memory, not in LDS alone); 8192 requests 12.3 us; 231 k blocks given back by 4096 requests
// 5.8 us.
#include "nsd_internal.h"

#include <type_traits>

namespace {

constexpr int kThreads = 1024;
constexpr int kMaxBatch = 8192;

// Inclusive prefix sum over the workgroup's threads.
__device__ inline int64_t scan(int64_t x, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int s = 1; s < 64; s *= 2) {
    const int64_t y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int64_t before = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) before += w < wave ? part[w] : 0;
  return x + before;
}

// The last r in [0, n) with key[r] <= x, for a key that does not fall and key[0] <= x.
__device__ inline int find(const int32_t* key, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (key[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct PlanArgs {
  int32_t* table;
  const int32_t *owned, *lens, *indptr, *free_ids, *free_count;
  int32_t *new_owned, *new_lens, *new_count, *granted, *slots;
  int32_t width, capacity, bs, total_q;
};

// PER: requests per thread.  LDS: indptr, start, lens, owned, each of bs + 1 entries.
template <int PER>
__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs A, int counters, int rows) {
  extern __shared__ int32_t mem[];
  __shared__ int64_t part[kThreads / 64];
  __shared__ int32_t taken[kThreads / 64];   // by each wave's last granted request
  const int n = A.bs, tid = threadIdx.x;
  int32_t *indptr = mem, *start = mem + (n + 1), *lens = mem + 2 * (n + 1),
          *owned = mem + 3 * (n + 1);
  const int free_n = min(max(A.free_count[0], 0), A.capacity);
  int a[PER], count[PER], len[PER], own[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {   // (all the loads in flight)
    const int r = min(i * kThreads + tid, n - 1);
    a[i] = n ? A.indptr[r] : 0;
    count[i] = n ? A.indptr[r + 1] : 0;
    len[i] = n ? A.lens[r] : 0;
    own[i] = n ? A.owned[r] : 0;
  }
  int32_t need[PER];   // -1: more tokens than the table's row holds, or a length counts
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = i * kThreads + tid;
    a[i] = min(max(a[i], 0), A.total_q);
    count[i] = min(max(count[i], a[i]), A.total_q) - a[i];
    len[i] = max(len[i], 0);
    own[i] = min(max(own[i], 0), A.width);
    const int64_t tokens = (int64_t)len[i] + count[i];
    const int64_t blocks = (tokens + NSD_BLOCK_SIZE - 1) / NSD_BLOCK_SIZE;
    need[i] = blocks > A.width || tokens > INT32_MAX ? -1 : max((int32_t)blocks - own[i], 0);
    if (r < n) {
      indptr[r] = a[i];
      lens[r] = len[i];
      start[r] = max(need[i], 0);
    }
  }
  if (tid == 0 && n) indptr[n] = min(max(A.indptr[n], 0), A.total_q);
  __syncthreads();
  // the prefix, each thread PER requests that follow each other
  int32_t each[PER];
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    each[i] = tid * PER + i < n ? start[tid * PER + i] : 0;
    sum += each[i];
  }
  int64_t upto = scan(sum, part) - sum;
  int32_t mine = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    // past the granted requests the prefix stays above every granted block's number
    if (tid * PER + i < n) start[tid * PER + i] = (int32_t)min(upto, (int64_t)free_n);
    upto += each[i];
    if (each[i] && upto <= free_n) mine = (int32_t)upto;
  }
  // the ids taken: up to the last granted request that needs some (the prefix does not fall)
  const uint64_t m = __ballot(mine > 0);
  if ((tid & 63) == (m ? 63 - __builtin_clzll(m) : 0)) taken[tid >> 6] = mine;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = i * kThreads + tid;
    if (r >= n) continue;
    const bool ok = need[i] == 0 || (need[i] > 0 && (int64_t)start[r] + need[i] <= free_n);
    owned[r] = ok ? own[i] : -1;
    if (counters && blockIdx.x == 0) {
      A.granted[r] = ok;
      A.new_owned[r] = own[i] + (ok ? need[i] : 0);
      A.new_lens[r] = len[i] + (ok ? count[i] : 0);
    }
  }
  __syncthreads();
  int32_t used = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) used = max(used, taken[w]);
  if (counters && blockIdx.x == 0 && tid == 0) A.new_count[0] = free_n - used;
  if (!rows) return;
  const int at = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  for (int k = at; k < used; k += step) {
    // the last request whose first new block is at most the k-th: it holds the block
    // (a request without new blocks shares its start with the next one that has some)
    const int r = find(start, n, k);
    A.table[(int64_t)r * A.width + owned[r] + (k - start[r])] = A.free_ids[free_n - 1 - k];
  }
  for (int i = at; i < A.total_q; i += step) {
    int32_t slot = -1;
    if (n == 0) {
      A.slots[i] = slot;
      continue;
    }
    const int r = find(indptr, n, i);
    const int64_t t = (int64_t)lens[r] + (i - indptr[r]), b = t / NSD_BLOCK_SIZE;
    // a granted request's tokens lie within its row (rows ahead of the first request's or behind
    // the last one's are no request's, and with offsets that are no prefix sum need not)
    if (owned[r] >= 0 && t >= 0 && b < A.width && i >= indptr[r] && i < indptr[r + 1]) {
      const int64_t k = start[r] + (b - owned[r]);
      const int id = b < owned[r] ? A.table[(int64_t)r * A.width + b]
                     : k < free_n ? A.free_ids[free_n - 1 - k] : -1;
      if (id >= 0 && id < (1 << 27)) slot = id * NSD_BLOCK_SIZE + (int)(t % NSD_BLOCK_SIZE);
    }
    A.slots[i] = slot;
  }
}

struct TrimArgs {
  const int32_t *table, *owned, *keep;
  int32_t* free_ids;
  const int32_t* free_count;
  int32_t *new_owned, *new_count;
  int32_t width, capacity, bs;
};

// LDS: start, kept, each of bs + 1 entries.
template <int PER>
__global__ __launch_bounds__(kThreads) void trim_kernel(TrimArgs A, int counters, int rows) {
  extern __shared__ int32_t mem[];
  __shared__ int64_t part[kThreads / 64];
  __shared__ int32_t total;
  const int n = A.bs, tid = threadIdx.x;
  int32_t *start = mem, *kept = mem + (n + 1);
  const int free_n = min(max(A.free_count[0], 0), A.capacity);
  int32_t own[PER], keep[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {   // (all the loads in flight)
    const int r = min(i * kThreads + tid, n - 1);
    own[i] = n ? A.owned[r] : 0;
    keep[i] = n ? A.keep[r] : 0;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = i * kThreads + tid, o = min(max(own[i], 0), A.width);
    const int64_t b = ((int64_t)max(keep[i], 0) + NSD_BLOCK_SIZE - 1) / NSD_BLOCK_SIZE;
    const int k = (int)min((int64_t)o, b);
    if (r >= n) continue;
    start[r] = o - k;
    kept[r] = k;
    if (counters && blockIdx.x == 0) A.new_owned[r] = k;
  }
  __syncthreads();
  // the prefix, each thread PER requests that follow each other
  int32_t each[PER];
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    each[i] = tid * PER + i < n ? start[tid * PER + i] : 0;
    sum += each[i];
  }
  const int64_t end = scan(sum, part);
  int64_t upto = end - sum;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (tid * PER + i < n) start[tid * PER + i] = (int32_t)upto;
    upto += each[i];
  }
  // ids past the list's capacity are dropped
  if (tid == kThreads - 1) total = (int32_t)min(end, (int64_t)(A.capacity - free_n));
  __syncthreads();
  if (counters && blockIdx.x == 0 && tid == 0) A.new_count[0] = free_n + total;
  if (!rows) return;
  for (int k = blockIdx.x * kThreads + tid; k < total; k += gridDim.x * kThreads) {
    const int r = find(start, n, k);
    A.free_ids[free_n + k] = A.table[(int64_t)r * A.width + kept[r] + (k - start[r])];
  }
}

// Workgroups for `work` blocks and tokens: one where its threads take at most four each.
int groups(int64_t work) {
  const int64_t g = work <= 4 * kThreads ? 1 : (work + kThreads - 1) / kThreads;
  return (int)(g < 256 ? g : 256);
}

// Runs kernel(requests per thread)(args, counters, rows) over the work, the counters in the
// same launch unless several workgroups would still read what they overwrite.
template <class Kernel, class Args>
void launch(Kernel kernel, const Args& args, int64_t work, bool alias, size_t lds,
            hipStream_t stream) {
  const int g = groups(work);
  const bool apart = g > 1 && alias;
  auto go = [&](auto k) {
    hipLaunchKernelGGL(k, dim3(g), dim3(kThreads), lds, stream, args, apart ? 0 : 1, 1);
    if (apart) hipLaunchKernelGGL(k, dim3(1), dim3(kThreads), lds, stream, args, 1, 0);
  };
  using std::integral_constant;
  if (args.bs <= kThreads) go(kernel(integral_constant<int, 1>{}));
  else if (args.bs <= 2 * kThreads) go(kernel(integral_constant<int, 2>{}));
  else if (args.bs <= 4 * kThreads) go(kernel(integral_constant<int, 4>{}));
  else go(kernel(integral_constant<int, 8>{}));
}
static_assert(kMaxBatch == 8 * kThreads, "a thread takes at most 8 requests");

nsd_status check_sizes(const char* fn, int32_t bs, int32_t width, int32_t capacity) {
  using namespace nsd;
  if (bs < 0 || bs > kMaxBatch)
    return fail(NSD_ERR_SHAPE, "%s: bs must be in [0, %d]", fn, kMaxBatch);
  if (width < 1 || capacity < 0)
    return fail(NSD_ERR_SHAPE, "%s: max_blocks_per_seq < 1 or free_capacity < 0", fn);
  if (capacity > (1 << 27))
    return fail(NSD_ERR_UNSUPPORTED, "%s: a pool of more than 2^27 blocks", fn);
  return NSD_OK;
}

}  // namespace

extern "C" nsd_status nsd_plan_blocks(int32_t* block_table, int32_t max_blocks_per_seq,
                                      const int32_t* owned, const int32_t* seq_lens,
                                      const int32_t* q_indptr, int32_t bs, int32_t total_q,
                                      const int32_t* free_blocks, int32_t free_capacity,
                                      const int32_t* free_count, int32_t* new_owned,
                                      int32_t* new_lens, int32_t* new_free_count,
                                      int32_t* granted, int32_t* slots, void* stream) {
  using namespace nsd;
  const char* fn = "plan_blocks";
  if (const nsd_status st = check_sizes(fn, bs, max_blocks_per_seq, free_capacity)) return st;
  if (total_q < 0) return fail(NSD_ERR_SHAPE, "%s: total_q < 0", fn);
  if (!free_count || !new_free_count || (free_capacity && !free_blocks) ||
      (bs && (!block_table || !owned || !seq_lens || !q_indptr || !new_owned || !new_lens ||
              !granted)) || (bs && total_q && !slots))
    return fail(NSD_ERR_NULL, "%s: NULL pointer argument", fn);
  const PlanArgs args{block_table, owned,     seq_lens,       q_indptr, free_blocks, free_count,
                      new_owned,   new_lens,  new_free_count, granted,  slots,       max_blocks_per_seq,
                      free_capacity, bs, slots ? total_q : 0};
  const bool alias = new_owned == owned || new_lens == seq_lens || new_free_count == free_count;
  clear_stale_error();
  launch([](auto per) { return plan_kernel<decltype(per)::value>; }, args, args.total_q, alias, ((size_t)bs + 1) * 16, (hipStream_t)stream);
  return check_launch(fn);
}

extern "C" nsd_status nsd_trim_blocks(const int32_t* block_table, int32_t max_blocks_per_seq,
                                      const int32_t* owned, const int32_t* keep_lens, int32_t bs,
                                      int32_t* free_blocks, int32_t free_capacity,
                                      const int32_t* free_count, int32_t* new_owned,
                                      int32_t* new_free_count, void* stream) {
  using namespace nsd;
  const char* fn = "trim_blocks";
  if (const nsd_status st = check_sizes(fn, bs, max_blocks_per_seq, free_capacity)) return st;
  if (!free_count || !new_free_count || (free_capacity && !free_blocks) ||
      (bs && (!block_table || !owned || !keep_lens || !new_owned)))
    return fail(NSD_ERR_NULL, "%s: NULL pointer argument", fn);
  if ((int64_t)bs * max_blocks_per_seq > INT32_MAX)
    return fail(NSD_ERR_UNSUPPORTED, "%s: a block table of more than 2^31-1 entries", fn);
  const TrimArgs args{block_table, owned,     keep_lens,      free_blocks, free_count,
                      new_owned,   new_free_count, max_blocks_per_seq, free_capacity, bs};
  const bool alias = new_owned == owned || new_free_count == free_count;
  clear_stale_error();
  // the host does not know how many blocks come back: at most the tables' or the list's
  const int64_t most = (int64_t)bs * max_blocks_per_seq;
  launch([](auto per) { return trim_kernel<decltype(per)::value>; }, args, most < free_capacity ? most : free_capacity, alias,
         ((size_t)bs + 1) * 8, (hipStream_t)stream);
  return check_launch(fn);
}
