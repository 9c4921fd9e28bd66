// Pages that sequences share.  A slot of the table lists the pages of one sequence
// (-1: none), refs counts the slots that hold a page, a page with count 0 is free.
//
//   fork     the pages of one slot in another, counted once more
//   free     the pages of a slot behind those it keeps, counted once less
//   grow     pages for new tokens, and a page of its own for a sequence whose last,
//            partly filled page others hold too
//   compact  the highest pages in use to the lowest free ones
//   copy     whole pages of row arrays
//
// Which pages are taken does not depend on the order of threads: the k-th page
// wanted is the k-th free one from below.  A workgroup makes a map of bits of kBlock
// pages in LDS, 64 at a ballot, scans the words' counts, and finds the k-th free page
// of its block by bisection, neighbouring k in neighbouring lanes, so that entries
// and counts are written side by side.
// Pools of one block that few pages are taken of take one launch.  Else a launch
// before writes the blocks' maps and counts (the second one changes refs, and several
// workgroups share a block).
// Bound by latency, a chain of dependent loads and bisections: 160 slots of a pool of
// 4800 pages grow in 11.5 us; two slots by 4096 pages each in a pool of 87000 in 5.3 +
// 7.5 us (by one workgroup a block 27).
#include <algorithm>

#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kThreads = 256;
constexpr int kBlockThreads = 1024;
constexpr int kBlock = 32 * kBlockThreads;  // pages

__device__ __forceinline__ bool in_pool(const Pages& p, int32_t page) { return (uint32_t)page < (uint32_t)p.n_pages; }
__host__ __device__ __forceinline__ int pages_of(const Pages& p, int32_t tokens) {
  return (int)(((int64_t)tokens + (1 << p.shift) - 1) >> p.shift);
}

__global__ __launch_bounds__(kThreads) void fork_kernel(Pages p, PageList l) {
  const int i = blockIdx.x, at = blockIdx.y * kThreads + threadIdx.x;
  if (at >= pages_of(p, l.b[i])) return;
  const int32_t page = p.table[(int64_t)l.slot[i] * p.max_pages + at];
  if (!in_pool(p, page)) return;
  p.table[(int64_t)l.a[i] * p.max_pages + at] = page;
  atomicAdd(p.refs + page, 1);
}

__global__ __launch_bounds__(kThreads) void free_kernel(Pages p, PageList l) {
  const int i = blockIdx.x, at = pages_of(p, l.b[i]) + blockIdx.y * kThreads + threadIdx.x;
  if (at >= pages_of(p, l.a[i])) return;
  int32_t* entry = p.table + (int64_t)l.slot[i] * p.max_pages + at;
  const int32_t page = *entry;
  if (!in_pool(p, page)) return;
  *entry = -1;
  atomicSub(p.refs + page, 1);
}

// Exclusive sums over a workgroup of T threads; total of all.
template <int T>
__device__ __forceinline__ int block_scan(int x, int* total) {
  __shared__ int s_wave[T / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(sum, o, 64);
    if (lane >= o) sum += v;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  *total = all;
  return before + sum - x;
}

// A block's pages: which are free, as bits (word t those from 32 t on), and the free
// ones before each word.  Pages behind the pool are not free.
struct Block {
  uint64_t map[kBlock / 64];
  int32_t before[kBlockThreads];
  __device__ uint32_t word(int t) const { return reinterpret_cast<const uint32_t*>(map)[t]; }
  // its pages' number in the block: the k-th free one, the k-th that is not free
  __device__ int free_page(int k) const { return find(k, false); }
  __device__ int used_page(int k) const { return find(k, true); }

  __device__ int find(int k, bool used) const {
    int lo = 0, hi = kBlockThreads - 1;  // the last word with at most k before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((used ? 32 * mid - before[mid] : before[mid]) <= k) lo = mid;
      else hi = mid - 1;
    }
    int n = k - (used ? 32 * lo - before[lo] : before[lo]), bit = 0;
    uint32_t bits = used ? ~word(lo) : word(lo);
#pragma unroll
    for (int half = 16; half > 0; half >>= 1) {  // its n-th bit
      const int c = __popc(bits & ((1u << half) - 1));
      if (n >= c) {
        n -= c;
        bits >>= half;
        bit += half;
      }
    }
    return 32 * lo + bit;
  }
};
__device__ __forceinline__ void map_block(const Pages& p, int block, Block* b) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = block * kBlock + (int)threadIdx.x;
  int count[32];
#pragma unroll
  for (int j = 0; j < 32; ++j)  // always loaded: a load for some lanes only would be waited for before the next
    count[j] = p.refs[min(first + kBlockThreads * j, p.n_pages - 1)];
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const uint64_t map = __ballot(count[j] == 0 && first + kBlockThreads * j < p.n_pages);
    if (lane == 0) b->map[kBlockThreads / 64 * j + wave] = map;
  }
  __syncthreads();
}
// The counts of the words before; returns all of the block's free pages.
__device__ __forceinline__ int scan_block(Block* b) {
  int total;
  b->before[threadIdx.x] = block_scan<kBlockThreads>(__popc(b->word(threadIdx.x)), &total);
  __syncthreads();
  return total;
}

// Free pages in the blocks before this one (blockIdx.x), and in the pool; counts: of a
// pool of more than one block.
__device__ __forceinline__ int free_before(const int32_t* counts, int mine, int* all) {
  if (gridDim.x == 1) {
    *all = mine;
    return 0;
  }
  int before = 0, sum = 0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kBlockThreads) {
    const int c = counts[i];
    sum += c;
    before += i < (int)blockIdx.x ? c : 0;
  }
  block_scan<kBlockThreads>(sum, all);
  int b;
  block_scan<kBlockThreads>(before, &b);
  return b;
}

// What growing takes.  first[i]: pages before sequence i's in the order they are
// taken, first[n]: all; old[i]: its last page, if that is copied, else -1.
struct Need {
  int32_t first[kMaxPageList + 1];
  int32_t old[kMaxPageList];
};

// By the first kMaxPageList threads of a workgroup of T (all come here).
template <int T>
__device__ __forceinline__ void find_need(const Pages& p, const PageList& l, Need* need) {
  __shared__ __attribute__((aligned(16))) int32_t s_last[kMaxPageList];
  const int i = threadIdx.x;
  int32_t last = -1, holders = 0;
  int fresh = 0;
  if (i < l.n && l.b[i] > l.a[i]) {
    fresh = pages_of(p, l.b[i]) - pages_of(p, l.a[i]);
    if (l.a[i] & ((1 << p.shift) - 1)) last = p.table[(int64_t)l.slot[i] * p.max_pages + (l.a[i] >> p.shift)];
    if (!in_pool(p, last)) last = -1;
    if (last >= 0) holders = p.refs[last];
  }
  if (i < kMaxPageList) s_last[i] = last;
  __syncthreads();
  int copied = 0;
  if (holders > 1) {
    int rank = 0;  // of the call's sequences before this one that hold the page
    for (int j = 0; j < i; j += 4) {
      const int4 v = *reinterpret_cast<const int4*>(&s_last[j]);
      rank += (v.x == last) + (j + 1 < i && v.y == last) + (j + 2 < i && v.z == last) + (j + 3 < i && v.w == last);
    }
    copied = rank < holders - 1;  // the last holder keeps it
  }
  int total;
  const int first = block_scan<T>(copied + fresh, &total);
  if (i < l.n) {
    need->first[i] = first;
    need->old[i] = copied ? last : -1;
  }
  if (i == 0) need->first[l.n] = total;
}

// The blocks' free pages and maps, and (one workgroup more) what growing takes.
__global__ __launch_bounds__(kBlockThreads) void count_kernel(Pages p, PageList l, int blocks, int32_t* counts,
                                                              uint64_t* maps, Need* need, int32_t* pairs, int n_pairs) {
  __shared__ Block s_block;
  const int at = blockIdx.x * kBlockThreads + threadIdx.x, all = gridDim.x * kBlockThreads;
  for (int64_t i = at; i < 2 * (int64_t)n_pairs; i += all) pairs[i] = -1;
  if ((int)blockIdx.x == blocks) {
    find_need<kBlockThreads>(p, l, need);
    return;
  }
  map_block(p, blockIdx.x, &s_block);
  const int total = scan_block(&s_block);
  if (threadIdx.x == 0) counts[blockIdx.x] = total;
  if (maps && threadIdx.x < kBlock / 64) maps[(int64_t)blockIdx.x * (kBlock / 64) + threadIdx.x] = s_block.map[threadIdx.x];
}

// The last of n ascending values (the first of them 0) that is at most x.
__device__ __forceinline__ int last_at_most(const int32_t* v, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (v[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// maps: NULL in the one launch of a pool of one block
__global__ __launch_bounds__(kBlockThreads) void grow_kernel(Pages p, PageList l, const int32_t* counts,
                                                             const uint64_t* maps, const Need* need, int32_t* pairs,
                                                             int32_t* state) {
  __shared__ Block s_block;
  __shared__ Need s_need;
  __shared__ PageList s_list;  // read at places that differ between threads
  const int tid = threadIdx.x;
  if (tid < l.n) {
    s_list.slot[tid] = l.slot[tid];
    s_list.a[tid] = l.a[tid];
  }
  if (!maps) {
    find_need<kBlockThreads>(p, l, &s_need);
    if (tid < 2 * l.n) pairs[tid] = -1;
    map_block(p, blockIdx.x, &s_block);
  } else {
    if (tid <= l.n) s_need.first[tid] = need->first[tid];
    if (tid < l.n) s_need.old[tid] = need->old[tid];
    if (tid < kBlock / 64) s_block.map[tid] = maps[(int64_t)blockIdx.x * (kBlock / 64) + tid];
    __syncthreads();
  }
  const int total = scan_block(&s_block);
  int all;
  const int before = free_before(counts, total, &all);
  const int want = s_need.first[l.n];
  if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) {
    state[0] = want > all ? want - all : 0;
    state[1] = want > all ? all : all - want;
  }
  if (want > all) return;
  const int mine = min(total, want - before);
  for (int k = blockIdx.y * kBlockThreads + tid; k < mine; k += gridDim.y * kBlockThreads) {
    const int page = blockIdx.x * kBlock + s_block.free_page(k);
    const int at = before + k, i = last_at_most(s_need.first, l.n, at), j = at - s_need.first[i];
    const int old = s_need.old[i], now = s_list.a[i];
    const bool copy = old >= 0 && j == 0;
    p.table[(int64_t)s_list.slot[i] * p.max_pages + (copy ? now >> p.shift : pages_of(p, now) + j - (old >= 0))] = page;
    p.refs[page] = 1;
    if (copy) {
      pairs[2 * i] = old;
      pairs[2 * i + 1] = page;
      atomicSub(p.refs + old, 1);
    }
  }
}

// The moves of compacting, pairs (from, to): the k-th free page from below takes
// the k-th page in use from above.  Of L pages in use as many lie at L and above as
// there are free ones below L; those are the moves there are.
__global__ __launch_bounds__(kBlockThreads) void moves_kernel(Pages p, const int32_t* counts, int most, int32_t* pairs,
                                                              int32_t* state) {
  __shared__ Block s_block;
  __shared__ int s_holes;
  const int tid = threadIdx.x, first = blockIdx.x * kBlock;
  map_block(p, blockIdx.x, &s_block);
  const int total = scan_block(&s_block);
  int all;
  const int before = free_before(counts, total, &all), in_use = p.n_pages - all;
  const int size = min(p.n_pages - first, kBlock), below = min(max(in_use - first, 0), size);  // pages below L
  if (tid == 0) {
    const uint32_t low = below & 31 ? s_block.word(below >> 5) & ((1u << (below & 31)) - 1) : 0;
    s_holes = below == kBlock ? total : s_block.before[below >> 5] + __popc(low);
  }
  __syncthreads();
  const int holes = s_holes;
  for (int i = tid; i < holes && before + i < most; i += kBlockThreads)
    pairs[2 * (int64_t)(before + i) + 1] = first + s_block.free_page(i);
  const int used_before = first - before;
  for (int u = size - total - 1 - tid; u >= below - holes; u -= kBlockThreads) {  // the highest ones first
    const int k = in_use - 1 - (used_before + u);
    if (k < most) pairs[2 * (int64_t)k] = first + s_block.used_page(u);
  }
  // the block that page L lies in (the last one, if no page is free)
  if (min(in_use, p.n_pages - 1) / kBlock != (int)blockIdx.x) return;
  const int n = min(before + holes, most);
  if (tid == 0) {
    state[0] = n;
    state[1] = in_use;
  }
  if (gridDim.x == 1)
    for (int64_t i = 2 * (int64_t)n + tid; i < 2 * (int64_t)most; i += kBlockThreads) pairs[i] = -1;
}

// Counts and table entries of the pages that move.
__global__ __launch_bounds__(kThreads) void remap_kernel(Pages p, const int32_t* pairs, const int32_t* state,
                                                         int64_t entries) {
  const int n = state[0];
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (at < n) {
    const int32_t from = pairs[2 * at], to = pairs[2 * at + 1];
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (at >= entries || n == 0) return;
  const int32_t page = p.table[at];
  if (!in_pool(p, page) || page < pairs[2 * (n - 1)]) return;
  int lo = 0, hi = n - 1;  // pairs go down from the highest page
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (pairs[2 * mid] <= page) hi = mid;
    else lo = mid + 1;
  }
  if (pairs[2 * lo] == page) p.table[at] = pairs[2 * lo + 1];
}

// Whole pages, 16 bytes (4, where an array's address allows no more) a thread.
template <class U>
__device__ __forceinline__ void copy_bytes(const uint8_t* from, uint8_t* to, int64_t bytes, int first, int step) {
  const int64_t units = bytes / (int)sizeof(U);
#pragma unroll 4
  for (int64_t i = first; i < units; i += step) reinterpret_cast<U*>(to)[i] = reinterpret_cast<const U*>(from)[i];
}

__global__ __launch_bounds__(kThreads) void copy_kernel(PageRows a, const int32_t* pairs) {
  const int32_t from = pairs[2 * (int64_t)blockIdx.x], to = pairs[2 * (int64_t)blockIdx.x + 1];
  if ((uint32_t)from >= (uint32_t)a.n_pages || (uint32_t)to >= (uint32_t)a.n_pages || from == to) return;
  const int first = blockIdx.y * kThreads + threadIdx.x, step = gridDim.y * kThreads;
  for (int i = 0; i < a.n; ++i) {
    const int64_t bytes = (int64_t)a.row_bytes[i] << a.shift;  // a multiple of 64
    if (((uintptr_t)a.rows[i] & 15) == 0)
      copy_bytes<uint4>(a.rows[i] + from * bytes, a.rows[i] + to * bytes, bytes, first, step);
    else
      copy_bytes<uint32_t>(a.rows[i] + from * bytes, a.rows[i] + to * bytes, bytes, first, step);
  }
}

int most_pages(const Pages& p, const PageList& l, const int32_t* from, const int32_t* to) {
  int most = 0;
  for (int i = 0; i < l.n; ++i) most = std::max(most, pages_of(p, to[i]) - (from ? pages_of(p, from[i]) : 0));
  return most;
}
unsigned blocks_of(int64_t items) { return (unsigned)((items + kThreads - 1) / kThreads); }
int pool_blocks(const Pages& p) { return (p.n_pages + kBlock - 1) / kBlock; }
size_t round256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

hipError_t launch_pages_fork(const Pages& p, const PageList& l, hipStream_t stream) {
  const int most = most_pages(p, l, nullptr, l.b);
  if (most == 0) return hipSuccess;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)l.n, blocks_of(most)), dim3(kThreads), 0, stream, p, l);
  return hipGetLastError();
}

hipError_t launch_pages_free(const Pages& p, const PageList& l, hipStream_t stream) {
  const int most = most_pages(p, l, l.b, l.a);
  if (most <= 0) return hipSuccess;
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)l.n, blocks_of(most)), dim3(kThreads), 0, stream, p, l);
  return hipGetLastError();
}

size_t pages_grow_workspace(const Pages& p) {
  return round256(sizeof(Need)) + round256((size_t)pool_blocks(p) * 4) + (size_t)pool_blocks(p) * (kBlock / 8);
}

hipError_t launch_pages_grow(const Pages& p, const PageList& l, int32_t* pairs, int32_t* state, void* workspace,
                             hipStream_t stream) {
  Need* need = (Need*)workspace;
  int32_t* counts = (int32_t*)((uint8_t*)workspace + round256(sizeof(Need)));
  const int blocks = pool_blocks(p);
  uint64_t* maps = (uint64_t*)((uint8_t*)counts + round256((size_t)blocks * 4));
  int64_t wanted = 0;
  for (int i = 0; i < l.n; ++i) wanted += pages_of(p, l.b[i]) - pages_of(p, l.a[i]) + 1;
  // workgroups that share a block: a round of bisections takes 2.5 us
  const int parts = (int)std::min<int64_t>(std::min<int64_t>(wanted, kBlock) / kBlockThreads + 1, 8);
  const bool one = blocks == 1 && parts <= 2;
  if (!one)
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)blocks + 1), dim3(kBlockThreads), 0, stream, p, l, blocks, counts, maps,
                       need, pairs, l.n);
  hipLaunchKernelGGL(grow_kernel, dim3((unsigned)blocks, one ? 1u : (unsigned)parts), dim3(kBlockThreads), 0, stream, p, l,
                     counts, one ? nullptr : maps, need, pairs, state);
  return hipGetLastError();
}

size_t pages_compact_workspace(const Pages& p) { return round256((size_t)pool_blocks(p) * 4); }

hipError_t launch_pages_compact(const Pages& p, int32_t slots, int32_t most, int32_t* pairs, int32_t* state,
                                void* workspace, hipStream_t stream) {
  const int blocks = pool_blocks(p);
  int32_t* counts = (int32_t*)workspace;
  if (blocks > 1)
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)blocks), dim3(kBlockThreads), 0, stream, p, PageList{}, blocks, counts,
                       nullptr, nullptr, pairs, most);
  hipLaunchKernelGGL(moves_kernel, dim3((unsigned)blocks), dim3(kBlockThreads), 0, stream, p, counts, most, pairs, state);
  const int64_t entries = (int64_t)slots * p.max_pages;
  hipLaunchKernelGGL(remap_kernel, dim3(blocks_of(std::max<int64_t>(entries, std::min(most, p.n_pages / 2 + 1)))),
                     dim3(kThreads), 0, stream, p, pairs, state, entries);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PageRows& a, int32_t n, const int32_t* pairs, hipStream_t stream) {
  int64_t bytes = 0;
  for (int i = 0; i < a.n; ++i) bytes = std::max<int64_t>(bytes, (int64_t)a.row_bytes[i] << a.shift);
  const unsigned pieces = (unsigned)std::min<int64_t>(std::max<int64_t>(bytes / (16 * kThreads * 4), 1), 16);
  constexpr int kMost = 1 << 16;  // pairs of a launch, which counts its threads in 32 bits
  for (int first = 0; first < n; first += kMost) {
    hipLaunchKernelGGL(copy_kernel, dim3((unsigned)std::min(n - first, kMost), pieces), dim3(kThreads), 0, stream, a,
                       pairs + 2 * (int64_t)first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (n - first <= kMost) break;  // first + kMost may pass 2^31
  }
  return hipSuccess;
}

}  // namespace pivot
