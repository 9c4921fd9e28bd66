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
// wanted is the k-th free one from below.  The pool is cut into blocks of kBlock
// pages: one launch counts each block's free pages, the next lets every block add
// up the counts before it and write its own pages where they belong.
#include <algorithm>

#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 4096;  // pages, 16 a thread
constexpr int kEach = kBlock / kThreads;

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

// A thread's 16 pages of a block, neighbours: bit e set where page e is free.
// Pages behind the pool are neither free nor live.
__device__ __forceinline__ uint32_t free_bits(const Pages& p, int block, uint32_t* live) {
  const int first = block * kBlock + kEach * threadIdx.x;
  uint32_t bits = 0, used = 0;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    if (first + e >= p.n_pages) break;
    if (p.refs[first + e] == 0) bits |= 1u << e;
    else used |= 1u << e;
  }
  *live = used;
  return bits;
}

// What growing takes.  need[i]: pages before sequence i's in the list of those
// taken, need[n]: all; copied[i]: whether its last page is copied.
struct Need {
  int32_t first[kMaxPageList + 1];
  int32_t copied[kMaxPageList];
};

__global__ __launch_bounds__(kThreads) void count_kernel(Pages p, int32_t* counts, int32_t* pairs, int n_pairs) {
  const int at = blockIdx.x * kThreads + threadIdx.x, all = gridDim.x * kThreads;
  for (int i = at; i < 2 * n_pairs; i += all) pairs[i] = -1;
  uint32_t live;
  const uint32_t bits = free_bits(p, blockIdx.x, &live);
  int total;
  block_scan<kThreads>(__popc(bits), &total);
  if (threadIdx.x == 0) counts[blockIdx.x] = total;
}

__global__ __launch_bounds__(kMaxPageList) void need_kernel(Pages p, PageList l, Need* need) {
  __shared__ int32_t s_last[kMaxPageList];
  const int i = threadIdx.x;
  int32_t last = -1;
  int fresh = 0;
  if (i < l.n && l.b[i] > l.a[i]) {
    fresh = pages_of(p, l.b[i]) - pages_of(p, l.a[i]);
    if (l.a[i] & ((1 << p.shift) - 1)) last = p.table[(int64_t)l.slot[i] * p.max_pages + (l.a[i] >> p.shift)];
    if (!in_pool(p, last)) last = -1;
  }
  s_last[i] = last;
  __syncthreads();
  int copied = 0;
  if (last >= 0) {
    int rank = 0;  // of the call's sequences before this one that hold the page
    for (int j = 0; j < i; ++j) rank += s_last[j] == last;
    copied = rank < p.refs[last] - 1;  // the last holder keeps it
  }
  int total;
  const int first = block_scan<kMaxPageList>(copied + fresh, &total);
  if (i < l.n) {
    need->first[i] = first;
    need->copied[i] = copied;
  }
  if (i == 0) need->first[l.n] = total;
}

// Free pages before this block, and in the pool.
__device__ __forceinline__ int free_before(const int32_t* counts, int blocks, int block, int* all) {
  int before = 0, sum = 0;
  for (int i = threadIdx.x; i < blocks; i += kThreads) {
    const int c = counts[i];
    sum += c;
    before += i < block ? c : 0;
  }
  block_scan<kThreads>(sum, all);
  int b;
  block_scan<kThreads>(before, &b);
  return b;
}

// The list of the pages that are taken, and their counts.
__global__ __launch_bounds__(kThreads) void take_kernel(Pages p, int n, const int32_t* counts, const Need* need,
                                                        int32_t* list, int32_t* state) {
  int all, total;
  const int before = free_before(counts, gridDim.x, blockIdx.x, &all);
  const int want = need->first[n];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    state[0] = want > all ? want - all : 0;
    state[1] = want > all ? all : all - want;
  }
  if (want > all || before >= want) return;
  uint32_t live, bits = free_bits(p, blockIdx.x, &live);
  int at = before + block_scan<kThreads>(__popc(bits), &total);
  for (; bits && at < want; bits &= bits - 1, ++at) {
    const int page = blockIdx.x * kBlock + kEach * threadIdx.x + __ffs(bits) - 1;
    list[at] = page;
    p.refs[page] = 1;
  }
}

__global__ __launch_bounds__(kThreads) void assign_kernel(Pages p, PageList l, const Need* need, const int32_t* list,
                                                          const int32_t* state, int32_t* pairs) {
  if (state[0] > 0) return;  // too few: nothing happens
  const int i = blockIdx.x, j = blockIdx.y * kThreads + threadIdx.x;
  const int first = need->first[i], n = need->first[i + 1] - first, copied = need->copied[i];
  if (j >= n) return;
  const int32_t page = list[first + j];
  const int at = copied && j == 0 ? l.a[i] >> p.shift : pages_of(p, l.a[i]) + j - copied;
  int32_t* entry = p.table + (int64_t)l.slot[i] * p.max_pages + at;
  if (copied && j == 0) {
    pairs[2 * i] = *entry;
    pairs[2 * i + 1] = page;
    atomicSub(p.refs + *entry, 1);
  }
  *entry = page;
}

// The moves of compacting, pairs (from, to): the k-th free page from below takes
// the k-th page in use from above.  Of L pages in use as many lie at L and above as
// there are free ones below L; those are the moves there are.
__global__ __launch_bounds__(kThreads) void moves_kernel(Pages p, const int32_t* counts, int most, int32_t* pairs,
                                                         int32_t* state) {
  int all, total;
  const int before = free_before(counts, gridDim.x, blockIdx.x, &all);
  const int first = blockIdx.x * kBlock, in_use = p.n_pages - all;
  uint32_t live, bits = free_bits(p, blockIdx.x, &live);
  const int free_at = before + block_scan<kThreads>(__popc(bits), &total);
  const int mine = first + kEach * (int)threadIdx.x;
  int holes = 0;
  for (int e = 0, at = free_at, used = min(mine, p.n_pages) - free_at; e < kEach && mine + e < p.n_pages; ++e) {
    if (bits >> e & 1) {
      if (mine + e < in_use) {
        ++holes;
        if (at < most) pairs[2 * at + 1] = mine + e;
      }
      ++at;
    } else {
      const int k = in_use - 1 - used;  // from above
      if (mine + e >= in_use && k < most) pairs[2 * k] = mine + e;
      ++used;
    }
  }
  block_scan<kThreads>(holes, &total);
  // the block that the L-th page lies in (the last one, if no page is free)
  if (threadIdx.x == 0 && min(in_use, p.n_pages - 1) / kBlock == (int)blockIdx.x) {
    state[0] = all == 0 ? 0 : min(before + total, most);
    state[1] = in_use;
  }
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

size_t pages_grow_workspace(const Pages& p, int64_t wanted) {
  return round256(sizeof(Need)) + round256((size_t)pool_blocks(p) * 4) + round256((size_t)wanted * 4);
}

hipError_t launch_pages_grow(const Pages& p, const PageList& l, int32_t* pairs, int32_t* state, void* workspace,
                             hipStream_t stream) {
  uint8_t* ws = (uint8_t*)workspace;
  Need* need = (Need*)ws;
  int32_t* counts = (int32_t*)(ws + round256(sizeof(Need)));
  int32_t* list = (int32_t*)((uint8_t*)counts + round256((size_t)pool_blocks(p) * 4));
  const unsigned blocks = (unsigned)pool_blocks(p);
  hipLaunchKernelGGL(count_kernel, dim3(blocks), dim3(kThreads), 0, stream, p, counts, pairs, l.n);
  hipLaunchKernelGGL(need_kernel, dim3(1), dim3(kMaxPageList), 0, stream, p, l, need);
  hipLaunchKernelGGL(take_kernel, dim3(blocks), dim3(kThreads), 0, stream, p, l.n, counts, need, list, state);
  hipLaunchKernelGGL(assign_kernel, dim3((unsigned)l.n, blocks_of(std::max(0, most_pages(p, l, l.a, l.b)) + 1)),
                     dim3(kThreads), 0, stream, p, l, need, list, state, pairs);
  return hipGetLastError();
}

size_t pages_compact_workspace(const Pages& p) { return round256((size_t)pool_blocks(p) * 4); }

hipError_t launch_pages_compact(const Pages& p, int32_t slots, int32_t most, int32_t* pairs, int32_t* state,
                                void* workspace, hipStream_t stream) {
  const unsigned blocks = (unsigned)pool_blocks(p);
  int32_t* counts = (int32_t*)workspace;
  hipLaunchKernelGGL(count_kernel, dim3(blocks), dim3(kThreads), 0, stream, p, counts, pairs, most);
  hipLaunchKernelGGL(moves_kernel, dim3(blocks), dim3(kThreads), 0, stream, p, counts, most, pairs, state);
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
