// The accepted path of a tree of drafted tokens: its nodes' rows move to the
// positions that follow the prefix, in place.
//
// A path is ascending, so its j-th node is node j or a later one.  Rows are moved some
// at a time, in order: all of them are read before the first is written, and what
// is written lies before everything that is read later.
// The nodes' weights, which lie by position and under no map, are one workgroup more.
// Bound by latency, three dependent loads (the path, the pages, the rows): 32
// sequences x 9 rows x 5 arrays in 3.7 us, with weights 3.75; with rows moved in order
// by the threads of their columns, eight at a time, 6.9.
#include <algorithm>

#include "cache4.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kThreads = 256;

template <class U>
__device__ __forceinline__ void move_path(uint8_t* rows, int bytes, const int64_t* from, const int64_t* to, int n) {
  const int units = bytes / (int)sizeof(U);
  int lg = 0;
  while ((1 << lg) < units && lg < 8) ++lg;  // threads of a row
  const int part = threadIdx.x & ((1 << lg) - 1), step = kThreads >> lg;
  const int rounds = (units + (1 << lg) - 1) >> lg;  // of a wide row: their columns do not meet
  for (int base = 0; base < n; base += step) {
    const int j = base + ((int)threadIdx.x >> lg);
    for (int round = 0; round < rounds; ++round) {
      const int i = part + (round << lg);
      const bool moves = j < n && i < units && from[j] != to[j];
      U v{};
      if (moves) v = reinterpret_cast<const U*>(rows + from[j] * bytes)[i];
      if (step > 1) __syncthreads();  // a thread alone with its column needs none
      if (moves) reinterpret_cast<U*>(rows + to[j] * bytes)[i] = v;
    }
  }
}

__global__ __launch_bounds__(kThreads) void accept_kernel(AcceptArgs a, RunTable t) {
  __shared__ int64_t s_from[PIVOT_TREE_MAX_NODES], s_to[PIVOT_TREE_MAX_NODES];
  __shared__ int s_length;
  const int b = blockIdx.x, arr = blockIdx.y, tid = threadIdx.x;
  const int32_t* path = a.path + (int64_t)b * a.n;
  const int64_t pos0 = t.pos0[b];
  // A row map leads entries outside the pool to some page of it.  Here that would
  // write rows of another sequence: a pool's table holds -1 where a sequence ends.
  auto held = [&](int64_t pos) -> int {
    return !a.map.pages ||
           (uint32_t)a.map.pages[(int64_t)b * a.map.max_pages + (pos >> a.map.shift)] < (uint32_t)a.map.n_pages;
  };
  if (tid == 0) s_length = a.n;
  __syncthreads();
  for (int j = tid; j < a.n; j += kThreads) {
    const int node = path[j], before = j > 0 ? path[j - 1] : -1;
    const bool ok = node >= j && node > before && node < a.limit - pos0 && node < t.n_rows[b] &&
                    (held(pos0 + node) & held(pos0 + j)) != 0;  // both loaded at once
    if (!ok) atomicMin(&s_length, j);
    s_from[j] = ok ? a.map.row(b, pos0 + node) : 0;
    s_to[j] = ok ? a.map.row(b, pos0 + j) : 0;
  }
  __syncthreads();
  const int n = s_length;
  if (arr == a.n_arrays) {  // the nodes' weights, by positions of the sequence
    __shared__ float s_acc[PIVOT_TREE_MAX_NODES];
    float* acc = a.acc + b * a.acc_stride + pos0;
    for (int j = tid; j < n; j += kThreads) s_acc[j] = acc[path[j]];
    __syncthreads();
    for (int j = tid; j < t.n_rows[b]; j += kThreads) acc[j] = j < n ? s_acc[j] : 0.f;
    return;
  }
  const int bytes = a.row_bytes[arr];
  if (((bytes | (uintptr_t)a.rows[arr]) & 15) == 0) move_path<uint4>(a.rows[arr], bytes, s_from, s_to, n);
  else move_path<uint32_t>(a.rows[arr], bytes, s_from, s_to, n);
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& a, const RunTable& t, hipStream_t stream) {
  const unsigned parts = (unsigned)a.n_arrays + (a.acc ? 1 : 0);
  hipLaunchKernelGGL(accept_kernel, dim3((unsigned)t.n, parts), dim3(kThreads), 0, stream, a, t);
  return hipGetLastError();
}

}  // namespace pivot
