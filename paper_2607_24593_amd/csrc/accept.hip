// The accepted path of a tree of drafted tokens: its nodes' rows move to the
// positions that follow the prefix, in place.
//
// A path is ascending and its j-th node is node j or a later one, so a row is read
// before any row of the path is written over it as long as one thread moves its
// column of all rows in order: no thread meets another's bytes, and there is
// nothing to wait for.
#include <algorithm>

#include "cache4.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 8;  // rows that a thread has in flight

template <class U>
__device__ __forceinline__ void move_path(const AcceptArgs& a, const RunTable& t, int b, const int32_t* path, uint8_t* rows,
                                          int bytes, int first, int step) {
  const int units = bytes / (int)sizeof(U);
  const int64_t pos0 = t.pos0[b];
  for (int i = first; i < units; i += step) {
    int before = -1;
    bool more = true;
    for (int j = 0; j < a.n && more; j += kAtOnce) {
      U v[kAtOnce];
      int node[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        node[e] = j + e < a.n ? path[j + e] : -1;
        more = more && node[e] >= j + e && node[e] > before && node[e] < a.limit - pos0;
        before = node[e];
        if (!more) node[e] = -1;
      }
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e)
        if (node[e] > j + e) v[e] = reinterpret_cast<const U*>(rows + a.map.row(b, pos0 + node[e]) * bytes)[i];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e)
        if (node[e] > j + e) reinterpret_cast<U*>(rows + a.map.row(b, pos0 + j + e) * bytes)[i] = v[e];
    }
  }
}

__global__ __launch_bounds__(kThreads) void accept_kernel(AcceptArgs a, RunTable t) {
  const int b = blockIdx.x, arr = blockIdx.y;
  const int32_t* path = a.path + (int64_t)b * a.n;
  const int bytes = a.row_bytes[arr];
  if (((bytes | (uintptr_t)a.rows[arr]) & 15) == 0)
    move_path<uint4>(a, t, b, path, a.rows[arr], bytes, threadIdx.x, kThreads);
  else
    move_path<uint32_t>(a, t, b, path, a.rows[arr], bytes, threadIdx.x, kThreads);
}

}  // namespace

hipError_t launch_accept(const AcceptArgs& a, const RunTable& t, hipStream_t stream) {
  hipLaunchKernelGGL(accept_kernel, dim3((unsigned)t.n, (unsigned)a.n_arrays), dim3(kThreads), 0, stream, a, t);
  return hipGetLastError();
}

}  // namespace pivot
