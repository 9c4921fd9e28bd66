// Eviction from a cache by accumulated attention weight.
//
// Of a sequence's n cached tokens the first `sink`, the last `recent` and the
// largest acc of the others stay, `keep` in all (all of them when n <= keep);
// equal weights go to the lower position.  The kept positions come out in
// ascending order, so the compacted cache keeps the tokens' order.
//
// evict_kernel finds the threshold T of the others by four 8-bit radix passes
// over order-preserving keys, then emits in one ordered pass: a token stays
// when its key is above T, or equals T and fewer than the remaining count of
// equal keys precede it.
#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWaves = kEvictThreads / kWave;

// Inclusive sum over the wave's lanes of two 16-bit counts packed in a word.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  return x;
}

__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a, RunTable t) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];
  __shared__ uint32_t wsum[kEvictWaves];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int n = t.n_k[b];
  const float* acc = a.acc + (int64_t)b * a.acc_stride;
  int32_t* out = a.out_keep + (int64_t)b * a.keep;
  float* out_acc = a.out_acc ? a.out_acc + (int64_t)b * a.keep : nullptr;
  if (n <= a.keep) {
    for (int j = tid; j < a.keep; j += kEvictThreads) {
      out[j] = j < n ? j : -1;
      if (out_acc) out_acc[j] = j < n ? acc[j] : 0.f;
    }
    return;
  }
  const int lo = a.sink, hi = n - a.recent;  // the others: [lo, hi), more than the places left for them
  uint32_t left = (uint32_t)(a.keep - a.sink - a.recent);
  uint32_t thr = 0;
  if (left > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
      for (int s = lo + tid; s < hi; s += kEvictThreads) {
        const uint32_t key = float_key(acc[s]);
        if ((key & mask) == thr) atomicAdd(&hist[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid < kWave) {  // lane l holds digits 255 - 4l .. 252 - 4l, from the top
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = hist[255 - 4 * lane - i], sum += c[i];
        uint32_t above = wave_scan(sum, lane) - sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < left && above + c[i] >= left) {
            found[0] = (uint32_t)(255 - 4 * lane - i);
            found[1] = left - above;
          }
          above += c[i];
        }
      }
      __syncthreads();
      thr |= found[0] << shift;
      left = found[1];
      __syncthreads();
    }
  } else {
    thr = 0xFFFFFFFFu;  // only a NaN could have this key, and none is wanted
  }
  // ordered emission, kEvictThreads * 4 positions at a time
  uint32_t sure0 = 0, tie0 = 0;
  for (int base = 0; base < n; base += kEvictThreads * 4) {
    const int s0 = base + 4 * tid;
    float v[4];
    uint32_t kind[4], mine = 0;  // 0 goes, 1 stays, 1 << 16 equals the threshold
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = s0 + i;
      kind[i] = 0;
      v[i] = 0.f;
      if (s < n) {
        v[i] = acc[s];
        if (s < lo || s >= hi) kind[i] = 1;
        else {
          const uint32_t key = float_key(v[i]);
          kind[i] = key > thr ? 1u : key == thr ? 1u << 16 : 0u;
        }
      }
      mine += kind[i];
    }
    const uint32_t incl = wave_scan(mine, lane);
    if (lane == 63) wsum[tid >> 6] = incl;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
      if (w < (tid >> 6)) before += wsum[w];
      total += wsum[w];
    }
    before += incl - mine;
    uint32_t sure = sure0 + (before & 0xFFFFu), tie = tie0 + (before >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool equal = kind[i] > 1;
      if (kind[i] == 1 || (equal && tie < left)) {
        const uint32_t j = sure + (tie < left ? tie : left);
        out[j] = s0 + i;
        if (out_acc) out_acc[j] = v[i];
      }
      sure += kind[i] & 0xFFFFu;
      tie += kind[i] >> 16;
    }
    sure0 += total & 0xFFFFu;
    tie0 += total >> 16;
    __syncthreads();
  }
}

// One array (blockIdx.y) of the moved rows: U bytes a thread, the threads of a
// row side by side.
template <class U>
__device__ __forceinline__ void move_row(const uint8_t* src, uint8_t* dst, int bytes, int part, int parts) {
  for (int i = part; i < bytes / (int)sizeof(U); i += parts)
    reinterpret_cast<U*>(dst)[i] = reinterpret_cast<const U*>(src)[i];
}

__global__ __launch_bounds__(256) void move_kernel(MoveArrays m, KeyMap from, KeyMap to, const int32_t* __restrict__ kept,
                                                   int batch, int keep, int rows_per_wg) {
  const int arr = blockIdx.y;
  const int parts = 256 / rows_per_wg;
  const int64_t r = (int64_t)blockIdx.x * rows_per_wg + threadIdx.x / parts;
  if (r >= (int64_t)batch * keep) return;
  const int32_t pos = kept[r];
  if (pos < 0) return;
  const int b = (int)(r / keep);
  const int bytes = m.row_bytes[arr];
  const uint8_t* src = m.src[arr] + from.row(b, pos) * bytes;
  uint8_t* dst = m.dst[arr] + to.row(b, r - (int64_t)b * keep) * bytes;
  const int part = threadIdx.x % parts;
  if (((bytes | (uintptr_t)m.src[arr] | (uintptr_t)m.dst[arr]) & 15) == 0) move_row<uint4>(src, dst, bytes, part, parts);
  else move_row<uint32_t>(src, dst, bytes, part, parts);
}

}  // namespace

size_t evict_workspace(const EvictArgs&, const RunTable&) { return 0; }

hipError_t launch_evict(const EvictArgs& a, const RunTable& t, void*, hipStream_t stream) {
  hipLaunchKernelGGL(evict_kernel, dim3((unsigned)t.n), dim3(kEvictThreads), 0, stream, a, t);
  return hipGetLastError();
}

hipError_t launch_move(const MoveArrays& m, const KeyMap& from, const KeyMap& to, const int32_t* kept, int batch,
                       int keep, hipStream_t stream) {
  const int rows_per_wg = 16;
  const int64_t rows = (int64_t)batch * keep;
  const unsigned gx = (unsigned)((rows + rows_per_wg - 1) / rows_per_wg);
  hipLaunchKernelGGL(move_kernel, dim3(gx, (unsigned)m.n), dim3(256), 0, stream, m, from, to, kept, batch, keep,
                     rows_per_wg);
  return hipGetLastError();
}

}  // namespace pivot
