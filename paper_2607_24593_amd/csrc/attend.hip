// Attention in the MQA form of latent attention, over the 4-bit cache.
//
//   z[r, h, s] = scale * q[r, h] . (latent[s], rope[s])     s in the row's set, or s <= its position
//   o[r, h]    = sum_s softmax(z)[s] latent[s],   lse = log sum_s exp(z)
//   acc[b, s] += sum_{r, h} softmax(z[r, h])[s]             optional
//
// A row with no key (an empty set, or only scores of -infinity) has o = 0 and
// lse = -infinity and adds nothing to acc.
//
// Scores are kept in base 2 (z log2 e), statistics and sums in fp32.
#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kTileKeys = 32;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLog2e = 1.4426950408889634f;

// Where a launch keeps the scores that the weights are summed from: for unit u
// (a query row of an index-set call, else a sequence) tiles of 32 keys, each
// tile [rows of the unit, 32] in fp32; base[u] counts words (dense units only:
// index-set units are all alike).
struct ScoreMap {
  float* s2;
  float2* stat;  // [rows * heads]: running maximum (base 2) and 1 / sum, 1 / sum = 0 for an empty row
  int64_t base[kMaxSeq];
};

__device__ __forceinline__ float block_max(float v, float* red, int tid) {
  v = wave_reduce(v, [](float a, float b) { return fmaxf(a, b); });
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}
__device__ __forceinline__ float block_sum(float v, float* red, int tid) {
  v = wave_reduce(v, [](float a, float b) { return a + b; });
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// One workgroup per (query row, head): a thread scores one key of a chunk of
// 256, then owns two of the 512 output values over the chunk's keys.
__global__ __launch_bounds__(256) void attend_kernel(AttendArgs a, RunTable t, ScoreMap sm) {
  __shared__ float q[kAttnDim];
  __shared__ float p[256];
  __shared__ int64_t krow[256];
  __shared__ float red[4];
  const int tid = threadIdx.x, head = blockIdx.x, r = blockIdx.y;
  const int b = run_of(t, r), i = r - t.row0[b];
  const int pos = t.pos0[b] + i;
  const uint16_t* qp = a.q + r * a.q_row + head * a.q_head;
  for (int e = tid; e < kAttnDim; e += 256) q[e] = __uint_as_float((uint32_t)qp[e] << 16);
  const float c = a.scale * kLog2e;
  const int n = a.idx ? a.topk : pos + 1;
  const int unit_rows = a.idx ? a.heads : t.n_rows[b] * a.heads;
  const int unit_row = a.idx ? head : i * a.heads + head;
  const int padded = a.idx ? (a.topk + kTileKeys - 1) / kTileKeys * kTileKeys
                           : (t.pos0[b] + t.n_rows[b] + kTileKeys - 1) / kTileKeys * kTileKeys;
  const int64_t base = a.idx ? (int64_t)r * unit_rows * padded : sm.base[b];
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int k0 = 0; k0 < (sm.s2 ? padded : n); k0 += 256) {
    const int k = k0 + tid;
    int key = -1;
    if (k < n) key = a.idx ? a.idx[(int64_t)r * a.topk + k] : k;
    if (key > pos) key = -1;
    float s = -INFINITY;
    int64_t row = 0;
    if (key >= 0) {
      row = a.map.row(b, key);
      float dot = 0.f;
      for (int j = 0; j < kLatent / 8; ++j) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(a.cache.codes + row * kCodeBytes + 4 * j);
        const uint4 v = decode8(w, scale_operand(a.cache.scales[row * kScaleBytes + j / 4]));
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dot = fmaf(q[8 * j + 2 * e], __uint_as_float(u[e] << 16), dot);
          dot = fmaf(q[8 * j + 2 * e + 1], __uint_as_float(u[e] & 0xFFFF0000u), dot);
        }
      }
      for (int e = 0; e < kRope; ++e)
        dot = fmaf(q[kLatent + e], __uint_as_float((uint32_t)a.cache.rope[row * kRope + e] << 16), dot);
      s = dot * c;
    }
    if (sm.s2 && k < padded)
      sm.s2[base + ((int64_t)(k / kTileKeys) * unit_rows + unit_row) * kTileKeys + k % kTileKeys] = s;
    const float top = fmaxf(m, block_max(s, red, tid));
    const float ref = top == -INFINITY ? 0.f : top;
    const float alpha = exp2f(m - ref);
    m = top;
    const float e = exp2f(s - ref);
    p[tid] = e;
    krow[tid] = row;
    l = l * alpha + block_sum(e, red, tid);
    o0 *= alpha;
    o1 *= alpha;
    const int count = min(256, n - k0);
    for (int j = 0; j < count; ++j) {
      if (p[j] == 0.f) continue;
      const uint32_t w = a.cache.codes[krow[j] * kCodeBytes + tid];
      const uint4 v = decode8(w, scale_operand(a.cache.scales[krow[j] * kScaleBytes + tid / 16]));
      o0 = fmaf(p[j], __uint_as_float(v.x << 16), o0);
      o1 = fmaf(p[j], __uint_as_float(v.x & 0xFFFF0000u), o1);
    }
    __syncthreads();
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t orow = (int64_t)r * a.heads + head;
  *reinterpret_cast<uint32_t*>(a.out + orow * kLatent + 2 * tid) =
      (uint32_t)bf16_rne(o0 * inv) | ((uint32_t)bf16_rne(o1 * inv) << 16);
  if (tid == 0) {
    if (a.lse) a.lse[orow] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
    if (sm.stat) sm.stat[orow] = {m == -INFINITY ? 0.f : m, inv};
  }
}

// Sum over a tile's rows of the softmax weights of its 32 keys: 8 rows at a
// time, each thread one key, the rows of a thread in ascending order.
__device__ __forceinline__ float tile_weight(const float* tile, const float2* stat, int rows, float* red, int tid) {
  const int k = tid & 31, first = tid >> 5;
  float w = 0.f;
  for (int r = first; r < rows; r += 8) {
    const float2 st = stat[r];
    w = fmaf(exp2f(tile[r * kTileKeys + k] - st.x), st.y, w);
  }
  red[tid] = w;
  __syncthreads();
  w = 0.f;
  if (tid < kTileKeys)
#pragma unroll
    for (int j = 0; j < 8; ++j) w += red[j * kTileKeys + k];
  return w;
}

__global__ __launch_bounds__(256) void dense_weights_kernel(AttendArgs a, RunTable t, ScoreMap sm) {
  __shared__ float red[256];
  const int b = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x;
  const int n = t.pos0[b] + t.n_rows[b], rows = t.n_rows[b] * a.heads;
  if (rows == 0 || tile * kTileKeys >= n) return;
  const float w = tile_weight(sm.s2 + sm.base[b] + (int64_t)tile * rows * kTileKeys,
                              sm.stat + (int64_t)t.row0[b] * a.heads, rows, red, tid);
  const int s = tile * kTileKeys + tid;
  if (tid < kTileKeys && s < n) a.acc[(int64_t)b * a.acc_stride + s] += w;
}

__global__ __launch_bounds__(256) void slot_weights_kernel(AttendArgs a, ScoreMap sm, float* __restrict__ slots,
                                                           int padded) {
  __shared__ float red[256];
  const int r = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x;
  const float w = tile_weight(sm.s2 + ((int64_t)r * padded + tile * kTileKeys) * a.heads,
                              sm.stat + (int64_t)r * a.heads, a.heads, red, tid);
  if (tid < kTileKeys) slots[(int64_t)r * padded + tile * kTileKeys + tid] = w;
}

// acc += the slots' weights: a workgroup owns kRange positions of a sequence
// and adds the sequence's rows one after the other (a position comes at most
// once in a set, so every sum has one order).
constexpr int kRange = 4096;
__global__ __launch_bounds__(256) void slot_add_kernel(AttendArgs a, RunTable t, const float* __restrict__ slots,
                                                       int padded) {
  __shared__ float sum[kRange];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int lo = blockIdx.x * kRange, n = t.pos0[b] + t.n_rows[b];
  if (t.n_rows[b] == 0 || lo >= n) return;
  for (int j = tid; j < kRange; j += 256) sum[j] = 0.f;
  __syncthreads();
  for (int i = 0; i < t.n_rows[b]; ++i) {
    const int64_t r = t.row0[b] + i;
    const int pos = t.pos0[b] + i;
    for (int k = tid; k < a.topk; k += 256) {
      const int key = a.idx[r * a.topk + k];
      if (key <= pos && (uint32_t)(key - lo) < (uint32_t)kRange && key >= 0)
        atomicAdd(&sum[key - lo], slots[r * padded + k]);
    }
    __syncthreads();
  }
  for (int j = tid; j < kRange && lo + j < n; j += 256)
    if (sum[j] != 0.f) a.acc[(int64_t)b * a.acc_stride + lo + j] += sum[j];
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  size_t scores, stats, slots;
  int padded;
  int64_t base[kMaxSeq];
  int rows, max_n;
  size_t bytes() const { return round256(scores) + round256(stats) + round256(slots); }
};

Plan plan_of(const AttendArgs& a, const RunTable& t) {
  Plan p{};
  int64_t words = 0;
  for (int b = 0; b < t.n; ++b) {
    const int n = t.pos0[b] + t.n_rows[b];
    p.base[b] = words;
    if (t.n_rows[b]) {
      words += (int64_t)((n + kTileKeys - 1) / kTileKeys) * kTileKeys * t.n_rows[b] * a.heads;
      if (n > p.max_n) p.max_n = n;
    }
    p.rows += t.n_rows[b];
  }
  p.padded = (a.topk + kTileKeys - 1) / kTileKeys * kTileKeys;
  if (a.idx) words = (int64_t)p.rows * p.padded * a.heads;
  if (a.acc) {
    p.scores = (size_t)words * 4;
    p.stats = (size_t)p.rows * a.heads * sizeof(float2);
    p.slots = a.idx ? (size_t)p.rows * p.padded * 4 : 0;
  }
  return p;
}

}  // namespace

size_t attend_workspace(const AttendArgs& a, const RunTable& t) { return plan_of(a, t).bytes(); }

hipError_t launch_attend(const AttendArgs& a, const RunTable& t, hipStream_t stream) {
  const Plan p = plan_of(a, t);
  if (p.rows == 0) return hipSuccess;
  ScoreMap sm{};
  float* slots = nullptr;
  if (a.acc) {
    uint8_t* ws = (uint8_t*)a.workspace;
    sm.s2 = (float*)ws;
    sm.stat = (float2*)(ws + round256(p.scores));
    slots = (float*)(ws + round256(p.scores) + round256(p.stats));
    for (int b = 0; b < t.n; ++b) sm.base[b] = p.base[b];
  }
  hipLaunchKernelGGL(attend_kernel, dim3((unsigned)a.heads, (unsigned)p.rows), dim3(256), 0, stream, a, t, sm);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.acc || (a.idx && a.topk == 0)) return e;
  if (!a.idx) {
    const unsigned tiles = (unsigned)((p.max_n + kTileKeys - 1) / kTileKeys);
    hipLaunchKernelGGL(dense_weights_kernel, dim3(tiles, (unsigned)t.n), dim3(256), 0, stream, a, t, sm);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(slot_weights_kernel, dim3((unsigned)(p.padded / kTileKeys), (unsigned)p.rows), dim3(256), 0, stream,
                     a, sm, slots, p.padded);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(slot_add_kernel, dim3((unsigned)((p.max_n + kRange - 1) / kRange), (unsigned)t.n), dim3(256), 0,
                     stream, a, t, slots, p.padded);
  return hipGetLastError();
}

}  // namespace pivot
