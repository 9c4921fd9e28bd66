// Eviction from a cache by accumulated attention weight.
//
// Of a sequence's n cached tokens the first `sink`, the last `recent` and the
// largest acc of the others stay, `keep` in all (all of them when n <= keep);
// equal weights go to the lower position.  The kept positions come out in
// ascending order, so the compacted cache keeps the tokens' order.
//
// The threshold T of the others is found by four 8-bit radix passes over
// order-preserving keys; then a token stays when its key is above T, or equals T
// and fewer than the remaining count of equal keys precede it.
//
// Up to kWhole = 32768 tokens one workgroup keeps a sequence's keys in registers
// and does it all: 8192 tokens in 9.6 us, 20000 in 20, 32 sequences of 3000 to
// 32768 side by side in 22.  There are instances of 8192 and of 32768 places, and
// a sequence pays for all of its instance's: 8193 tokens take 17.4 us.  With 20000
// one CU's vector instructions take 26200 of 47800 cycles on every SIMD; the rest
// are waits for barriers, LDS and the first loads.  A longer sequence is cut into chunks, a workgroup each, with a launch
// per pass and one that emits; every workgroup adds up the chunks' counts of the
// pass before by itself.  That is five launches, 25 us at 32769 tokens and 33 at
// 131072, where one workgroup takes 200; at 20000 it is 25.
// The rows then move at a copy's rate: 131072 rows of 532 bytes in 30 us, 4.7 TB/s.
#include <algorithm>

#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWaves = kEvictThreads / kWave;
constexpr int kStep = 4 * kEvictThreads;  // positions: 4 adjacent ones a thread
constexpr int kWhole = 8 * kStep;
constexpr int kMaxChunks = 64;
constexpr int kCopies = 32;

// Accumulated weights lie close together: most share their first digit, and a
// wave's 64 additions to one counter would take turns.  So every counter has 32
// copies side by side in the banks, one for each lane of half a wave.
struct EvictShared {
  uint32_t copies[256 * kCopies];
  uint32_t hist[256];
  uint32_t found[2];
  uint32_t wsum[8 * kEvictWaves];
};

// What the launches of one sequence hand on.
struct EvictState {
  uint32_t thr[4], left[4];               // after each pass
  uint32_t above[4][kMaxChunks];          // a chunk's keys that the pass found above the threshold
  uint32_t hist[4][kMaxChunks][256];
};

// How a sequence's tokens are selected: the first lo and those from hi on stay,
// and `places` of the others, which are more.
struct Tokens {
  int n, lo, hi;
  uint32_t places;
  const float* acc;
  __device__ __forceinline__ Tokens(const EvictArgs& a, const RunTable& t, int b)
      : n(t.n_k[b]), lo(a.sink), hi(n - a.recent), places((uint32_t)(a.keep - a.sink - a.recent)),
        acc(a.acc + (int64_t)b * a.acc_stride) {}
  // Keys of positions s .. s + 3: 0 where they are not of the others, which is below
  // every number and cannot reach the threshold.
  __device__ __forceinline__ void load(uint32_t (&key)[4], int s) const {
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (s + 3 < n && ((uintptr_t)(acc + s) & 15) == 0) {
      const float4 x = *reinterpret_cast<const float4*>(acc + s);
      v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (s + i < n) v[i] = acc[s + i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = s + i >= lo && s + i < hi ? float_key(v[i]) : 0u;
  }
};

__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  return wave_total_at63(x, 0u, [](uint32_t a, uint32_t b) { return a + b; });
}

// Counts of digit `shift` of the keys that each(f) calls f with and that agree
// with thr above it, to sh.hist; begins and ends with a barrier.
template <class Each>
__device__ __forceinline__ void histogram(EvictShared& sh, int shift, uint32_t thr, Each&& each) {
  const int tid = threadIdx.x, lane = tid & 63;
#pragma unroll
  for (int i = 0; i < 256 * kCopies / kEvictThreads; i += 4)
    *reinterpret_cast<uint4*>(&sh.copies[i * kEvictThreads + 4 * tid]) = uint4{0, 0, 0, 0};
  __syncthreads();
  const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
  each([&](uint32_t key) {
    if ((key & mask) == thr) atomicAdd(&sh.copies[(key >> shift & 255) * kCopies + (lane & (kCopies - 1))], 1u);
  });
  __syncthreads();
  // 4 threads a counter, 8 copies each
  const uint4 x = *reinterpret_cast<const uint4*>(&sh.copies[8 * tid]),
              y = *reinterpret_cast<const uint4*>(&sh.copies[8 * tid + 4]);
  uint32_t sum = (x.x + x.y + x.z + x.w) + (y.x + y.y + y.z + y.w);
  sum += lane_xor1(sum);
  sum += lane_xor2(sum);
  if ((tid & 3) == 0) sh.hist[tid >> 2] = sum;
  __syncthreads();
}

// The digit of sh.hist that the `left`-th largest key has; left: among the keys
// with that digit.  Ends with a barrier.
__device__ __forceinline__ uint32_t digit_of(EvictShared& sh, uint32_t& left) {
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < kWave) {  // lane l holds digits 255 - 4l .. 252 - 4l, from the top
    uint32_t c[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = sh.hist[255 - 4 * lane - i], sum += c[i];
    uint32_t above = wave_scan(sum) - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (above < left && above + c[i] >= left) {
        sh.found[0] = (uint32_t)(255 - 4 * lane - i);
        sh.found[1] = left - above;
      }
      above += c[i];
    }
  }
  __syncthreads();
  left = sh.found[1];
  return sh.found[0];
}

// Emits the tokens that stay of C steps of positions from base on, in order;
// sure / tie: how many before them stay for sure / equal the threshold.  Both
// counts go through the sums in one word (C steps have at most 32768 of each).
template <int C>
__device__ __forceinline__ void emit(EvictShared& sh, const EvictArgs& a, const Tokens& k, int b,
                                     const uint32_t (&key)[C][4], int base, uint32_t thr, uint32_t left, uint32_t& sure0,
                                     uint32_t& tie0) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* out = a.out_keep + (int64_t)b * a.keep;
  float* out_acc = a.out_acc ? a.out_acc + (int64_t)b * a.keep : nullptr;
  auto kind = [&](int c, int i) -> uint32_t {
    const int s = base + c * kStep + 4 * tid + i;
    return s >= k.n ? 0u : s < k.lo || s >= k.hi ? 1u : key[c][i] > thr ? 1u : key[c][i] == thr ? 1u << 16 : 0u;
  };
  uint32_t before[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const uint32_t mine = kind(c, 0) + kind(c, 1) + kind(c, 2) + kind(c, 3);
    const uint32_t incl = wave_scan(mine);
    if (lane == 63) sh.wsum[c * kEvictWaves + wave] = incl;
    before[c] = incl - mine;
  }
  __syncthreads();
  if (tid < kWave) {  // exclusive sums over steps and waves
    constexpr int E = (C * kEvictWaves + 63) / 64;  // a lane's
    const bool has = E * lane < C * kEvictWaves;
    uint32_t x[E], mine = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = has ? sh.wsum[E * lane + i] : 0u, mine += x[i];
    const uint32_t incl = wave_scan(mine);
    uint32_t sum = incl - mine;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (has) sh.wsum[E * lane + i] = sum;
      sum += x[i];
    }
    if (lane == 63) sh.found[0] = incl;
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < C; ++c) {
    before[c] += sh.wsum[c * kEvictWaves + wave];
    uint32_t sure = sure0 + (before[c] & 0xFFFFu), tie = tie0 + (before[c] >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t q = kind(c, i);
      if (q == 1 || (q > 1 && tie < left)) {
        const uint32_t j = sure + (tie < left ? tie : left);
        const int s = base + c * kStep + 4 * tid + i;
        out[j] = s;
        if (out_acc) out_acc[j] = k.acc[s];
      }
      sure += q & 0xFFFFu;
      tie += q >> 16;
    }
  }
  sure0 += sh.found[0] & 0xFFFFu;
  tie0 += sh.found[0] >> 16;
}

// Up to C <= 8 steps of tokens, or all of them kept.
template <int C>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictArgs a, RunTable t) {
  __shared__ __attribute__((aligned(16))) EvictShared sh;
  const int b = blockIdx.x, tid = threadIdx.x;
  const Tokens k(a, t, b);
  if (k.n <= a.keep) {
    for (int j = tid; j < a.keep; j += kEvictThreads) {
      a.out_keep[(int64_t)b * a.keep + j] = j < k.n ? j : -1;
      if (a.out_acc) a.out_acc[(int64_t)b * a.keep + j] = j < k.n ? k.acc[j] : 0.f;
    }
    return;
  }
  if (k.n > C * kStep) return;
  uint32_t key[C][4];
#pragma unroll
  for (int c = 0; c < C; ++c) k.load(key[c], c * kStep + 4 * tid);
  uint32_t thr = 0, left = k.places;
  if (left > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      histogram(sh, shift, thr, [&](auto&& f) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) f(key[c][i]);
      });
      thr |= digit_of(sh, left) << shift;
    }
  } else {
    thr = 0xFFFFFFFFu;  // none of the others stays: only a NaN has this key, and none is wanted
  }
  uint32_t sure = 0, tie = 0;
  __syncthreads();
  emit(sh, a, k, b, key, 0, thr, left, sure, tie);
}

// Longer sequences: chunk blockIdx.x of sequence blockIdx.y.
struct Chunk {
  int n, begin, end;
  __device__ __forceinline__ Chunk(int tokens) {
    const int len = (tokens + kMaxChunks * kStep - 1) / (kMaxChunks * kStep) * kStep;
    n = (tokens + len - 1) / len;
    begin = (int)blockIdx.x * len;
    end = min(tokens - begin, len) + begin;
  }
};

// The pass's digit from all chunks' counts.
__device__ __forceinline__ uint32_t resolve(EvictShared& sh, const EvictState& st, int pass, int chunks, uint32_t& left) {
  const int bin = threadIdx.x & 255, part = threadIdx.x >> 8;
  uint32_t sum = 0;
  for (int c = part; c < chunks; c += 4) sum += st.hist[pass][c][bin];
  sh.copies[threadIdx.x] = sum;
  __syncthreads();
  if (part == 0) sh.hist[bin] = sum + sh.copies[256 + bin] + sh.copies[512 + bin] + sh.copies[768 + bin];
  __syncthreads();
  return digit_of(sh, left);
}

__global__ __launch_bounds__(kEvictThreads) void evict_pass_kernel(EvictArgs a, RunTable t, EvictState* states, int pass) {
  __shared__ __attribute__((aligned(16))) EvictShared sh;
  const int b = blockIdx.y, tid = threadIdx.x, chunk = blockIdx.x;
  const Tokens k(a, t, b);
  if (k.n <= a.keep || k.n <= kWhole || k.places == 0) return;
  const Chunk ch(k.n);
  if (chunk >= ch.n) return;
  EvictState& st = states[b];
  uint32_t thr = pass >= 2 ? st.thr[pass - 2] : 0, left = pass >= 2 ? st.left[pass - 2] : k.places;
  if (pass > 0) {
    const uint32_t digit = resolve(sh, st, pass - 1, ch.n, left);
    thr |= digit << (32 - 8 * pass);
    if (chunk == 0 && tid == 0) st.thr[pass - 1] = thr, st.left[pass - 1] = left;
    if (tid < kWave) {
      uint32_t above = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) above += 4 * tid + i > (int)digit ? st.hist[pass - 1][chunk][4 * tid + i] : 0u;
      above = wave_scan(above);
      if (tid == kWave - 1) st.above[pass - 1][chunk] = above;
    }
  }
  histogram(sh, 24 - 8 * pass, thr, [&](auto&& f) {
    for (int base = ch.begin; base < ch.end; base += kStep) {
      uint32_t key[4];
      k.load(key, base + 4 * tid);
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // the others only: emission counts on from the chunks' sums
        const int s = base + 4 * tid + i;
        if (s >= k.lo && s < k.hi) f(key[i]);
      }
    }
  });
  if (tid < 256) st.hist[pass][chunk][tid] = sh.hist[tid];
}

__global__ __launch_bounds__(kEvictThreads) void evict_emit_kernel(EvictArgs a, RunTable t, const EvictState* states) {
  __shared__ __attribute__((aligned(16))) EvictShared sh;
  const int b = blockIdx.y, tid = threadIdx.x, chunk = blockIdx.x;
  const Tokens k(a, t, b);
  if (k.n <= a.keep || k.n <= kWhole) return;
  const Chunk ch(k.n);
  if (chunk >= ch.n) return;
  const EvictState& st = states[b];
  uint32_t thr = 0xFFFFFFFFu, left = 0, sure = 0, tie = 0;
  if (k.places > 0) {
    left = st.left[2];
    const uint32_t digit = resolve(sh, st, 3, ch.n, left);
    thr = st.thr[2] | digit;
    // the chunks before: a wave's lanes are chunks, the waves share the digits above
    uint32_t above = 0;
    const int lane = tid & 63, wave = tid >> 6;
    if (lane < chunk) {
      for (int d = wave; d < 256; d += kEvictWaves) above += d > (int)digit ? st.hist[3][lane][d] : 0u;
      if (wave < 3) above += st.above[wave][lane];
    }
    const uint32_t equal = wave == 0 && lane < chunk ? st.hist[3][lane][digit] : 0u;
    above = wave_scan(above);
    const uint32_t equals = wave_scan(equal);
    __syncthreads();
    if (lane == 63) {
      sh.wsum[wave] = above;
      if (wave == 0) sh.found[0] = equals;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) sure += sh.wsum[w];
    tie = sh.found[0];
    __syncthreads();
  }
  sure += (uint32_t)(min(ch.begin, k.lo) + max(0, ch.begin - k.hi));
  for (int base = ch.begin; base < ch.end; base += kStep) {
    uint32_t key[1][4];
    k.load(key[0], base + 4 * tid);
    emit(sh, a, k, b, key, base, thr, left, sure, tie);
    __syncthreads();
  }
}

// kMoveRows kept rows of one sequence in every array.  A row's two
// places are found once; 16 bytes (or 4, where that is all the row or its
// pointers allow) a thread, the threads of a row side by side.
constexpr int kMoveRows = 64;

template <class U>
__device__ __forceinline__ void move_rows(const uint8_t* src, uint8_t* dst, int bytes, const int64_t* from,
                                          const int64_t* to) {
  const int units = bytes / (int)sizeof(U);
  int lg = 0;
  while ((1 << lg) < units && lg < 8) ++lg;  // threads of a row
  const int part = threadIdx.x & ((1 << lg) - 1);
#pragma unroll 4
  for (int r = threadIdx.x >> lg; r < kMoveRows; r += 256 >> lg) {
    if (from[r] < 0) continue;
    const U* x = reinterpret_cast<const U*>(src + from[r] * bytes);
    U* y = reinterpret_cast<U*>(dst + to[r] * bytes);
    for (int i = part; i < units; i += 1 << lg) y[i] = x[i];
  }
}

__global__ __launch_bounds__(256) void move_kernel(MoveArrays m, KeyMap from, KeyMap to, const int32_t* __restrict__ kept,
                                                   int b0, int keep, unsigned groups) {
  __shared__ int64_t s_from[kMoveRows], s_to[kMoveRows];
  const int b = b0 + (int)(blockIdx.x / groups), j = (int)(blockIdx.x % groups) * kMoveRows + threadIdx.x;
  if (threadIdx.x < kMoveRows) {
    const int32_t pos = j < keep ? kept[(int64_t)b * keep + j] : -1;
    const int64_t row = pos < 0 ? -1 : to.held_row(b, j);
    s_from[threadIdx.x] = row < 0 ? -1 : from.row(b, pos);
    s_to[threadIdx.x] = row;
  }
  __syncthreads();
  for (int arr = 0; arr < m.n; ++arr) {
    const int bytes = m.row_bytes[arr];
    if (((bytes | (uintptr_t)m.src[arr] | (uintptr_t)m.dst[arr]) & 15) == 0)
      move_rows<uint4>(m.src[arr], m.dst[arr], bytes, s_from, s_to);
    else
      move_rows<uint32_t>(m.src[arr], m.dst[arr], bytes, s_from, s_to);
  }
}

}  // namespace

size_t evict_workspace(const EvictArgs& a, const RunTable& t) {
  for (int b = 0; b < t.n; ++b)
    if (t.n_k[b] > kWhole && t.n_k[b] > a.keep) return (size_t)t.n * sizeof(EvictState);
  return 0;
}

hipError_t launch_evict(const EvictArgs& a, const RunTable& t, void* workspace, hipStream_t stream) {
  int chunks = 0, whole = 0, longest = 0;
  for (int b = 0; b < t.n; ++b) {
    const int steps = (int)(((int64_t)t.n_k[b] + kStep - 1) / kStep);
    if (t.n_k[b] > kWhole && t.n_k[b] > a.keep) chunks = std::max(chunks, std::min(steps, kMaxChunks));
    else {
      ++whole;
      if (t.n_k[b] > a.keep) longest = std::max(longest, t.n_k[b]);
    }
  }
  hipError_t e = hipSuccess;
  if (whole > 0) {
    const auto kernel = longest <= 2 * kStep ? evict_kernel<2> : evict_kernel<8>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)t.n), dim3(kEvictThreads), 0, stream, a, t);
    e = hipGetLastError();
  }
  if (chunks == 0) return e;
  const dim3 grid((unsigned)chunks, (unsigned)t.n);
  for (int pass = 0; pass < 4 && e == hipSuccess && a.keep > a.sink + a.recent; ++pass) {
    hipLaunchKernelGGL(evict_pass_kernel, grid, dim3(kEvictThreads), 0, stream, a, t, (EvictState*)workspace, pass);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_emit_kernel, grid, dim3(kEvictThreads), 0, stream, a, t, (const EvictState*)workspace);
  return hipGetLastError();
}

hipError_t launch_move(const MoveArrays& m, const KeyMap& from, const KeyMap& to, const int32_t* kept, int batch,
                       int keep, hipStream_t stream) {
  const unsigned groups = (unsigned)((keep + kMoveRows - 1) / kMoveRows);  // of a sequence
  // a launch counts its threads in 32 bits, and drops what is above without an error
  const int most = (int)(((1u << 24) - 1) / groups);  // sequences
  for (int b = 0; b < batch; b += most) {
    hipLaunchKernelGGL(move_kernel, dim3(groups * (unsigned)std::min(batch - b, most)), dim3(256), 0, stream, m, from, to,
                       kept, b, keep, groups);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pivot
