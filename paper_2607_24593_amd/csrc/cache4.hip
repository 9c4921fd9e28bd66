// Writing tokens into the 4-bit latent cache and reading rows back.
//
// A block of 32 latent values x shares the scale 2^e, the smallest power of
// two with max|x| / 2^e <= 6 (6 is the largest E2M1 value, so nothing
// saturates); its codes are the E2M1 values nearest to x / 2^e, ties to even.
// Dividing by a power of two is exact, so is the product on reading: a value
// read back is the code's value times 2^e in bf16 (infinite where 3.5 * 2^126 and
// more was rounded up to 4 * 2^126).  A block of zeros has the
// scale byte 0, a block that holds an infinity or a NaN the byte 255 (all of
// it reads as NaN).
//
// One wave per token, 8 values a lane: 1152 bytes read and 400 written (or the
// reverse), each once and in whole cache lines; bound by bytes, or by the
// latency of one round of loads for a few tokens.  8192 tokens: written in 4.2 us
// (3.0 TB/s), read in 4.8; 131072 paged rows read in 40 us, 5.1 TB/s; one token of
// 32 sequences: 3.6 and 2.8.
#include <algorithm>

#include "cache4.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kWavesPerWg = 4;

struct __attribute__((packed, aligned(2))) Bf8 {
  uint32_t w[4];
};

__device__ __forceinline__ uint32_t max_u32(uint32_t a, uint32_t b) { return a > b ? a : b; }

__global__ __launch_bounds__(256) void cache4_write_kernel(Cache4Write a, RunTable t) {
  const int lane = threadIdx.x & 63;
  const int r = blockIdx.x * kWavesPerWg + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const int b = run_of(t, r);
  const int64_t row = a.map.held_row(b, (int64_t)t.pos0[b] + (r - t.row0[b]));
  const Bf8 v = *reinterpret_cast<const Bf8*>(a.latent + r * a.ld_latent + 8 * lane);
  const uint16_t rope = a.rope[r * a.ld_rope + lane];
  // |x| of bf16 orders as its bits do, infinities and NaN last
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max_u32(top, max_u32(v.w[i] & 0x7FFFu, (v.w[i] >> 16) & 0x7FFFu));
  top = max_u32(top, lane_xor1(top));
  top = max_u32(top, lane_xor2(top));
  // max|x| = 2^(E - 127) (1 + m / 128) <= 6 * 2^e for e = E - 127 - 2, one more when m / 128 > 1/2
  const int fit = (int)(top >> 7) - 2 + ((top & 0x7F) > 64 ? 1 : 0);
  const uint32_t byte = top >= 0x7F80u ? 255u : (uint32_t)max(fit, 0);
  const float s = scale_operand(byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(v2bf, v.w[0]), s, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(v2bf, v.w[1]), s, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(v2bf, v.w[2]), s, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(v2bf, v.w[3]), s, 3);
  if (byte == 255u) code = 0;
  if (row < 0) return;
  *reinterpret_cast<uint32_t*>(a.cache.codes + row * kCodeBytes + 4 * lane) = code;
  if ((lane & 3) == 0) a.cache.scales[row * kScaleBytes + (lane >> 2)] = (uint8_t)byte;
  a.cache.rope[row * kRope + lane] = rope;
}

__global__ __launch_bounds__(256) void cache4_read_kernel(Cache4Read a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = a.first + (int64_t)blockIdx.x * kWavesPerWg + (threadIdx.x >> 6);
  if (r >= (int64_t)a.batch * a.n) return;
  const int b = (int)(r / a.n);
  const int32_t pos = a.idx[r];
  uint4 v = {0, 0, 0, 0};
  uint16_t rope = 0;
  if (pos >= 0 && pos < a.capacity) {
    const int64_t row = a.map.row(b, pos);
    const uint32_t code = *reinterpret_cast<const uint32_t*>(a.cache.codes + row * kCodeBytes + 4 * lane);
    v = decode8(code, scale_operand(a.cache.scales[row * kScaleBytes + (lane >> 2)]));
    rope = a.cache.rope[row * kRope + lane];
  }
  uint16_t* out = a.out + r * kAttnDim;  // 1152-byte rows: 16-byte aligned
  *reinterpret_cast<uint4*>(out + 8 * lane) = v;
  out[kLatent + lane] = rope;
}

}  // namespace

hipError_t launch_cache4_write(const Cache4Write& a, const RunTable& t, hipStream_t stream) {
  const unsigned grid = (unsigned)((a.rows + kWavesPerWg - 1) / kWavesPerWg);
  hipLaunchKernelGGL(cache4_write_kernel, dim3(grid), dim3(64 * kWavesPerWg), 0, stream, a, t);
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4Read& a, hipStream_t stream) {
  Cache4Read part = a;
  const int64_t end = (int64_t)a.batch * a.n;
  for (; part.first < end; part.first += kMaxCacheRows) {
    const unsigned grid = (unsigned)((std::min<int64_t>(end - part.first, kMaxCacheRows) + kWavesPerWg - 1) / kWavesPerWg);
    hipLaunchKernelGGL(cache4_read_kernel, dim3(grid), dim3(64 * kWavesPerWg), 0, stream, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pivot
