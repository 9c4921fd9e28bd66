// Root-mean-square norm of x + residual with E4M3FN output: the fp8 rows and
// scales that the index calls (and fp8 products) take.
//
//   h = x + residual                        fp32 sum; stored rounded to x's type
//   y = h * rsqrt(mean(h^2) + eps) * weight  fp32, of the unrounded h
//   per group of the row: scale = max|y| / 448 (1 if max|y| is 0, else at least 2^-149),
//                         code = RNE(y / scale)
//
// One workgroup per row, the row held in registers: x, residual and weight are
// read once and every output is written once, so the kernel is bound by bytes
// (by latency for a few rows).  max|y| needs no second pass: with one scale
// per row it is max|h w| times the rsqrt, reduced together with the sum of
// squares (where max|h w| is no normal number the row's y are reduced instead);
// with a scale per 128 values, 16 neighbouring lanes hold a group.
// 8192 x 6144 fp32 values: 122 us, 5.4 TB/s, a copy's rate; 260 rows of bf16 in
// groups: 5.1 of 5120 values, 6.4 of 5003, whose odd rows start anywhere; one row
// of 4096: 2.8.
#include <algorithm>

#include "device_common.h"
#include "dpp.h"
#include "ops.h"

namespace pivot {

namespace {

constexpr int kV = 8;  // values a thread holds side by side
constexpr int kNormGroup = 128;

// Eight values from an address aligned to the element only: rows of odd width
// start anywhere, and the hardware takes unaligned vector accesses.
struct __attribute__((packed, aligned(2))) Bf8 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) F8 {
  float v[8];
};
struct __attribute__((packed, aligned(1))) C8 {
  uint32_t w[2];
};

__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float widen(float f) { return f; }
__device__ __forceinline__ void narrow(float f, uint16_t& o) { o = bf16_rne(f); }
__device__ __forceinline__ void narrow(float f, float& o) { o = f; }

// v[0..7] = p[e .. e+7], zero past n
template <class T>
__device__ __forceinline__ void load8(const T* p, int e, int n, float (&v)[kV]) {
  if (e + kV <= n) {
    if constexpr (sizeof(T) == 2) {
      const Bf8 b = *reinterpret_cast<const Bf8*>(p + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(b.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(b.w[i] & 0xFFFF0000u);
      }
    } else {
      const F8 b = *reinterpret_cast<const F8*>(p + e);
#pragma unroll
      for (int i = 0; i < kV; ++i) v[i] = b.v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] = e + i < n ? widen(p[e + i]) : 0.f;
  }
}

template <class T>
__device__ __forceinline__ void store8(T* p, int e, int n, const float (&v)[kV]) {
  if (e + kV <= n) {
    if constexpr (sizeof(T) == 2) {
      Bf8 b;
#pragma unroll
      for (int i = 0; i < 4; ++i) b.w[i] = (uint32_t)bf16_rne(v[2 * i]) | ((uint32_t)bf16_rne(v[2 * i + 1]) << 16);
      *reinterpret_cast<Bf8*>(p + e) = b;
    } else {
      F8 b;
#pragma unroll
      for (int i = 0; i < kV; ++i) b.v[i] = v[i];
      *reinterpret_cast<F8*>(p + e) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (e + i < n) narrow(v[i], p[e + i]);
  }
}

__device__ __forceinline__ float scale_of(float amax) { return amax > 0.f ? fmaxf(amax / 448.f, 0x1p-149f) : 1.f; }

// y / s for y = h rstd w, with r = 1 / s: one correction step, so the quotient is
// that of the division up to its last bit's rounding.  Below 2^-126 the reciprocal
// may be infinite, so there the division itself is taken; such a scale is rounded
// to few bits, and the quotient may pass 448 by half of them.
__device__ __forceinline__ void quotients(float (&y)[kV], float s) {
  if (s >= 0x1p-126f) {
    const float r = 1.f / s;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const float q = y[i] * r;
      y[i] = fmaf(fmaf(-q, s, y[i]), r, q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const float q = y[i] / s;
      y[i] = q > 448.f ? 448.f : q < -448.f ? -448.f : q;
    }
  }
}

template <class T, int NT, int IT, bool GROUPS>
__global__ __launch_bounds__(NT) void norm_kernel(const T* x, int64_t ld_x, const T* res, int64_t ld_res,
                                                   const T* __restrict__ weight, float eps, int dim, T* res_out,
                                                   uint8_t* __restrict__ codes, float* __restrict__ scale) {
  constexpr int NW = NT / kWave;
  __shared__ float part[2][NW];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  x += row * ld_x;
  float h[IT][kV], w[IT][kV];
  float sq = 0.f, top = 0.f;
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = (it * NT + tid) * kV;
    if (e >= dim) {
#pragma unroll
      for (int i = 0; i < kV; ++i) h[it][i] = w[it][i] = 0.f;
      continue;
    }
    load8(x, e, dim, h[it]);
    if (res) {
      float r[kV];
      load8(res + row * ld_res, e, dim, r);
#pragma unroll
      for (int i = 0; i < kV; ++i) h[it][i] += r[i];
    }
    load8(weight, e, dim, w[it]);
    if (res_out) store8(res_out + row * (int64_t)dim, e, dim, h[it]);
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      sq = fmaf(h[it][i], h[it][i], sq);
      if constexpr (!GROUPS) top = fmaxf(top, fabsf(h[it][i] * w[it][i]));
    }
  }
  sq = wave_reduce(sq, [](float a, float b) { return a + b; });
  top = wave_reduce(top, [](float a, float b) { return fmaxf(a, b); });
  if constexpr (NW > 1) {
    if ((tid & 63) == 0) part[0][tid >> 6] = sq, part[1][tid >> 6] = top;
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) sq += part[0][i], top = fmaxf(top, part[1][i]);
  }
  const float rstd = 1.0f / sqrtf(sq / (float)dim + eps);
  uint8_t* out = codes + row * (int64_t)dim;
  const int groups = GROUPS ? (dim + kNormGroup - 1) / kNormGroup : 1;
#pragma unroll
  for (int it = 0; it < IT; ++it)
#pragma unroll
    for (int i = 0; i < kV; ++i) h[it][i] = h[it][i] * rstd * w[it][i];  // y
  float s = 1.f;
  if constexpr (!GROUPS) {
    float amax = top * rstd;
    if (!(top >= 0x1p-126f && top < INFINITY)) {  // the same in all threads: h w left fp32's range, y need not have
      amax = 0.f;
#pragma unroll
      for (int it = 0; it < IT; ++it)
#pragma unroll
        for (int i = 0; i < kV; ++i) amax = fmaxf(amax, fabsf(h[it][i]));
      amax = wave_reduce(amax, [](float a, float b) { return fmaxf(a, b); });
      if constexpr (NW > 1) {
        __syncthreads();
        if ((tid & 63) == 0) part[0][tid >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) amax = fmaxf(amax, part[0][i]);
      }
    }
    s = scale_of(amax);
    if (tid == 0) scale[row] = s;
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int e = (it * NT + tid) * kV;
    if constexpr (GROUPS) {  // every lane takes part: those past the row hold zeros
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < kV; ++i) a = fmaxf(a, fabsf(h[it][i]));
      a = fmaxf(a, lane_xor1(a));
      a = fmaxf(a, lane_xor2(a));
      a = fmaxf(a, lane_xor4(a));
      a = fmaxf(a, lane_xor8(a));
      s = scale_of(a);
      if (e < dim && (tid & 15) == 0) scale[row * groups + e / kNormGroup] = s;
    }
    if (e >= dim) continue;
    float (&y)[kV] = h[it];
    quotients(y, s);
    C8 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
      c.w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], lo, true);
    }
    if (e + kV <= dim) {
      *reinterpret_cast<C8*>(out + e) = c;
    } else {
#pragma unroll
      for (int i = 0; i < kV; ++i)
        if (e + i < dim) out[e + i] = (uint8_t)(c.w[i / 4] >> (8 * (i % 4)));
    }
  }
}

template <class T, bool GROUPS>
hipError_t launch(const NormArgs& a, hipStream_t stream) {
  const int groups = GROUPS ? (a.dim + kNormGroup - 1) / kNormGroup : 1;
  // a launch counts its threads in 32 bits, and drops what is above without an error
  constexpr int64_t kMost = 1 << 21;
  for (int64_t row = 0; row < a.rows; row += kMost) {
    const T* x = (const T*)a.x + row * a.ld_x;
    const T* res = a.residual ? (const T*)a.residual + row * a.ld_residual : nullptr;
    T* res_out = a.residual_out ? (T*)a.residual_out + row * a.dim : nullptr;
    const dim3 grid((unsigned)std::min<int64_t>(a.rows - row, kMost));
#define PIVOT_NORM(NT, IT)                                                                                      \
  hipLaunchKernelGGL((norm_kernel<T, NT, IT, GROUPS>), grid, dim3(NT), 0, stream, x, a.ld_x, res, a.ld_residual, \
                     (const T*)a.weight, a.eps, a.dim, res_out, a.codes + row * a.dim, a.scale + row * groups)
    // The fewest threads that hold a row with 8 values each, and 32 a thread only
    // where 8 are not enough.  Us for 8192 bf16 rows: of 2048 values, 256 threads 20.9
    // and 1024 40.3; of 512, 12.2 and 34.7; of 8192, 8 values a thread 93.7 and 32
    // 144.9.  64 rows: of 2048 3.5 and 3.6, of 8192 4.5 and 5.1.
    if (a.dim <= 2048) PIVOT_NORM(256, 1);
    else if (a.dim <= 8192) PIVOT_NORM(1024, 1);
    else PIVOT_NORM(1024, 4);
#undef PIVOT_NORM
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_norm(int dtype, const NormArgs& a, hipStream_t stream) {
  if (dtype == PIVOT_DT_BF16)
    return a.group ? launch<uint16_t, true>(a, stream) : launch<uint16_t, false>(a, stream);
  return a.group ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace pivot
