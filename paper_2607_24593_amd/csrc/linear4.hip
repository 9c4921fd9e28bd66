// Products of few rows with weights in 4 bits:
//
//   y[r, n] = s[r, .] sum_k x[r, k] w[n, k]
//
// w in OCP MXFP4 (E2M1 codes, a power-of-two scale per 32 values of k), x in bf16
// or in E4M3FN with a scale per row or per 128 values.  Codes and fp8 values are
// widened to bf16, which is exact (two and four significant bits), so every
// product is exact and only the sums round, in fp32.
#include <algorithm>

#include "cache4.h"
#include "ops.h"

namespace pivot {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kWaves = 8;
constexpr int kChunk = 128;  // values of k that a wave multiplies at a time: one scale per lane

struct __attribute__((packed, aligned(2))) Bf8 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(1))) Fp8x8 {
  uint32_t w[2];
};

// Eight E4M3FN codes as bf16.
__device__ __forceinline__ uint4 widen8(const Fp8x8& v) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto f = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)v.w[i >> 1], true)
                         : __builtin_amdgcn_cvt_pk_f32_fp8((int)v.w[i >> 1], false);
    o[i] = (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xFFFF0000u);
  }
  return uint4{o[0], o[1], o[2], o[3]};
}

// How a launch is cut: `kw` of a workgroup's 8 waves share k, the others take
// other tiles of 16 weight rows; `splits` workgroups share k.
struct Cut {
  int kw, splits;
  int tiles;   // of 16 weight rows
  int groups;  // workgroups along n
};

template <int MT, int KC, bool GROUPS>
__global__ __launch_bounds__(64 * kWaves, 2) void linear4_kernel(Linear4Args a, Cut cut, float* parts) {
  __shared__ __attribute__((aligned(16))) v4f s_part[2][kWaves][MT][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int nw = kWaves / cut.kw, wk = w % cut.kw, wn = w / cut.kw;
  const int row0 = blockIdx.z * 16 * MT;
  const int k0 = ((int)blockIdx.y * cut.kw + wk) * KC * kChunk;
  const int blocks = a.k / kBlk;  // scales of a weight row

  // the wave's part of x: column m = lane & 15 of every product, 8 values from
  // k0 + 128 c + 32 g + 8 u on in product (c, u)
  uint4 x[MT][KC][4];
  float xs[MT][KC];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = min(row0 + 16 * t + r, a.rows - 1);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int k = k0 + kChunk * c + kBlk * g;
      const bool in = k < a.k;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint4 v = {0, 0, 0, 0};
        if (in) {
          if (a.x_fp8) {
            v = widen8(*reinterpret_cast<const Fp8x8*>((const uint8_t*)a.x + m * a.ld_x + k + 8 * u));
          } else {
            const Bf8 b = *reinterpret_cast<const Bf8*>((const uint16_t*)a.x + m * a.ld_x + k + 8 * u);
            v = uint4{b.w[0], b.w[1], b.w[2], b.w[3]};
          }
        }
        x[t][c][u] = v;
      }
      if constexpr (GROUPS) {
        const int i = k0 / kChunk + c, n = (a.k + kChunk - 1) / kChunk;
        xs[t][c] = i < n ? a.x_scale[m * n + i] : 0.f;
      }
    }
  }

  const int per = (cut.tiles + cut.groups - 1) / cut.groups;  // tiles of a workgroup
  const int first = (int)blockIdx.x * per, last = min(first + per, cut.tiles);
  const int steps = (last - first + nw - 1) / nw;
  for (int i = 0; i < steps; ++i) {
    const int tile = first + i * nw + wn;
    const int64_t n = min(16 * tile + r, a.n - 1);
    uint4 code[KC];
    uint32_t byte[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int k = k0 + kChunk * c + kBlk * g;
      const bool in = k < a.k;
      const int at = in ? k : 0;
      code[c] = *reinterpret_cast<const uint4*>(a.codes + n * (a.k / 2) + at / 2);
      byte[c] = a.scales[n * blocks + at / kBlk];
      if (!in) {
        code[c] = uint4{0, 0, 0, 0};
        byte[c] = 127;
      }
    }
    v4f sum[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) sum[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      v4f part[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) part[t] = GROUPS ? v4f{0.f, 0.f, 0.f, 0.f} : sum[t];
      const uint32_t words[4] = {code[c].x, code[c].y, code[c].z, code[c].w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const v8bf wide = __builtin_bit_cast(v8bf, decode8(words[u], scale_operand(byte[c])));
#pragma unroll
        for (int t = 0; t < MT; ++t)
          part[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide, __builtin_bit_cast(v8bf, x[t][c][u]), part[t], 0, 0, 0);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if constexpr (GROUPS) {
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[t][e] = fmaf(part[t][e], xs[t][c], sum[t][e]);
        } else {
          sum[t] = part[t];
        }
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) s_part[i & 1][w][t][lane] = sum[t];
    __syncthreads();
    // the sums over the waves that share k: items (n tile, m tile), one a wave
    for (int item = w; item < nw * MT; item += kWaves) {
      const int tn = item / MT, t = item % MT;
      v4f total = s_part[i & 1][tn * cut.kw][t][lane];
      for (int j = 1; j < cut.kw; ++j) total += s_part[i & 1][tn * cut.kw + j][t][lane];
      const int m = row0 + 16 * t + r, at = 16 * (first + i * nw + tn) + 4 * g;
      if (first + i * nw + tn >= last || m >= a.rows) continue;
      if (parts) {
        float* to = parts + ((int64_t)blockIdx.y * a.rows + m) * a.n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (at + e < a.n) to[at + e] = total[e];
        continue;
      }
      const float s = a.x_fp8 && !GROUPS ? a.x_scale[m] : 1.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (at + e >= a.n) break;
        const float y = total[e] * s;
        if (a.out_fp32) ((float*)a.out)[m * a.ld_out + at + e] = y;
        else ((uint16_t*)a.out)[m * a.ld_out + at + e] = bf16_rne(y);
      }
    }
  }
}

// The sums of the workgroups that share k, in their order.
__global__ __launch_bounds__(256) void linear4_join_kernel(Linear4Args a, int splits, const float* parts) {
  const int n = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  if (n >= a.n) return;
  float y = 0.f;
  for (int s = 0; s < splits; ++s) y += parts[((int64_t)s * a.rows + m) * a.n + n];
  if (a.x_fp8 && a.group == 0) y *= a.x_scale[m];
  if (a.out_fp32) ((float*)a.out)[m * a.ld_out + n] = y;
  else ((uint16_t*)a.out)[m * a.ld_out + n] = bf16_rne(y);
}

// Rows of 32 weights to codes and a scale, 8 values a lane (cache4.hip says how).
template <class T>
__global__ __launch_bounds__(256) void linear4_pack_kernel(const T* __restrict__ w, int64_t ld, int32_t k, int64_t items,
                                                           int64_t first, uint8_t* codes, uint8_t* scales) {
  const int64_t i = first + (int64_t)blockIdx.x * 256 + threadIdx.x;  // 8 values each
  const int64_t at = i < items ? i : items - 1;
  const int64_t n = at / (k / 8);
  const int j = (int)(at - n * (k / 8));
  float v[8], top = 0.f;
  bool finite = true;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T x = w[n * ld + 8 * j + e];
    if constexpr (sizeof(T) == 2) v[e] = __uint_as_float((uint32_t)x << 16);
    else v[e] = x;
    finite = finite && fabsf(v[e]) < INFINITY;
    top = fmaxf(top, fabsf(v[e]));
  }
  uint32_t bits = finite ? __float_as_uint(top) : 0x7F800000u;  // |x| orders as its bits do
  bits = max(bits, (uint32_t)__shfl_xor((int)bits, 1, 64));
  bits = max(bits, (uint32_t)__shfl_xor((int)bits, 2, 64));
  // max|x| = 2^(E - 127) (1 + f) <= 6 * 2^e for e = E - 127 - 2, one more when f > 1/2
  const int fit = (int)(bits >> 23) - 2 + ((bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  const uint32_t byte = bits >= 0x7F800000u ? 255u : (uint32_t)max(fit, 0);
  const float s = scale_operand(byte);
  uint32_t code = 0;
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], s, 0);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], s, 1);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], s, 2);
  code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], s, 3);
  if (byte == 255u) code = 0;
  if (i >= items) return;
  *reinterpret_cast<uint32_t*>(codes + n * (k / 2) + 4 * j) = code;
  if ((j & 3) == 0) scales[n * (k / kBlk) + j / 4] = (uint8_t)byte;
}

struct Plan {
  int mt, kc;
  Cut cut;
};

Plan plan_of(const Linear4Args& a) {
  Plan p{};
  p.mt = a.rows <= 16 ? 1 : a.rows <= 32 ? 2 : 4;
  const int most = 8 / p.mt;  // chunks of k whose x a wave keeps
  const int chunks = (a.k + kChunk - 1) / kChunk;
  p.cut.splits = (chunks + kWaves * most - 1) / (kWaves * most);
  const int mine = (chunks + p.cut.splits - 1) / p.cut.splits;  // of a workgroup
  p.kc = (mine + kWaves - 1) / kWaves;
  const int waves = (mine + p.kc - 1) / p.kc;
  p.cut.kw = waves > 4 ? 8 : waves > 2 ? 4 : waves;
  p.cut.tiles = (a.n + 15) / 16;
  const int nw = kWaves / p.cut.kw;
  p.cut.groups = std::min((p.cut.tiles + nw - 1) / nw, 512);
  return p;
}

template <int MT, int KC>
void launch(const Linear4Args& a, const Plan& p, float* parts, hipStream_t stream) {
  const dim3 grid((unsigned)p.cut.groups, (unsigned)p.cut.splits, (unsigned)((a.rows + 16 * MT - 1) / (16 * MT)));
  if (a.group)
    hipLaunchKernelGGL((linear4_kernel<MT, KC, true>), grid, dim3(64 * kWaves), 0, stream, a, p.cut, parts);
  else
    hipLaunchKernelGGL((linear4_kernel<MT, KC, false>), grid, dim3(64 * kWaves), 0, stream, a, p.cut, parts);
}

}  // namespace

size_t linear4_workspace(const Linear4Args& a) {
  const Plan p = plan_of(a);
  return p.cut.splits > 1 ? (size_t)p.cut.splits * a.rows * a.n * 4 : 0;
}

hipError_t launch_linear4(const Linear4Args& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(a);
  float* parts = p.cut.splits > 1 ? (float*)workspace : nullptr;
  switch (10 * p.mt + p.kc) {
    case 11: launch<1, 1>(a, p, parts, stream); break;
    case 12: launch<1, 2>(a, p, parts, stream); break;
    case 13: launch<1, 3>(a, p, parts, stream); break;
    case 14: launch<1, 4>(a, p, parts, stream); break;
    case 15: launch<1, 5>(a, p, parts, stream); break;
    case 16: launch<1, 6>(a, p, parts, stream); break;
    case 17: launch<1, 7>(a, p, parts, stream); break;
    case 18: launch<1, 8>(a, p, parts, stream); break;
    case 21: launch<2, 1>(a, p, parts, stream); break;
    case 22: launch<2, 2>(a, p, parts, stream); break;
    case 23: launch<2, 3>(a, p, parts, stream); break;
    case 24: launch<2, 4>(a, p, parts, stream); break;
    case 41: launch<4, 1>(a, p, parts, stream); break;
    default: launch<4, 2>(a, p, parts, stream); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !parts) return e;
  hipLaunchKernelGGL(linear4_join_kernel, dim3((unsigned)((a.n + 255) / 256), (unsigned)a.rows), dim3(256), 0, stream, a,
                     p.cut.splits, parts);
  return hipGetLastError();
}

hipError_t launch_linear4_pack(bool fp32, int32_t n, int32_t k, const void* w, int64_t ld, uint8_t* codes,
                               uint8_t* scales, hipStream_t stream) {
  const int64_t items = (int64_t)n * (k / 8), most = int64_t(1) << 30;  // a launch counts its threads in 32 bits
  for (int64_t first = 0; first < items; first += most) {
    const unsigned grid = (unsigned)((std::min(items - first, most) + 255) / 256);
    if (fp32)
      hipLaunchKernelGGL(linear4_pack_kernel<float>, dim3(grid), dim3(256), 0, stream, (const float*)w, ld, k, items,
                         first, codes, scales);
    else
      hipLaunchKernelGGL(linear4_pack_kernel<uint16_t>, dim3(grid), dim3(256), 0, stream, (const uint16_t*)w, ld, k,
                         items, first, codes, scales);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pivot
