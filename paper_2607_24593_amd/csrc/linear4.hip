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
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

constexpr int kCus = 256;
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
// other tiles of 16 weight rows; `splits` workgroups share k; `groups` share the
// tiles.
struct Cut {
  int kw, splits, tiles, groups;
};

// Sixteen bytes (four; one, as a word) of every lane from base + off into LDS at byte
// address dst + 16 (4) * lane, base and dst the same in all lanes of the wave.  The
// waves wait for these loads themselves.  A scalar register that a vector instruction
// wrote (readfirstlane) may be read by a memory instruction five wait states later;
// the compiler does not see into the statement, so it waits itself.
__device__ __forceinline__ const void* uniform(const void* p) {
  const uint64_t v = (uint64_t)p;
  return (const void*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}
__device__ __forceinline__ void load_lds16(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(dst), "v"(off), "s"(uniform(base)) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("s_nop 4\n\tglobal_load_lds_dword %1, %2" ::"{m0}"(dst), "v"(off), "s"(uniform(base)) : "memory");
}
__device__ __forceinline__ void load_lds1(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("s_nop 4\n\tglobal_load_lds_ubyte %1, %2" ::"{m0}"(dst), "v"(off), "s"(uniform(base)) : "memory");
}

// A workgroup of 8 waves keeps its part of x in registers, KC chunks of 128 values
// of 16 MT rows a wave, and passes all of its weight tiles by it.  A wave's part of a
// tile (16 rows x KC chunks: 1 KB of codes a chunk, then the scales) is loaded into
// its own ring in LDS, some tiles ahead.  It is read as the first operand of the
// matrix instruction (lane: row r, block g; the blocks of a row change places by bits
// of the row, so that 8 rows lie in different banks) and its place is loaded again at
// once.
// Chunks of a wave come in pairs, neighbours in k, loaded as 8 rows x 128 bytes, whole
// lines of memory; an odd last one as 16 rows x 64.
// The waves' sums over k meet in LDS.  The waves do not wait for each other there:
// sums of kSums tiles have room, a wave counts its arrival at a tile, and the wave
// whose turn it is adds a tile's sums up kLag tiles later.
// Few rows are bound by the weights' bytes: 2 rows x 4096 x 73728 in 31 us, 5.1 TB/s
// (met at a barrier every tile 50 us, loaded as 16 rows x 64 bytes 34).  More rows
// also by x, which every workgroup loads (64 rows, half of 6144 values: 3 us at 64
// bytes a cycle), the waves' sums and the parts that are joined: 64 rows x 6144 x
// 24576 in 31 + 5 us.  One token x 4096 x 4096 takes 6 us, latency.
// WORDS: the scales of a row's chunk are an aligned word (k a multiple of 128, the
// array 4-byte aligned), else single bytes, each a word in LDS.
constexpr int kLds = 160 * 1024 - 512;
template <int MT, int KC, bool WORDS>
struct Ring {
  static constexpr int kSums = MT == 1 ? 4 : 3, kLag = kSums > 2 ? kSums - 2 : 1;
  static constexpr int kSumBytes = kSums * kWaves * MT * 1024;
  static constexpr int kScaleLoads = WORDS ? (KC + 3) / 4 : KC;
  static constexpr int kLoads = KC + kScaleLoads;  // of a tile
  static constexpr int kTile = 1024 * KC + 256 * kScaleLoads;
  static constexpr int kFit = (kLds - kSumBytes) / (kWaves * kTile);
  static constexpr int T = kFit > 6 ? 6 : kFit;  // tiles on their way
  static_assert(T >= 1 && (T - 1) * kLoads < 64, "the wait's counter has 6 bits");
  static_assert(kWaves * kTile + kWaves * 4096 <= kLds, "a block of x has room behind slot 0");
};
constexpr int kDirectRows = 4;  // up to here x is loaded straight into registers
constexpr int64_t kMaxStride = 1 << 24;  // 64 rows so far apart have offsets of 32 bits

// Four neighbouring outputs of row m from column n on, times s.
__device__ __forceinline__ void put(const Linear4Args& a, int m, int n, v4f y, float s) {
  const int64_t at = m * a.ld_out + n;
  if (a.out_fp32) {
    float* to = (float*)a.out + at;
    if (n + 4 <= a.n && ((uintptr_t)to & 15) == 0) {
      *reinterpret_cast<v4f*>(to) = y * s;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.n) to[e] = y[e] * s;
    }
    return;
  }
  uint16_t* to = (uint16_t*)a.out + at;
  const v4bf v = {(__bf16)(y[0] * s), (__bf16)(y[1] * s), (__bf16)(y[2] * s), (__bf16)(y[3] * s)};
  if (n + 4 <= a.n && ((uintptr_t)to & 7) == 0) {
    *reinterpret_cast<v4bf*>(to) = v;
  } else {
    const uint2 bits = __builtin_bit_cast(uint2, v);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.n) to[e] = (uint16_t)((e < 2 ? bits.x : bits.y) >> (16 * (e & 1)));
  }
}

// What x holds.
enum Rows : int { kRowsBf16, kRowsFp8, kRowsGroups };

template <int MT, int KC, int X, bool WORDS>
__global__ __launch_bounds__(64 * kWaves, 2) void linear4_kernel(Linear4Args a, Cut cut, v4f* parts) {
  using R = Ring<MT, KC, WORDS>;
  constexpr bool GROUPS = X == kRowsGroups, FP8 = X != kRowsBf16;
  constexpr int PAIRED = KC / 2 * 2;  // chunks that come in pairs
  constexpr int T = R::T;
  constexpr int CHAINS = MT == 1 ? 4 : MT == 2 ? 2 : 1;  // sums that do not wait for each other
  __shared__ __attribute__((aligned(16))) uint8_t s_lds[kLds];
  __shared__ uint32_t s_arrived[R::kSums], s_added[R::kSums];
  __shared__ float s_row[16 * MT];  // the rows' scales: a load in the loop would wait for the weights on their way
  // slot 0 of all waves, the sums, the other slots
  constexpr int SUMS = kWaves * R::kTile;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int nw = kWaves / cut.kw, wk = w % cut.kw, wn = w / cut.kw;
  const int row0 = blockIdx.z * 16 * MT;
  auto chunk = [&](int c) {  // the wave's c-th
    return (int)blockIdx.y * cut.kw * KC + (c < PAIRED ? wk * PAIRED + c : cut.kw * PAIRED + wk);
  };
  const int blocks = a.k / kBlk;  // scales of a weight row

  // the tiles that do not divide go to the first workgroups
  const int each = cut.tiles / cut.groups, rest = cut.tiles % cut.groups, group = blockIdx.x;
  const int first = group * each + min(group, rest), last = first + each + (group < rest);
  const int steps = (last - first + nw - 1) / nw;
  if (threadIdx.x < R::kSums) s_arrived[threadIdx.x] = s_added[threadIdx.x] = 0;
  if (X == kRowsFp8 && threadIdx.x < 16 * MT) s_row[threadIdx.x] = a.x_scale[min(row0 + (int)threadIdx.x, a.rows - 1)];

  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_lds;
  auto slot_at = [&](int slot) { return (slot * kWaves + w) * R::kTile + (slot ? R::kSumBytes : 0); };
  // a load's bytes of a lane: row lane / 8 (or / 4), and one of the row's pieces
  const int row8 = lane >> 3, piece8 = (lane & 7) ^ row8, row4 = lane >> 2, piece4 = (lane & 3) ^ (row4 >> 1 & 3);
  auto load = [&](int i, int slot) {
    const int tile = min(first + i * nw + wn, cut.tiles - 1), most = a.n - 1 - 16 * tile;
    const int64_t at = (int64_t)16 * tile * blocks;
    const uint32_t to = lds + slot_at(slot);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const bool pair = c < PAIRED;  // c even: rows 0 .. 7 of both chunks, c odd: rows 8 .. 15
      const int row = min(pair ? row8 + 8 * (c & 1) : row4, most);
      const int block = min(4 * chunk(pair ? c & ~1 : c) + (pair ? piece8 : piece4), blocks - 1);
      load_lds16(a.codes + at * 16, (uint32_t)((row * blocks + block) * 16), to + 1024 * c);
    }
#pragma unroll
    for (int c = 0; c < R::kScaleLoads; ++c) {
      const int row = min(row4, most) * blocks;
      if constexpr (WORDS) {  // words of chunks 4 c ..
        int mine = chunk(4 * c);
#pragma unroll
        for (int e = 1; e < 4; ++e)
          if (4 * c + e < KC) mine = (lane & 3) == e ? chunk(4 * c + e) : mine;
        load_lds4(a.scales + at, (uint32_t)(row + min(4 * mine, blocks - 4)), to + 1024 * KC + 256 * c);
      } else {
        load_lds1(a.scales + at, (uint32_t)(row + min(4 * chunk(c) + (lane & 3), blocks - 1)), to + 1024 * KC + 256 * c);
      }
    }
  };
  // the wave's part of x: column m = lane & 15 of every product, 8 values from
  // 128 chunk(c) + 32 g + 8 u on in product (c, u)
  uint4 x[MT][KC][4];
  float xs[MT][KC];
  constexpr int E = FP8 ? 1 : 2;  // bytes of a value
  // Of few rows most lanes read the same bytes; of more every lane would read a line
  // of its own, 64 steps for 1 KB (64 rows of 6144: 11 us).  Those go through LDS,
  // four lanes a row's 64 bytes.
  const bool direct = a.rows <= kDirectRows || a.ld_x > kMaxStride || (((uintptr_t)a.x | (uintptr_t)(a.ld_x * E)) & 15) != 0;
  if (steps > 0) load(0, 0);
  if (direct) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) x[t][c][u] = uint4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int64_t m = row0 + 16 * t + r;
      if (m >= a.rows) continue;  // a load takes as long as its lanes are many
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int k = min(kChunk * chunk(c) + kBlk * g, a.k - kBlk) + 8 * u;
          if constexpr (FP8) {
            const Fp8x8 b = *reinterpret_cast<const Fp8x8*>((const uint8_t*)a.x + m * a.ld_x + k);
            x[t][c][u] = uint4{b.w[0], b.w[1], 0, 0};
          } else {
            const Bf8 b = *reinterpret_cast<const Bf8*>((const uint16_t*)a.x + m * a.ld_x + k);
            x[t][c][u] = uint4{b.w[0], b.w[1], b.w[2], b.w[3]};
          }
        }
    }
  } else {
    constexpr int BLOCKS = MT * KC;
    constexpr int PIECES = FP8 ? 2 : 4;  // loads of 16 rows x 64 bytes
    constexpr int AREA = (kLds - SUMS) / kWaves / 1024;  // of a wave, behind slot 0
    constexpr int DEPTH = AREA / PIECES < BLOCKS ? AREA / PIECES : BLOCKS;
    auto load_x = [&](int b) {
      const int m = min(row0 + 16 * (b / KC) + row4, a.rows - 1) - row0;
      const uint8_t* from = (const uint8_t*)a.x + (int64_t)row0 * a.ld_x * E;
      const uint32_t to = lds + SUMS + (w * AREA + b % DEPTH * PIECES) * 1024;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {  // 32 bf16 values, 64 fp8 values of a row
        const int kb = 4 * chunk(b % KC) + (FP8 ? 2 * p + (piece4 >> 1) : p);
        load_lds16(from, (uint32_t)(m * (int)(a.ld_x * E) + min(kb, blocks - 1) * kBlk * E + 16 * (FP8 ? piece4 & 1 : piece4)),
                   to + 1024 * p);
      }
    };
#pragma unroll
    for (int b = 0; b < DEPTH; ++b) load_x(b);
    const int swap = r >> 1 & 3;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      // of the loads those of the DEPTH - 1 blocks behind this one may be on their way
      if (b + DEPTH <= BLOCKS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * PIECES < 63 ? (DEPTH - 1) * PIECES : 63) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const uint8_t* from = s_lds + SUMS + (w * AREA + b % DEPTH * PIECES) * 1024 + 64 * r;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint4& to = x[b / KC][b % KC][u];
        if constexpr (FP8) {
          const uint2 v = *reinterpret_cast<const uint2*>(from + 1024 * (g >> 1) + ((2 * (g & 1) + (u >> 1)) ^ swap) * 16 + 8 * (u & 1));
          to = uint4{v.x, v.y, 0, 0};
        } else {
          to = *reinterpret_cast<const uint4*>(from + 1024 * g + (u ^ swap) * 16);
        }
      }
      if (b + DEPTH < BLOCKS) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // read before the place is loaded again
          uint4& v = x[b / KC][b % KC][u];
          asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)::"memory");
        }
        load_x(b + DEPTH);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // every wave has read its rows
  }
#pragma unroll
  for (int i = 1; i < T; ++i)
    if (i < steps) load(i, i);
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const bool in = 4 * chunk(c) + g < blocks;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if constexpr (FP8) x[t][c][u] = widen8(Fp8x8{{x[t][c][u].x, x[t][c][u].y}});
        if (!in) x[t][c][u] = uint4{0, 0, 0, 0};
      }
      if constexpr (GROUPS) {
        const int64_t m = min(row0 + 16 * t + r, a.rows - 1);
        const int n = (a.k + kChunk - 1) / kChunk;
        xs[t][c] = chunk(c) < n ? a.x_scale[m * n + chunk(c)] : 0.f;
      }
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // the counters are 0

  v4f* s_sum = reinterpret_cast<v4f*>(s_lds + SUMS);  // [kSums][wave][MT][lane]
  auto wait_for = [](const uint32_t* counter, uint32_t count) {
    while ((uint32_t)__builtin_amdgcn_readfirstlane((int)__hip_atomic_load(counter, __ATOMIC_RELAXED,
                                                                           __HIP_MEMORY_SCOPE_WORKGROUP)) < count)
      __builtin_amdgcn_s_sleep(1);
    asm volatile("" ::: "memory");
  };
  auto count = [&](uint32_t* counter) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (lane == 0) __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  };
  const int items = nw * MT;  // (n tile, m tile) of a step

  int slot = 0;
  for (int i = 0; i < steps + R::kLag; ++i) {
    if (i < steps) {
      // of the loads those of the T - 1 tiles behind this one may be on their way
      if (i + T <= steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((T - 1) * R::kLoads) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const uint8_t* tile = s_lds + slot_at(slot);
      uint4 code[KC];
      uint32_t byte[KC];
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c < PAIRED)
          code[c] = *reinterpret_cast<const uint4*>(tile + 1024 * ((c & ~1) + (r >> 3)) + 128 * (r & 7) + ((4 * (c & 1) + g) ^ (r & 7)) * 16);
        else
          code[c] = *reinterpret_cast<const uint4*>(tile + 1024 * c + (4 * r + (g ^ (r >> 1 & 3))) * 16);
        if constexpr (WORDS)
          byte[c] = *reinterpret_cast<const uint32_t*>(tile + 1024 * KC + 256 * (c / 4) + (4 * r + c % 4) * 4);
        else
          byte[c] = *reinterpret_cast<const uint32_t*>(tile + 1024 * KC + 256 * c + (4 * r + g) * 4);
      }
      // read before the place is loaded again
#pragma unroll
      for (int c = 0; c < KC; ++c)
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(code[c].x), "+v"(code[c].y), "+v"(code[c].z), "+v"(code[c].w), "+v"(byte[c])::"memory");
      if (i + T < steps) load(i + T, slot);
      slot = slot + 1 == T ? 0 : slot + 1;
      v4f sum[MT][CHAINS];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int q = 0; q < CHAINS; ++q) sum[t][q] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        uint32_t scale = WORDS ? byte[c] >> (8 * g) & 255u : byte[c];
        if (4 * chunk(c) + g >= blocks) {
          code[c] = uint4{0, 0, 0, 0};
          scale = 127;
        }
        const uint32_t words[4] = {code[c].x, code[c].y, code[c].z, code[c].w};
        v4f part[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) part[t] = GROUPS ? v4f{0.f, 0.f, 0.f, 0.f} : sum[t][c % CHAINS];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const v8bf wide = __builtin_bit_cast(v8bf, decode8(words[u], scale_operand(scale)));
#pragma unroll
          for (int t = 0; t < MT; ++t)
            part[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide, __builtin_bit_cast(v8bf, x[t][c][u]), part[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          if constexpr (GROUPS) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[t][c % CHAINS][e] = fmaf(part[t][e], xs[t][c], sum[t][c % CHAINS][e]);
          } else {
            sum[t][c % CHAINS] = part[t];
          }
        }
      }
      const int at = i % R::kSums;
      if (i >= R::kSums) wait_for(&s_added[at], (uint32_t)(i / R::kSums * items));  // the tile before here is put out
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int q = 1; q < CHAINS; ++q) sum[t][0] += sum[t][q];
        s_sum[((at * kWaves + w) * MT + t) * 64 + lane] = sum[t][0];
      }
      count(&s_arrived[at]);
    }
    const int done = i - R::kLag, at = done % R::kSums;
    if (done < 0) continue;
    for (int item = (w + done) % kWaves; item < items; item += kWaves) {
      wait_for(&s_arrived[at], (uint32_t)((done / R::kSums + 1) * kWaves));
      const int tn = item / MT, t = item % MT;
      const v4f* from = s_sum + ((at * kWaves + tn * cut.kw) * MT + t) * 64 + lane;
      v4f total = from[0];
      if (cut.kw == kWaves) {  // all read before the first is added
        v4f others[kWaves - 1];
#pragma unroll
        for (int j = 1; j < kWaves; ++j) others[j - 1] = from[j * MT * 64];
#pragma unroll
        for (int j = 1; j < kWaves; ++j) total += others[j - 1];
      } else {
        for (int j = 1; j < cut.kw; ++j) total += from[j * MT * 64];
      }
      count(&s_added[at]);
      const int tile = first + done * nw + tn;
      if (tile >= last) continue;
      if (parts) {  // the registers as they lie: the joining kernel has the same lanes
        parts[(((int64_t)blockIdx.y * gridDim.z + blockIdx.z) * MT + t) * cut.tiles * 64 + (int64_t)tile * 64 + lane] = total;
        continue;
      }
      const int m = row0 + 16 * t + r;
      if (m < a.rows) put(a, m, 16 * tile + 4 * g, total, X == kRowsFp8 ? s_row[16 * t + r] : 1.f);
    }
  }
}

// The sums of the workgroups that share k, in their order: a wave a tile of 16 rows x
// 16 weight rows (blockIdx.y: 16 rows).
__global__ __launch_bounds__(256) void linear4_join_kernel(Linear4Args a, int splits, int tiles, int64_t stride,
                                                           const v4f* parts) {
  const int lane = threadIdx.x & 63, tile = blockIdx.x * 4 + (threadIdx.x >> 6), m = 16 * blockIdx.y + (lane & 15);
  if (tile >= tiles) return;
  const v4f* from = parts + (int64_t)blockIdx.y * tiles * 64 + (int64_t)tile * 64 + lane;
  v4f y = from[0];
  for (int s = 1; s < splits; ++s) y += from[s * stride];
  if (m >= a.rows) return;
  put(a, m, 16 * tile + 4 * (lane >> 4), y, a.x_fp8 && a.group == 0 ? a.x_scale[m] : 1.f);
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

// As few workgroups share k as have registers for its part of x (a part more costs 8
// bytes a sum, written and read): 26 rows x 5024 x 8203 take 14 + 4 us in two parts
// and 15 in one.  Then one workgroup a CU, which has the LDS to itself.
Plan plan_of(const Linear4Args& a) {
  Plan p{};
  p.mt = a.rows <= 16 ? 1 : a.rows <= 32 ? 2 : 4;
  const int most = p.mt == 1 ? 8 : p.mt == 2 ? 5 : a.group ? 2 : 3;  // chunks of k whose x a wave has registers for
  const int chunks = (a.k + kChunk - 1) / kChunk;
  p.cut.splits = (chunks + kWaves * most - 1) / (kWaves * most);
  const int mine = (chunks + p.cut.splits - 1) / p.cut.splits;  // of a workgroup
  p.kc = (mine + kWaves - 1) / kWaves;
  const int waves = (mine + p.kc - 1) / p.kc;
  p.cut.kw = waves > 4 ? 8 : waves > 2 ? 4 : waves;
  p.cut.tiles = (a.n + 15) / 16;
  const int nw = kWaves / p.cut.kw;
  const int rows = (a.rows + 16 * p.mt - 1) / (16 * p.mt);
  p.cut.groups = std::max(1, std::min((p.cut.tiles + nw - 1) / nw, kCus / (p.cut.splits * rows)));
  return p;
}

// Sums of a workgroup's part of k, four a lane.
int64_t part_of(const Linear4Args& a, const Plan& p) {
  const int64_t blocks = (a.rows + 16 * p.mt - 1) / (16 * p.mt);
  return blocks * p.mt * p.cut.tiles * 64;
}

template <int MT, int KC, int X>
void launch_words(const Linear4Args& a, const Plan& p, v4f* parts, hipStream_t stream) {
  const dim3 grid((unsigned)p.cut.groups, (unsigned)p.cut.splits, (unsigned)((a.rows + 16 * MT - 1) / (16 * MT)));
  if (a.k % kChunk == 0 && ((uintptr_t)a.scales & 3) == 0)
    hipLaunchKernelGGL((linear4_kernel<MT, KC, X, true>), grid, dim3(64 * kWaves), 0, stream, a, p.cut, parts);
  else
    hipLaunchKernelGGL((linear4_kernel<MT, KC, X, false>), grid, dim3(64 * kWaves), 0, stream, a, p.cut, parts);
}
template <int MT, int KC>
void launch(const Linear4Args& a, const Plan& p, v4f* parts, hipStream_t stream) {
  if (!a.x_fp8) launch_words<MT, KC, kRowsBf16>(a, p, parts, stream);
  else if (!a.group) launch_words<MT, KC, kRowsFp8>(a, p, parts, stream);
  else if constexpr (MT * KC <= 10) launch_words<MT, KC, kRowsGroups>(a, p, parts, stream);
}

}  // namespace

size_t linear4_workspace(const Linear4Args& a) {
  const Plan p = plan_of(a);
  return p.cut.splits > 1 ? (size_t)p.cut.splits * part_of(a, p) * sizeof(v4f) : 0;
}

hipError_t launch_linear4(const Linear4Args& a, void* workspace, hipStream_t stream) {
  const Plan p = plan_of(a);
  v4f* parts = p.cut.splits > 1 ? (v4f*)workspace : nullptr;
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
    case 25: launch<2, 5>(a, p, parts, stream); break;
    case 41: launch<4, 1>(a, p, parts, stream); break;
    case 42: launch<4, 2>(a, p, parts, stream); break;
    default: launch<4, 3>(a, p, parts, stream); break;
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !parts) return e;
  hipLaunchKernelGGL(linear4_join_kernel, dim3((unsigned)((p.cut.tiles + 3) / 4), (unsigned)((a.rows + 15) / 16)), dim3(256),
                     0, stream, a, p.cut.splits, p.cut.tiles, part_of(a, p), parts);
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
