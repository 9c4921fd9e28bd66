// Attention in the MQA form of latent attention, over the 4-bit cache.
//
//   z[r, h, s] = scale * q[r, h] . (latent[s], rope[s])     s in the row's set, or s <= its position
//   o[r, h]    = sum_s softmax(z)[s] latent[s],   lse = log sum_s exp(z)
//   acc[b, s] += sum_{r, h} softmax(z[r, h])[s]             optional
//
// A row with no key (an empty set, or only scores of -infinity) has o = 0 and
// lse = -infinity and adds nothing to acc.  Rows that are a tree of drafted tokens
// attend to the positions before the tree's first, and to those of its nodes that
// their masks name.
//
// Scores are kept in base 2 (z log2 e), statistics and sums in fp32.
#include <algorithm>
#include <type_traits>
#include <utility>

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

typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

#define LDS(type, p) ((__attribute__((address_space(3))) type*)(p))

// Sixteen (or four) bytes of every lane from memory into LDS at byte address dst
// + 16 (4) * lane, dst the same in all lanes of the wave.  Written out, because
// the compiler waits for all such loads before any read of LDS that it cannot
// tell apart from their target; the tile loop waits for them itself, before the
// barrier that hands the tile over.
__device__ __forceinline__ void load_lds16(const void* src, uint32_t dst) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(dst), "v"(src) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* src, uint32_t dst) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" ::"{m0}"(dst), "v"(src) : "memory");
}

// f(0), f(1), ..., f(N - 1) with the index a constant
template <class F, int... I>
__device__ __forceinline__ void unroll(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unroll(F&& f) {
  unroll(f, std::make_integer_sequence<int, N>{});
}
// Pieces [0, PIECES) of other work, spread over the steps of a loop of STEPS:
// those that belong after step S.
template <int STEPS, int PIECES, int S, class F>
__device__ __forceinline__ void pieces_after(F&& piece) {
  constexpr int lo = S * PIECES / STEPS, hi = (S + 1) * PIECES / STEPS;
  unroll<hi - lo>([&](auto i) { piece(std::integral_constant<int, lo + i>{}); });
}

// The largest / the sum of a value over the four lane groups of 16 lanes.
__device__ __forceinline__ float groups_max(float x) {
  auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(e[0]), __uint_as_float(e[1]));
  e = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(e[0]), __uint_as_float(e[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(e[0]) + __uint_as_float(e[1]);
  e = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(e[0]) + __uint_as_float(e[1]);
}

// A reduction over groups of LANES consecutive lanes, the result in all of them.
template <int LANES, class Op>
__device__ __forceinline__ float row_reduce(float x, Op op) {
  x = op(x, lane_xor1(x));
  x = op(x, lane_xor2(x));
  x = op(x, lane_xor4(x));
  if constexpr (LANES >= 16) x = op(x, lane_xor8(x));
  if constexpr (LANES == 32) {
    const auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(e[0]), __uint_as_float(e[1]));
  }
  return x;
}

// Two bf16 values, 0 for those that are infinite or NaN.
__device__ __forceinline__ uint32_t finite(uint32_t v) {
  if ((v & 0x7F80u) == 0x7F80u) v &= 0xFFFF0000u;
  if ((v & 0x7F800000u) == 0x7F800000u) v &= 0xFFFFu;
  return v;
}

// LDS.  As loaded, 1024 bytes of one wave's load (4 keys' codes, 8 keys' position
// values) are a group, the groups 1088 bytes apart; the 16-byte chunks of a row
// change places by two bits of the key.  Together the two put one chunk of 16
// keys, which a score operand reads at once, into 16 different bank groups.
constexpr int kGroup = 1024 + 64;
constexpr int kCodesBytes = kTileKeys / 4 * kGroup, kRopeBytes = kTileKeys / 8 * kGroup;
constexpr int kScalesBytes = kTileKeys / 8 * 256;  // 8 keys' scales twice, as 64 lanes load them
// The widened latent values are rows of 64 chunks of 8 values, chunk c of key k
// at c ^ swizzle(k): 4 neighbouring chunks of keys 4 n .. 4 n + 3, which a
// transposed read takes, lie in different banks.
constexpr int kValueBytes = kTileKeys * 2 * kLatent;
__device__ __forceinline__ int swizzle(int key) { return (key & 3) << 2 | (key >> 2 & 3); }
// Weights: rows of 32 high parts, then 32 low parts.
constexpr int kWeightStride = 4 * kTileKeys + 16;
constexpr int kQueryStride = 2 * kRope + 64 + 16;
constexpr int kWaves = 8;

// What one launch's workgroups are: for every unit (query row of an index-set call,
// else sequence) tiles of 16 RG rows x splits of the unit's keys.  Units of an
// index-set call are alike; a sequence has as many splits as its length asks for,
// and its workgroups follow those of the sequence before it (first).
struct Work {
  int units, tiles_per_split;
  int row_tiles, splits;  // of a unit, for sequences the most
  int32_t first[kMaxSeq + 1];
  float4* part_o;
  float2* part_ml;  // reference, sum
};

// How the output lies in the waves' registers.  RG = 8: 64 rows x 128 values a
// wave, else all rows x 64 values (tiles of values x rows: 32 x 32, for RG = 1
// 16 x 16): of the shapes with as many registers the ones with the least reads of
// weights and values.
template <int RG>
struct Output {
  static constexpr int XT = RG == 8 || RG == 1 ? 4 : 2;  // tiles of values
  static constexpr int YT = RG >= 4 ? 2 : 1;             // tiles of rows
  static constexpr int QUADS = RG == 1 ? XT : 4 * XT * YT;  // registers / 4, (y XT + x) 4 + i
  __device__ static __forceinline__ int row(int w, int lane, int y) {
    return RG == 1 ? lane & 15 : (RG == 8 ? 64 * (w >> 2) : 0) + 32 * y + (lane & 31);
  }
  // the first of four values
  __device__ static __forceinline__ int value(int w, int lane, int x, int i) {
    return RG == 1 ? 64 * w + 16 * x + 4 * (lane >> 4)
                   : (RG == 8 ? 128 * (w & 3) : 64 * w) + 32 * x + 8 * i + 4 * (lane >> 5);
  }
};

// A workgroup of 8 waves attends 16 RG rows (heads of one query; in a prefix call
// heads of consecutive queries of a sequence) to one split of their keys, 32 at
// a time, in four stages:
//   load    the tile's rows into LDS, a tile ahead;
//   score   transposed, keys x rows, the codes widened to bf16 in registers
//           (exact: a code has two significant bits); a lane has 4 keys of a row,
//           so maxima and sums need two lane swaps.  The reference m of a row only
//           moves when a score passes it by more than 32 (weights, sums and output
//           have fp32's range, so none comes near its end), and the output is
//           hardly ever rescaled.  A weight goes to LDS as two bf16, 16 bits of
//           it: one bf16 would round it by up to 2^-8, as much as the output's own
//           rounding, and fp16 would lose the small ones;
//   widen   codes to bf16 in LDS, 4 keys a wave;
//   output  transposed, values x rows, the values read transposed from LDS.
// RG = 8: a wave scores its 16 rows against all 32 keys; the stages of an
// iteration (output of tile i; score and widen of i + 1; load of i + 2) need
// nothing of each other, so one barrier per tile is enough, and the two waves of
// a SIMD take them in different orders: one widens codes for its scores while the
// other's output keeps the matrix core busy.  Operands are read from LDS some
// steps ahead, and the vector work of other stages is cut into pieces issued
// between the output's matrix products, which run on their own once issued;
// scheduling barriers keep the two from being sorted apart.  Bound by vector
// instructions (the codes' conversion at half rate, 4460 of 7900 cycles a tile:
// every wave converts all 32 keys for its own rows, and the tile is widened once
// more into LDS) next to 3200 cycles of matrix products: 1003 queries x 128 heads x
// 2048 keys in 814 us, 703 TFLOP/s.
// RG <= 4: 16 rows' products with 16 keys are shared by 4 / RG waves, so that all
// 8 have some; their parts go through LDS, and a tile takes an iteration more: the
// load of tile i + 2 + AHEAD, the products of i + 2, the weights and the widening
// of i + 1, the output of i, again with one barrier.  All operands are read from
// LDS first, then used.  With RG = 1 a tile takes 3200 cycles, a third of them
// reads of LDS: 8 sequences of 9001 to 40000 keys x 16 heads in 43 us, 1.8 TB/s.
// The sequence that workgroup i belongs to: the last one with first <= i (one
// without workgroups shares its first with the next).
__device__ __forceinline__ int owner_of(const int32_t* first, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// splits of a sequence's keys
__host__ __device__ inline int splits_of(const RunTable& t, int b, int tiles_per_split) {
  const int tiles = (t.n_k[b] + kTileKeys - 1) / kTileKeys;
  return tiles > tiles_per_split ? (tiles + tiles_per_split - 1) / tiles_per_split : 1;
}

// What a kernel is compiled for: causal calls of both kinds, trees over the prefix,
// trees over index sets.  At 128 rows both kernels of trees spill three registers, one
// of which every tile reloads (the causal one spills none); one kernel for both kinds
// spills as many, and takes 2 to 4% longer (64 nodes x 128 heads x 131072 keys 3.27
// instead of 3.16 ms).
enum Call : int { kCausal, kTreePrefix, kTreeSets };
struct NoTree {};
template <bool TREE>
using TreeOf = std::conditional_t<TREE, TreeMask, NoTree>;

template <int RG, int CALL>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_kernel(AttendArgs a, RunTable t, ScoreMap sm, Work wk,
                                                                TreeOf<CALL != kCausal> tree) {
  constexpr bool TREE = CALL != kCausal;
  constexpr bool ONE = RG == 8;                // one barrier per tile
  constexpr int ROWS = 16 * RG;
  constexpr int KT = kTileKeys;
  constexpr int NKT = ONE ? 2 : 1;             // key tiles of 16 per wave
  constexpr int DG = ONE ? 1 : 4 / RG;         // waves that share 16 rows' products with 16 keys
  constexpr int TT = 4 / DG;                   // a wave's part of them: blocks of 128 latent values
  constexpr int KPT = ONE ? 1 : RG, LPR = kTileKeys / KPT;  // a thread's scores of a tile, threads of a row
  using O = Output<RG>;
  constexpr int AHEAD = ONE ? 1 : RG == 1 ? 3 : 2;  // tiles in flight; RG <= 4: as many as LDS has room for
  constexpr int NS = AHEAD + (ONE ? 1 : 2);    // tiles' codes held
  constexpr int WB = ROWS * kWeightStride;
  __shared__ __attribute__((aligned(16))) uint8_t s_val[2 * kValueBytes];
  __shared__ __attribute__((aligned(16))) uint8_t s_codes[NS * kCodesBytes];
  __shared__ __attribute__((aligned(16))) uint8_t s_rope[NS * kRopeBytes];
  __shared__ __attribute__((aligned(16))) uint8_t s_scale[NS * kScalesBytes];
  __shared__ __attribute__((aligned(16))) int s_pos[NS * KT];
  __shared__ __attribute__((aligned(16))) uint8_t s_w[2 * WB];
  // the part of the queries that finds no register: the position values and the
  // last 32 latent ones
  __shared__ __attribute__((aligned(16))) uint8_t s_qr[ONE ? ROWS * kQueryStride : 16];
  // partial scores of two tiles
  constexpr int PR = kTileKeys + 4;  // words from one row to the next
  __shared__ __attribute__((aligned(16))) float s_part[ONE ? 4 : 2 * DG * ROWS * PR];
  __shared__ int s_entry[ONE ? 1 : 4 * 64], s_page[ONE ? 1 : 4 * 64];  // of 8 tiles' keys, on their way
  __shared__ float s_alpha[2][ROWS], s_max[ROWS], s_sum[ROWS];
  // of a tree: the word that a row's mask starts at (prefix calls), the mask of the
  // unit's query (index sets), the masks and their words; here, and not in registers,
  // because few tiles need them (masks held in registers cost the tile loop 20%)
  __shared__ int s_tree[TREE ? ROWS : 1];
  __shared__ uint32_t s_mask[TREE ? kTreeWords : 1];
  __shared__ const uint32_t* s_bits;
  __shared__ int s_words;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool sets = CALL == kCausal ? a.idx != nullptr : CALL == kTreeSets;
  const int part = blockIdx.x;
  const int unit = sets ? part / (wk.row_tiles * wk.splits) : owner_of(wk.first, t.n, part);
  const int b = sets ? run_of(t, unit) : unit;
  const int unit_rows = sets ? a.heads : t.n_rows[b] * a.heads;
  const int row_tiles = (unit_rows + ROWS - 1) / ROWS;
  const int splits = sets ? wk.splits : splits_of(t, b, wk.tiles_per_split);
  const int in_unit = part - (sets ? unit * row_tiles * splits : wk.first[b]);
  const int split = in_unit % splits, rt = row_tiles - 1 - in_unit / splits;  // the rows with the most keys first
  const int first = rt * ROWS;
  const int rows = min(ROWS, unit_rows - first);
  const int i_first = sets ? unit - t.row0[b] : 0;                       // the unit's first query in its sequence
  const int pos_last = TREE ? t.n_k[b] - 1 : t.pos0[b] + (sets ? i_first : (first + rows - 1) / a.heads);
  // kept scores cover the unit's keys for every row
  const int n = sets ? a.topk : sm.s2 ? t.n_k[b] : pos_last + 1;
  const int all_tiles = (n + KT - 1) / KT;
  const int t0 = split * wk.tiles_per_split, t1 = min(all_tiles, t0 + wk.tiles_per_split);
  if (t0 >= t1 && splits > 1) {
    if (tid < ROWS) wk.part_ml[(int64_t)part * ROWS + tid] = {-INFINITY, 0.f};
    return;
  }

  const int kt = ONE ? 0 : w / RG & 1;         // the wave's (first) 16 keys of a tile,
  const int row0 = ONE ? 16 * w : 16 * (w % RG);  // its rows of scores,
  const int dg = ONE ? 0 : w / (2 * RG);       // and its part of the products

  // Keys 8 (w mod 4) + (lane & 7) of a tile, found in three steps, so that no step
  // waits for its load: the set's entry; the page of its position; the cache row.
  // Waves 0 .. 3 load position values and scales of these keys, waves 4 .. 7 their
  // codes.
  // RG = 8: a step a tile.  Both loads are made in every call (where there is no set or no page table, of
  // any readable word): a choice between a load's result and another value would
  // be made, and waited for, where the load is.
  const bool paged = a.map.pages != nullptr;
  const int32_t* any_word = reinterpret_cast<const int32_t*>(a.cache.codes);
  const int32_t* idx = sets ? a.idx + (int64_t)unit * a.topk : any_word;
  const int32_t* pages = paged ? a.map.pages + (int64_t)b * a.map.max_pages : any_word;
  const int w4 = w & 3;
  const bool code_wave = w >= 4;
  auto fetch = [&](int ln, int tile) {
    const int k = min(tile * KT + 8 * w4 + (ln & 7), n - 1);
    return idx[sets ? k : 0];
  };
  // of key (ln & 7) of the tile with set entry `entry`: pos: the position whose
  // row is loaded (0 for keys that do not count), at: the one that masks the key
  auto place = [&](int ln, int tile, int entry, int& pos, int& at) {
    const int k = tile * KT + 8 * w4 + (ln & 7);
    entry = sets ? entry : k;
    const bool ok = ((uint32_t)entry <= (uint32_t)pos_last) & (tile < t1) & (k < n);
    pos = ok ? entry : 0;
    at = ok ? entry : 0x7FFFFFFF;
    return pages[paged ? pos >> a.map.shift : 0];
  };
  auto locate = [&](int pos, int page) -> int {
    if (!paged) return (int)(b * a.map.stride) + pos;
    return (min(max(page, 0), a.map.n_pages - 1) << a.map.shift) | (pos & ((1 << a.map.shift) - 1));
  };
  const uint32_t codes0 = (uint32_t)(uintptr_t)LDS(uint8_t, s_codes), rope0 = (uint32_t)(uintptr_t)LDS(uint8_t, s_rope),
                 scale0 = (uint32_t)(uintptr_t)LDS(uint8_t, s_scale);
  int at = 0, pos = 0, page = 0, entry = 0;  // of the next tile to be loaded; the entry of the one after
  int row1 = 0, row2 = 0, row_at = 0;  // the rows of the lane's two loads; the masking position
  auto load_piece = [&](int ln, int tile, int slot, auto piece) {
    constexpr int P = piece;
    if constexpr (P == 0) {
      const int row = locate(pos, page);
      row_at = at;
      row1 = __shfl(row, ln >> (code_wave ? 4 : 3), 64);
      row2 = __shfl(row, code_wave ? 4 + (ln >> 4) : ln >> 2 & 7, 64);
    } else if constexpr (P == 1) {  // before this tile's loads, so that it does not wait for them
      page = place(ln, tile + 1, entry, pos, at);
    } else if constexpr (P == 2) {
      entry = fetch(ln, tile + 2);
    } else if constexpr (P == 3) {  // 8 keys' position values, or 4 keys' codes
      const int key = ln >> (code_wave ? 4 : 3);
      const int64_t r = row1;
      const uint8_t* base = code_wave ? a.cache.codes : reinterpret_cast<const uint8_t*>(a.cache.rope);
      const int chunk = code_wave ? (ln & 15) ^ key : (ln & 7) ^ (key >> 1);
      load_lds16(base + (r << (code_wave ? 8 : 7)) + (chunk << 4),
                 code_wave ? codes0 + slot * kCodesBytes + 2 * w4 * kGroup : rope0 + slot * kRopeBytes + w4 * kGroup);
    } else {
      if (code_wave) {
        const int key = ln >> 4;
        const int64_t r = row2;
        load_lds16(a.cache.codes + r * kCodeBytes + (((ln & 15) ^ key) << 4),
                   codes0 + slot * kCodesBytes + (2 * w4 + 1) * kGroup);
      } else {
        const int64_t r = row2;
        load_lds4(a.cache.scales + r * kScaleBytes + 4 * (ln & 3), scale0 + slot * kScalesBytes + w4 * 256);
        s_pos[slot * KT + 8 * w4 + (ln & 7)] = row_at;
      }
    }
  };
  constexpr int LOADS = 5;
  // RG <= 4: a step for the keys of 8 tiles, one a lane; waves 0 .. 3 load entries
  // and pages into LDS, so that the only loads in the loop are those that the
  // counts in meet() know.
  int row_of = 0, at_of = 0;  // of the 8 tiles that are loaded
  auto fetch8 = [&](int tile) {  // where the lane's entry of the 8 tiles from this one is
    const int k = min((tile + (lane >> 3)) * KT + 8 * w4 + (lane & 7), n - 1);
    return idx + (sets ? k : 0);
  };
  auto place8 = [&](int tile, int e) {  // pos and at of the 8 tiles from this one
    const int k = (tile + (lane >> 3)) * KT + 8 * w4 + (lane & 7);
    e = sets ? e : k;
    const bool ok = ((uint32_t)e <= (uint32_t)pos_last) & (tile + (lane >> 3) < t1) & (k < n);
    pos = ok ? e : 0;
    at = ok ? e : 0x7FFFFFFF;
  };
  auto page8 = [&] { return pages + (paged ? pos >> a.map.shift : 0); };
  int key_row1 = 0, key_row2 = 0, key_pos = 0;  // the rows of the lane's two loads; the masking position
  auto rows_of = [&](int ln, int i) {           // of tile t0 + i, one of the 8
    key_row1 = __shfl(row_of, 8 * (i & 7) + (ln >> (code_wave ? 4 : 3)), 64);
    key_row2 = __shfl(row_of, 8 * (i & 7) + (code_wave ? 4 + (ln >> 4) : ln >> 2 & 7), 64);
    key_pos = __shfl(at_of, 8 * (i & 7) + (ln & 7), 64);
  };
  auto next_rows = [&](int ln, int i) {  // the same, after steps that are due
    if ((i & 7) == 0) {
      row_of = locate(pos, s_page[64 * w4 + ln]);
      at_of = at;
      place8(t0 + i + 8, s_entry[64 * w4 + ln]);
    } else if ((i & 7) == 1 && !code_wave) {  // every wave has read the ones before
      load_lds4(page8(), (uint32_t)(uintptr_t)LDS(int, s_page) + 256 * w4);
      load_lds4(fetch8(t0 + i - 1 + 16), (uint32_t)(uintptr_t)LDS(int, s_entry) + 256 * w4);
    }
    rows_of(ln, i);
  };
  auto load_rows = [&](int ln, int slot) {
    const int64_t r1 = key_row1, r2 = key_row2;
    if (code_wave) {
      const int key = ln >> 4, chunk = (ln & 15) ^ key;
      load_lds16(a.cache.codes + r1 * kCodeBytes + (chunk << 4), codes0 + slot * kCodesBytes + 2 * w4 * kGroup);
      load_lds16(a.cache.codes + r2 * kCodeBytes + (chunk << 4), codes0 + slot * kCodesBytes + (2 * w4 + 1) * kGroup);
    } else {
      const int key = ln >> 3, chunk = (ln & 7) ^ (key >> 1);
      load_lds16(reinterpret_cast<const uint8_t*>(a.cache.rope) + r1 * 2 * kRope + (chunk << 4),
                 rope0 + slot * kRopeBytes + w4 * kGroup);
      load_lds4(a.cache.scales + r2 * kScaleBytes + 4 * (ln & 3), scale0 + slot * kScalesBytes + w4 * 256);
      s_pos[slot * KT + 8 * w4 + (ln & 7)] = key_pos;
    }
  };

  const float c = a.scale * kLog2e;
  // The wave's query rows as the second operand of the score products: lane (row
  // r, group g) has values 8 u .. + 7 of block 4 g + t in product 4 t + u, then
  // 8 g .. + 7 of each 32 position values.
  constexpr int QK = ONE ? kLatent / 32 - 1 : 4 * TT;  // latent products whose query part stays in registers
  constexpr int QR = ONE ? 0 : DG == 1 ? 2 : 1;        // and those of position values
  v4i q[QK + QR];
  // the last position that a row of scores attends to (RG = 8: the lane's, else the
  // thread's); rows past the last one take its query, masked
  int limit;
  {
    const int mine = row0 + (lane & 15), flat = first + min(mine, rows - 1), g = lane >> 4;
    const int i = sets ? 0 : flat / a.heads, head = flat - i * a.heads;
    if constexpr (TREE) {  // the last position before the tree, for padded rows too
      limit = tree.base[b] - 1;
      const int r = min(tid, rows - 1);
      if (tid < ROWS) s_tree[tid] = (t.row0[b] + i_first + (sets ? 0 : (first + r) / a.heads)) * tree.words;
      if (sets && tid < tree.words) s_mask[tid] = tree.bits[(int64_t)(t.row0[b] + i_first) * tree.words + tid];
      if (tid == 0) {
        s_bits = tree.bits;
        s_words = tree.words;
      }
      asm volatile("" : "+v"(limit));  // kept as it is, not as the base
    } else if constexpr (ONE) {
      limit = mine < rows ? t.pos0[b] + i_first + i : -1;
    } else {
      const int r = tid / LPR;
      limit = r < rows ? t.pos0[b] + i_first + (sets ? 0 : (first + r) / a.heads) : -1;
    }
    const uint16_t* from = a.q + ((int64_t)t.row0[b] + i_first + i) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
    for (int k = 0; k < 4 * TT; ++k) {
      const v4i v = *reinterpret_cast<const v4i*>(from + 32 * (4 * g + TT * dg + k / 4) + 8 * (k % 4));
      if (k < QK) q[k] = v;
      else *reinterpret_cast<v4i*>(s_qr + mine * kQueryStride + 2 * kRope + 16 * g) = v;  // its own wave's
    }
    if constexpr (ONE) {
#pragma unroll
      for (int k = 0; k < kRope / 32; ++k)
        *reinterpret_cast<v4i*>(s_qr + mine * kQueryStride + 64 * k + 16 * g) =
            *reinterpret_cast<const v4i*>(from + kLatent + 32 * k + 8 * g);
    } else {
#pragma unroll
      for (int k = 0; k < QR; ++k)
        q[QK + k] = DG == 4 && dg >= 2 ? v4i{0, 0, 0, 0} : *reinterpret_cast<const v4i*>(from + kLatent + 32 * (QR == 2 ? k : dg & 1) + 8 * g);
    }
  }
  float m = -INFINITY, l = 0.f;
  v16f o[O::XT][O::YT];
  v4f o1[4];
#pragma unroll
  for (int x = 0; x < O::XT; ++x)
#pragma unroll
    for (int y = 0; y < O::YT; ++y)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[x][y][i] = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) o1[x] = v4f{0.f, 0.f, 0.f, 0.f};
  float* s2 = nullptr;  // the workgroup's rows in the unit's first tile of kept scores
  if (sm.s2) {
    const int64_t padded = (a.topk + KT - 1) / KT * KT;
    s2 = sm.s2 + (sets ? (int64_t)unit * unit_rows * padded : sm.base[b]) + (int64_t)first * KT;
  }

  // ---- the other stages
  // 8 values a lane of the wave's j-th key, widened
  auto put_values = [&](int ln, int j, int vslot, uint32_t word, int byte) {
    *reinterpret_cast<uint4*>(s_val + vslot * kValueBytes + (4 * w + j) * 2 * kLatent +
                              (16 * ln ^ (swizzle(4 * w + j) << 4))) = decode8(word, scale_operand(byte));
  };
  // one of the wave's 4 keys: read, then widened
  uint32_t word[2];
  int byte[2];
  auto widen_piece = [&](int ln, int slot, int vslot, auto piece) {
    constexpr int j = piece / 2;
    if constexpr (piece % 2 == 0) {
      word[j & 1] = *reinterpret_cast<const uint32_t*>(s_codes + slot * kCodesBytes + w * kGroup + ((4 * ln) ^ (j << 4)) +
                                                       j * kCodeBytes);
      byte[j & 1] = s_scale[slot * kScalesBytes + (w >> 1) * 256 + (4 * (w & 1) + j) * kScaleBytes + (ln >> 2)];
    } else {
      put_values(ln, j, vslot, word[j & 1], byte[j & 1]);
    }
  };
  constexpr int WIDENS = 8;
  // The wave's 4 keys once widened: a NaN or an infinity (byte 255; 2^128 and more,
  // which bytes from 253 on can give) makes the key's scores NaN or infinite, its
  // weight NaN or 0; as a value it must not reach the rows that do not attend to
  // the key (0 * NaN), so 0 stands for it.
  auto drop_infinite = [&](int ln, int slot, int vslot) {
    if (!__any(s_scale[slot * kScalesBytes + (w >> 1) * 256 + (w & 1) * 64 + ln] >= 253)) return;
#pragma unroll 1
    for (int j = 0; j < 16; ++j) {
      uint32_t& v = *reinterpret_cast<uint32_t*>(s_val + vslot * kValueBytes + 4 * w * 2 * kLatent + 256 * j + 4 * ln);
      v = finite(v);
    }
  };

  // scores of the wave's rows and keys, operands read ahead
  v4f s[NKT];
  auto score = [&](int ln, int slot) {
    constexpr int STEPS = 4 * 4 * NKT;  // products; those of the key tiles take turns, so that none waits for the one before
    const int key = ln & 15, g = ln >> 4;
    const uint8_t* codes = s_codes + slot * kCodesBytes;
    const uint32_t at0 = (uint32_t)((key >> 2) * kGroup + (key & 3) * kCodeBytes + 64 * g + ((key & 3) << 4));
    const uint8_t* rope = s_rope + slot * kRopeBytes + (key >> 3) * kGroup + (key & 7) * 2 * kRope +
                          ((g ^ ((key >> 1) & 3)) << 4);
    const uint8_t* scale = s_scale + slot * kScalesBytes + (key >> 3) * 256 + (key & 7) * kScaleBytes + 4 * g;
    v4i x[4][NKT];  // [128 values][key tile]
    uint32_t sk[NKT];
    auto read = [&](auto tt) {
#pragma unroll
      for (int j = 0; j < NKT; ++j) x[tt][j] = *reinterpret_cast<const v4i*>(codes + (at0 ^ (tt << 4)) + 4 * j * kGroup);
    };
#pragma unroll
    for (int j = 0; j < NKT; ++j) sk[j] = *reinterpret_cast<const uint32_t*>(scale + 2 * j * 256);
    read(std::integral_constant<int, 0>{});
    // the position part first: its operands need not share the registers with the others'
    {
      v4i xr[NKT][2], qr[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int j = 0; j < NKT; ++j) xr[j][k] = *reinterpret_cast<const v4i*>(rope + 2 * j * kGroup + 64 * k);
        qr[k] = *reinterpret_cast<const v4i*>(s_qr + (row0 + key) * kQueryStride + 64 * k + 16 * g);
      }
#pragma unroll
      for (int j = 0; j < NKT; ++j) s[j] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < NKT; ++j)
          s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, xr[j][k]),
                                                         __builtin_bit_cast(v8bf, qr[k]), s[j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    v8bf wide[2];  // the widened operand of this product and of the next
    auto widen = [&](auto v) {
      constexpr int tt = v / (4 * NKT), u = v / NKT % 4, j = v % NKT;
      wide[v & 1] = __builtin_bit_cast(v8bf, decode8((uint32_t)x[tt][j][u], scale_operand(sk[j] >> (8 * tt) & 255u)));
    };
    widen(std::integral_constant<int, 0>{});
    v4i last;
    unroll<STEPS>([&](auto v) {
      constexpr int tt = v / (4 * NKT), u = v / NKT % 4, j = v % NKT;
      if constexpr (v % (4 * NKT) == 0 && tt + 1 < 4) read(std::integral_constant<int, tt + 1>{});
      if constexpr (v == 3 * 4 * NKT)
        last = *reinterpret_cast<const v4i*>(s_qr + (row0 + key) * kQueryStride + 2 * kRope + 16 * g);
      if constexpr (v + 1 < STEPS) widen(std::integral_constant<int, v + 1>{});
      const v4i qu = 4 * tt + u < QK ? q[4 * tt + u < QK ? 4 * tt + u : 0] : last;
      s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[v & 1], __builtin_bit_cast(v8bf, qu), s[j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // Of the keys at s_pos[first + 16 (e / 4) + e % 4], e < n, the nodes of the tree that
  // a row's mask names, as bits (padded rows share the last row's mask: nothing of
  // theirs is put out).  A loop that is not unrolled: few tiles need it, and no
  // registers are left around it.
  auto named = [&](int row, int first_key, int n_keys) {
    uint32_t bits = 0;
    if constexpr (TREE) {
#pragma unroll 1
      for (int e = 0; e < n_keys; ++e) {
        const int node = s_pos[first_key + 16 * (e >> 2) + (e & 3)] - limit - 1;
        if ((uint32_t)node < (uint32_t)(32 * s_words)) {
          const uint32_t word = sets ? s_mask[node >> 5] : s_bits[s_tree[row] + (node >> 5)];
          bits |= (word >> (node & 31) & 1u) << e;
        }
      }
    }
    return bits;
  };

  // the scores in base 2, masked, and the row's largest; tile: the unit's tile, for the kept scores
  float top = 0.f;
  auto finish_scores = [&](int ln, int tile, int slot) {
    const int key = ln & 15, g = ln >> 4;
    top = -INFINITY;
    uint32_t seen = 0;  // nodes of a tree
    if constexpr (TREE) {
      bool drafts = tile * KT + KT - 1 > limit;
      if (sets) {
        drafts = false;
#pragma unroll
        for (int j = 0; j < NKT; ++j) {
          const v4i key_at = *reinterpret_cast<const v4i*>(&s_pos[slot * KT + 16 * j + 4 * g]);
#pragma unroll
          for (int i = 0; i < 4; ++i) drafts = drafts || (key_at[i] > limit && key_at[i] != 0x7FFFFFFF);
        }
      }
      if (__any(drafts)) seen = named(row0 + key, slot * KT + 4 * g, 4 * NKT);
    }
#pragma unroll
    for (int j = 0; j < NKT; ++j) {
      const int k4 = 16 * j + 4 * g;
      const v4i key_at = *reinterpret_cast<const v4i*>(&s_pos[slot * KT + k4]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = key_at[i] <= limit || (TREE && (seen >> (4 * j + i) & 1u));
        s[j][i] = in ? s[j][i] * c : -INFINITY;
        top = fmaxf(top, s[j][i]);
      }
      if (s2 && tile < t1 && row0 + key < rows)
        *reinterpret_cast<v4f*>(s2 + (int64_t)tile * unit_rows * KT + ((row0 + key) * KT + k4)) = s[j];
    }
    top = groups_max(top);
  };
  // the scores' weights to s_w[wslot]
  float ref = 0.f, alpha = 1.f, e[NKT][4];
  v4bf hi[NKT];
  auto weigh_piece = [&](int ln, int wslot, auto piece) {
    const int key = ln & 15, g = ln >> 4, mine = row0 + key;
    if constexpr (piece == 0) {
      const bool move = top > m + 32.f;
      const float next = move ? top : m;
      alpha = move ? __builtin_amdgcn_exp2f(m - next) : 1.f;
      ref = next == -INFINITY ? 0.f : next;
      m = next;
      s_alpha[wslot][mine] = alpha;
      l *= alpha;
    } else {
      constexpr int j = (piece - 1) / 3, P = (piece - 1) % 3;
      if constexpr (P == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) e[j][i] = __builtin_amdgcn_exp2f(s[j][i] - ref);
      } else if constexpr (P == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) hi[j][i] = (__bf16)e[j][i];
        l += (e[j][0] + e[j][1]) + (e[j][2] + e[j][3]);
      } else {
        v4bf lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) lo[i] = (__bf16)(e[j][i] - (float)hi[j][i]);
        uint8_t* to = s_w + wslot * WB + mine * kWeightStride + 32 * j + 8 * g;
        *reinterpret_cast<v4bf*>(to) = hi[j];
        *reinterpret_cast<v4bf*>(to + 2 * KT) = lo;
      }
    }
  };
  constexpr int WEIGHS = 1 + 3 * NKT;

  // RG <= 4: what a wave reads from LDS for the stages of an iteration
  v4i x[TT], xr[QR ? QR : 1];  // score: its keys' codes and position values
  uint32_t sk = 0;             // and scales
  float zp[KPT][DG];           // weigh: the scores' parts
  int key_at[KPT];
  uint32_t codes4[4];          // widen: its 4 keys
  int scale4[4];
  constexpr int OS = RG == 1 ? 4 : 2 * O::XT;  // output: steps of 16 (RG = 1: all 32) keys, 32 (16) values, all rows
  v4s v0[OS], v1[OS];
  v8bf wt[2][2][O::YT];  // [16 keys][high, low][32 rows]; RG = 1: [0][high, low][0]
  float al[O::YT];
  auto read_score = [&](int ln, int slot) {
    const int key = ln & 15, g = ln >> 4;
    const uint8_t* codes = s_codes + slot * kCodesBytes + 4 * kt * kGroup;
    const uint32_t at0 = (uint32_t)((key >> 2) * kGroup + (key & 3) * kCodeBytes + 64 * g + ((key & 3) << 4));
    const uint8_t* rope = s_rope + slot * kRopeBytes + (key >> 3) * kGroup + (key & 7) * 2 * kRope +
                          ((g ^ ((key >> 1) & 3)) << 4) + 2 * kt * kGroup;
    sk = *reinterpret_cast<const uint32_t*>(s_scale + slot * kScalesBytes + (key >> 3) * 256 + (key & 7) * kScaleBytes +
                                            4 * g + 2 * kt * 256);
#pragma unroll
    for (int k = 0; k < QR; ++k) xr[k] = *reinterpret_cast<const v4i*>(rope + 64 * (QR == 2 ? k : dg & 1));
#pragma unroll
    for (int i = 0; i < TT; ++i) x[i] = *reinterpret_cast<const v4i*>(codes + (at0 ^ ((TT * dg + i) << 4)));
  };
  // the wave's part of the scores of its rows and keys, to s_part[buf]
  auto score_part = [&](int ln, int buf) {
    v4f sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < QR; ++k) {
      if (DG == 4 && dg >= 2) xr[k] = v4i{0, 0, 0, 0};  // two of four waves have no position values left
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, xr[k]), __builtin_bit_cast(v8bf, q[QK + k]),
                                                    sum, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      const float by = scale_operand(sk >> (8 * (TT * dg + i)) & 255u);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, decode8((uint32_t)x[i][u], by)),
                                                      __builtin_bit_cast(v8bf, q[4 * i + u]), sum, 0, 0, 0);
    }
    *reinterpret_cast<v4f*>(&s_part[((buf * DG + dg) * ROWS + row0 + (ln & 15)) * PR + 16 * kt + 4 * (ln >> 4)]) = sum;
  };
  auto read_part = [&](int td, int slot, int buf) {
    const int row = td / LPR, k0 = td % LPR * KPT;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      key_at[i] = s_pos[slot * KT + k0 + i];
#pragma unroll
      for (int d = 0; d < DG; ++d) zp[i][d] = s_part[((buf * DG + d) * ROWS + row) * PR + k0 + i];
    }
  };
  // the weights of KPT scores of one row to s_w[wslot]; slot: of their keys
  auto weigh_part = [&](int td, int wslot, int slot) {
    const int row = td / LPR, k0 = td % LPR * KPT;
    float z[KPT], e[KPT], top = -INFINITY;
    uint32_t seen = 0;  // nodes of a tree
    if constexpr (TREE) {
      bool drafts = false;
#pragma unroll
      for (int i = 0; i < KPT; ++i) drafts = drafts || (key_at[i] > limit && key_at[i] != 0x7FFFFFFF);
      if (__any(drafts)) seen = named(row, slot * KT + k0, KPT);
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      z[i] = zp[i][0];
#pragma unroll
      for (int d = 1; d < DG; ++d) z[i] += zp[i][d];
      const bool in = key_at[i] <= limit || (TREE && (seen >> i & 1u));
      z[i] = in ? z[i] * c : -INFINITY;
      top = fmaxf(top, z[i]);
    }
    top = row_reduce<LPR>(top, [](float x, float y) { return fmaxf(x, y); });
    const bool move = top > m + 32.f;
    const float next = move ? top : m;
    const float alpha = move ? __builtin_amdgcn_exp2f(m - next) : 1.f;
    const float ref = next == -INFINITY ? 0.f : next;
    m = next;
    l *= alpha;
    if (k0 == 0) s_alpha[wslot][row] = alpha;
    __bf16* to = reinterpret_cast<__bf16*>(s_w + wslot * WB + row * kWeightStride) + k0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      e[i] = __builtin_amdgcn_exp2f(z[i] - ref);
      l += e[i];
      const __bf16 hi = (__bf16)e[i];
      to[i] = hi;
      to[KT + i] = (__bf16)(e[i] - (float)hi);
      zp[i][0] = z[i];
    }
  };
  auto keep_scores = [&](int td, int tile) {
    const int row = td / LPR, k0 = td % LPR * KPT;
    if (s2 && tile < t1 && row < rows) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) s2[(int64_t)tile * unit_rows * KT + (row * KT + k0 + i)] = zp[i][0];
    }
  };
  auto read_codes = [&](int ln, int slot) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      codes4[j] = *reinterpret_cast<const uint32_t*>(s_codes + slot * kCodesBytes + w * kGroup + ((4 * ln) ^ (j << 4)) +
                                                     j * kCodeBytes);
      scale4[j] = s_scale[slot * kScalesBytes + (w >> 1) * 256 + (4 * (w & 1) + j) * kScaleBytes + (ln >> 2)];
    }
  };
  auto widen_codes = [&](int ln, int vslot) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      put_values(ln, j, vslot, codes4[j], scale4[j]);
  };
  auto read_output = [&](int ln, int vslot, int wslot) {
    const uint8_t* wgt = s_w + wslot * WB;
    const int g = ln >> 4, quad = (ln & 15) >> 2, h = ln >> 5;
    if constexpr (RG == 1) {
      // keys 8 g + 4 r + quad, chunks 8 w + 2 x + (ln & 3) / 2
      const uint8_t* base = s_val + vslot * kValueBytes + (8 * g + quad) * 2 * kLatent + 256 * (w >> 1) + 8 * (ln & 1);
      const uint32_t at0 = (uint32_t)(((8 * (w & 1) + ((ln & 3) >> 1)) ^ (4 * quad + (2 * g & 3))) << 4);
#pragma unroll
      for (int i = 0; i < OS; ++i) {
        v0[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, base + (at0 ^ (i << 5))));
        v1[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, base + (at0 ^ (i << 5) ^ 16) + 4 * 2 * kLatent));
      }
      const uint8_t* wp = wgt + (ln & 15) * kWeightStride + 16 * g;
#pragma unroll
      for (int part = 0; part < 2; ++part)
        wt[0][part][0] = __builtin_bit_cast(v8bf, *reinterpret_cast<const v4i*>(wp + part * 2 * KT));
      al[0] = s_alpha[wslot][ln & 15];
    } else if constexpr (!ONE) {
      // keys 16 k + 8 h + 4 r + quad, chunks 8 w + 4 x + 2 (g & 1) + (ln & 3) / 2
      const uint8_t* base = s_val + vslot * kValueBytes + (8 * h + quad) * 2 * kLatent + 256 * (w >> 1) + 8 * (ln & 1);
      const uint32_t at0 = (uint32_t)((((8 * (w & 1)) + 2 * (g & 1) + ((ln & 3) >> 1)) ^ (4 * quad + 2 * h)) << 4);
#pragma unroll
      for (int i = 0; i < OS; ++i) {
        const uint8_t* from = base + i / O::XT * 16 * 2 * kLatent;
        const uint32_t d = (uint32_t)(i % O::XT << 6);
        v0[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, from + (at0 ^ d)));
        v1[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, from + (at0 ^ d ^ 16) + 4 * 2 * kLatent));
      }
#pragma unroll
      for (int y = 0; y < O::YT; ++y) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int part = 0; part < 2; ++part)
            wt[k][part][y] = __builtin_bit_cast(
                v8bf, *reinterpret_cast<const v4i*>(wgt + O::row(w, ln, y) * kWeightStride + 32 * k + 16 * h + part * 2 * KT));
        al[y] = s_alpha[wslot][O::row(w, ln, y)];
      }
    }
  };
  auto add_output = [&] {
#pragma unroll
    for (int y = 0; y < O::YT; ++y)
      if (RG < 4 || __any(al[y] != 1.f)) {
#pragma unroll
        for (int i = 0; i < O::XT; ++i) {
          if constexpr (RG == 1) o1[i] *= al[y];
          else o[i][y] *= al[y];
        }
      }
#pragma unroll
    for (int part = 0; part < 2; ++part)  // all with the high parts, then with the low ones
#pragma unroll
      for (int i = 0; i < OS; ++i) {
        const v8bf v = __builtin_bit_cast(v8bf, __builtin_shufflevector(v0[i], v1[i], 0, 1, 2, 3, 4, 5, 6, 7));
        if constexpr (RG == 1) {
          o1[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, wt[0][part][0], o1[i], 0, 0, 0);
        } else {
#pragma unroll
          for (int y = 0; y < O::YT; ++y)
            o[i % O::XT][y] =
                __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, wt[i / O::XT][part][y], o[i % O::XT][y], 0, 0, 0);
        }
      }
  };

  // RG = 8: values are read one step ahead, other stages' pieces issued between the products
  auto output = [&](int ln, int vslot, int wslot, auto after) {
    const uint8_t* wgt = s_w + wslot * WB;
    const int g = ln >> 4, quad = (ln & 15) >> 2, h = ln >> 5;
    // keys 16 k + 8 h + 4 r + quad, chunks 16 (w & 3) + 4 x + 2 (g & 1) + (ln & 3) / 2
    const uint8_t* base = s_val + vslot * kValueBytes + (8 * h + quad) * 2 * kLatent +
                          256 * (w & 3) + 8 * (ln & 1);
    const uint32_t at0 =
        (uint32_t)(((2 * (g & 1) + ((ln & 3) >> 1)) ^ (4 * quad + 2 * h)) << 4);
    constexpr int STEPS = 2 * O::XT;  // a step: 16 keys, 32 values, all rows; values are read one ahead
    v4s v0[STEPS], v1[STEPS];
    auto read_value = [&](auto i) {
      const uint8_t* from = base + i / O::XT * 16 * 2 * kLatent;
      const uint32_t d = (uint32_t)(i % O::XT << 6);
      v0[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, from + (at0 ^ d)));
      v1[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, from + (at0 ^ d ^ 16) + 4 * 2 * kLatent));
    };
    v8bf wt[2][2][O::YT];  // [16 keys][high, low][32 rows]
    auto read_weight = [&](int k, int part, int y) {
      wt[k][part][y] = __builtin_bit_cast(
          v8bf, *reinterpret_cast<const v4i*>(wgt + O::row(w, ln, y) * kWeightStride + 32 * k + 16 * h + part * 2 * KT));
    };
#pragma unroll
    for (int y = 0; y < O::YT; ++y) read_weight(0, 0, y);
    read_value(std::integral_constant<int, 0>{});
#pragma unroll
    for (int y = 0; y < O::YT; ++y) read_weight(0, 1, y);
#pragma unroll
    for (int y = 0; y < O::YT; ++y) {
      const float al = s_alpha[wslot][O::row(w, ln, y)];
      if (__any(al != 1.f)) {
#pragma unroll
        for (int x = 0; x < O::XT; ++x) o[x][y] *= al;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    unroll<STEPS>([&](auto i) {
      constexpr int k = i / O::XT, x = i % O::XT;
      const v8bf v = __builtin_bit_cast(v8bf, __builtin_shufflevector(v0[i], v1[i], 0, 1, 2, 3, 4, 5, 6, 7));
      unroll<2 * O::YT>([&](auto u) {  // all rows with the high parts, then with the low ones
        constexpr int part = u / O::YT, y = u % O::YT;
        o[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, wt[k][part][y], o[x][y], 0, 0, 0);
        if constexpr (u == 0 && i + 1 < STEPS) read_value(std::integral_constant<int, (i + 1) % STEPS>{});
        if constexpr (i + 1 == O::XT) read_weight(1, part, y);  // in place of the one that was used last here
        after(std::integral_constant<int, 2 * O::YT * i + u>{}, std::integral_constant<int, 2 * O::YT * STEPS>{});
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };

  const int count = t1 - t0;
  if (count > 0) {
    if constexpr (ONE) {
      const int entry0 = fetch(lane, t0);
      entry = fetch(lane, t0 + 1);
      page = place(lane, t0, entry0, pos, at);
      unroll<LOADS>([&](auto p) { load_piece(lane, t0, 0, p); });
    } else {
      const int entry0 = *fetch8(t0), entry8 = *fetch8(t0 + 8);
      place8(t0, entry0);
      row_of = locate(pos, *page8());
      at_of = at;
      place8(t0 + 8, entry8);
      // as after a step of tile 0
      if (!code_wave) load_lds4(fetch8(t0 + 16), (uint32_t)(uintptr_t)LDS(int, s_entry) + 256 * w4);
      if (!code_wave) load_lds4(page8(), (uint32_t)(uintptr_t)LDS(int, s_page) + 256 * w4);
      for (int i = 0; i < NS; ++i) {
        rows_of(lane, i);
        load_rows(lane, i);
      }
    }
  }
  // the query is in registers before the loop (its waits would fall inside it)
#pragma unroll
  for (int k = 0; k < QK + QR; ++k) asm volatile("s_waitcnt vmcnt(0)" : "+v"(q[k]));
  // RG = 8: every load is done, the entry and the page too (named here, so that the
  // compiler waits for them nowhere else), and all waves are here.  Written out:
  // the waves of a workgroup may come to it by two ways.
  const auto meet = [&] {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : "+v"(entry), "+v"(page)::"memory");
  };
  // RG <= 4: of the loads those that were issued AHEAD or more iterations ago are
  // done.  Each iteration since has issued at least 2 of them, and a store where
  // the wave keeps scores.
  const bool stores = s2 && w * (64 / LPR) < rows;
  const auto meet_ahead = [&] {
    if (stores) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * (AHEAD - 1)) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (AHEAD - 1)) : "memory");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  if (count > 0) {
    meet();
    if constexpr (ONE) {
      unroll<LOADS>([&](auto p) { load_piece(lane, t0 + 1, 1, p); });
      if (w < 4) {
        score(lane, 0);
        finish_scores(lane, t0, 0);
        unroll<WEIGHS>([&](auto p) { weigh_piece(lane, 0, p); });
      }
    } else {
      read_score(lane, 0);
      score_part(lane, 0);
      meet();
      read_score(lane, 1);
      read_part(tid, 0, 0);
      score_part(lane, 1);
      weigh_part(tid, 0, 0);
      keep_scores(tid, t0);
    }
    unroll<WIDENS>([&](auto p) { widen_piece(lane, 0, 0, p); });
  }
  // Iteration i puts out tile i (past the last tile masked ones, of row 0).
  int slot = 0;  // of tile i's codes
  for (int i = 0; i < count; ++i) {
    int ln = lane;
    if constexpr (RG >= 4) asm volatile("" : "+v"(ln));  // no registers are left to keep addresses in: made anew for every tile
    drop_infinite(ln, slot, i & 1);
    const int next = slot + 1 == NS ? 0 : slot + 1, after_next = next + 1 == NS ? 0 : next + 1;  // of i + 1, i + 2
    if constexpr (ONE) {
      // tile i + 2 is loaded, i + 1 scored; waves 0 .. 3 meet the others before they
      // score tile i + 1, waves 4 .. 7 after they scored tile i
      const bool early = w < 4;
      const int st = early ? i + 1 : i, ss = early ? next : slot;
      if (early) meet();
      score(ln, ss);
      finish_scores(ln, t0 + st, ss);
      unroll<WEIGHS>([&](auto p) { weigh_piece(ln, st & 1, p); });
      if (!early) meet();
      output(ln, i & 1, i & 1, [&](auto step, auto steps) {
        pieces_after<steps, LOADS + WIDENS, step>([&](auto p) {
          if constexpr (p < LOADS) load_piece(ln, t0 + i + 2, after_next, p);
          else widen_piece(ln, next, (i + 1) & 1, std::integral_constant<int, p - LOADS>{});
        });
      });
    } else {
      // tile i + 2 + AHEAD is loaded, i + 2 multiplied, i + 1 weighed and widened
      meet_ahead();
      next_rows(ln, i + NS);
      read_part(64 * w + ln, next, (i + 1) & 1);
      read_score(ln, after_next);
      read_codes(ln, next);
      if constexpr (RG < 4) read_output(ln, i & 1, i & 1);
      __builtin_amdgcn_sched_barrier(0);
      weigh_part(64 * w + ln, (i + 1) & 1, next);
      score_part(ln, i & 1);
      widen_codes(ln, (i + 1) & 1);
      if constexpr (RG == 4) read_output(ln, i & 1, i & 1);  // no registers for it before
      add_output();
      keep_scores(64 * w + ln, t0 + i + 1);
      load_rows(ln, slot);
    }
    slot = next;
  }
  // no load into LDS may outlive the workgroup
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

  // the rows' statistics
  __syncthreads();
  if constexpr (ONE) {
    l = groups_sum(l);
    if (lane < 16) {
      s_sum[row0 + lane] = l;
      s_max[row0 + lane] = m;
    }
  } else {
    l = row_reduce<LPR>(l, [](float x, float y) { return x + y; });
    if (tid % LPR == 0) {
      s_sum[tid / LPR] = l;
      s_max[tid / LPR] = m;
    }
  }
  __syncthreads();
  if (splits > 1) {
    if (tid < ROWS) wk.part_ml[(int64_t)part * ROWS + tid] = {s_max[tid], s_sum[tid]};
    // the registers as they lie: the joining kernel has the same lanes
    float4* po = wk.part_o + (int64_t)part * O::QUADS * (64 * kWaves) + tid;
    if constexpr (RG == 1) {
#pragma unroll
      for (int x = 0; x < 4; ++x) po[x * 64 * kWaves] = float4{o1[x][0], o1[x][1], o1[x][2], o1[x][3]};
    } else {
#pragma unroll
      for (int y = 0; y < O::YT; ++y)
#pragma unroll
        for (int x = 0; x < O::XT; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            po[((O::XT * y + x) * 4 + i) * 64 * kWaves] =
                float4{o[x][y][4 * i], o[x][y][4 * i + 1], o[x][y][4 * i + 2], o[x][y][4 * i + 3]};
    }
    return;
  }
  const int64_t orow = ((int64_t)t.row0[b] + i_first) * a.heads + first;
  if (tid < rows) {
    const float sum = s_sum[tid], top = s_max[tid];
    if (a.lse) a.lse[orow + tid] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    if (sm.stat) sm.stat[orow + tid] = {top == -INFINITY ? 0.f : top, sum == 0.f ? 0.f : 1.f / sum};
  }
  // A row tile of every wave at a time through LDS, so that whole rows are
  // written; chunks of 8 values change places by the row against bank conflicts.
  constexpr int OR = RG == 1 ? 16 : RG == 8 ? 64 : 32;  // rows at a time
  static_assert(OR * 2 * kLatent <= sizeof(s_val), "the rows fit");
#pragma unroll
  for (int y = 0; y < O::YT; ++y) {
    const int row = O::row(w, lane, y), at_row = RG == 8 ? (row & 31) + 32 * (w >> 2) : row - 32 * y;
    const float sum = s_sum[row], inv = sum == 0.f ? 0.f : 1.f / sum;
    auto put = [&](int value, float a0, float a1, float a2, float a3) {
      const v4bf v = {(__bf16)(a0 * inv), (__bf16)(a1 * inv), (__bf16)(a2 * inv), (__bf16)(a3 * inv)};
      *reinterpret_cast<v4bf*>(s_val + at_row * 2 * kLatent + (((value >> 3) ^ (at_row & 63)) << 4) + (value & 4) * 2) = v;
    };
    if constexpr (RG == 1) {
#pragma unroll
      for (int x = 0; x < O::XT; ++x) put(O::value(w, lane, x, 0), o1[x][0], o1[x][1], o1[x][2], o1[x][3]);
    } else {
#pragma unroll
      for (int x = 0; x < O::XT; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          put(O::value(w, lane, x, i), o[x][y][4 * i], o[x][y][4 * i + 1], o[x][y][4 * i + 2], o[x][y][4 * i + 3]);
    }
    __syncthreads();
    for (int r = w; r < OR; r += kWaves) {
      const int out = RG == 8 ? 64 * (r >> 5) + 32 * y + (r & 31) : 32 * y + r;
      if (out < rows)
        *reinterpret_cast<uint4*>(a.out + (orow + out) * kLatent + 8 * lane) =
            *reinterpret_cast<const uint4*>(s_val + r * 2 * kLatent + ((lane ^ (r & 63)) << 4));
    }
    if (y + 1 < O::YT) __syncthreads();
  }
}

// Joins the splits of a row tile (blockIdx.y).  An item is four registers of one
// wave of the attention kernel, 1 KB a split; the items of one group hold the same
// rows and share the splits' weights.  Bound by the bytes of the splits' outputs.
template <int RG>
struct Join {
  static constexpr int kRows = RG == 1 ? 16 : 32;
  static constexpr int kGroups = 16 * RG / kRows;
  static constexpr int kItems = kWaves * Output<RG>::QUADS / kGroups;
  static constexpr int kSharing = RG == 8 ? 4 : kWaves;  // waves of the attention kernel with the same rows
};
// Waves that share an item, each with every so-many-th split, their sums added up
// in LDS: many splits mean few row tiles, and one wave for 128 splits leaves the
// chip empty (1 x 128 rows x 128 splits: 202 us, with 8 waves 16); with 8 splits of
// 32 x 128 rows 8 waves of one split each take 50 us, one wave for all 17.
__host__ __device__ inline int join_waves(int splits) { return splits > 32 ? 8 : splits > 16 ? 4 : splits > 8 ? 2 : 1; }

template <int RG>
__global__ __launch_bounds__(64 * kWaves) void join_kernel(AttendArgs a, RunTable t, ScoreMap sm, Work wk) {
  using O = Output<RG>;
  using J = Join<RG>;
  constexpr int ROWS = 16 * RG;
  constexpr int LR = J::kRows;
  constexpr int SL = 64 * kWaves / LR;   // splits whose weights are made side by side
  extern __shared__ float s_w[];         // [splits][LR] weights
  __shared__ float s_red[SL][LR];
  __shared__ float4 s_sum[kWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, part_wave = tid >> 6;
  const int unit = blockIdx.y / wk.row_tiles, rt = blockIdx.y % wk.row_tiles;
  const bool sets = a.idx != nullptr;
  const int b = sets ? run_of(t, unit) : unit;
  const int unit_rows = sets ? a.heads : t.n_rows[b] * a.heads;
  const int first = rt * ROWS;
  const int splits = sets ? wk.splits : splits_of(t, b, wk.tiles_per_split);
  if (first >= unit_rows || splits == 1) return;
  const int rows = min(ROWS, unit_rows - first);
  const int64_t orow = ((int64_t)t.row0[b] + (sets ? unit - t.row0[b] : 0)) * a.heads + first;
  const int row_tiles = (unit_rows + ROWS - 1) / ROWS;
  const int64_t part = (sets ? unit * row_tiles * splits : wk.first[b]) + (row_tiles - 1 - rt) * splits;
  // a group of rows, and of its registers (item: wave of the attention kernel,
  // then quad) the one that this wave joins with per - 1 others
  const int per = join_waves(wk.splits), blocks = J::kItems * per / kWaves;
  const int group = blockIdx.x / blocks, item = (blockIdx.x % blocks * kWaves + part_wave) / per;
  const int y = group % O::YT, q = item / J::kSharing;
  const int w = group / O::YT * J::kSharing + item % J::kSharing;
  const int x = RG == 1 ? q : q / 4, quad = (RG == 1 ? 0 : 4 * O::XT * y) + q;
  const int row0 = O::row(w, 0, y);  // the first of the group's rows
  {
    const int r = tid % LR, s0 = tid / LR;
    const float2* ml = wk.part_ml + part * ROWS + row0 + r;
    float top = -INFINITY;
    for (int s = s0; s < splits; s += SL) top = fmaxf(top, ml[(int64_t)s * ROWS].x);
    s_red[s0][r] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SL; ++k) top = fmaxf(top, s_red[k][r]);
    __syncthreads();
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int s = s0; s < splits; s += SL) {
      const float2 v = ml[(int64_t)s * ROWS];
      const float e = __builtin_amdgcn_exp2f(v.x - ref);
      s_w[s * LR + r] = e;
      sum = fmaf(e, v.y, sum);
    }
    s_red[s0][r] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < SL; ++k) sum += s_red[k][r];
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    for (int s = s0; s < splits; s += SL) s_w[s * LR + r] *= inv;
    // a group's first block writes its rows' statistics
    if (s0 == 0 && row0 + r < rows && blockIdx.x % blocks == 0) {
      if (a.lse) a.lse[orow + row0 + r] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
      if (sm.stat) sm.stat[orow + row0 + r] = {ref, inv};
    }
    __syncthreads();
  }
  const float4* po = wk.part_o + (part * O::QUADS + quad) * (64 * kWaves) + 64 * w + lane;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = part_wave % per; s < splits; s += per) {
    const float e = s_w[s * LR + lane % LR];
    float4 v = {0.f, 0.f, 0.f, 0.f};
    if (e != 0.f) v = po[(int64_t)s * O::QUADS * (64 * kWaves)];  // an empty split wrote no output
    sum.x = fmaf(e, v.x, sum.x);
    sum.y = fmaf(e, v.y, sum.y);
    sum.z = fmaf(e, v.z, sum.z);
    sum.w = fmaf(e, v.w, sum.w);
  }
  s_sum[part_wave][lane] = sum;
  __syncthreads();
  if (part_wave % per == 0) {
    for (int k = 1; k < per; ++k) {
      const float4 v = s_sum[part_wave + k][lane];
      sum.x += v.x;
      sum.y += v.y;
      sum.z += v.z;
      sum.w += v.w;
    }
    const int row = O::row(w, lane, y);
    if (row < rows) {
      const v4bf v = {(__bf16)sum.x, (__bf16)sum.y, (__bf16)sum.z, (__bf16)sum.w};
      *reinterpret_cast<v4bf*>(a.out + (orow + row) * kLatent + O::value(w, lane, x, quad % 4)) = v;
    }
  }
}

// Sum over a tile's rows from `least` on, those that attend to the thread's key,
// of the softmax weights of its 32 keys: 8 rows at a time, each thread one key,
// the rows of a thread in ascending order.  The rows before are left out, not
// added as zeros: the masked scores of a NaN row give NaN.
__device__ __forceinline__ float tile_weight(const float* tile, const float2* stat, int least, int rows, float* red,
                                             int tid) {
  const int k = tid & 31, first = tid >> 5;
  float w = 0.f;
  for (int r = first + (max(least - first, 0) + 7) / 8 * 8; r < rows; r += 8) {
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
  const int n = t.n_k[b], rows = t.n_rows[b] * a.heads;
  if (rows == 0 || tile * kTileKeys >= n) return;
  const int least = max(tile * kTileKeys + (tid & 31) - t.pos0[b], 0) * a.heads;
  const float w = tile_weight(sm.s2 + sm.base[b] + (int64_t)tile * rows * kTileKeys,
                              sm.stat + (int64_t)t.row0[b] * a.heads, least, rows, red, tid);
  const int s = tile * kTileKeys + tid;
  if (tid < kTileKeys && s < n) a.acc[(int64_t)b * a.acc_stride + s] += w;
}

// The same for trees, where a call has many rows: T / 8 rows at a time, each thread 4
// keys, four loads on their way.  Rows whose mask does not name a node are left out,
// not added as zeros.  Bound by the scores' bytes: 192 rows x 196000 keys in 25 us, 6
// TB/s (one key a thread: 52).  T = 1024 from 1024 rows a sequence on, where a
// workgroup of 256 threads passes a tile in many rounds, 32 rows each; below, 1024
// threads have too few rows to share.  Calls with 256 and 1024 threads, us: 3328 rows a
// sequence x 1026 keys 91, 68; x 6026 keys 145, 123; x 40026 keys 610, 599; 32 x 3328
// rows x 1026 keys 626, 617; 8192 rows x 16064 keys 613, 583; 2048 rows x 100064 keys
// 879, 869; 38400 rows x 2300 keys 1010, 694; 4 x 1024 rows x 20008 keys 371, 364; 32 x
// 896 rows x 1507 keys 203, 202; 8 x 640 rows x 3040 keys 101, 102; 8 x 192 rows x 24012
// keys 212, 233; 64 x 128 rows x 2008 keys 104, 121.
template <int T>
__global__ __launch_bounds__(T) void tree_weights_kernel(AttendArgs a, RunTable t, ScoreMap sm, TreeMask tree) {
  constexpr int R = T / 8;  // rows at a time
  __shared__ float red[T / 64][kTileKeys];
  const int b = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x;
  const int n = t.n_k[b], rows = t.n_rows[b] * a.heads;
  if (rows == 0 || tile * kTileKeys >= n) return;
  const v4f* scores = reinterpret_cast<const v4f*>(sm.s2 + sm.base[b] + (int64_t)tile * rows * kTileKeys) + tid;
  const float2* stat = sm.stat + (int64_t)t.row0[b] * a.heads;
  v4f w = {0.f, 0.f, 0.f, 0.f};
  // the tree's nodes that the thread's keys are (before it: negative), the two words of
  // a mask that hold them
  const int node = tile * kTileKeys + 4 * (tid & 7) - tree.base[b], word = max(node, 0) >> 5;
  const bool drafts = tile * kTileKeys + kTileKeys > tree.base[b];
  const int w0 = min(word, tree.words - 1), w1 = min(word + 1, tree.words - 1);
  for (int r = tid >> 3; r < rows; r += 4 * R) {
    v4f z[4];
    float2 st[4];
    uint32_t m0[4], m1[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = min(r + R * j, rows - 1);
      z[j] = scores[(at - (tid >> 3)) * (kTileKeys / 4)];
      st[j] = stat[at];
      if (drafts) {
        const uint32_t* mask = tree.bits + (int64_t)(t.row0[b] + at / a.heads) * tree.words;
        m0[j] = mask[w0];
        m1[j] = mask[w1];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t bits = (uint64_t)m1[j] << 32 | m0[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bool seen = r + R * j < rows;
        if (drafts && node + i >= 0) seen = seen && (bits >> (node + i - 32 * word) & 1) && node + i < n - tree.base[b];
        if (seen) w[i] = fmaf(__builtin_amdgcn_exp2f(z[j][i] - st[j].x), st[j].y, w[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // the wave's 8 rows, then the waves
    w[i] += lane_xor8(w[i]);
    w[i] = groups_sum(w[i]);
    if ((tid & 63) < 8) red[tid >> 6][4 * (tid & 7) + i] = w[i];
  }
  __syncthreads();
  const int s = tile * kTileKeys + tid;
  if (tid < kTileKeys && s < n) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < T / 64; ++j) sum += red[j][tid];
    a.acc[(int64_t)b * a.acc_stride + s] += sum;
  }
}

__global__ __launch_bounds__(256) void slot_weights_kernel(AttendArgs a, ScoreMap sm, float* __restrict__ slots,
                                                           int padded) {
  __shared__ float red[256];
  const int r = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x;
  const float w = tile_weight(sm.s2 + ((int64_t)r * padded + tile * kTileKeys) * a.heads,
                              sm.stat + (int64_t)r * a.heads, 0, a.heads, red, tid);
  if (tid < kTileKeys) slots[(int64_t)r * padded + tile * kTileKeys + tid] = w;
}

// acc += the slots' weights: a workgroup owns kRange positions of a sequence
// and adds rows one after the other (a position comes at most once in a set, so
// every sum has one order).  A step is 2048 entries of a row, 2 a thread; the
// entries of the next kAhead steps are loaded while these are added.  Many rows are
// cut into `groups` whose sums are added up in order afterwards: one group of 1003
// rows x 2048 takes 1160 us, 62 groups 46 with their addition.  32 sequences of 2 rows x 2048 take 14.
constexpr int kRange = 8192;
constexpr int kAddThreads = 1024;
constexpr int kAhead = 4;
template <bool TREE>
__global__ __launch_bounds__(kAddThreads) void slot_add_kernel(AttendArgs a, RunTable t, const float* __restrict__ slots,
                                                               int padded, int groups, float* parts, TreeOf<TREE> tree) {
  __shared__ float sum[kRange];
  const int b = blockIdx.y, tid = threadIdx.x, group = blockIdx.x % groups;
  const int lo = blockIdx.x / groups * kRange, n = t.n_k[b];
  if (t.n_rows[b] == 0 || lo >= n) return;
  const int each = (t.n_rows[b] + groups - 1) / groups, row0 = group * each;
  const int rows = max(0, min(each, t.n_rows[b] - row0));
  const int passes = (a.topk + 2 * kAddThreads - 1) / (2 * kAddThreads), steps = rows * passes;
  int key[2][kAhead][2];
  float w[2][kAhead][2];
  auto load = [&](int first, int (&keys)[kAhead][2], float (&ws)[kAhead][2]) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = (first + j) / passes, base = (first + j - i * passes) * 2 * kAddThreads;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = base + e * kAddThreads + tid;
        const int64_t r = t.row0[b] + row0 + i;
        const bool ok = first + j < steps && k < a.topk;
        keys[j][e] = ok ? a.idx[r * a.topk + k] : -1;
        ws[j][e] = ok ? slots[r * padded + k] : 0.f;
      }
    }
  };
  auto add = [&](int first, const int (&keys)[kAhead][2], const float (&ws)[kAhead][2]) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (first + j >= steps) return;
      const int i = (first + j) / passes, pos = t.pos0[b] + row0 + i;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = keys[j][e];
        bool seen = at >= 0 && at <= pos;
        if constexpr (TREE) {
          const int node = at - tree.base[b];
          seen = at >= 0 && at < n;
          if (seen && node >= 0)
            seen = (tree.bits[(int64_t)(t.row0[b] + row0 + i) * tree.words + (node >> 5)] >> (node & 31) & 1u) != 0u;
        }
        if (seen && (uint32_t)(at - lo) < (uint32_t)kRange) atomicAdd(&sum[at - lo], ws[j][e]);
      }
      __syncthreads();
    }
  };
  load(0, key[0], w[0]);
  for (int j = tid; j < kRange; j += kAddThreads) sum[j] = 0.f;
  __syncthreads();
  for (int first = 0; first < steps; first += 2 * kAhead) {
    load(first + kAhead, key[1], w[1]);
    add(first, key[0], w[0]);
    load(first + 2 * kAhead, key[0], w[0]);
    add(first + kAhead, key[1], w[1]);
  }
  if (groups > 1) {
    float* part = parts + ((int64_t)b * groups + group) * (gridDim.x / groups * kRange) + lo;
    for (int j = tid; j < kRange; j += kAddThreads) part[j] = sum[j];
    return;
  }
  for (int j = tid; j < kRange && lo + j < n; j += kAddThreads)
    if (sum[j] != 0.f) a.acc[(int64_t)b * a.acc_stride + lo + j] += sum[j];
}

__global__ __launch_bounds__(256) void group_add_kernel(AttendArgs a, RunTable t, int groups, const float* parts,
                                                        int64_t stride) {
  const int b = blockIdx.y, at = blockIdx.x * 256 + threadIdx.x;
  if (t.n_rows[b] == 0 || at >= t.n_k[b]) return;
  float sum = 0.f;
#pragma unroll 8
  for (int g = 0; g < groups; ++g) sum += parts[((int64_t)b * groups + g) * stride + at];
  if (sum != 0.f) a.acc[(int64_t)b * a.acc_stride + at] += sum;
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  size_t scores, stats, slots, sums, part_o, part_ml;
  int ranges, groups;  // of the slots' sums
  int padded;
  int64_t base[kMaxSeq];
  int rows, max_n;
  int64_t workgroups;
  int rg;       // row groups of 16 per workgroup
  Work wk;
  size_t bytes() const {
    return round256(scores) + round256(stats) + round256(slots) + round256(sums) + round256(part_o) + round256(part_ml);
  }
};

constexpr int kCus = 256;
constexpr int kLeastTiles = 4;

Plan plan_of(const AttendArgs& a, const RunTable& t) {
  Plan p{};
  int64_t words = 0;
  int max_rows = 0;
  p.padded = (a.topk + kTileKeys - 1) / kTileKeys * kTileKeys;
  for (int b = 0; b < t.n; ++b) {
    const int n = t.n_k[b];
    p.base[b] = words;
    if (t.n_rows[b]) {
      words += (int64_t)((n + kTileKeys - 1) / kTileKeys) * kTileKeys * t.n_rows[b] * a.heads;
      if (n > p.max_n) p.max_n = n;
      if (t.n_rows[b] > max_rows) max_rows = t.n_rows[b];
    }
    p.rows += t.n_rows[b];
  }
  if (p.rows == 0) return p;
  if (a.idx) words = (int64_t)p.rows * p.padded * a.heads;
  if (a.acc) {
    p.scores = (size_t)words * 4;
    p.stats = (size_t)p.rows * a.heads * sizeof(float2);
    p.slots = a.idx ? (size_t)p.rows * p.padded * 4 : 0;
    // groups of 16 rows or more, as far as workgroups of two a CU are not many enough
    p.ranges = (p.max_n + kRange - 1) / kRange;
    p.groups = std::max(1, std::min(max_rows / 16, 2 * kCus / (t.n * p.ranges)));
    p.sums = a.idx && p.groups > 1 ? (size_t)t.n * p.groups * p.ranges * kRange * 4 : 0;
  }
  const int64_t unit_rows = a.idx ? a.heads : (int64_t)max_rows * a.heads;
  p.rg = unit_rows > 64 ? 8 : unit_rows > 32 ? 4 : unit_rows > 16 ? 2 : 1;
  p.wk.units = a.idx ? p.rows : t.n;
  const int max_tiles = a.idx ? p.padded / kTileKeys : (p.max_n + kTileKeys - 1) / kTileKeys;
  const auto row_tiles_of = [&](int64_t rows) { return (rows + 16 * p.rg - 1) / (16 * p.rg); };
  const auto workgroups = [&](int64_t each) {
    if (a.idx) return p.rows * row_tiles_of(a.heads) * (max_tiles > each ? (max_tiles + each - 1) / each : 1);
    int64_t w = 0;
    for (int b = 0; b < t.n; ++b) w += row_tiles_of((int64_t)t.n_rows[b] * a.heads) * splits_of(t, b, (int)each);
    return w;
  };
  // A split has at least kLeastTiles.  Where even so workgroups of half the rows
  // would all run at once, they are taken: a tile of 16 rows takes 1.3 us, one of
  // 128 rows 3.3 (2 queries of 128 heads on 2048 keys: 28 us with 128 rows a
  // workgroup, 17 with 16).
  int64_t each = kLeastTiles;
  while (p.rg > 1 && 2 * workgroups(each) <= kCus) p.rg /= 2;
  // Splits of as few tiles as give no more workgroups than run at once: one more
  // would wait for another to end.
  while (each < max_tiles && workgroups(each) > kCus) each += 1 + each / 32;
  if (each >= max_tiles) each = max_tiles > 0 ? max_tiles : 1;
  const int R = 16 * p.rg;
  p.wk.row_tiles = (int)row_tiles_of(unit_rows);
  p.wk.tiles_per_split = (int)each;
  p.wk.splits = max_tiles > 0 ? (int)((max_tiles + each - 1) / each) : 1;
  p.workgroups = workgroups(each);
  if (!a.idx) {
    int32_t w = 0;
    for (int b = 0; b < t.n; ++b) {
      p.wk.first[b] = w;
      w += (int32_t)(row_tiles_of((int64_t)t.n_rows[b] * a.heads) * splits_of(t, b, (int)each));
    }
    p.wk.first[t.n] = w;
  }
  if (p.wk.splits > 1) {
    p.part_o = (size_t)p.workgroups * R * kLatent * 4;
    p.part_ml = (size_t)p.workgroups * R * sizeof(float2);
  }
  return p;
}

template <int RG, int CALL>
hipError_t launch_rows(const AttendArgs& a, const RunTable& t, const ScoreMap& sm, const Work& wk, unsigned workgroups,
                       const TreeOf<CALL != kCausal>& tree, hipStream_t stream) {
  hipLaunchKernelGGL((attend_kernel<RG, CALL>), dim3(workgroups), dim3(64 * kWaves), 0, stream, a, t, sm, wk, tree);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || wk.splits == 1) return e;
  using J = Join<RG>;
  hipLaunchKernelGGL(join_kernel<RG>, dim3((unsigned)(J::kGroups * J::kItems * join_waves(wk.splits) / kWaves),
                          (unsigned)(wk.units * wk.row_tiles)),
                     dim3(64 * kWaves), (size_t)wk.splits * J::kRows * 4, stream, a, t, sm, wk);
  return hipGetLastError();
}

}  // namespace

size_t attend_workspace(const AttendArgs& a, const RunTable& t) { return plan_of(a, t).bytes(); }

namespace {

template <int CALL>
hipError_t launch_call(const AttendArgs& a, const RunTable& t, const TreeOf<CALL != kCausal>& tree, hipStream_t stream) {
  constexpr bool TREE = CALL != kCausal;
  Plan p = plan_of(a, t);
  if (p.rows == 0) return hipSuccess;
  ScoreMap sm{};
  uint8_t* ws = (uint8_t*)a.workspace;
  if (a.acc) {
    sm.s2 = (float*)ws;
    sm.stat = (float2*)(ws + round256(p.scores));
    for (int b = 0; b < t.n; ++b) sm.base[b] = p.base[b];
  }
  float* slots = (float*)(ws + round256(p.scores) + round256(p.stats));
  float* sums = (float*)((uint8_t*)slots + round256(p.slots));
  uint8_t* parts = (uint8_t*)sums + round256(p.sums);
  p.wk.part_o = (float4*)parts;
  p.wk.part_ml = (float2*)(parts + round256(p.part_o));
  const unsigned wgs = (unsigned)p.workgroups;
  hipError_t e = p.rg == 8   ? launch_rows<8, CALL>(a, t, sm, p.wk, wgs, tree, stream)
                 : p.rg == 4 ? launch_rows<4, CALL>(a, t, sm, p.wk, wgs, tree, stream)
                 : p.rg == 2 ? launch_rows<2, CALL>(a, t, sm, p.wk, wgs, tree, stream)
                             : launch_rows<1, CALL>(a, t, sm, p.wk, wgs, tree, stream);
  if (e != hipSuccess || !a.acc || (a.idx && a.topk == 0)) return e;
  if (!a.idx) {
    const unsigned tiles = (unsigned)((p.max_n + kTileKeys - 1) / kTileKeys);
    if constexpr (TREE) {
      int most = 0;
      for (int b = 0; b < t.n; ++b) most = std::max(most, t.n_rows[b]);
      if (most * a.heads >= 1024)
        hipLaunchKernelGGL(tree_weights_kernel<1024>, dim3(tiles, (unsigned)t.n), dim3(1024), 0, stream, a, t, sm, tree);
      else
        hipLaunchKernelGGL(tree_weights_kernel<256>, dim3(tiles, (unsigned)t.n), dim3(256), 0, stream, a, t, sm, tree);
    } else
      hipLaunchKernelGGL(dense_weights_kernel, dim3(tiles, (unsigned)t.n), dim3(256), 0, stream, a, t, sm);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(slot_weights_kernel, dim3((unsigned)(p.padded / kTileKeys), (unsigned)p.rows), dim3(256), 0, stream,
                     a, sm, slots, p.padded);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(slot_add_kernel<TREE>, dim3((unsigned)(p.ranges * p.groups), (unsigned)t.n), dim3(kAddThreads), 0,
                     stream, a, t, slots, p.padded, p.groups, sums, tree);
  e = hipGetLastError();
  if (e != hipSuccess || p.groups == 1) return e;
  hipLaunchKernelGGL(group_add_kernel, dim3((unsigned)((p.max_n + 255) / 256), (unsigned)t.n), dim3(256), 0, stream, a, t,
                     p.groups, sums, (int64_t)p.ranges * kRange);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, const RunTable& t, const TreeMask* tree, hipStream_t stream) {
  if (!tree) return launch_call<kCausal>(a, t, NoTree{}, stream);
  return a.idx ? launch_call<kTreeSets>(a, t, *tree, stream) : launch_call<kTreePrefix>(a, t, *tree, stream);
}

}  // namespace pivot
