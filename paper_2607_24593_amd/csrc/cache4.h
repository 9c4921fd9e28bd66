// The 4-bit latent cache: one row per token, shared by all heads.
//   codes  [rows, 256]  512 latent values, OCP E2M1, the even value in the low nibble
//   scales [rows, 16]   one E8M0 byte (2^(byte - 127), 255 = NaN) per 32 values
//   rope   [rows, 64]   position values, bf16
// 400 bytes a token, against 1152 in bf16.  The three arrays keep every part
// aligned to its own size, so a gathered row touches as many 64-byte sectors
// (4 + 1 + 2) as a packed row of 400 bytes would.
#pragma once

#include "device_common.h"

namespace pivot {

constexpr int kLatent = 512;                // latent values per token (the attention's values)
constexpr int kRope = 64;                   // position values per token
constexpr int kAttnDim = kLatent + kRope;   // key and query width
constexpr int kBlk = 32;                    // latent values per scale
constexpr int kCodeBytes = kLatent / 2;
constexpr int kScaleBytes = kLatent / kBlk;

struct Cache4 {
  uint8_t* codes;
  uint8_t* scales;
  uint16_t* rope;
};

// Sequences of one launch (at most kMaxSeq), passed by value: rows of sequence
// b are row0[b] .. row0[b] + n_rows[b] - 1 of the launch's packed arrays, row i
// at position pos0[b] + i of n_k[b] cached tokens.
struct RunTable {
  int32_t n;
  int32_t pos0[kMaxSeq];
  int32_t n_k[kMaxSeq];
  int32_t n_rows[kMaxSeq];
  int32_t row0[kMaxSeq];
};

// The sequence that owns packed row r (r < the launch's rows): the last one
// with row0 <= r, by bisection; empty sequences share their row0 with the next.
__device__ __forceinline__ int run_of(const RunTable& t, int r) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.row0[mid] <= r) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

// A scale byte as the float whose exponent field it is; the conversion
// instructions read only that field (0 stands for 2^-127, 255 for NaN).
__device__ __forceinline__ float scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes (one word) times a scale, as bf16: exact, since a code has two
// significant bits, or infinite from 2^128 on.
__device__ __forceinline__ uint4 decode8(uint32_t w, float scale) {
  uint4 o;
  o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return o;
}

}  // namespace pivot
