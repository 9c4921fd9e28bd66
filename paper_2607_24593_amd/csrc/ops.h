// Host-side launchers of the operators around the index calls (internal to
// libpivot.so): norm, 4-bit cache, attention over it, eviction.
#pragma once

#include "cache4.h"
#include "pivot.h"

namespace pivot {

constexpr int kNormMaxDim = 32768;

struct NormArgs {
  const void* x;
  int64_t ld_x;
  const void* residual;
  int64_t ld_residual;
  const void* weight;
  float eps;
  int32_t rows, dim, group;
  void* residual_out;
  uint8_t* codes;
  float* scale;
};
hipError_t launch_norm(int dtype, const NormArgs& a, hipStream_t stream);

// Quantise `rows` <= kMaxCacheRows packed tokens into the cache rows of their
// positions (RunTable), and read rows back as bf16, a wave a row.  A launch counts
// its threads in 32 bits, and drops what is above without an error.
constexpr int kMaxCacheRows = 1 << 25;
struct Cache4Write {
  const uint16_t* latent;
  int64_t ld_latent;
  const uint16_t* rope;
  int64_t ld_rope;
  Cache4 cache;
  KeyMap map;
  int32_t rows;
};
hipError_t launch_cache4_write(const Cache4Write& a, const RunTable& t, hipStream_t stream);

struct Cache4Read {
  Cache4 cache;
  KeyMap map;
  int64_t capacity;      // positions past it read as zeros, as negative ones do
  int64_t first;         // of the launch's rows
  const int32_t* idx;    // [batch, n]
  int32_t batch, n;
  uint16_t* out;         // [batch, n, 576]
};
hipError_t launch_cache4_read(const Cache4Read& a, hipStream_t stream);

// Attention of query rows over cached tokens (attend.hip).
struct AttendArgs {
  const uint16_t* q;       // row r, head h at r * q_row + h * q_head
  int64_t q_row, q_head;
  int32_t heads;
  Cache4 cache;
  KeyMap map;
  const int32_t* idx;      // [rows, topk] positions, or nullptr: every position up to the row's own
  int32_t topk;
  float scale;
  uint16_t* out;           // [rows, heads, 512]
  float* lse;              // [rows, heads] or nullptr
  float* acc;              // [sequences, acc_stride] or nullptr
  int64_t acc_stride;
  void* workspace;
};
// Workspace bytes of one launch over the table's sequences.
size_t attend_workspace(const AttendArgs& a, const RunTable& t);
hipError_t launch_attend(const AttendArgs& a, const RunTable& t, hipStream_t stream);

// Which tokens stay (evict.hip): per sequence, the first `sink`, the last
// `recent` and the largest acc of the others, `keep` in all, ascending.
struct EvictArgs {
  const float* acc;
  int64_t acc_stride;
  int32_t keep, sink, recent;
  int32_t* out_keep;  // [sequences, keep], -1 past the kept ones
  float* out_acc;     // [sequences, keep] or nullptr, 0 past the kept ones
};
size_t evict_workspace(const EvictArgs& a, const RunTable& t);
hipError_t launch_evict(const EvictArgs& a, const RunTable& t, void* workspace, hipStream_t stream);

// rows keep[b][j] >= 0 of every array, moved from position keep[b][j] of the
// source map to position j of the destination map.
struct MoveArrays {
  int32_t n;
  const uint8_t* src[PIVOT_EVICT_MAX_ARRAYS];
  uint8_t* dst[PIVOT_EVICT_MAX_ARRAYS];
  int32_t row_bytes[PIVOT_EVICT_MAX_ARRAYS];
};
hipError_t launch_move(const MoveArrays& m, const KeyMap& from, const KeyMap& to, const int32_t* kept, int batch,
                       int keep, hipStream_t stream);

}  // namespace pivot
