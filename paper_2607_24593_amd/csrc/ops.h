// Host-side launchers of the operators around the index calls (internal to
// libpivot.so): norm, 4-bit cache, attention over it, eviction, products with
// 4-bit weights, shared pages.
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
// Rows that are trees of drafted tokens: row r of the launch attends to positions
// below base[b], and to node j of its sequence, at position base[b] + j, where bit
// j mod 32 of word r * words + j / 32 is set.
constexpr int kTreeWords = PIVOT_TREE_MAX_NODES / 32;
struct TreeMask {
  const uint32_t* bits;
  int32_t words;
  int32_t base[kMaxSeq];
};
// Workspace bytes of one launch over the table's sequences, n_k[b] the positions
// that the launch's rows of sequence b may attend to (0 .. n_k[b] - 1).
size_t attend_workspace(const AttendArgs& a, const RunTable& t);
hipError_t launch_attend(const AttendArgs& a, const RunTable& t, const TreeMask* tree, hipStream_t stream);

// Rows of accepted nodes, moved within their arrays: row pos0[b] + path[b][j] of
// sequence b to row pos0[b] + j, up to the first j whose entry is not in
// [j, min(limit - pos0[b], n_rows[b])) or not above the entry before it, or where the
// map has no page for either row.  With acc the weights of the tree's n_rows[b] nodes
// move alike, and those behind the path become 0.
struct AcceptArgs {
  const int32_t* path;  // [sequences, n]
  int32_t n;
  int64_t limit;        // positions of a sequence that the map holds
  KeyMap map;
  int32_t n_arrays;
  uint8_t* rows[PIVOT_EVICT_MAX_ARRAYS];
  int32_t row_bytes[PIVOT_EVICT_MAX_ARRAYS];
  float* acc;           // [sequences, acc_stride], or NULL
  int64_t acc_stride;
};
hipError_t launch_accept(const AcceptArgs& a, const RunTable& t, hipStream_t stream);

// y = x w^T with weights in 4 bits (linear4.hip), at most kLinearRows rows.
constexpr int kLinearRows = 1024;
struct Linear4Args {
  const void* x;
  int64_t ld_x;
  const float* x_scale;
  int32_t x_fp8, group, rows, n, k;
  const uint8_t* codes;
  const uint8_t* scales;
  void* out;
  int64_t ld_out;
  int32_t out_fp32;
};
size_t linear4_workspace(const Linear4Args& a);
hipError_t launch_linear4(const Linear4Args& a, void* workspace, hipStream_t stream);
hipError_t launch_linear4_pack(bool fp32, int32_t n, int32_t k, const void* w, int64_t ld, uint8_t* codes,
                               uint8_t* scales, hipStream_t stream);

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

// Pages that sequences share (pages.hip).
constexpr int kMaxPageList = PIVOT_PAGES_MAX_LIST;
struct Pages {
  int32_t* table;   // [slots, max_pages]
  int32_t* refs;    // [n_pages]
  int32_t max_pages, n_pages, shift;
};
// Entries of a call, passed by value: a fork from slot[i] to slot a[i] of b[i]
// tokens; a growth of slot[i] from a[i] to b[i] tokens; a freeing of slot[i] from
// a[i] tokens to b[i].
struct PageList {
  int32_t n;
  int32_t slot[kMaxPageList], a[kMaxPageList], b[kMaxPageList];
};
struct PageRows {
  int32_t n_pages, shift, n;
  uint8_t* rows[PIVOT_EVICT_MAX_ARRAYS];
  int32_t row_bytes[PIVOT_EVICT_MAX_ARRAYS];
};
hipError_t launch_pages_fork(const Pages& p, const PageList& l, hipStream_t stream);
hipError_t launch_pages_free(const Pages& p, const PageList& l, hipStream_t stream);
size_t pages_grow_workspace(const Pages& p);
hipError_t launch_pages_grow(const Pages& p, const PageList& l, int32_t* pairs, int32_t* state, void* workspace,
                             hipStream_t stream);
size_t pages_compact_workspace(const Pages& p);
hipError_t launch_pages_compact(const Pages& p, int32_t slots, int32_t most, int32_t* pairs, int32_t* state,
                                void* workspace, hipStream_t stream);
hipError_t launch_pages_copy(const PageRows& a, int32_t n, const int32_t* pairs, hipStream_t stream);

}  // namespace pivot
