// C ABI of the operators around the index calls: argument checks, the split of
// a call into launches of at most kMaxSeq sequences, and the launches.
#include <algorithm>
#include <cmath>

#include "ops.h"
#include "status.h"

using namespace pivot;

namespace {

constexpr int kMaxLaunchRows = 16384;                     // query rows per attention launch
constexpr int64_t kScoreBudget = int64_t(1) << 30;        // scores kept at once for the weights
constexpr size_t kAlign = 256;

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A row map over `batch` sequences whose longest holds `longest` rows.
pivot_status check_map(const pivot_row_map& m, int batch, int64_t longest, const char* what) {
  if (m.rows < 1 || m.rows > 0x7FFFFFFF)
    return fail(PIVOT_ERR_INVALID_ARG, "%s: rows=%lld must be in [1, 2^31)", what, (long long)m.rows);
  if (m.block_table) {
    const int P = m.page_size;
    if (P < 16 || P > 65536 || (P & (P - 1)))
      return fail(PIVOT_ERR_INVALID_ARG, "%s: page_size=%d must be a power of two in [16, 65536]", what, P);
    if (m.max_pages < 1) return fail(PIVOT_ERR_INVALID_ARG, "%s: max_pages must be >= 1", what);
    if (m.rows < P || m.rows % P)
      return fail(PIVOT_ERR_INVALID_ARG, "%s: rows=%lld must be a positive multiple of page_size", what,
                  (long long)m.rows);
    if (longest > (int64_t)m.max_pages * P)
      return fail(PIVOT_ERR_INVALID_ARG, "%s: %lld tokens exceed max_pages*page_size", what, (long long)longest);
    return PIVOT_OK;
  }
  if (m.seq_stride < 1) return fail(PIVOT_ERR_INVALID_ARG, "%s: seq_stride must be >= 1", what);
  if (longest > m.seq_stride)
    return fail(PIVOT_ERR_INVALID_ARG, "%s: %lld tokens exceed seq_stride=%lld", what, (long long)longest,
                (long long)m.seq_stride);
  if (m.seq_stride > m.rows || (int64_t)batch > m.rows / m.seq_stride)
    return fail(PIVOT_ERR_INVALID_ARG, "%s: batch * seq_stride exceeds rows=%lld", what, (long long)m.rows);
  return PIVOT_OK;
}

// The kernels' map of sequences b0, b0 + 1, ...: `first` is the row that a
// contiguous map's arrays start at.
KeyMap key_map(const pivot_row_map& m, int b0, int64_t* first) {
  KeyMap k{};
  *first = 0;
  if (m.block_table) {
    k.pages = m.block_table + (int64_t)b0 * m.max_pages;
    k.max_pages = m.max_pages;
    k.shift = __builtin_ctz((unsigned)m.page_size);
    k.n_pages = (int32_t)(m.rows / m.page_size);
  } else {
    k.stride = m.seq_stride;
    *first = (int64_t)b0 * m.seq_stride;
  }
  return k;
}
int64_t capacity(const pivot_row_map& m) {
  return m.block_table ? (int64_t)m.max_pages * m.page_size : m.seq_stride;
}

pivot_status check_cache(const pivot_cache4& c, int batch, int64_t longest) {
  if (!c.codes || !c.scales || !c.rope) return fail(PIVOT_ERR_INVALID_ARG, "cache: codes, scales and rope are required");
  if (!aligned(c.codes, 16) || !aligned(c.scales, 16) || !aligned(c.rope, 16))
    return fail(PIVOT_ERR_INVALID_ARG, "cache: codes, scales and rope must be 16-byte aligned");
  return check_map(c.map, batch, longest, "cache");
}

Cache4 cache_at(const pivot_cache4& c, int64_t row) {
  return Cache4{(uint8_t*)c.codes + row * kCodeBytes, (uint8_t*)c.scales + row * kScaleBytes,
                (uint16_t*)c.rope + row * kRope};
}

// Rows of sequence b of a call (cu: packed runs, or n_q rows each).
int run_rows(const int32_t* cu, int n_q, int b) { return cu ? cu[b + 1] - cu[b] : n_q; }

pivot_status check_runs(int batch, int n_q, const int32_t* cu, const int32_t* pos0, const int32_t* n_k) {
  if (batch < 1) return fail(PIVOT_ERR_INVALID_ARG, "batch must be >= 1");
  if (!pos0) return fail(PIVOT_ERR_INVALID_ARG, "the positions (host array) are required");
  if (cu) {
    if (cu[0] != 0) return fail(PIVOT_ERR_INVALID_ARG, "cu_q[0] must be 0");
    for (int b = 0; b < batch; ++b)
      if (cu[b + 1] < cu[b]) return fail(PIVOT_ERR_INVALID_ARG, "cu_q must be nondecreasing (at %d)", b);
  } else if (n_q < 0) {
    return fail(PIVOT_ERR_INVALID_ARG, "n_q must be >= 0");
  } else if ((int64_t)n_q * batch > 0x7FFFFFFF) {
    return fail(PIVOT_ERR_UNSUPPORTED, "more than 2^31 rows");
  }
  for (int b = 0; b < batch; ++b) {
    const int64_t end = (int64_t)pos0[b] + run_rows(cu, n_q, b);
    if (pos0[b] < 0) return fail(PIVOT_ERR_INVALID_ARG, "position %d of sequence %d is negative", pos0[b], b);
    if (n_k && end > n_k[b])
      return fail(PIVOT_ERR_INVALID_ARG, "n_k[%d]=%d < q_pos0+n_q=%lld", b, n_k[b], (long long)end);
    if (std::max<int64_t>(end, n_k ? n_k[b] : 0) > PIVOT_MAX_KEYS)
      return fail(PIVOT_ERR_UNSUPPORTED, "sequence %d exceeds PIVOT_MAX_KEYS=%d", b, PIVOT_MAX_KEYS);
  }
  return PIVOT_OK;
}

// A call's launches: runs of sequences with at most `most` rows in all (a
// sequence's rows may be cut), `row_limit(b)` of which may be of sequence b
// when the piece is empty.  f(table, first sequence, first packed row).
template <class Cost, class F>
pivot_status for_pieces(int batch, int n_q, const int32_t* cu, const int32_t* pos0, const int32_t* n_k, int most,
                        int64_t budget, Cost cost, F f) {
  int b = 0, done = 0;  // rows [0, done) of sequence b are launched
  int64_t row = 0;
  while (b < batch) {
    RunTable t{};
    const int b0 = b;
    const int64_t row0 = row;
    int rows = 0;
    int64_t left = budget;
    while (b < batch && t.n < kMaxSeq) {
      const int want = run_rows(cu, n_q, b) - done;
      const int64_t each = cost(b);
      int64_t fit = std::min<int64_t>(want, most - rows);
      if (each > 0) fit = std::min<int64_t>(fit, left / each);
      if (fit < 1 && rows == 0 && want > 0) fit = 1;
      const int take = (int)std::max<int64_t>(fit, 0);
      if (take == 0 && want > 0) break;
      const int u = t.n++;
      t.pos0[u] = pos0[b] + done;
      t.n_k[u] = n_k ? n_k[b] : pos0[b] + done + take;
      t.n_rows[u] = take;
      t.row0[u] = rows;
      rows += take;
      row += take;
      left -= each * take;
      if (take < want) {
        done += take;
        break;
      }
      ++b;
      done = 0;
    }
    const pivot_status s = f(t, b0, row0, rows);
    if (s != PIVOT_OK) return s;
  }
  return PIVOT_OK;
}

// The checks of an attention call that concern shapes, not pointers.
pivot_status check_attend_shape(const pivot_attend_args* a) {
  if (!a) return fail(PIVOT_ERR_INVALID_ARG, "args is NULL");
  if (a->heads < 1 || a->heads > PIVOT_ATTEND_MAX_HEADS)
    return fail(PIVOT_ERR_UNSUPPORTED, "heads=%d must be in [1, %d]", a->heads, PIVOT_ATTEND_MAX_HEADS);
  if (!a->n_k) return fail(PIVOT_ERR_INVALID_ARG, "n_k (host array) is required");
  const pivot_status s = check_runs(a->batch, a->n_q, a->cu_q, a->q_pos0, a->n_k);
  if (s != PIVOT_OK) return s;
  if (a->topk < 0 || a->topk > PIVOT_MAX_KEYS) return fail(PIVOT_ERR_INVALID_ARG, "topk=%d", a->topk);
  if (!std::isfinite(a->scale)) return fail(PIVOT_ERR_INVALID_ARG, "scale must be finite");
  return PIVOT_OK;
}

AttendArgs attend_shape(const pivot_attend_args* a) {
  AttendArgs k{};
  k.heads = a->heads;
  k.topk = a->topk;
  k.scale = a->scale;
  k.idx = a->idx;
  k.acc = a->acc;
  return k;
}

// Launches of an attention call; f(launch arguments, table, b0, row0).  The table's
// n_k are the positions that its rows may attend to: up to the last one's own, in a
// tree up to the sequence's last node.
template <class F>
pivot_status attend_pieces(const pivot_attend_args* a, bool tree, F f) {
  const auto cost = [&](int b) -> int64_t {  // bytes of kept scores per query row
    if (!a->acc) return 0;
    const int64_t keys = a->idx ? a->topk : a->n_k[b];
    return (keys + 31) / 32 * 32 * 4 * a->heads;
  };
  return for_pieces(a->batch, a->n_q, a->cu_q, a->q_pos0, a->n_k, kMaxLaunchRows, kScoreBudget, cost,
                    [&](const RunTable& piece, int b0, int64_t row0, int rows) -> pivot_status {
                      if (rows == 0) return PIVOT_OK;
                      RunTable t = piece;
                      for (int u = 0; u < t.n; ++u)
                        t.n_k[u] = tree ? a->q_pos0[b0 + u] + run_rows(a->cu_q, a->n_q, b0 + u) : t.pos0[u] + t.n_rows[u];
                      return f(t, b0, row0);
                    });
}

pivot_status check_tree(const pivot_attend_args* a, const pivot_tree* tree) {
  if (!tree) return fail(PIVOT_ERR_INVALID_ARG, "tree is NULL");
  if (tree->words < 1 || tree->words > kTreeWords)
    return fail(PIVOT_ERR_UNSUPPORTED, "words=%d must be in [1, %d]", tree->words, kTreeWords);
  for (int b = 0; b < a->batch; ++b)
    if (run_rows(a->cu_q, a->n_q, b) > 32 * tree->words)
      return fail(PIVOT_ERR_INVALID_ARG, "sequence %d has %d nodes, a mask %d bits", b, run_rows(a->cu_q, a->n_q, b),
                  32 * tree->words);
  return PIVOT_OK;
}

size_t attend_need(const pivot_attend_args* a, bool tree) {
  size_t need = 0;
  const AttendArgs k = attend_shape(a);
  attend_pieces(a, tree, [&](const RunTable& t, int, int64_t) -> pivot_status {
    need = std::max(need, attend_workspace(k, t));
    return PIVOT_OK;
  });
  return need;
}

// The call with its shapes (and the tree's) checked.
pivot_status attend(const pivot_attend_args* a, const pivot_tree* tree) {
  int64_t rows = 0, longest = 0;
  for (int b = 0; b < a->batch; ++b) {
    rows += run_rows(a->cu_q, a->n_q, b);
    longest = std::max<int64_t>(longest, a->n_k[b]);
  }
  if (rows == 0) return PIVOT_OK;
  const pivot_status s = check_cache(a->cache, a->batch, longest);
  if (s != PIVOT_OK) return s;
  if (!a->q || !a->out) return fail(PIVOT_ERR_INVALID_ARG, "q and out are required");
  if (!aligned(a->q, 16) || !aligned(a->out, 16)) return fail(PIVOT_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (a->q_head_stride < kAttnDim || a->q_head_stride % 8 || a->q_row_stride % 8 ||
      a->q_row_stride < (int64_t)(a->heads - 1) * a->q_head_stride + kAttnDim)
    return fail(PIVOT_ERR_INVALID_ARG, "q strides (%lld, %lld): multiples of 8 values that keep rows apart",
                (long long)a->q_row_stride, (long long)a->q_head_stride);
  if (a->acc && a->acc_stride < longest)
    return fail(PIVOT_ERR_INVALID_ARG, "acc_stride=%lld < %lld tokens", (long long)a->acc_stride, (long long)longest);
  if (tree && (!tree->mask || !aligned(tree->mask, 4)))
    return fail(PIVOT_ERR_INVALID_ARG, "the tree's mask is required, 4-byte aligned");
  const size_t need = attend_need(a, tree != nullptr);
  if (need > 0) {
    if (!a->workspace || a->workspace_bytes < need)
      return fail(PIVOT_ERR_WORKSPACE, "the call needs %zu workspace bytes", need);
    if (!aligned(a->workspace, kAlign)) return fail(PIVOT_ERR_INVALID_ARG, "workspace must be %zu-byte aligned", kAlign);
  }
  return attend_pieces(a, tree != nullptr, [&](const RunTable& t, int b0, int64_t row0) -> pivot_status {
    AttendArgs k = attend_shape(a);
    int64_t first;
    k.map = key_map(a->cache.map, b0, &first);
    k.cache = cache_at(a->cache, first);
    k.q = (const uint16_t*)a->q + row0 * a->q_row_stride;
    k.q_row = a->q_row_stride;
    k.q_head = a->q_head_stride;
    if (a->idx) k.idx = a->idx + row0 * a->topk;
    k.out = (uint16_t*)a->out + row0 * a->heads * kLatent;
    k.lse = a->lse ? a->lse + row0 * a->heads : nullptr;
    k.acc = a->acc ? a->acc + (int64_t)b0 * a->acc_stride : nullptr;
    k.acc_stride = a->acc_stride;
    k.workspace = a->workspace;
    TreeMask m{};
    if (tree) {
      m.bits = tree->mask + row0 * tree->words;
      m.words = tree->words;
      for (int u = 0; u < t.n; ++u) m.base[u] = a->q_pos0[b0 + u];
    }
    return hip_check(launch_attend(k, t, tree ? &m : nullptr, (hipStream_t)a->stream), "attention kernels");
  });
}

pivot_status check_evict_shape(const pivot_evict_args* a) {
  if (!a) return fail(PIVOT_ERR_INVALID_ARG, "args is NULL");
  if (a->batch < 1) return fail(PIVOT_ERR_INVALID_ARG, "batch must be >= 1");
  if (!a->n_k) return fail(PIVOT_ERR_INVALID_ARG, "n_k (host array) is required");
  if (a->keep < 1 || a->sink < 0 || a->recent < 0 || (int64_t)a->sink + a->recent > a->keep)
    return fail(PIVOT_ERR_INVALID_ARG, "keep=%d must be >= 1 and >= sink=%d + recent=%d", a->keep, a->sink, a->recent);
  if (a->keep > PIVOT_MAX_KEYS || (int64_t)a->keep * a->batch > 0x7FFFFFFF)
    return fail(PIVOT_ERR_UNSUPPORTED, "keep=%d of %d sequences", a->keep, a->batch);
  for (int b = 0; b < a->batch; ++b) {
    if (a->n_k[b] < 0) return fail(PIVOT_ERR_INVALID_ARG, "n_k[%d] < 0", b);
    if (a->n_k[b] > PIVOT_MAX_KEYS)
      return fail(PIVOT_ERR_UNSUPPORTED, "n_k[%d]=%d exceeds PIVOT_MAX_KEYS=%d", b, a->n_k[b], PIVOT_MAX_KEYS);
  }
  return PIVOT_OK;
}

EvictArgs evict_shape(const pivot_evict_args* a) {
  EvictArgs k{};
  k.acc_stride = a->acc_stride;
  k.keep = a->keep;
  k.sink = a->sink;
  k.recent = a->recent;
  return k;
}

RunTable evict_table(const pivot_evict_args* a, int b0) {
  RunTable t{};
  t.n = std::min(kMaxSeq, a->batch - b0);
  for (int u = 0; u < t.n; ++u) t.n_k[u] = a->n_k[b0 + u];
  return t;
}

pivot_status check_rows(int n_arrays, const pivot_rows* arrays) {
  if (n_arrays < 1 || n_arrays > PIVOT_EVICT_MAX_ARRAYS || !arrays)
    return fail(PIVOT_ERR_INVALID_ARG, "n_arrays=%d must be in [1, %d]", n_arrays, PIVOT_EVICT_MAX_ARRAYS);
  for (int i = 0; i < n_arrays; ++i) {
    const pivot_rows& r = arrays[i];
    if (!r.rows) return fail(PIVOT_ERR_INVALID_ARG, "array %d: null pointer", i);
    if (r.row_bytes < 4 || r.row_bytes % 4 || !aligned(r.rows, 4))
      return fail(PIVOT_ERR_INVALID_ARG, "array %d: rows of %d bytes (a multiple of 4, 4-byte aligned)", i, r.row_bytes);
  }
  return PIVOT_OK;
}

// nodes: of each tree, where the call has acc, else NULL.
pivot_status accept(int32_t batch, int32_t n, const int32_t* path, const int32_t* pos0, const int32_t* nodes,
                    int32_t n_arrays, const pivot_rows* arrays, const pivot_row_map* map, float* acc, int64_t acc_stride,
                    void* stream) {
  if (batch < 1 || n < 0) return fail(PIVOT_ERR_INVALID_ARG, "batch must be >= 1 and n >= 0");
  if (n > PIVOT_TREE_MAX_NODES) return fail(PIVOT_ERR_UNSUPPORTED, "n=%d exceeds %d nodes", n, PIVOT_TREE_MAX_NODES);
  if (!pos0 || !map) return fail(PIVOT_ERR_INVALID_ARG, "pos0 (host array) and map are required");
  int64_t longest = 0;
  for (int b = 0; b < batch; ++b) {
    if (pos0[b] < 0) return fail(PIVOT_ERR_INVALID_ARG, "position %d of sequence %d is negative", pos0[b], b);
    if (nodes && nodes[b] < 0) return fail(PIVOT_ERR_INVALID_ARG, "%d nodes of sequence %d", nodes[b], b);
    if (nodes && nodes[b] > PIVOT_TREE_MAX_NODES)
      return fail(PIVOT_ERR_UNSUPPORTED, "%d nodes of sequence %d exceed %d", nodes[b], b, PIVOT_TREE_MAX_NODES);
    const int64_t end = (int64_t)pos0[b] + (nodes ? nodes[b] : 0);
    if (end > PIVOT_MAX_KEYS) return fail(PIVOT_ERR_UNSUPPORTED, "sequence %d exceeds PIVOT_MAX_KEYS=%d", b, PIVOT_MAX_KEYS);
    longest = std::max(longest, end);
  }
  if (acc && acc_stride < longest)
    return fail(PIVOT_ERR_INVALID_ARG, "acc_stride=%lld < %lld tokens", (long long)acc_stride, (long long)longest);
  pivot_status s = check_map(*map, batch, longest, "map");
  if (s != PIVOT_OK) return s;
  s = check_rows(n_arrays, arrays);
  if (s != PIVOT_OK || (n == 0 && !acc)) return s;
  if (n > 0 && (!path || !aligned(path, 4))) return fail(PIVOT_ERR_INVALID_ARG, "path is required, 4-byte aligned");
  for (int b0 = 0; b0 < batch; b0 += kMaxSeq) {
    RunTable t{};
    t.n = std::min(kMaxSeq, batch - b0);
    for (int u = 0; u < t.n; ++u) {
      t.pos0[u] = pos0[b0 + u];
      t.n_rows[u] = nodes ? nodes[b0 + u] : 0x7FFFFFFF;
    }
    AcceptArgs k{};
    int64_t first;
    k.path = path + (int64_t)b0 * n;
    k.n = n;
    k.limit = capacity(*map);
    k.map = key_map(*map, b0, &first);
    k.n_arrays = n_arrays;
    for (int i = 0; i < n_arrays; ++i) {
      k.rows[i] = (uint8_t*)arrays[i].rows + first * arrays[i].row_bytes;
      k.row_bytes[i] = arrays[i].row_bytes;
    }
    k.acc = acc ? acc + (int64_t)b0 * acc_stride : nullptr;
    k.acc_stride = acc_stride;
    s = hip_check(launch_accept(k, t, (hipStream_t)stream), "accept kernel");
    if (s != PIVOT_OK) return s;
  }
  return PIVOT_OK;
}

pivot_status check_pages(const pivot_pages* p) {
  if (!p) return fail(PIVOT_ERR_INVALID_ARG, "pages is NULL");
  const int P = p->page_size;
  if (P < 16 || P > 65536 || (P & (P - 1)))
    return fail(PIVOT_ERR_INVALID_ARG, "page_size=%d must be a power of two in [16, 65536]", P);
  if (p->slots < 1 || p->max_pages < 1 || (int64_t)p->slots * p->max_pages > 0x7FFFFFFF)
    return fail(PIVOT_ERR_INVALID_ARG, "a table of %d slots x %d pages", p->slots, p->max_pages);
  if (p->n_pages < 1 || (int64_t)p->n_pages * P > 0x7FFFFFFF)
    return fail(PIVOT_ERR_INVALID_ARG, "a pool of %d pages", p->n_pages);
  return PIVOT_OK;
}
pivot_status check_pool(const pivot_pages* p) {
  if (!p->table || !p->refs || !aligned(p->table, 4) || !aligned(p->refs, 4))
    return fail(PIVOT_ERR_INVALID_ARG, "table and refs are required, 4-byte aligned");
  return PIVOT_OK;
}

pivot_status check_list(const pivot_pages* p, int n) {
  const pivot_status s = check_pages(p);
  if (s != PIVOT_OK) return s;
  if (n < 0) return fail(PIVOT_ERR_INVALID_ARG, "n must be >= 0");
  if (n > PIVOT_PAGES_MAX_LIST) return fail(PIVOT_ERR_UNSUPPORTED, "n=%d exceeds %d", n, PIVOT_PAGES_MAX_LIST);
  return PIVOT_OK;
}
// Which slots a list holds: as bits while they fit (a sort of 160 entries takes 3 us),
// else sorted.
struct SlotSet {
  static constexpr int kBits = 1 << 15;
  uint64_t bits[kBits / 64];
  int32_t sorted[PIVOT_PAGES_MAX_LIST];
  int n;
  bool small;
  // False, and the slot, if one comes twice.
  bool fill(const pivot_pages* p, int count, const int32_t* slot, int32_t* twice) {
    n = count;
    small = p->slots <= kBits;
    if (small) {
      std::fill(bits, bits + (p->slots + 63) / 64, 0);
      for (int i = 0; i < n; ++i) {
        uint64_t& word = bits[slot[i] >> 6];
        const uint64_t bit = uint64_t(1) << (slot[i] & 63);
        if (word & bit) return *twice = slot[i], false;
        word |= bit;
      }
      return true;
    }
    std::copy(slot, slot + n, sorted);
    std::sort(sorted, sorted + n);
    for (int i = 1; i < n; ++i)
      if (sorted[i] == sorted[i - 1]) return *twice = sorted[i], false;
    return true;
  }
  bool holds(int32_t slot) const {
    return small ? bits[slot >> 6] >> (slot & 63) & 1 : std::binary_search(sorted, sorted + n, slot);
  }
};
pivot_status check_slots(const pivot_pages* p, int n, const int32_t* slot, SlotSet* distinct, const char* what) {
  if (!slot) return fail(PIVOT_ERR_INVALID_ARG, "%s (host array) is required", what);
  for (int i = 0; i < n; ++i)
    if (slot[i] < 0 || slot[i] >= p->slots) return fail(PIVOT_ERR_INVALID_ARG, "%s[%d]=%d of %d", what, i, slot[i], p->slots);
  int32_t twice = 0;
  if (distinct && !distinct->fill(p, n, slot, &twice)) return fail(PIVOT_ERR_INVALID_ARG, "%s holds slot %d twice", what, twice);
  return PIVOT_OK;
}
// 0 <= low[i] <= high[i] <= what a slot can hold (low NULL: 0).
pivot_status check_tokens(const pivot_pages* p, int n, const int32_t* low, const int32_t* high) {
  if (!high) return fail(PIVOT_ERR_INVALID_ARG, "the numbers of tokens (host arrays) are required");
  for (int i = 0; i < n; ++i) {
    if ((low && low[i] < 0) || high[i] < (low ? low[i] : 0))
      return fail(PIVOT_ERR_INVALID_ARG, "entry %d: %d and %d tokens", i, low ? low[i] : 0, high[i]);
    if (high[i] > (int64_t)p->max_pages * p->page_size)
      return fail(PIVOT_ERR_INVALID_ARG, "entry %d: %d tokens exceed max_pages*page_size", i, high[i]);
    if (high[i] > PIVOT_MAX_KEYS)
      return fail(PIVOT_ERR_UNSUPPORTED, "entry %d: %d tokens exceed PIVOT_MAX_KEYS=%d", i, high[i], PIVOT_MAX_KEYS);
  }
  return PIVOT_OK;
}

// The pages that a growth takes are counted in 32 bits.
pivot_status check_growth(const pivot_pages* p, int n, const int32_t* tokens, const int32_t* new_tokens) {
  const pivot_status s = check_tokens(p, n, tokens, new_tokens);
  if (s != PIVOT_OK) return s;
  int64_t want = 0;
  for (int i = 0; i < n; ++i) want += (int64_t)(new_tokens[i] - tokens[i]) / p->page_size + 2;
  if (want > (1 << 30)) return fail(PIVOT_ERR_UNSUPPORTED, "growth by %lld pages", (long long)want);
  return PIVOT_OK;
}

Pages pages_at(const pivot_pages* p) {
  return Pages{p->table, p->refs, p->max_pages, p->n_pages, __builtin_ctz((unsigned)p->page_size)};
}
PageList page_list(int n, const int32_t* slot, const int32_t* a, const int32_t* b) {
  PageList l{};
  l.n = n;
  std::copy(slot, slot + n, l.slot);
  std::copy(a, a + n, l.a);
  std::copy(b, b + n, l.b);
  return l;
}
// The checks of a product that concern shapes, not pointers.
pivot_status check_linear4(const pivot_linear4_args* a) {
  if (!a) return fail(PIVOT_ERR_INVALID_ARG, "args is NULL");
  if (a->x_dtype != PIVOT_DT_BF16 && a->x_dtype != PIVOT_DT_FP8_E4M3)
    return fail(PIVOT_ERR_UNSUPPORTED, "x_dtype %d: bf16 or fp8", a->x_dtype);
  if (a->out_dtype != PIVOT_DT_BF16 && a->out_dtype != PIVOT_DT_FP32)
    return fail(PIVOT_ERR_UNSUPPORTED, "out_dtype %d: bf16 or fp32", a->out_dtype);
  if (a->n_rows < 0 || a->n < 0) return fail(PIVOT_ERR_INVALID_ARG, "n_rows and n must be >= 0");
  if (a->n > PIVOT_LINEAR4_MAX_N) return fail(PIVOT_ERR_UNSUPPORTED, "n=%d exceeds %d", a->n, PIVOT_LINEAR4_MAX_N);
  if (a->k < 1) return fail(PIVOT_ERR_INVALID_ARG, "k must be >= 1");
  if (a->k % kBlk || a->k > PIVOT_LINEAR4_MAX_K)
    return fail(PIVOT_ERR_UNSUPPORTED, "k=%d must be a multiple of %d up to %d", a->k, kBlk, PIVOT_LINEAR4_MAX_K);
  if (a->group != 0 && (a->group != 128 || a->x_dtype != PIVOT_DT_FP8_E4M3))
    return fail(PIVOT_ERR_UNSUPPORTED, "group=%d: 0 (the row), or 128 with fp8", a->group);
  if (a->ld_x < a->k || a->ld_out < a->n)
    return fail(PIVOT_ERR_INVALID_ARG, "rows overlap (ld_x=%lld, ld_out=%lld)", (long long)a->ld_x, (long long)a->ld_out);
  return PIVOT_OK;
}

// Launches of a product: f(arguments of at most kLinearRows rows, its first row).
template <class F>
pivot_status linear4_pieces(const pivot_linear4_args* a, F f) {
  Linear4Args k{};
  k.ld_x = a->ld_x;
  k.x_fp8 = a->x_dtype == PIVOT_DT_FP8_E4M3;
  k.group = a->group;
  k.n = a->n;
  k.k = a->k;
  k.codes = (const uint8_t*)a->codes;
  k.scales = (const uint8_t*)a->scales;
  k.ld_out = a->ld_out;
  k.out_fp32 = a->out_dtype == PIVOT_DT_FP32;
  for (int64_t r = 0; r < a->n_rows && a->n > 0; r += kLinearRows) {
    k.rows = (int32_t)std::min<int64_t>(kLinearRows, a->n_rows - r);
    const pivot_status s = f(k, r);
    if (s != PIVOT_OK) return s;
  }
  return PIVOT_OK;
}

}  // namespace

extern "C" {

pivot_status pivot_rmsnorm_fp8(int32_t dtype, int32_t n_rows, int32_t dim, const void* x, int64_t ld_x,
                               const void* residual, int64_t ld_residual, const void* weight, float eps, int32_t group,
                               void* residual_out, uint8_t* codes, float* scale, void* stream) {
  if (dtype != PIVOT_DT_BF16 && dtype != PIVOT_DT_FP32)
    return fail(PIVOT_ERR_UNSUPPORTED, "dtype %d: x is bf16 or fp32", dtype);
  if (n_rows < 0) return fail(PIVOT_ERR_INVALID_ARG, "n_rows must be >= 0");
  if (dim < 1) return fail(PIVOT_ERR_INVALID_ARG, "dim must be >= 1");
  if (dim > kNormMaxDim) return fail(PIVOT_ERR_UNSUPPORTED, "dim=%d exceeds %d", dim, kNormMaxDim);
  if (group != 0 && group != 128) return fail(PIVOT_ERR_UNSUPPORTED, "group=%d: 0 (the row) or 128", group);
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(PIVOT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (ld_x < dim || (residual && ld_residual < dim))
    return fail(PIVOT_ERR_INVALID_ARG, "rows of %d values overlap (ld_x=%lld, ld_residual=%lld)", dim, (long long)ld_x,
                (long long)ld_residual);
  if (n_rows == 0) return PIVOT_OK;
  if (!x || !weight || !codes || !scale) return fail(PIVOT_ERR_INVALID_ARG, "x, weight, codes and scale are required");
  const uintptr_t e = dtype == PIVOT_DT_BF16 ? 2 : 4;
  if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, e) || !aligned(residual_out, e) || !aligned(scale, 4))
    return fail(PIVOT_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
  // a padded row's sums would land on other rows that are still to be read
  if (residual_out && n_rows > 1 && ((residual_out == x && ld_x != dim) || (residual_out == residual && ld_residual != dim)))
    return fail(PIVOT_ERR_INVALID_ARG, "residual_out may only be an input whose rows are not padded");
  const NormArgs a{x, ld_x, residual, ld_residual, weight, eps, n_rows, dim, group, residual_out, codes, scale};
  return hip_check(launch_norm(dtype, a, (hipStream_t)stream), "norm kernel");
}

pivot_status pivot_cache4_write(const pivot_cache4* c, int32_t batch, int32_t n_new, const int32_t* cu,
                                const int32_t* pos0, const void* latent, int64_t ld_latent, const void* rope,
                                int64_t ld_rope, void* stream) {
  if (!c) return fail(PIVOT_ERR_INVALID_ARG, "cache is NULL");
  pivot_status s = check_runs(batch, n_new, cu, pos0, nullptr);
  if (s != PIVOT_OK) return s;
  int64_t longest = 0, rows = 0;
  for (int b = 0; b < batch; ++b) {
    const int n = run_rows(cu, n_new, b);
    rows += n;
    if (n) longest = std::max<int64_t>(longest, (int64_t)pos0[b] + n);
  }
  if (rows == 0) return PIVOT_OK;
  s = check_cache(*c, batch, longest);
  if (s != PIVOT_OK) return s;
  if (!latent || !rope) return fail(PIVOT_ERR_INVALID_ARG, "latent and rope are required");
  if (!aligned(latent, 2) || !aligned(rope, 2)) return fail(PIVOT_ERR_INVALID_ARG, "latent and rope hold bf16 values");
  if (ld_latent < kLatent || ld_rope < kRope)
    return fail(PIVOT_ERR_INVALID_ARG, "rows overlap (ld_latent=%lld, ld_rope=%lld)", (long long)ld_latent,
                (long long)ld_rope);
  return for_pieces(batch, n_new, cu, pos0, nullptr, kMaxCacheRows, 0, [](int) -> int64_t { return 0; },
                    [&](const RunTable& t, int b0, int64_t row0, int n) -> pivot_status {
                      if (n == 0) return PIVOT_OK;
                      int64_t first;
                      const KeyMap map = key_map(c->map, b0, &first);
                      const Cache4Write w{(const uint16_t*)latent + row0 * ld_latent, ld_latent,
                                          (const uint16_t*)rope + row0 * ld_rope, ld_rope, cache_at(*c, first), map, n};
                      return hip_check(launch_cache4_write(w, t, (hipStream_t)stream), "cache write kernel");
                    });
}

pivot_status pivot_cache4_read(const pivot_cache4* c, int32_t batch, int32_t n, const int32_t* idx, void* out,
                               void* stream) {
  if (!c) return fail(PIVOT_ERR_INVALID_ARG, "cache is NULL");
  if (batch < 1 || n < 0) return fail(PIVOT_ERR_INVALID_ARG, "batch must be >= 1 and n >= 0");
  if ((int64_t)batch * n > 0x7FFFFFFF) return fail(PIVOT_ERR_UNSUPPORTED, "more than 2^31 rows");
  if (n == 0) return PIVOT_OK;
  const pivot_status s = check_cache(*c, batch, 0);
  if (s != PIVOT_OK) return s;
  if (!idx || !out) return fail(PIVOT_ERR_INVALID_ARG, "idx and out are required");
  if (!aligned(out, 16)) return fail(PIVOT_ERR_INVALID_ARG, "out must be 16-byte aligned");
  int64_t first;
  const KeyMap map = key_map(c->map, 0, &first);
  const Cache4Read r{cache_at(*c, first), map, capacity(c->map), 0, idx, batch, n, (uint16_t*)out};
  return hip_check(launch_cache4_read(r, (hipStream_t)stream), "cache read kernel");
}

size_t pivot_cache4_attend_workspace_size(const pivot_attend_args* a) {
  return check_attend_shape(a) == PIVOT_OK ? attend_need(a, false) : 0;
}

pivot_status pivot_cache4_attend(const pivot_attend_args* a) {
  const pivot_status s = check_attend_shape(a);
  return s == PIVOT_OK ? attend(a, nullptr) : s;
}

size_t pivot_cache4_attend_tree_workspace_size(const pivot_attend_args* a, const pivot_tree* t) {
  return check_attend_shape(a) == PIVOT_OK && check_tree(a, t) == PIVOT_OK ? attend_need(a, true) : 0;
}

pivot_status pivot_cache4_attend_tree(const pivot_attend_args* a, const pivot_tree* t) {
  pivot_status s = check_attend_shape(a);
  if (s == PIVOT_OK) s = check_tree(a, t);
  return s == PIVOT_OK ? attend(a, t) : s;
}

pivot_status pivot_tree_accept(int32_t batch, int32_t n, const int32_t* path, const int32_t* pos0, int32_t n_arrays,
                               const pivot_rows* arrays, const pivot_row_map* map, void* stream) {
  return accept(batch, n, path, pos0, nullptr, n_arrays, arrays, map, nullptr, 0, stream);
}

pivot_status pivot_tree_accept_acc(int32_t batch, int32_t n, const int32_t* path, const int32_t* pos0,
                                   const int32_t* nodes, int32_t n_arrays, const pivot_rows* arrays,
                                   const pivot_row_map* map, float* acc, int64_t acc_stride, void* stream) {
  if (!nodes) return fail(PIVOT_ERR_INVALID_ARG, "nodes (host array) is required");
  if (!acc || !aligned(acc, 4)) return fail(PIVOT_ERR_INVALID_ARG, "acc is required, 4-byte aligned");
  return accept(batch, n, path, pos0, nodes, n_arrays, arrays, map, acc, acc_stride, stream);
}

size_t pivot_evict_workspace_size(const pivot_evict_args* a) {
  if (check_evict_shape(a) != PIVOT_OK) return 0;
  size_t need = 0;
  const EvictArgs k = evict_shape(a);
  for (int b0 = 0; b0 < a->batch; b0 += kMaxSeq) need = std::max(need, evict_workspace(k, evict_table(a, b0)));
  return need;
}

pivot_status pivot_evict(const pivot_evict_args* a) {
  pivot_status s = check_evict_shape(a);
  if (s != PIVOT_OK) return s;
  int64_t longest = 0;
  for (int b = 0; b < a->batch; ++b) longest = std::max<int64_t>(longest, a->n_k[b]);
  if (!a->acc || !a->out_keep) return fail(PIVOT_ERR_INVALID_ARG, "acc and out_keep are required");
  if (a->acc_stride < longest)
    return fail(PIVOT_ERR_INVALID_ARG, "acc_stride=%lld < %lld tokens", (long long)a->acc_stride, (long long)longest);
  if (a->n_arrays < 0 || a->n_arrays > PIVOT_EVICT_MAX_ARRAYS)
    return fail(PIVOT_ERR_INVALID_ARG, "n_arrays=%d must be in [0, %d]", a->n_arrays, PIVOT_EVICT_MAX_ARRAYS);
  if (a->n_arrays > 0) {
    s = check_map(a->from, a->batch, longest, "from");
    if (s != PIVOT_OK) return s;
    s = check_map(a->to, a->batch, std::min<int64_t>(a->keep, longest), "to");
    if (s != PIVOT_OK) return s;
  }
  for (int i = 0; i < a->n_arrays; ++i) {
    const pivot_move& m = a->arrays[i];
    if (!m.src || !m.dst) return fail(PIVOT_ERR_INVALID_ARG, "array %d: null pointer", i);
    if (m.row_bytes < 4 || m.row_bytes % 4 || !aligned(m.src, 4) || !aligned(m.dst, 4))
      return fail(PIVOT_ERR_INVALID_ARG, "array %d: rows of %d bytes (a multiple of 4, 4-byte aligned)", i, m.row_bytes);
    if (m.src == m.dst && !(a->from.block_table && a->to.block_table))
      return fail(PIVOT_ERR_INVALID_ARG, "array %d: rows move within one array only between pages", i);
  }
  const size_t need = pivot_evict_workspace_size(a);
  if (need > 0) {
    if (!a->workspace || a->workspace_bytes < need)
      return fail(PIVOT_ERR_WORKSPACE, "the call needs %zu workspace bytes", need);
    if (!aligned(a->workspace, kAlign)) return fail(PIVOT_ERR_INVALID_ARG, "workspace must be %zu-byte aligned", kAlign);
  }
  for (int b0 = 0; b0 < a->batch; b0 += kMaxSeq) {
    EvictArgs k = evict_shape(a);
    k.acc = a->acc + (int64_t)b0 * a->acc_stride;
    k.out_keep = a->out_keep + (int64_t)b0 * a->keep;
    k.out_acc = a->out_acc ? a->out_acc + (int64_t)b0 * a->keep : nullptr;
    s = hip_check(launch_evict(k, evict_table(a, b0), a->workspace, (hipStream_t)a->stream), "evict kernel");
    if (s != PIVOT_OK) return s;
  }
  if (a->n_arrays == 0) return PIVOT_OK;
  int64_t from0, to0;
  MoveArrays m{};
  const KeyMap from = key_map(a->from, 0, &from0), to = key_map(a->to, 0, &to0);
  m.n = a->n_arrays;
  for (int i = 0; i < m.n; ++i) {
    m.src[i] = (const uint8_t*)a->arrays[i].src;
    m.dst[i] = (uint8_t*)a->arrays[i].dst;
    m.row_bytes[i] = a->arrays[i].row_bytes;
  }
  return hip_check(launch_move(m, from, to, a->out_keep, a->batch, a->keep, (hipStream_t)a->stream), "move kernel");
}

size_t pivot_linear4_workspace_size(const pivot_linear4_args* a) {
  if (check_linear4(a) != PIVOT_OK) return 0;
  size_t need = 0;
  linear4_pieces(a, [&](const Linear4Args& k, int64_t) -> pivot_status {
    need = std::max(need, linear4_workspace(k));
    return PIVOT_OK;
  });
  return need;
}

pivot_status pivot_linear4(const pivot_linear4_args* a) {
  const pivot_status s = check_linear4(a);
  if (s != PIVOT_OK) return s;
  if (a->n_rows == 0 || a->n == 0) return PIVOT_OK;
  const bool fp8 = a->x_dtype == PIVOT_DT_FP8_E4M3, fp32 = a->out_dtype == PIVOT_DT_FP32;
  if (!a->x || !a->codes || !a->scales || !a->out || (fp8 && !a->x_scale))
    return fail(PIVOT_ERR_INVALID_ARG, "x, codes, scales, out and fp8's x_scale are required");
  if (!aligned(a->codes, 16)) return fail(PIVOT_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  if ((!fp8 && !aligned(a->x, 2)) || (fp8 && !aligned(a->x_scale, 4)) || !aligned(a->out, fp32 ? 4 : 2))
    return fail(PIVOT_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
  const size_t need = pivot_linear4_workspace_size(a);
  if (need > 0) {
    if (!a->workspace || a->workspace_bytes < need)
      return fail(PIVOT_ERR_WORKSPACE, "the call needs %zu workspace bytes", need);
    if (!aligned(a->workspace, kAlign)) return fail(PIVOT_ERR_INVALID_ARG, "workspace must be %zu-byte aligned", kAlign);
  }
  return linear4_pieces(a, [&](Linear4Args k, int64_t r) -> pivot_status {
    const int64_t scales = a->group ? (a->k + 127) / 128 : 1;
    k.x = (const uint8_t*)a->x + r * a->ld_x * (fp8 ? 1 : 2);
    k.x_scale = fp8 ? a->x_scale + r * scales : nullptr;
    k.out = (uint8_t*)a->out + r * a->ld_out * (fp32 ? 4 : 2);
    return hip_check(launch_linear4(k, a->workspace, (hipStream_t)a->stream), "linear kernels");
  });
}

pivot_status pivot_linear4_pack(int32_t dtype, int32_t n, int32_t k, const void* w, int64_t ld_w, void* codes,
                                void* scales, void* stream) {
  if (dtype != PIVOT_DT_BF16 && dtype != PIVOT_DT_FP32)
    return fail(PIVOT_ERR_UNSUPPORTED, "dtype %d: weights are bf16 or fp32", dtype);
  if (n < 0 || k < 1) return fail(PIVOT_ERR_INVALID_ARG, "n must be >= 0 and k >= 1");
  if (k % kBlk || k > PIVOT_LINEAR4_MAX_K)
    return fail(PIVOT_ERR_UNSUPPORTED, "k=%d must be a multiple of %d up to %d", k, kBlk, PIVOT_LINEAR4_MAX_K);
  if (ld_w < k) return fail(PIVOT_ERR_INVALID_ARG, "rows overlap (ld_w=%lld)", (long long)ld_w);
  if (n == 0) return PIVOT_OK;
  if (!w || !codes || !scales) return fail(PIVOT_ERR_INVALID_ARG, "w, codes and scales are required");
  if (!aligned(w, dtype == PIVOT_DT_BF16 ? 2 : 4) || !aligned(codes, 4))
    return fail(PIVOT_ERR_INVALID_ARG, "w must be aligned to its elements, codes to 4 bytes");
  return hip_check(launch_linear4_pack(dtype == PIVOT_DT_FP32, n, k, w, ld_w, (uint8_t*)codes, (uint8_t*)scales,
                                       (hipStream_t)stream),
                   "pack kernel");
}

pivot_status pivot_pages_fork(const pivot_pages* p, int32_t n, const int32_t* src, const int32_t* dst,
                              const int32_t* tokens, void* stream) {
  pivot_status s = check_list(p, n);
  if (s != PIVOT_OK) return s;
  if (n == 0) return PIVOT_OK;
  SlotSet slots;
  if ((s = check_slots(p, n, src, nullptr, "src")) != PIVOT_OK) return s;
  if ((s = check_slots(p, n, dst, &slots, "dst")) != PIVOT_OK) return s;
  for (int i = 0; i < n; ++i)
    if (slots.holds(src[i]))
      return fail(PIVOT_ERR_INVALID_ARG, "slot %d is both src and dst", src[i]);
  if ((s = check_tokens(p, n, nullptr, tokens)) != PIVOT_OK) return s;
  if ((s = check_pool(p)) != PIVOT_OK) return s;
  return hip_check(launch_pages_fork(pages_at(p), page_list(n, src, dst, tokens), (hipStream_t)stream), "fork kernel");
}

pivot_status pivot_pages_free(const pivot_pages* p, int32_t n, const int32_t* slot, const int32_t* tokens,
                              const int32_t* keep, void* stream) {
  pivot_status s = check_list(p, n);
  if (s != PIVOT_OK) return s;
  if (n == 0) return PIVOT_OK;
  SlotSet slots;
  if ((s = check_slots(p, n, slot, &slots, "slot")) != PIVOT_OK) return s;
  if (!keep) return fail(PIVOT_ERR_INVALID_ARG, "the numbers of tokens (host arrays) are required");
  if ((s = check_tokens(p, n, keep, tokens)) != PIVOT_OK) return s;
  if ((s = check_pool(p)) != PIVOT_OK) return s;
  return hip_check(launch_pages_free(pages_at(p), page_list(n, slot, tokens, keep), (hipStream_t)stream), "free kernel");
}

size_t pivot_pages_grow_workspace_size(const pivot_pages* p, int32_t n, const int32_t* tokens, const int32_t* new_tokens) {
  if (check_list(p, n) != PIVOT_OK || n == 0 || !tokens || check_growth(p, n, tokens, new_tokens) != PIVOT_OK) return 0;
  return pages_grow_workspace(pages_at(p));
}

pivot_status pivot_pages_grow(const pivot_pages* p, int32_t n, const int32_t* slot, const int32_t* tokens,
                              const int32_t* new_tokens, int32_t* copies, int32_t* state, void* workspace,
                              size_t workspace_bytes, void* stream) {
  pivot_status s = check_list(p, n);
  if (s != PIVOT_OK) return s;
  if (n == 0) return fail(PIVOT_ERR_INVALID_ARG, "n must be >= 1");
  SlotSet slots;
  if ((s = check_slots(p, n, slot, &slots, "slot")) != PIVOT_OK) return s;
  if (!tokens) return fail(PIVOT_ERR_INVALID_ARG, "the numbers of tokens (host arrays) are required");
  if ((s = check_growth(p, n, tokens, new_tokens)) != PIVOT_OK) return s;
  if ((s = check_pool(p)) != PIVOT_OK) return s;
  if (!copies || !state || !aligned(copies, 4) || !aligned(state, 4))
    return fail(PIVOT_ERR_INVALID_ARG, "copies and state are required, 4-byte aligned");
  const size_t need = pivot_pages_grow_workspace_size(p, n, tokens, new_tokens);
  if (!workspace || workspace_bytes < need) return fail(PIVOT_ERR_WORKSPACE, "the call needs %zu workspace bytes", need);
  if (!aligned(workspace, kAlign)) return fail(PIVOT_ERR_INVALID_ARG, "workspace must be %zu-byte aligned", kAlign);
  return hip_check(launch_pages_grow(pages_at(p), page_list(n, slot, tokens, new_tokens), copies, state, workspace,
                                     (hipStream_t)stream),
                   "grow kernels");
}

size_t pivot_pages_compact_workspace_size(const pivot_pages* p) {
  return check_pages(p) == PIVOT_OK ? pages_compact_workspace(pages_at(p)) : 0;
}

pivot_status pivot_pages_compact(const pivot_pages* p, int32_t max_moves, int32_t* moves, int32_t* state, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  pivot_status s = check_pages(p);
  if (s != PIVOT_OK) return s;
  if (max_moves < 0) return fail(PIVOT_ERR_INVALID_ARG, "max_moves must be >= 0");
  if ((s = check_pool(p)) != PIVOT_OK) return s;
  if (!state || (!moves && max_moves > 0) || !aligned(moves, 4) || !aligned(state, 4))
    return fail(PIVOT_ERR_INVALID_ARG, "moves and state are required, 4-byte aligned");
  const size_t need = pivot_pages_compact_workspace_size(p);
  if (!workspace || workspace_bytes < need) return fail(PIVOT_ERR_WORKSPACE, "the call needs %zu workspace bytes", need);
  if (!aligned(workspace, kAlign)) return fail(PIVOT_ERR_INVALID_ARG, "workspace must be %zu-byte aligned", kAlign);
  return hip_check(launch_pages_compact(pages_at(p), p->slots, max_moves, moves, state, workspace, (hipStream_t)stream),
                   "compact kernels");
}

pivot_status pivot_pages_copy(const pivot_pages* p, int32_t n, const int32_t* pairs, int32_t n_arrays,
                              const pivot_rows* arrays, void* stream) {
  pivot_status s = check_pages(p);
  if (s != PIVOT_OK) return s;
  if (n < 0) return fail(PIVOT_ERR_INVALID_ARG, "n must be >= 0");
  if ((s = check_rows(n_arrays, arrays)) != PIVOT_OK || n == 0) return s;
  if (!pairs || !aligned(pairs, 4)) return fail(PIVOT_ERR_INVALID_ARG, "pairs is required, 4-byte aligned");
  PageRows k{};
  k.n_pages = p->n_pages;
  k.shift = __builtin_ctz((unsigned)p->page_size);
  k.n = n_arrays;
  for (int i = 0; i < n_arrays; ++i) {
    k.rows[i] = (uint8_t*)arrays[i].rows;
    k.row_bytes[i] = arrays[i].row_bytes;
  }
  return hip_check(launch_pages_copy(k, n, pairs, (hipStream_t)stream), "copy kernel");
}

}  // extern "C"
