// Declarations shared by the host entry points of the pages (pages_api.cpp,
// hermes_api.cpp) and their kernels (pages.hip, page_attention.hip).
#pragma once

#include "hermes_internal.h"

namespace hermes {

// A pool as the kernels see it.
struct PagePool {
  uint8_t *pages;
  int32_t *status;          // or null
  int64_t page_bytes;
  int32_t block_bytes;      // of one KV head's block in a page
  int32_t log_rows;         // page_rows = 1 << log_rows
  int32_t n_pages;
  int32_t Hq, Hkv;
};

// A call's sequences, as in hermes_page_batch.
struct PageSeqs {
  const int32_t *row_start, *kv_len, *tables;
  int32_t n_seqs, n_rows, max_pages;
};

struct PageAppendArgs {
  PagePool pool;
  PageSeqs seqs;
  const uint16_t *q, *k, *v;
  uint16_t *q_out;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *rope;      // [axes][n_rows], or null: k as it is
  int32_t axes;
  int32_t section[3];       // axes 3: frequency pairs of the t, h, w sections
  int32_t share;            // waves that share a row: 1 or 4
  double inv_freq[kMaxHalfDim];
};

struct PageReadArgs {
  PagePool pool;
  PageSeqs seqs;
  uint16_t *k, *v;          // [n_rows][Hkv][d], either may be null
};

struct PagePackArgs {
  PagePool pool;
  const int32_t *tables;    // [n_list][max_pages]
  int32_t *kv_len;          // [n_list]
  int32_t max_pages, n_list;
  const uint16_t *k[kMaxLayers], *v[kMaxLayers];
  int32_t len[kMaxLayers];
};

// How an attention call is cut.  An item is a tile of `rows` packed rows (row, query
// head of the KV head) of one (sequence, KV head), against all keys its rows see.
// The items, in order, are cut into `units` runs of equal cost, a workgroup each, at
// least `step` keys long: the lengths are on the device, so the kernel finds its run.
// Where cuts would save less than they cost, there are none (`tiles` > 0): every pair
// has `tiles` units, each for a tile (for more, if the pair has more tiles than that).
// rows of 16 and 32 take page_attn_few, more page_attn_many.
struct PagePlan {
  int32_t rows, units, step, tiles;
  int32_t item_keys;        // what an item's start and end cost, in keys
  double inv_units, inv_group;   // 1 / units, 1 / (query heads of a KV head)
};

// What page_combine has to know of a cut item, written by the unit that holds its
// first cut: the units that have parts of it, its first packed row and its rows.
struct PageCut {
  int32_t first, last;      // units (last < first: no item is first cut here)
  int32_t slot;             // of the first unit's part: 0 or 1 (the others: 0)
  int32_t kv, r0;           // KV head, first stacked row of the sequence
  int32_t p0, P;            // the item's first packed row, the sequence's packed rows
  int32_t pad_;
};

struct PageAttnArgs {
  PagePool pool;
  PageSeqs seqs;
  const uint16_t *q;
  int64_t q_stride;
  uint16_t *out;            // [n_rows][Hq][d]
  float *lse;               // [n_rows][Hq] or null
  float scale_log2;         // sm_scale * log2(e)
  PagePlan plan;
  // Parts of cut items: unit u has two, 2 u for the item it starts with and 2 u + 1
  // for the one it ends with, each rows x d fp32 (unnormalised O) and (max, sum) pairs
  // (log2 domain).
  PageCut *cuts;            // [units]
  float *opart;
  float *mlpart;
};

hipError_t launch_page_append(const PageAppendArgs &a, int head_dim, int format, hipStream_t s);
hipError_t launch_page_read(const PageReadArgs &a, int head_dim, int format, hipStream_t s);
hipError_t launch_page_pack(const PagePackArgs &a, int head_dim, int format, hipStream_t s);
hipError_t launch_page_attend(const PageAttnArgs &a, int head_dim, int format, hipStream_t s);

// Host checks of a pool and a batch (HERMES_OK or an error), and the kernels'
// view of them.  check_page_memory also looks at the pool's pointers.
int check_page_pool(const hermes_page_pool *p);
int check_page_memory(const hermes_page_pool *p);
PagePool page_pool_of(const hermes_page_pool *p);

#ifdef __HIP__
// Sequence b of a batch: its first stacked row, its rows and its length, with
// whatever does not fit clamped and noted in the pool's status word.
struct PageSeq {
  int r0, n, len;
};
__device__ __forceinline__ void page_note(const PagePool &p, int bit) {
  if (p.status != nullptr) atomicOr(p.status, bit);
}
__device__ __forceinline__ PageSeq page_seq_of(const PagePool &p, const PageSeqs &s, int a0, int a1, int len) {
  PageSeq x;
  x.r0 = min(max(a0, 0), s.n_rows);
  const int r1 = min(max(a1, x.r0), s.n_rows);
  x.n = r1 - x.r0;
  if (x.r0 != a0 || r1 != a1) page_note(p, HERMES_PAGE_BAD_ROWS);
  x.len = len;
  if (len < 0 || len > (int64_t)s.max_pages << p.log_rows) {
    x.len = 0;
    page_note(p, HERMES_PAGE_BAD_LENGTH);
  }
  return x;
}
__device__ __forceinline__ PageSeq page_seq(const PagePool &p, const PageSeqs &s, int b) {
  const bool starts = s.row_start != nullptr;
  return page_seq_of(p, s, starts ? s.row_start[b] : b, starts ? s.row_start[b + 1] : b + 1, s.kv_len[b]);
}
// Byte offsets inside a KV head's block (see hermes.h): K row r, V rows 4 r4 ..
// 4 r4 + 3, and their scales.
template <int D, bool FP4>
struct PageBlock {
  static constexpr int kRow = FP4 ? D / 2 : 2 * D;          // bytes of a row of K (or of V)
  static constexpr int kPiece = kRow / 16;                  // of a piece of V
  static constexpr int kScales = D / 32;                    // of a row's scales
  __device__ static __forceinline__ int k(int r) { return r * kRow; }
  __device__ static __forceinline__ int v(int rows, int r4) { return rows * kRow + r4 * 4 * kRow; }
  __device__ static __forceinline__ int ks(int rows, int r) { return 2 * rows * kRow + r * kScales; }
  __device__ static __forceinline__ int vs(int rows, int r4) {
    return 2 * rows * kRow + rows * kScales + r4 * 4 * kScales;
  }
};
#endif

}  // namespace hermes
