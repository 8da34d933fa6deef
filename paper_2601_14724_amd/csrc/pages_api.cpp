// Host side of the pages: argument checks, the cut of an attention call, and the
// launches on the caller's stream.  Nothing here keeps state or allocates.
#include <cmath>
#include <cstdint>
#include <cstring>

#include "pages_internal.h"

using namespace hermes;

namespace hermes {

namespace {

constexpr double kLog2e = 1.4426950408889634;

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int64_t block_bytes(const hermes_page_pool *p) {
  const int64_t d = p->head_dim, row = p->format == HERMES_PAGE_FP4 ? d / 2 + d / 32 : 2 * d;
  return 2 * row * p->page_rows;
}

int check_batch(const hermes_page_pool *p, const hermes_page_batch *b) {
  if (b == nullptr || b->n_seqs < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_len < 0) return HERMES_EINVAL;
  // (a row a wave: a launch's threads have to stay below 2^32)
  if (b->n_rows > 1 << 25 || (b->row_start == nullptr && b->n_rows != b->n_seqs)) return HERMES_EINVAL;
  if (b->n_seqs == 0 || b->n_rows == 0) return HERMES_OK;
  if (b->max_pages < 1 || (int64_t)b->max_pages * p->page_rows > INT32_MAX - 256) return HERMES_EINVAL;
  if ((int64_t)b->n_seqs * p->n_kv_heads > 1 << 24) return HERMES_EINVAL;
  return HERMES_OK;
}

// What an attention call asks of a (good) batch beside that: the cost of all items has to
// be exact as a double (items of 16 rows, one more a pair; it keeps n_rows G below 2^28).
int check_attend_batch(const hermes_page_pool *p, const hermes_page_batch *b) {
  if (b->n_seqs == 0 || b->n_rows == 0) return HERMES_OK;
  const double G = (double)p->n_q_heads / p->n_kv_heads, keys = (double)b->max_pages * p->page_rows;
  const double items = (double)b->n_rows * p->n_q_heads / 16.0 + (double)b->n_seqs * p->n_kv_heads;
  if (items * (G * (keys + 1024.0) + (double)b->n_rows * G) > 4.0e15) return HERMES_EINVAL;
  return HERMES_OK;
}

int check_batch_memory(const hermes_page_batch *b) {
  if (b->kv_len == nullptr || b->tables == nullptr) return HERMES_EINVAL;
  if (!aligned(b->row_start, 4) || !aligned(b->kv_len, 4) || !aligned(b->tables, 4)) return HERMES_EINVAL;
  return HERMES_OK;
}

// rows of bf16 `width` wide, `stride` apart
bool good_rows(const void *p, int64_t stride, int64_t width) {
  return p != nullptr && aligned(p, 16) && stride >= width && stride % 8 == 0;
}

PageSeqs seqs_of(const hermes_page_batch *b) {
  return PageSeqs{b->row_start, b->kv_len, b->tables, b->n_seqs, b->n_rows, b->max_pages};
}

int64_t over(int64_t x, int64_t y) { return (x + y - 1) / y; }

constexpr int kWholeSteps = 16;   // steps of a round's longest items without cuts, at most

// The cut of an attention call, from what the host knows of it.
PagePlan plan_of(const hermes_page_pool *p, const hermes_page_batch *b) {
  const int64_t G = p->n_q_heads / p->n_kv_heads;
  const int64_t max_rows = b->row_start == nullptr ? 1 : b->max_rows > 0 && b->max_rows < b->n_rows ? b->max_rows : b->n_rows;
  const int64_t table = (int64_t)b->max_pages * p->page_rows;
  const int64_t max_len = b->max_len > 0 && b->max_len < table ? b->max_len : table;
  const int64_t P = max_rows * G;
  PagePlan x;
  x.rows = P <= 16 ? 16 : P <= 32 ? 32 : P <= 64 ? 64 : P <= 128 ? 128 : 256;
  // (0 / half / this / twice, us: 40 ragged sequences of 64 rows 243 / 123 / 110 / 119; one row of
  // 64 sequences to 9 K tokens, FP4 200 / 94 / 75 / 79; of 11 to 10 K, bf16 71 / 46 / 45 / 46.5)
  x.item_keys = x.rows > 32 ? 320 : p->format == HERMES_PAGE_FP4 ? 1024 : 512;
  // Without cuts a launch takes rounds of items; with cuts its steps are shared out, whatever
  // the lengths, at the price of a second launch and of the parts (5 to 10 us).  So there
  // are none where the longest items' rounds are short, in keys, and cuts would save
  // little of them even if all were as long.  Without and with, us, 28 + 4 heads of 128 in FP4:
  // one row of 28 sequences of 2000 tokens 15.8 / 20.0, of 4 of 2500 15.9 / 13.1; 64 rows of 10
  // of 300 20.5 / 31.6, of 4 of 1500 54.6 / 33.6.  (Near its bounds the rule is not always
  // right: one bf16 row on 2000 tokens 26.3 / 15.8 goes without, one row of 256 sequences of 1900
  // 51.3 / 72.8 with.)
  // A workgroup of eight waves fits a CU; of the few-row kernel also two of four, which hide
  // the start of one item behind another's keys where there are items enough (256 sequences of
  // 1000 tokens 33.6 us, 45.6 with eight waves; 128 of 1000 18.7 and 24.6).  A step is 32 keys for
  // each wave, or a tile for each key group.
  const bool few = x.rows <= 32;
  const int64_t tiles = over(P, x.rows), all = (int64_t)b->n_seqs * p->n_kv_heads * tiles;
  const int64_t items = all < 1 << 24 ? all : 1 << 24;   // (as good as more: cut, and products below 2^63)
  const bool four = few && items >= 2 * kStreamSlots;
  const int64_t slots = four ? 2 * kStreamSlots : kStreamSlots, step = few ? 256 : x.rows <= 128 ? 128 : 64;
  const int64_t longest = over(items, slots) * max_len * (four ? 2 : 1), shared = over(items * max_len, kStreamSlots);
  if (longest <= kWholeSteps * step && longest - shared <= (few ? 8 : 4) * step) {
    x.step = (int32_t)(four ? step / 2 : step);
    x.tiles = (int32_t)tiles;
    x.units = (int32_t)items;
  } else {
    const int64_t steps = items * over(max_len, step);
    x.step = (int32_t)step;
    x.tiles = 0;
    x.units = (int32_t)(steps < kStreamSlots ? steps : kStreamSlots);
  }
  x.inv_units = 1.0 / x.units;
  x.inv_group = 1.0 / (double)G;
  return x;
}

// Workspace: the cuts, then O and (max, sum) of 2 units parts.
size_t cuts_bytes(const PagePlan &x) { return (sizeof(PageCut) * (size_t)x.units + 255) / 256 * 256; }
size_t workspace_of(const hermes_page_pool *p, const PagePlan &x) {
  if (x.tiles > 0) return 0;
  return cuts_bytes(x) + sizeof(float) * 2 * (size_t)x.units * x.rows * (p->head_dim + 2);
}

void fill_rope(const hermes_page_pool *p, PageAppendArgs *a) {
  const double base = p->rope_theta > 0.0 ? p->rope_theta : 1.0e6;
  const int half = p->head_dim / 2;
  for (int j = 0; j < half; ++j) a->inv_freq[j] = std::pow(base, (-2.0 * (double)j) / (double)p->head_dim);
  a->axes = p->rope_axes == 3 ? 3 : 1;
  const int *sec = p->mrope_section;
  if (sec[0] == 0 && sec[1] == 0 && sec[2] == 0) {
    a->section[0] = half / 4;
    a->section[1] = (half - half / 4) / 2;
    a->section[2] = half - a->section[0] - a->section[1];
  } else {
    for (int i = 0; i < 3; ++i) a->section[i] = sec[i];
  }
}

}  // namespace

int check_page_pool(const hermes_page_pool *p) {
  if (p == nullptr) return HERMES_EINVAL;
  if (p->n_kv_heads < 1 || p->n_q_heads < p->n_kv_heads || p->n_q_heads % p->n_kv_heads != 0) return HERMES_EINVAL;
  if (p->n_q_heads > 1 << 16) return HERMES_EINVAL;
  if (p->head_dim != 64 && p->head_dim != 128) return HERMES_ENOTSUP;
  if (p->format != HERMES_PAGE_BF16 && p->format != HERMES_PAGE_FP4) return HERMES_EINVAL;
  if (p->page_rows < 16 || p->page_rows > 256 || (p->page_rows & (p->page_rows - 1)) != 0) return HERMES_EINVAL;
  if (p->n_pages < 1) return HERMES_EINVAL;
  if (!std::isfinite(p->sm_scale) || !std::isfinite(p->rope_theta)) return HERMES_EINVAL;
  if (p->sm_scale > 0.0 && (p->sm_scale < 1e-30 || p->sm_scale > 1e30)) return HERMES_EINVAL;   // (an fp32 with an inverse)
  if (p->rope_axes != 0 && p->rope_axes != 1 && p->rope_axes != 3) return HERMES_EINVAL;
  if (p->rope_axes == 3) {
    const int *sec = p->mrope_section;
    if (sec[0] < 0 || sec[1] < 0 || sec[2] < 0) return HERMES_EINVAL;
    const int64_t sum = (int64_t)sec[0] + sec[1] + sec[2];
    if (sum != 0 && sum != p->head_dim / 2) return HERMES_EINVAL;
  }
  return HERMES_OK;
}

int check_page_memory(const hermes_page_pool *p) {
  const int rc = check_page_pool(p);
  if (rc != HERMES_OK) return rc;
  if (p->pages == nullptr || !aligned(p->pages, 16) || !aligned(p->status, 4)) return HERMES_EINVAL;
  return HERMES_OK;
}

PagePool page_pool_of(const hermes_page_pool *p) {
  PagePool x;
  x.pages = static_cast<uint8_t *>(p->pages);
  x.status = p->status;
  x.block_bytes = (int32_t)block_bytes(p);
  x.page_bytes = block_bytes(p) * p->n_kv_heads;
  x.log_rows = 0;
  while ((1 << x.log_rows) < p->page_rows) ++x.log_rows;
  x.n_pages = p->n_pages;
  x.Hq = p->n_q_heads;
  x.Hkv = p->n_kv_heads;
  return x;
}

}  // namespace hermes

extern "C" {

size_t hermes_page_bytes(const hermes_page_pool *pool) {
  if (check_page_pool(pool) != HERMES_OK) return 0;
  return (size_t)(block_bytes(pool) * pool->n_kv_heads);
}

size_t hermes_page_workspace_bytes(const hermes_page_pool *pool, const hermes_page_batch *batch) {
  if (check_page_pool(pool) != HERMES_OK || check_batch(pool, batch) != HERMES_OK) return 0;
  if (check_attend_batch(pool, batch) != HERMES_OK) return 0;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return 0;
  return workspace_of(pool, plan_of(pool, batch));
}

int hermes_page_append(const hermes_page_pool *pool, const hermes_page_batch *batch, const void *q,
                       int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                       const int32_t *rope, void *q_out, void *stream) {
  int rc = check_page_memory(pool);
  if (rc == HERMES_OK) rc = check_batch(pool, batch);
  if (rc != HERMES_OK) return rc;
  if ((q == nullptr) != (q_out == nullptr) || (q != nullptr && rope == nullptr)) return HERMES_EINVAL;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return HERMES_OK;
  if ((rc = check_batch_memory(batch)) != HERMES_OK) return rc;
  const int64_t qw = (int64_t)pool->n_q_heads * pool->head_dim, kw = (int64_t)pool->n_kv_heads * pool->head_dim;
  if (!good_rows(k, k_stride, kw) || !good_rows(v, v_stride, kw) || !aligned(rope, 4)) return HERMES_EINVAL;
  if (q != nullptr) {
    if (!good_rows(q, q_stride, qw) || !aligned(q_out, 16)) return HERMES_EINVAL;
    if (q == q_out && q_stride != qw) return HERMES_EINVAL;
  }
  PageAppendArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pool = page_pool_of(pool);
  a.seqs = seqs_of(batch);
  a.q = static_cast<const uint16_t *>(q);
  a.k = static_cast<const uint16_t *>(k);
  a.v = static_cast<const uint16_t *>(v);
  a.q_out = static_cast<uint16_t *>(q_out);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.rope = rope;
  a.share = batch->n_rows < 4 * kStreamSlots ? 4 : 1;   // (a row a wave fills the CUs from there on)
  if (rope != nullptr) fill_rope(pool, &a);
  return launch_page_append(a, pool->head_dim, pool->format, static_cast<hipStream_t>(stream)) == hipSuccess
             ? HERMES_OK : HERMES_EHIP;
}

int hermes_page_attend(const hermes_page_pool *pool, const hermes_page_batch *batch, const void *q,
                       int64_t q_stride, void *out, float *lse, void *workspace, size_t ws_bytes, void *stream) {
  int rc = check_page_memory(pool);
  if (rc == HERMES_OK) rc = check_batch(pool, batch);
  if (rc == HERMES_OK) rc = check_attend_batch(pool, batch);
  if (rc != HERMES_OK) return rc;
  if (batch->n_seqs == 0 || batch->n_rows == 0) return HERMES_OK;
  if ((rc = check_batch_memory(batch)) != HERMES_OK) return rc;
  const int64_t qw = (int64_t)pool->n_q_heads * pool->head_dim;
  if (!good_rows(q, q_stride, qw) || out == nullptr || !aligned(out, 16) || !aligned(lse, 4)) return HERMES_EINVAL;
  PageAttnArgs a;
  std::memset(&a, 0, sizeof(a));
  a.plan = plan_of(pool, batch);
  const size_t need = workspace_of(pool, a.plan);
  if (need > 0) {
    if (workspace == nullptr || !aligned(workspace, 16)) return HERMES_EINVAL;
    if (ws_bytes < need) return HERMES_ECAPACITY;
    a.cuts = static_cast<PageCut *>(workspace);
    a.opart = reinterpret_cast<float *>(static_cast<char *>(workspace) + cuts_bytes(a.plan));
    a.mlpart = a.opart + 2 * (size_t)a.plan.units * a.plan.rows * pool->head_dim;
  }
  a.pool = page_pool_of(pool);
  a.seqs = seqs_of(batch);
  a.q = static_cast<const uint16_t *>(q);
  a.q_stride = q_stride;
  a.out = static_cast<uint16_t *>(out);
  a.lse = lse;
  const double scale = pool->sm_scale > 0.0 ? pool->sm_scale : 1.0 / std::sqrt((double)pool->head_dim);
  a.scale_log2 = (float)(scale * kLog2e);
  return launch_page_attend(a, pool->head_dim, pool->format, static_cast<hipStream_t>(stream)) == hipSuccess
             ? HERMES_OK : HERMES_EHIP;
}

int hermes_page_read(const hermes_page_pool *pool, const hermes_page_batch *batch, void *k, void *v, void *stream) {
  int rc = check_page_memory(pool);
  if (rc == HERMES_OK) rc = check_batch(pool, batch);
  if (rc != HERMES_OK) return rc;
  if (!aligned(k, 16) || !aligned(v, 16)) return HERMES_EINVAL;
  if (batch->n_seqs == 0 || batch->n_rows == 0 || (k == nullptr && v == nullptr)) return HERMES_OK;
  if ((rc = check_batch_memory(batch)) != HERMES_OK) return rc;
  PageReadArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pool = page_pool_of(pool);
  a.seqs = seqs_of(batch);
  a.k = static_cast<uint16_t *>(k);
  a.v = static_cast<uint16_t *>(v);
  return launch_page_read(a, pool->head_dim, pool->format, static_cast<hipStream_t>(stream)) == hipSuccess
             ? HERMES_OK : HERMES_EHIP;
}

}  // extern "C"
