// Host side of what stands around a generated token: products with weights in 4 bits, the
// choice over beams, and the reordering of their pages.  Argument checks, sizes and launches;
// nothing here keeps state or allocates.
#include <cstdint>
#include <cstring>

#include "tokens_internal.h"

using namespace hermes;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
constexpr int64_t kMaxStride = INT64_C(1) << 32;   // (an end of rows is counted in 64 bits)
int64_t over(int64_t x, int64_t y) { return (x + y - 1) / y; }

bool overlap(const void *p, int64_t n, const void *q, int64_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p != nullptr && q != nullptr && a < b + (uintptr_t)m && b < a + (uintptr_t)n;
}

int check_weight(const hermes_weight *w) {
  if (w == nullptr || w->n_out < 1 || w->n_out > 1 << 24 || w->n_in < 1 || w->n_in > 1 << 20) return HERMES_EINVAL;
  return HERMES_OK;
}

WeightView view_of(const hermes_weight *w) {
  WeightView v;
  v.n_out = w->n_out;
  v.n_in = w->n_in;
  v.tiles_out = (int32_t)over(w->n_out, 16);
  v.tiles_in = (int32_t)over(w->n_in, 128);
  v.quads = (int32_t)over(v.tiles_in, 4);
  v.codes = static_cast<uint8_t *>(w->data);
  v.scales = v.codes + (int64_t)v.tiles_out * v.tiles_in * 1024;
  return v;
}

int64_t bytes_of(const WeightView &v) {
  return (int64_t)v.tiles_out * v.tiles_in * 1024 + (int64_t)v.tiles_out * v.quads * 256;
}

// The cut of a product.  Fitted to 140 sizes (1, 8, 16, 32 and 64 rows, 64 to 14336 outputs, 1200 to 14336
// inputs), each with every cut, and checked with 255: 0.5 to 4% slower than the best cut on average.  More tiles a
// wave read x less often (64 rows on 14336 x 3584: 16.0 us with four, 22.6 with two, 36 with one), fewer
// leave more waves (16 on 2048 x 3584: 4.8 with one, 5.9 with two); `split` makes waves where outputs are few
// (one row on 4608 x 3584: 5.4 us with eight, 12 with one).  Parts make workgroups where even so most CUs
// would have none, or each too long a chain, at the price of a launch and of their sums: 64 rows on
// 1024 x 14336 20.8 us without, 10.8 with; 16 on 4608 x 14336 17.4 and 14.2; 64 on 1024 x 3584 8.1 and 7.8;
// and 16 on 1024 x 8000 6.8 and 7.0.
// Where outputs are many, or inputs few, waves share x (`common`): 64 rows on 14336 x 3584 15.8 us without and
// 18.6 with, on 18000 x 3584 24.9 and 23.8, on 131072 x 3584 87 and 58; 16 rows on 2048 x 384 3.1 and 2.8, on
// 2048 x 512 3.1 and 3.3, on 9000 x 1200 5.4 and 5.1, on 9000 x 2236 7.9 and 8.3; few inputs of 5 to 8 rows go as
// 16 do (8 on 131072 x 250 9.7 and 7.6, on 2048 x 384 2.9 and 2.8), of up to 4 not (131072 x 128 4.9 and 5.4).  A wave has the fewest tiles that
// leave two workgroups a CU at most (64 rows on 24000 x 896: one tile 9.1, two 10.3, four more than 11.3; on
// 131072 x 3584 two 73, four 58): 3 to 6% slower than the best cut of 111 sizes with 16, 32 and 64 rows,
// 14336 to 131072 outputs and 896 to 8000 inputs.
WeightPlan plan_of(const WeightView &v, int32_t n_rows) {
  WeightPlan p;
  p.row_quads = n_rows <= 4 ? 1 : n_rows <= 8 && v.tiles_in > 3 ? 2 : n_rows <= 16 ? 4 : n_rows <= 32 ? 8 : 16;
  p.common = 0;
  const int most = p.row_quads < 16 ? 3 : 2;    // waves that share inputs, their log
  if (p.row_quads >= 4 && v.tiles_in >= (p.row_quads < 16 ? 40 : 20) && v.tiles_out <= 600) {
    p.tiles = v.tiles_out <= 64 ? 1 : v.tiles_out <= 128 ? 2 : 4;
    p.log_split = most;
    const int64_t groups = over(v.tiles_out, p.tiles) * over(n_rows, 64), longest = v.tiles_in >> most;
    const int64_t parts = kStreamSlots / groups, cap = p.row_quads < 16 ? 6 : 16;
    p.parts = (int32_t)(parts < cap ? parts : cap);
    if (p.parts > longest) p.parts = (int32_t)longest;
    if (p.parts > 1) return p;
  }
  const int64_t all = v.tiles_out * over(n_rows, 64);     // tiles of all rows
  if (p.row_quads >= 4 && (all > 1024 || v.tiles_in <= 3 || (all > 512 && v.tiles_in <= 12))) {
    p.common = 1;
    p.parts = 1;
    p.log_split = 0;
    p.tiles = all <= 8 * kStreamSlots ? 1 : all <= 16 * kStreamSlots ? 2 : 4;
    return p;
  }
  int waves;                // enough of them to fill the device
  if (p.row_quads == 1) {
    p.tiles = v.tiles_out > 1024 && v.tiles_in > 10 ? 2 : 1;
    waves = 3072;
  } else {
    p.tiles = v.tiles_out > 320 && v.tiles_in > (p.row_quads == 2 ? 10 : 4) ? 4 : v.tiles_out > 192 && v.tiles_in > 4 ? 2 : 1;
    waves = p.row_quads < 16 ? 1536 : 512;
  }
  const int64_t groups = over(v.tiles_out, p.tiles);
  p.parts = 1;
  p.log_split = 0;
  while (p.log_split < most && groups << p.log_split < waves && 2 << p.log_split <= v.tiles_in) ++p.log_split;
  return p;
}

int64_t sums_of(const WeightView &v, const WeightPlan &p, int32_t n_rows) {
  return p.parts > 1 ? (int64_t)64 * p.parts * n_rows * v.tiles_out : 0;
}

int check_beams(const hermes_beam_config *c) {
  if (c == nullptr || c->n_seqs < 0 || c->n_beams < 1 || c->n_beams > kMaxBeams || c->n_vocab < 1) return HERMES_EINVAL;
  if (c->n_keep < 1 || c->n_keep > kMaxKeep) return HERMES_EINVAL;
  if ((int64_t)c->n_seqs * c->n_beams > 1 << 15 || (int64_t)c->n_beams * c->n_vocab > 1 << 30) return HERMES_EINVAL;
  if (c->logits_type != HERMES_BF16 && c->logits_type != HERMES_FP32) return HERMES_EINVAL;
  if (c->end_token < -1 || c->end_token >= c->n_vocab) return HERMES_EINVAL;
  if (c->pad_token < 0 || c->pad_token >= c->n_vocab) return HERMES_EINVAL;
  return HERMES_OK;
}

// A wave takes so many chunks of a row that some thousands of waves are left, and a row has 16 parts, of
// four waves, at most.
void cut_of(const hermes_beam_config *c, BeamArgs *a) {
  const int64_t rows = (int64_t)c->n_seqs * c->n_beams;
  a->chunks = (int32_t)over(c->n_vocab, kBeamChunk);
  const int64_t even = rows * a->chunks / 32768, least = over(a->chunks, 64), per = even < 16 ? even : 16;
  a->per = (int32_t)(per > least ? per : least);
  a->parts = (int32_t)over(a->chunks, 4 * a->per);
}

struct BeamRoom { int64_t sum, peak, top, all; };
BeamRoom beam_room(const BeamArgs &a, int64_t rows) {
  BeamRoom r;
  r.sum = 0;
  r.peak = 8 * rows * a.parts;
  r.top = r.peak + 4 * rows * a.parts;
  r.all = over(r.top + 4 * rows * a.chunks, 16) * 16;
  return r;
}

}  // namespace

extern "C" {

size_t hermes_weight_bytes(const hermes_weight *w) {
  return check_weight(w) == HERMES_OK ? (size_t)bytes_of(view_of(w)) : 0;
}

int hermes_weight_pack(const hermes_weight *w, const void *dense, int64_t stride, void *stream) {
  const int rc = check_weight(w);
  if (rc != HERMES_OK) return rc;
  if (w->data == nullptr || !aligned(w->data, 16)) return HERMES_EINVAL;
  if (dense == nullptr || !aligned(dense, 2) || stride < w->n_in || stride > kMaxStride) return HERMES_EINVAL;
  WeightPackArgs a;
  a.w = view_of(w);
  a.dense = static_cast<const uint16_t *>(dense);
  a.stride = stride;
  if (overlap(w->data, bytes_of(a.w), dense, 2 * ((w->n_out - 1) * stride + w->n_in))) return HERMES_EINVAL;
  return launch_weight_pack(a, static_cast<hipStream_t>(stream)) == hipSuccess ? HERMES_OK : HERMES_EHIP;
}

size_t hermes_weight_workspace_bytes(const hermes_weight *w, int32_t n_rows) {
  if (check_weight(w) != HERMES_OK || n_rows < 1 || n_rows > 1 << 20) return 0;
  const WeightView v = view_of(w);
  return (size_t)sums_of(v, plan_of(v, n_rows), n_rows);
}

int hermes_weight_product(const hermes_weight *w, const void *x, int64_t x_stride, int32_t n_rows,
                          const void *bias, const void *add, void *out, int32_t out_type, void *workspace,
                          size_t ws_bytes, void *stream) {
  const int rc = check_weight(w);
  if (rc != HERMES_OK) return rc;
  if (n_rows < 0 || n_rows > 1 << 20) return HERMES_EINVAL;
  if (out_type != HERMES_BF16 && out_type != HERMES_FP32) return HERMES_EINVAL;
  if (w->data == nullptr || !aligned(w->data, 16)) return HERMES_EINVAL;
  if (n_rows == 0) return HERMES_OK;
  if (x == nullptr || !aligned(x, 16) || x_stride < w->n_in || x_stride > 1 << 24 || x_stride % 8 != 0) return HERMES_EINVAL;
  if (out == nullptr || !aligned(out, 16) || !aligned(bias, 2) || !aligned(add, 2)) return HERMES_EINVAL;
  WeightProductArgs a;
  std::memset(&a, 0, sizeof(a));
  a.w = view_of(w);
  const int64_t n = (int64_t)n_rows * w->n_out, size = out_type == HERMES_FP32 ? 4 : 2;
  if (overlap(out, n * size, x, 2 * ((n_rows - 1) * x_stride + w->n_in))) return HERMES_EINVAL;
  if (overlap(out, n * size, bias, 2 * (int64_t)w->n_out) || overlap(out, n * size, w->data, bytes_of(a.w))) return HERMES_EINVAL;
  if (overlap(out, n * size, add, 2 * n) && (add != out || out_type != HERMES_BF16)) return HERMES_EINVAL;
  a.x = static_cast<const uint16_t *>(x);
  a.bias = static_cast<const uint16_t *>(bias);
  a.add = static_cast<const uint16_t *>(add);
  a.out = out;
  a.x_stride = x_stride;
  a.n_rows = n_rows;
  a.fp32 = out_type == HERMES_FP32;
  a.plan = plan_of(a.w, n_rows);
  const int64_t need = sums_of(a.w, a.plan, n_rows);
  if (need > 0) {
    if (workspace == nullptr || !aligned(workspace, 16)) return HERMES_EINVAL;
    if (ws_bytes < (size_t)need) return HERMES_ECAPACITY;
    a.sums = static_cast<float *>(workspace);
  }
  return launch_weight_product(a, static_cast<hipStream_t>(stream)) == hipSuccess ? HERMES_OK : HERMES_EHIP;
}

size_t hermes_beam_workspace_bytes(const hermes_beam_config *cfg) {
  if (check_beams(cfg) != HERMES_OK) return 0;
  BeamArgs a;
  cut_of(cfg, &a);
  return (size_t)beam_room(a, (int64_t)cfg->n_seqs * cfg->n_beams).all;
}

int hermes_beam_select(const hermes_beam_config *cfg, const void *logits, int64_t stride, const float *score,
                       const int32_t *done, float *score_out, int32_t *parent_out, int32_t *token_out,
                       int32_t *done_out, void *workspace, size_t ws_bytes, void *stream) {
  const int rc = check_beams(cfg);
  if (rc != HERMES_OK) return rc;
  if (cfg->n_seqs == 0) return HERMES_OK;
  const int64_t rows = (int64_t)cfg->n_seqs * cfg->n_beams, size = cfg->logits_type == HERMES_FP32 ? 4 : 2;
  if (logits == nullptr || !aligned(logits, size) || stride < cfg->n_vocab || stride > kMaxStride) return HERMES_EINVAL;
  if (score == nullptr || !aligned(score, 4) || !aligned(done, 4)) return HERMES_EINVAL;
  const int64_t in_bytes = size * ((rows - 1) * stride + cfg->n_vocab), out_bytes = 4 * (int64_t)cfg->n_seqs * cfg->n_keep;
  const void *outs[] = {score_out, parent_out, token_out, done_out};
  for (int i = 0; i < 4; ++i) {
    if (outs[i] == nullptr && i < 3) return HERMES_EINVAL;
    if (!aligned(outs[i], 4) || overlap(outs[i], out_bytes, logits, in_bytes)) return HERMES_EINVAL;
    if (overlap(outs[i], out_bytes, score, 4 * rows) || overlap(outs[i], out_bytes, done, 4 * rows)) return HERMES_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out_bytes, outs[j], out_bytes)) return HERMES_EINVAL;
  }
  BeamArgs a;
  std::memset(&a, 0, sizeof(a));
  cut_of(cfg, &a);
  const BeamRoom room = beam_room(a, rows);
  if (workspace == nullptr || !aligned(workspace, 16)) return HERMES_EINVAL;
  if (ws_bytes < (size_t)room.all) return HERMES_ECAPACITY;
  char *ws = static_cast<char *>(workspace);
  a.sum = reinterpret_cast<double *>(ws + room.sum);
  a.peak = reinterpret_cast<float *>(ws + room.peak);
  a.top = reinterpret_cast<float *>(ws + room.top);
  a.logits = logits;
  a.score = score;
  a.done = done;
  a.score_out = score_out;
  a.parent_out = parent_out;
  a.token_out = token_out;
  a.done_out = done_out;
  a.stride = stride;
  a.n_seqs = cfg->n_seqs;
  a.n_beams = cfg->n_beams;
  a.n_vocab = cfg->n_vocab;
  a.n_keep = cfg->n_keep;
  a.end_token = cfg->end_token;
  a.pad_token = cfg->pad_token;
  return launch_beam_select(a, cfg->logits_type == HERMES_FP32, static_cast<hipStream_t>(stream)) == hipSuccess
             ? HERMES_OK : HERMES_EHIP;
}

int hermes_page_reorder(const hermes_page_pool *pool, const hermes_page_beams *beams, void *stream) {
  const int rc = check_page_memory(pool);
  if (rc != HERMES_OK) return rc;
  const hermes_page_beams *b = beams;
  if (b == nullptr || b->n_groups < 0 || b->n_beams < 1 || b->n_beams > kMaxBeams) return HERMES_EINVAL;
  if (b->grow < 0 || b->grow > 1 << 20) return HERMES_EINVAL;
  if (b->n_groups == 0) return HERMES_OK;
  if (b->n_seqs < 1 || b->n_groups % b->n_seqs != 0 || (int64_t)b->n_groups * b->n_beams > 1 << 22) return HERMES_EINVAL;
  if (b->max_pages < 1 || (int64_t)b->max_pages * pool->page_rows > INT32_MAX - 256) return HERMES_EINVAL;
  const void *all[] = {b->parent, b->room, b->tables, b->kv_len, b->tables_out, b->kv_len_out};
  const int64_t rows = (int64_t)b->n_groups * b->n_beams;
  const int64_t bytes[] = {4 * (int64_t)b->n_seqs * b->n_beams, 8 * (int64_t)b->n_groups, 4 * rows * b->max_pages,
                           4 * rows, 4 * rows * b->max_pages, 4 * rows};
  for (int i = 0; i < 6; ++i) {
    if (all[i] == nullptr || !aligned(all[i], 4)) return HERMES_EINVAL;
    for (int j = 0; i >= 4 && j < i; ++j)
      if (overlap(all[i], bytes[i], all[j], bytes[j])) return HERMES_EINVAL;
  }
  PageReorderArgs a;
  std::memset(&a, 0, sizeof(a));
  a.pool = page_pool_of(pool);
  a.parent = b->parent;
  a.room = b->room;
  a.tables = b->tables;
  a.kv_len = b->kv_len;
  a.tables_out = b->tables_out;
  a.kv_len_out = b->kv_len_out;
  a.n_groups = b->n_groups;
  a.n_seqs = b->n_seqs;
  a.n_beams = b->n_beams;
  a.max_pages = b->max_pages;
  a.grow = b->grow;
  const bool fp4 = pool->format == HERMES_PAGE_FP4;
  a.row_bytes = fp4 ? pool->head_dim / 2 : 2 * pool->head_dim;
  a.scale_bytes = fp4 ? pool->head_dim / 32 : 0;
  // A group's copies, about a third of its beams' pages, are shared by workgroups as far as all are on the
  // device at once, for 64 KiB of pages each (28 layers of eight sequences, eight beams of 34 KiB pages: 15.2 us with
  // one, 12.3 with four; of 16 sequences 22.5, and 18.0 with two; one layer of eight 10.7, and 6.6 with five).
  const int64_t room = 4 * kStreamSlots / b->n_groups, use = over(b->n_beams * a.pool.page_bytes, 1 << 16);
  const int64_t shares = room < use ? room : use;
  a.shares = (int32_t)(shares < 1 ? 1 : shares > 8 ? 8 : shares);
  return launch_page_reorder(a, static_cast<hipStream_t>(stream)) == hipSuccess ? HERMES_OK : HERMES_EHIP;
}

}  // extern "C"
