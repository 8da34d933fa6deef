// Declarations shared by the host entry points around a generated token (tokens_api.cpp)
// and their kernels (weights.hip, beams.hip, page_reorder.hip).
#pragma once

#include "pages_internal.h"

namespace hermes {

// A weight in memory (see hermes.h): tiles of 16 outputs and 128 inputs.
struct WeightView {
  uint8_t *codes;           // [tiles_out][tiles_in][64][16]
  uint8_t *scales;          // [tiles_out][quads][64][4]
  int32_t n_out, n_in;
  int32_t tiles_out, tiles_in, quads;   // quads: tiles_in / 4, rounded up
};

struct WeightPackArgs {
  WeightView w;
  const uint16_t *dense;
  int64_t stride;
};

// How a product is cut: a workgroup takes 4 row_quads rows, and its waves (eight, or four with
// 64 rows) waves / split x tiles tiles of outputs, `split` waves sharing the inputs of each.
struct WeightPlan {
  int32_t row_quads;        // 1, 2, 4, 8 or 16
  int32_t tiles;            // 1, 2 or 4 (2 at most with row_quads 1)
  int32_t log_split;        // split: 1, 2, 4 or 8 (4 at most with 64 rows)
  int32_t parts;            // workgroups that share the inputs; more than one: joined by a second launch
  int32_t common;           // four waves that share x in LDS (row_quads 4 and more, split and parts 1)
};

struct WeightProductArgs {
  WeightView w;
  const uint16_t *x;
  const uint16_t *bias, *add;   // or null
  void *out;
  float *sums;              // [parts][n_rows][16 tiles_out], with more than one part
  int64_t x_stride;
  int32_t n_rows;
  int32_t fp32;             // out is fp32, else bf16
  WeightPlan plan;
};

constexpr int kBeamChunk = 512;     // tokens of a chunk
constexpr int kMaxBeams = 64, kMaxKeep = 64;

struct BeamArgs {
  const void *logits;
  const float *score;
  const int32_t *done;      // or null
  float *score_out;
  int32_t *parent_out, *token_out, *done_out;   // done_out or null
  int64_t stride;
  int32_t n_seqs, n_beams, n_vocab, n_keep, end_token, pad_token;
  int32_t chunks;           // of a row
  int32_t per, parts;       // chunks of a wave; parts of a row, of four waves (16 at most)
  float *top;               // [rows][chunks]: a chunk's greatest logit
  double *sum;              // [rows][parts]: sum of exp(logit - peak)
  float *peak;              // [rows][parts]
};

struct PageReorderArgs {
  PagePool pool;
  const int32_t *parent, *room, *tables, *kv_len;
  int32_t *tables_out, *kv_len_out;
  int32_t n_groups, n_seqs, n_beams, max_pages, grow;
  int32_t row_bytes, scale_bytes;   // of a row of K (or V) of a head, and of its scales
  int32_t shares;           // workgroups of a group (they share its copies)
};
constexpr int kRoomPages = 65536;   // of a group, at most

hipError_t launch_weight_pack(const WeightPackArgs &a, hipStream_t s);
hipError_t launch_weight_product(const WeightProductArgs &a, hipStream_t s);
hipError_t launch_beam_select(const BeamArgs &a, bool fp32, hipStream_t s);
hipError_t launch_page_reorder(const PageReorderArgs &a, hipStream_t s);

}  // namespace hermes
