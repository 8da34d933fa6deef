// beam_select of logits given on standard input; the four outputs come back.
//   beams <sequences> <beams> <vocabulary> <keep> <fp32> <stride> <end> <pad> <done given> <chunks a wave>
#include "more.h"

#include "beams.hip"

using namespace hermes;

int main(int, char **argv) {
  auto number = [&](int i) { return std::atoi(argv[i]); };
  BeamArgs a = {};
  a.n_seqs = number(1);
  a.n_beams = number(2);
  a.n_vocab = number(3);
  a.n_keep = number(4);
  const bool fp32 = number(5) != 0;
  a.stride = number(6);
  a.end_token = number(7);
  a.pad_token = number(8);
  a.per = number(10);
  a.chunks = (a.n_vocab + kBeamChunk - 1) / kBeamChunk;
  a.parts = (a.chunks + 4 * a.per - 1) / (4 * a.per);
  const size_t rows = (size_t)a.n_seqs * a.n_beams, n = (rows - 1) * a.stride + a.n_vocab, k = (size_t)a.n_seqs * a.n_keep;
  a.logits = fp32 ? static_cast<const void *>(input<float>(n)) : input<uint16_t>(n);
  a.score = input<float>(rows);
  a.done = number(9) != 0 ? input<int32_t>(rows) : nullptr;
  a.sum = static_cast<double *>(guarded(8 * rows * a.parts, 8));
  a.peak = static_cast<float *>(guarded(4 * rows * a.parts, 4));
  a.top = static_cast<float *>(guarded(4 * rows * a.chunks, 4));
  a.score_out = static_cast<float *>(guarded(4 * k, 4));
  a.parent_out = static_cast<int32_t *>(guarded(4 * k, 4));
  a.token_out = static_cast<int32_t *>(guarded(4 * k, 4));
  a.done_out = static_cast<int32_t *>(guarded(4 * k, 4));
  launch_beam_select(a, fp32, nullptr);
  output(a.score_out, k);
  output(a.parent_out, k);
  output(a.token_out, k);
  output(a.done_out, k);
}
