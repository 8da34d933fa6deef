// weight_pack and weight_product in memory that ends where their inputs end.
//   weights <outputs> <inputs> <rows> <rows by four> <tiles> <split> <bias> <add> <fp32> <parts> <common>
#include "more.h"

#include "weights.hip"

using namespace hermes;

int main(int, char **argv) {
  auto number = [&](int i) { return std::atoi(argv[i]); };
  auto over = [](int x, int y) { return (x + y - 1) / y; };
  WeightView w = {};
  w.n_out = number(1);
  w.n_in = number(2);
  w.tiles_out = over(w.n_out, 16);
  w.tiles_in = over(w.n_in, 128);
  w.quads = over(w.tiles_in, 4);
  const size_t codes = (size_t)w.tiles_out * w.tiles_in * 1024;
  w.codes = static_cast<uint8_t *>(guarded(codes + (size_t)w.tiles_out * w.quads * 256, 16));
  w.scales = w.codes + codes;
  const int stride = w.n_in + 3;
  WeightPackArgs p = {w, static_cast<uint16_t *>(guarded(2 * ((size_t)(w.n_out - 1) * stride + w.n_in), 2)), stride};
  launch_weight_pack(p, nullptr);
  WeightProductArgs a = {};
  a.w = w;
  a.n_rows = number(3);
  a.plan = {number(4), number(5), __builtin_ctz(number(6)), number(10), number(11)};
  a.fp32 = number(9);
  a.x_stride = over(w.n_in, 8) * 8;
  const size_t n = (size_t)a.n_rows * w.n_out;
  // (the last row ends with its last input: begins 16-byte aligned, and ends at most 14 bytes before the guard)
  a.x = static_cast<uint16_t *>(guarded(2 * ((a.n_rows - 1) * a.x_stride + w.n_in), 16));
  if (number(7)) a.bias = static_cast<uint16_t *>(guarded(2 * (size_t)w.n_out, 2));
  if (number(8)) a.add = static_cast<uint16_t *>(guarded(2 * n, 2));
  a.out = guarded(n * (a.fp32 ? 4 : 2), 16);
  if (a.plan.parts > 1) a.sums = static_cast<float *>(guarded(64 * (size_t)a.plan.parts * a.n_rows * w.tiles_out, 16));
  launch_weight_product(a, nullptr);
  std::puts("done");
}
