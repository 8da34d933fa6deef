// page_reorder of groups given on standard input; tables, lengths, pages and status come back.
//   reorder <groups> <sequences> <beams> <max pages> <grow> <log rows> <pages> <heads> <row bytes> <scale bytes> <shares>
#include "more.h"

#include "page_reorder.hip"

using namespace hermes;

int main(int, char **argv) {
  auto number = [&](int i) { return std::atoi(argv[i]); };
  PageReorderArgs a = {};
  a.n_groups = number(1);
  a.n_seqs = number(2);
  a.n_beams = number(3);
  a.max_pages = number(4);
  a.grow = number(5);
  a.pool.log_rows = number(6);
  a.pool.n_pages = number(7);
  a.pool.Hkv = a.pool.Hq = number(8);
  a.row_bytes = number(9);
  a.scale_bytes = number(10);
  a.shares = number(11);
  a.pool.block_bytes = 2 * (a.row_bytes + a.scale_bytes) << a.pool.log_rows;
  a.pool.page_bytes = (int64_t)a.pool.block_bytes * a.pool.Hkv;
  const size_t rows = (size_t)a.n_groups * a.n_beams, bytes = a.pool.page_bytes * a.pool.n_pages;
  a.parent = input<int32_t>((size_t)a.n_seqs * a.n_beams);
  a.room = input<int32_t>(2 * a.n_groups);
  a.tables = input<int32_t>(rows * a.max_pages);
  a.kv_len = input<int32_t>(rows);
  a.pool.pages = input<uint8_t>(bytes, 16);
  a.tables_out = static_cast<int32_t *>(guarded(4 * rows * a.max_pages, 4));
  a.kv_len_out = static_cast<int32_t *>(guarded(4 * rows, 4));
  std::memset(a.tables_out, 0x55, 4 * rows * a.max_pages);
  int32_t status = 0;
  a.pool.status = &status;
  launch_page_reorder(a, nullptr);
  output(a.tables_out, rows * a.max_pages);
  output(a.kv_len_out, rows);
  output(a.pool.pages, bytes);
  output(&status, 1);
}
