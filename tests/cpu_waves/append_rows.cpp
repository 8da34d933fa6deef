// page_append of a batch in which only rows `first` .. `first` + `live` - 1 of 80 are a
// sequence's, and are all that is in memory: what lies before or behind them cannot be read.
//   append_rows <sequences> <first> <axes> <waves that share a row>
#include <sys/mman.h>

#include <cstdio>

#include "pages.hip"

using namespace hermes;

constexpr int kRows = 80, kLive = 64, Hq = 14, Hkv = 2, D = 64;

// `bytes` of memory between two pages that cannot be touched, at their end or their start
static char *room(size_t bytes, bool at_end) {
  const size_t size = (bytes + 4095) / 4096 * 4096;
  char *m = static_cast<char *>(mmap(nullptr, size + 8192, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0)) + 4096;
  if (mprotect(m, size, PROT_READ | PROT_WRITE) != 0) std::abort();
  return m + (at_end ? size - bytes : 0);
}

int main(int, char **argv) {
  const int seqs = std::atoi(argv[1]), first = std::atoi(argv[2]), axes = std::atoi(argv[3]);
  PageAppendArgs a = {};
  a.pool.block_bytes = 2 * 16 * 2 * D;
  a.pool.page_bytes = a.pool.block_bytes * Hkv;
  a.pool.log_rows = 4;
  a.pool.n_pages = kLive;
  a.pool.Hq = Hq;
  a.pool.Hkv = Hkv;
  a.pool.pages = reinterpret_cast<uint8_t *>(room(a.pool.page_bytes * a.pool.n_pages, true));
  std::vector<int32_t> start(seqs + 1), len(seqs), table(seqs * 4);
  for (int b = 0; b <= seqs; ++b) start[b] = first + kLive * b / seqs;
  for (int b = 0; b < seqs; ++b) len[b] = start[b + 1] - start[b];
  for (size_t i = 0; i < table.size(); ++i) table[i] = i % kLive;
  a.seqs = {start.data(), len.data(), table.data(), seqs, kRows, 4};
  const bool at_end = first == 0;
  auto rows = [&](int heads) {
    return reinterpret_cast<uint16_t *>(room(kLive * heads * D * 2, at_end)) - (int64_t)first * heads * D;
  };
  a.q = rows(Hq);
  a.k = rows(Hkv);
  a.v = rows(Hkv);
  a.q_out = rows(Hq);
  a.q_stride = Hq * D;
  a.k_stride = a.v_stride = Hkv * D;
  a.axes = axes;
  a.section[0] = a.section[1] = 8;
  a.section[2] = 16;
  // positions of the live rows of the last axis end the memory, or those of the first begin it
  const int span = (axes - 1) * kRows + kLive;
  a.rope = reinterpret_cast<int32_t *>(room(4 * span, at_end)) - first;
  a.share = std::atoi(argv[4]);
  launch_page_append(a, D, HERMES_PAGE_BF16, nullptr);
  std::puts("done");
}
