// Plans of attention calls of any size that the host takes: built so that an overflow of
// whole numbers ends the program.
#include <cstdio>
#include <random>

#include "pages_api.cpp"

namespace hermes {
static bool good = true;
hipError_t launch_page_append(const PageAppendArgs &, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_page_read(const PageReadArgs &, int, int, hipStream_t) { return hipSuccess; }
hipError_t launch_page_attend(const PageAttnArgs &a, int, int, hipStream_t) {
  const PagePlan &p = a.plan;
  if (p.units < 1 || p.units > 1 << 24 || p.tiles < 0 || p.step < 64 || p.step > 256) good = false;
  if (p.tiles == 0 && p.units > kStreamSlots) good = false;
  return hipSuccess;
}
}  // namespace hermes

int main() {
  std::mt19937_64 rng(1);
  auto any = [&](double bits) { return (int32_t)std::exp2(std::uniform_real_distribution<double>(0, bits)(rng)); };
  void *const here = reinterpret_cast<void *>(16);
  int taken = 0;
  for (int i = 0; i < 3000000; ++i) {
    hermes_page_pool p = {};
    p.n_kv_heads = any(6);
    p.n_q_heads = p.n_kv_heads * any(8);
    p.head_dim = rng() % 2 ? 64 : 128;
    p.format = rng() % 2;
    p.page_rows = 16 << rng() % 5;
    p.n_pages = 1;
    p.pages = here;
    hermes_page_batch b = {};
    b.n_seqs = any(24.5);
    b.n_rows = any(25.5);
    b.max_rows = rng() % 2 ? 0 : any(26);
    b.max_len = rng() % 2 ? 0 : any(31);
    b.max_pages = any(27);
    b.kv_len = b.tables = static_cast<int32_t *>(here);
    b.row_start = static_cast<int32_t *>(here);
    if (rng() % 4 == 0) {
      b.row_start = nullptr;
      b.n_rows = b.n_seqs;
    }
    const size_t bytes = hermes_page_workspace_bytes(&p, &b);
    if (bytes > (size_t)1 << 27) good = false;
    const int64_t stride = (int64_t)p.n_q_heads * p.head_dim;
    if (hermes_page_attend(&p, &b, here, stride, here, nullptr, here, bytes, nullptr) == HERMES_OK) ++taken;
  }
  std::printf("%s, %s taken\n", good ? "good" : "bad", taken > 500000 ? "many" : "few");
}
