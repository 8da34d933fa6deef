// The walk of an attention call's units over its items, with cuts, where the starts of the
// sequences fall again and again (0, n, 0, n, ...), so that taken as they are the sequences
// hold far more rows than the batch: every item has to be one of the batch's, the sequences'
// rows have to be apart, and a cut item's parts have to be those of units that there are.
//   walk_items <sequences> <rows> <query heads> <length> <units to walk, from both ends>
#include <cstdio>
#include <cstdlib>
#include <set>

#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, ...) (c)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, ...) (c)
#define __builtin_amdgcn_exp2f(x) (x)
#define __builtin_amdgcn_perm(a, b, c) ((a) ^ (b))
#define __builtin_amdgcn_permlane32_swap(a, b, ...) (Pair{{a, b}})
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) (s4{})
#define __builtin_amdgcn_sched_group_barrier(...)
#define __builtin_amdgcn_s_setprio(x)
#define __float_as_uint(x) (x)
#define __uint_as_float(x) (x)

#include <hip/hip_runtime.h>

struct Pair {
  float x[2];
  float operator[](int i) const { return x[i]; }
};
inline float __shfl_xor(float x, int) { return x; }

#include "page_attention.hip"

using namespace hermes;

int main(int, char **argv) {
  const int seqs = std::atoi(argv[1]), n = std::atoi(argv[2]), Hq = std::atoi(argv[3]), keys = std::atoi(argv[4]);
  const int ends = std::atoi(argv[5]);
  std::vector<int32_t> start(seqs + 1), len(seqs, keys);
  for (int b = 0; b <= seqs; ++b) start[b] = b % 2 * n;
  int32_t status = 0;
  PageAttnArgs a = {};
  a.pool.status = &status;
  a.pool.log_rows = 8;
  a.pool.Hq = Hq;
  a.pool.Hkv = 1;
  a.seqs = {start.data(), len.data(), nullptr, seqs, n, (keys + 255) / 256};
  a.plan.rows = 16;
  a.plan.units = kStreamSlots;
  a.plan.step = 256;
  a.plan.item_keys = 1024;
  a.plan.inv_units = 1.0 / a.plan.units;
  a.plan.inv_group = 1.0 / Hq;
  std::vector<PageCut> cuts(a.plan.units);
  for (PageCut &c : cuts) c = PageCut{0, -1, 0, 0, 0, 0, 0, 0};
  a.cuts = cuts.data();
  std::set<int> found;
  bool good = true;
  long long rows = 0, items = 0;
  for (int unit = 0; unit < a.plan.units && good; ++unit) {
    if (unit >= ends && unit < a.plan.units - ends) continue;
    cpu::launch(dim3(1), dim3(64), [&] {
      walk_items<1>(a, unit, [&](const Item &it, int lo, int hi, bool, int) {
        __syncthreads();
        if (threadIdx.x != 0) return;
        const PageSeq s = it.seq;
        if (it.b < 0 || it.b >= seqs || s.r0 < 0 || s.n < 1 || s.r0 + s.n > n || it.P != s.n * Hq || it.p0 < 0 || it.p0 >= it.P ||
            lo < 0 || hi > s.len)
          good = false;
        ++items;
        if (found.insert(it.b).second) rows += s.n;
      });
    });
  }
  for (const PageCut &c : cuts)
    if (c.first < 0 || c.last >= a.plan.units) good = false;
  good = good && items > 0 && rows <= n;
  std::printf("%s, status %d\n", good ? "in bounds" : "out of bounds", status);
}
