// Causal attention over pages for gfx950 (MFMA bf16, 64-wide waves).
//
// page_attn_few    up to 32 packed rows (row, query head of the KV head) an item
// page_attn_many   64, 128 or 256 packed rows an item
// page_combine     joins the parts of items that were cut
//
// S = scale q k^T over the keys a row sees, O = softmax(S) V, in one pass over the
// keys with a running maximum and sum (fp32), lse = ln sum exp S.  P = 2^(S - max) is
// rounded to bf16 for the second product, whose other operand is V in bf16 (its sum is
// not): each p off by 2^-8 of itself at most, which takes O's error in the 2-norm from
// 1.7e-3 (O's own rounding to bf16) to 1.9e-3 to 2.4e-3.  P as a sum of two bf16 numbers
// would double that product.
//
// The cut.  Lengths and rows are on the device and ragged, so the cut is made there:
// every workgroup (unit) adds up the items' costs and takes an equal run of them,
// [u q, (u + 1) q) of N with q = ceil(N / units).  The cost of item i of a
// (sequence, KV head) pair is, in 1/G keys, G max(T - n, 0) + min((i + 1) rows, n G)
// + item_keys G: the keys its last row sees, and a constant for its start and end.
// That is an arithmetic progression, so the sums over a sequence's items, and the
// item that holds a point, need no loop over items.  A cut inside an item falls on a
// multiple of the step.  Items that lie in one unit are written at once; of a cut
// item each unit leaves a part (fp32), at most two a unit.
#include <type_traits>

#include "pages_internal.h"

namespace hermes {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int KS = 32;                  // keys of a wave's step (page_attn_few)
constexpr float kLowest = -3.0e38f;     // running maximum before the first key (finite: -inf minus it stays -inf)
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t f2bf(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale, int byte) {
  switch (byte) {   // (the byte is an immediate)
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  }
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// ---------------------------------------------------------------------- the cut
struct Item {
  PageSeq seq;
  int b, kv;
  int P, p0;                // packed rows of the sequence, the item's first
  int64_t start, end;       // where the item lies in the run of all items
};

// A sequence's costs: sum(i) of its first i items a KV head.
struct SeqCost {
  int64_t base, P, rows, items;
  __device__ __forceinline__ SeqCost(const PageSeq &s, int G, const PagePlan &plan) {
    base = (int64_t)G * (max(s.len - s.n, 0) + plan.item_keys);
    P = (int64_t)s.n * G;
    rows = plan.rows;
    items = (P + rows - 1) / rows;
  }
  __device__ __forceinline__ int64_t sum(int64_t i) const {
    if (i < items) return i * base + rows * (i * (i + 1) / 2);
    return items == 0 ? 0 : items * base + rows * (items * (items - 1) / 2) + P;
  }
};

__device__ __forceinline__ int64_t pair64(uint32_t lo, uint32_t hi) { return (int64_t)((uint64_t)hi << 32 | lo); }
__device__ __forceinline__ int64_t scalar64(int64_t x) {
  return pair64(__builtin_amdgcn_readfirstlane((int)(uint32_t)x), __builtin_amdgcn_readfirstlane((int)(x >> 32)));
}
__device__ __forceinline__ int64_t lane64(int64_t x, int lane) {
  return pair64(__builtin_amdgcn_readlane((int)(uint32_t)x, lane), __builtin_amdgcn_readlane((int)(x >> 32), lane));
}
// x of the lane that a data-parallel move names, 0 where it names none
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved64(int64_t x) {
  return pair64(__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false),
                __builtin_amdgcn_update_dpp(0, (int)(x >> 32), CTRL, ROWS, 0xF, false));
}
// inclusive sums over the lanes: within rows of 16 by shifts of 1, 2, 4 and 8, then the
// last lane of row 0 to row 1 and of 2 to 3, then lane 31 to rows 2 and 3
__device__ __forceinline__ int64_t wave_sums(int64_t x) {
  x += moved64<0x111, 0xF>(x);
  x += moved64<0x112, 0xF>(x);
  x += moved64<0x114, 0xF>(x);
  x += moved64<0x118, 0xF>(x);
  x += moved64<0x142, 0xA>(x);
  x += moved64<0x143, 0xC>(x);
  return x;
}
// x / y of scalars, 0 <= x, 0 < y (64-bit divisions are some 100 instructions, and the
// start of a short call waits for them)
__device__ __forceinline__ int64_t over64(int64_t x, int64_t y) {
  if (((x | y) >> 32) == 0) return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)x / (uint32_t)y));
  return scalar64((int64_t)((uint64_t)x / (uint64_t)y));
}

// The items of a call, a sequence a lane.
struct Items {
  const PagePool &pool;
  const PageSeqs &seqs;
  const PagePlan &plan;
  int G;
  __device__ __forceinline__ Items(const PageAttnArgs &a)
      : pool(a.pool), seqs(a.seqs), plan(a.plan), G(a.pool.Hq / a.pool.Hkv) {}
  // Lane l has sequence b0 + l: its bounds, and the sum of the costs up to it.  A start that
  // falls counts as the greatest before it, so that no two sequences share rows: the host has
  // bounded the cost of n_rows rows, and starts on the device could ask for those of every
  // sequence.  from: the row where the sequences before b0 end.
  struct Scan {
    PageSeq seq;
    int64_t sums;
  };
  __device__ __forceinline__ Scan scan(int b0, int from) const {
    const int lane = threadIdx.x & 63, b = b0 + lane;
    const bool on = b < seqs.n_seqs, starts = on && seqs.row_start != nullptr;
    int a0 = starts ? seqs.row_start[b] : b, a1 = starts ? seqs.row_start[b + 1] : b + 1;
    const int len = on ? seqs.kv_len[b] : 0;
    if (__builtin_expect(__any(starts && (a1 < a0 || a0 < from)), 0)) {
      page_note(pool, HERMES_PAGE_BAD_ROWS);
      a1 = max(max(a0, a1), from);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) a1 = max(a1, __shfl_up(a1, d));
      const int before = __shfl_up(a1, 1);
      a0 = lane > 0 ? before : max(a0, from);
    }
    Scan x = {{0, 0, 0}, 0};
    if (on) {
      x.seq = page_seq_of(pool, seqs, a0, a1, len);
      const SeqCost c(x.seq, G, plan);
      x.sums = pool.Hkv * c.sum(c.items);
    }
    x.sums = wave_sums(x.sums);
    return x;
  }
  // the row where the 64 sequences of a scan end (more follow)
  __device__ __forceinline__ int end_of(const Scan &s) const {
    return __builtin_amdgcn_readlane(s.seq.r0 + s.seq.n, 63);
  }
  // the cost of all; s: scan(0, 0)
  __device__ __forceinline__ int64_t total(Scan s) const {
    int64_t n = lane64(s.sums, 63);
    for (int b = 64; b < seqs.n_seqs; b += 64) {
      s = scan(b, end_of(s));
      n += lane64(s.sums, 63);
    }
    return n;
  }
  // The item that holds x (x < total); s: scan(0, 0).
  __device__ __forceinline__ Item find(int64_t x, Scan s) const {
    int64_t before = 0;
    int b = 0, l;
    for (;;) {
      const unsigned long long past = __ballot(before + s.sums > x);
      l = past != 0ull ? __builtin_ctzll(past) : 63;
      if (past != 0ull || b + 64 >= seqs.n_seqs) break;
      before += lane64(s.sums, 63);
      b += 64;
      s = scan(b, end_of(s));
    }
    before += l > 0 ? lane64(s.sums, l - 1) : 0;
    const PageSeq seq = {__builtin_amdgcn_readlane(s.seq.r0, l), __builtin_amdgcn_readlane(s.seq.n, l),
                         __builtin_amdgcn_readlane(s.seq.len, l)};
    return in_sequence(b + l, seq, before, x);
  }
  // Sequence b; from: the row where the one before ends.
  __device__ __forceinline__ PageSeq sequence(int b, int from) const {
    const bool starts = seqs.row_start != nullptr;
    int a0 = starts ? seqs.row_start[b] : b, a1 = starts ? seqs.row_start[b + 1] : b + 1;
    if (a0 < from || a1 < a0) {
      page_note(pool, HERMES_PAGE_BAD_ROWS);
      a0 = max(a0, from);
      a1 = max(a0, a1);
    }
    const PageSeq s = page_seq_of(pool, seqs, a0, a1, seqs.kv_len[b]);
    return {__builtin_amdgcn_readfirstlane(s.r0), __builtin_amdgcn_readfirstlane(s.n),
            __builtin_amdgcn_readfirstlane(s.len)};
  }
  // The item that holds x, in sequence b, whose items start at `before`.
  __device__ __forceinline__ Item in_sequence(int b, const PageSeq &seq, int64_t before, int64_t x) const {
    Item it;
    it.b = b;
    it.seq = seq;
    const SeqCost c(seq, G, plan);
    it.P = (int)c.P;
    const int64_t head = c.sum(c.items);
    int64_t rest = x - before;
    if (pool.Hkv <= 64) {                 // (a lane a head, for a division)
      const int lane = threadIdx.x & 63;
      const unsigned long long past = __ballot(lane + 1 >= pool.Hkv || (lane + 1) * head > rest);
      it.kv = __builtin_ctzll(past);
    } else {
      it.kv = (int)over64(rest, head);
    }
    rest -= it.kv * head;
    int64_t i = 0, j = c.items;           // sum(i) <= rest < sum(j)
    while (j - i > 1) {
      const int64_t m = (i + j) / 2;
      if (c.sum(m) <= rest) i = m; else j = m;
    }
    it.p0 = __builtin_amdgcn_readfirstlane((int)i * plan.rows);
    it.start = before + it.kv * head + c.sum(i);
    it.end = before + it.kv * head + c.sum(i + 1);
    return it;
  }
  // The item after `it`, if any (it.end < total).
  __device__ __forceinline__ Item next(const Item &it) const {
    const SeqCost c(it.seq, G, plan);
    const int64_t all = pool.Hkv * c.sum(c.items), head = c.sum(c.items);
    const int64_t before = it.start - it.kv * head - c.sum(it.p0 / plan.rows);
    if (it.end < before + all) return in_sequence(it.b, it.seq, before, it.end);
    int b = it.b + 1;                      // (sequences without rows have no items)
    PageSeq seq = sequence(b, it.seq.r0 + it.seq.n);
    while (b + 1 < seqs.n_seqs && seq.n == 0) seq = sequence(++b, seq.r0);
    return in_sequence(b, seq, it.end, it.end);
  }
};

// A unit's walk over its items: body(item, lo, hi, whole, slot) for each, with the keys
// [lo, hi) of it that are the unit's.  The first wave finds the items and leaves them in
// LDS for all: so the waves take the same way through the barriers whatever the lengths'
// memory holds, and the walk's state takes no registers from the body.  (body has a barrier
// after which no wave reads the item again.)
struct Walk {
  Item it;
  int64_t lo, hi, q;        // the unit's run, and the length of all units' runs
  int more;                 // whether `it` is an item
};
template <int WAVES, typename F>
__device__ __forceinline__ void walk_items(const PageAttnArgs &a, int unit, F &&body) {
  __shared__ Walk walk;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Items items(a);
  const int tiles = a.plan.tiles;           // > 0: no cuts, `tiles` units for each pair
  if (wave == 0) {
    Walk w;
    if (tiles > 0) {
      const int pair = unit / tiles;
      w.it.b = pair / a.pool.Hkv;
      w.it.kv = pair - w.it.b * a.pool.Hkv;
      w.it.seq = items.sequence(w.it.b, 0);   // (starts that fall: two pairs may write one row)
      w.it.P = w.it.seq.n * items.G;
      w.it.p0 = (unit - pair * tiles) * a.plan.rows;
      w.it.start = w.lo = 0;
      w.it.end = w.hi = w.q = 1;
      w.more = w.it.p0 < w.it.P;
    } else {
      const Items::Scan first = items.scan(0, 0);
      const int64_t N = items.total(first);
      w.q = max((int64_t)((double)N * a.plan.inv_units) + 1, (int64_t)a.plan.step * items.G);
      w.lo = unit * w.q;
      w.hi = min(w.lo + w.q, N);
      w.more = w.lo < w.hi;
      if (w.more) w.it = items.find(w.lo, first);
    }
    walk = w;
  }
  for (int slot = 0;; slot = 1) {
    __syncthreads();
    const bool more = __builtin_amdgcn_readfirstlane(walk.more) != 0;
    const int64_t start = scalar64(walk.it.start), end = scalar64(walk.it.end);
    const int64_t lo = scalar64(walk.lo), hi = scalar64(walk.hi);
    if (tiles == 0 && slot == 0 && wave == WAVES - 1) {   // (the wave with the fewest steps)
      // does this unit hold its first item's first cut?
      PageCut cut = {0, -1, 0, 0, 0, 0, 0, 0};
      const int64_t q = scalar64(walk.q);
      if (more && start < lo && start >= lo - q)
        cut = PageCut{unit - 1, (int)over64(end - 1, q), start == lo - q ? 0 : 1, walk.it.kv, walk.it.seq.r0,
                      walk.it.p0, walk.it.P, 0};
      if ((threadIdx.x & 63) == 0) a.cuts[unit] = cut;
    }
    if (!more) return;
    {
      Item it;
      it.b = __builtin_amdgcn_readfirstlane(walk.it.b);
      it.kv = __builtin_amdgcn_readfirstlane(walk.it.kv);
      it.p0 = __builtin_amdgcn_readfirstlane(walk.it.p0);
      it.P = __builtin_amdgcn_readfirstlane(walk.it.P);
      it.seq.r0 = __builtin_amdgcn_readfirstlane(walk.it.seq.r0);
      it.seq.n = __builtin_amdgcn_readfirstlane(walk.it.seq.n);
      it.seq.len = __builtin_amdgcn_readfirstlane(walk.it.seq.len);
      // the keys its last row sees
      const int last = (min(it.p0 + a.plan.rows, it.P) - 1) / items.G;
      const int seen = max(0, it.seq.len - it.seq.n + last + 1);
      auto key_at = [&](int64_t x) {
        const int64_t keys = (int64_t)((double)(x - start) * a.plan.inv_group);
        return (int)min(keys & -(int64_t)a.plan.step, (int64_t)seen);   // (a step is a power of two)
      };
      const bool head = start >= lo, tail = end <= hi;
      const int k0 = head ? 0 : key_at(lo), k1 = tail ? seen : key_at(hi);
      body(it, __builtin_amdgcn_readfirstlane(k0), __builtin_amdgcn_readfirstlane(k1), head && tail, slot);
    }
    if (wave == 0) {
      Item it = walk.it;
      it.start = scalar64(it.start);
      it.end = scalar64(it.end);
      it.p0 = __builtin_amdgcn_readfirstlane(it.p0);
      it.P = __builtin_amdgcn_readfirstlane(it.P);
      if (tiles > 0) {                      // (more rows than the hint said)
        const int64_t p0 = it.p0 + (int64_t)tiles * a.plan.rows;
        walk.more = p0 < it.P;
        walk.it.p0 = (int)p0;
      } else if (it.end >= scalar64(walk.hi)) {
        walk.more = 0;
      } else {
        it.b = __builtin_amdgcn_readfirstlane(it.b);
        it.kv = __builtin_amdgcn_readfirstlane(it.kv);
        it.seq.r0 = __builtin_amdgcn_readfirstlane(it.seq.r0);
        it.seq.n = __builtin_amdgcn_readfirstlane(it.seq.n);
        it.seq.len = __builtin_amdgcn_readfirstlane(it.seq.len);
        walk.it = items.next(it);
      }
    }
  }
}

// Workgroups are dispatched to the 8 XCDs round-robin; consecutive units, which read
// the same sequence, are given to the same XCD, and share its L2.
__device__ __forceinline__ int xcd_remap(int i, int n) {
  const int q = n / 8, r = n % 8, x = i % 8, k = i / 8;
  return x < r ? x * (q + 1) + k : r * (q + 1) + (x - r) * q + k;
}

// ------------------------------------------------------------------- a few rows
// MFMA layout (v_mfma_f32_16x16x32_bf16): lane l = 16 u + n supplies A[m = n][k = 8 u
// .. + 7] and B[k = 8 u .. + 7][n]; result register j holds D[m = 4 u + j][n].
//
// A wave takes 32 keys a step, as two groups of 16, straight from the page into
// registers: no LDS and no barrier between steps.
//   S^T = K Q^T: lane (u, n) holds key n of a group and a quarter u of its channels.
//   The k index of an MFMA may be any order of the channels that K and Q agree on,
//   so with FP4 a lane's channels are one run, 16 bytes, one block with one scale.
//   The result gives lane (u, n) row n and the keys 4 u .. 4 u + 3 of both groups.
//   O^T = V^T P^T: those eight keys are the lane's k index of the second product, so P
//   goes from one MFMA to the next without leaving its lane, and V comes as four
//   rows' pieces of d / 16 channels, again 16 bytes a lane and group (FP4, d 128).
// Both loads of a group are one contiguous KiB of the page.
//
// Bound by HBM where there is much to read: 16 sequences of 9 K to 36 K tokens, 4 KV
// heads of 128 in FP4, 195 MB: 47 us, of which the keys take about 39 (5 TB/s), the start (cut,
// tables, first loads) 4 and the joins 4.5.  28 layers of 2 K to 6 K tokens, 63 MB: 23.6 us, as
// much start and join as keys; a dependent chain of loads, not traffic, bounds those.
//
// What a lane holds of a step's 32 keys, as it lies in the page: WK words of K and
// WV of V for each group of 16 keys, and with FP4 the scales.
template <int D, bool FP4>
struct Step {
  static constexpr int WK = FP4 ? D / 32 : D / 8, WV = FP4 ? D / 32 : D / 8;
  uint32_t k[2][WK], v[2][WV];
  uint32_t ks[2], vs[2];
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t *w, const uint8_t *p) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 x = reinterpret_cast<const uint4 *>(p)[i];
      w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
    }
  } else if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  } else {
    static_assert(N == 2, "two words");
    const uint2 x = *reinterpret_cast<const uint2 *>(p);
    w[0] = x.x, w[1] = x.y;
  }
}

template <int D, bool FP4, int RT, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void page_attn_few(PageAttnArgs a) {
  using B = PageBlock<D, FP4>;
  constexpr int KK = D / 32;                // MFMAs of S for each group of keys
  constexpr int PC = D / 16;                // channels of a piece of V
  // Steps in flight beside the one computed.  A step of bf16 at head size 128 is 64 registers
  // a lane: with one more of them 32 rows spill (11 sequences, 8 rows of 32 + 8 heads: 80 us, 58
  // without).
  constexpr int AHEAD = FP4 ? 2 : D == 128 && RT == 2 ? 0 : 1;
  const PagePool &pool = a.pool;
  const int Hq = pool.Hq, G = Hq / pool.Hkv;
  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n16 = lane & 15, u = lane >> 4;
  const int rows_log = pool.log_rows, page_rows = 1 << rows_log;
  const float c = a.scale_log2, inv_c = 1.f / c;

  // lane's byte offsets in a KV head's block, from the first row of a group of 16
  const int k_ofs = n16 * B::kRow + (FP4 ? u * (D / 8) : u * 16);
  const int v_ofs = B::v(page_rows, u) + n16 * 4 * B::kPiece;
  const int ks_ofs = B::ks(page_rows, n16) + u * (D / 4) / 32;
  const int vs_ofs = B::vs(page_rows, u) + n16 * PC / 32 * 4;

  // the waves' states of 16 rows (32 rows: in two buffers, so that a wave may leave its second
  // ones while others still read the first)
  __shared__ __attribute__((aligned(16))) float so_[RT][NW][16][D + 4];
  __shared__ float2 sml_[RT][NW][16];

  walk_items<NW>(a, unit, [&](const Item &it, int lo, int hi, bool whole, int slot) {
    // keys [lo, hi); row i of the sequence sees those below base + i + 1
    const PageSeq seq = it.seq;
    const int kv = it.kv;
    const int p0 = it.p0, P = it.P;
    const int first = __builtin_amdgcn_readfirstlane(p0 / G), base = seq.len - seq.n;
    const int32_t *table = a.seqs.tables + (int64_t)it.b * a.seqs.max_pages;

    bf16x8 qf[RT][KK];
    int vis[RT];                            // keys this lane's row sees
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int p = p0 + 16 * t + n16;
      const int i = p < P ? p / G : 0, g = p < P ? p - i * G : 0;
      vis[t] = p < P ? base + i + 1 : 0;
      const uint16_t *q = a.q + (int64_t)(seq.r0 + i) * a.q_stride + (int64_t)(kv * G + g) * D;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        qf[t][kk] = p < P ? *reinterpret_cast<const bf16x8 *>(q + (FP4 ? u * (D / 4) + 8 * kk : 32 * kk + 8 * u)) : bf16x8{};
    }
    f32x4 o[RT][PC];
    float m_run[RT], m_lim[RT], l_run[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int i = 0; i < PC; ++i) o[t][i] = f32x4{};
      m_run[t] = kLowest;
      m_lim[t] = (kLowest + 8.f) * inv_c;
      l_run[t] = 0.f;
    }
    const int all_see = base + first + 1;   // keys that every row of the tile sees

    // wave w takes the steps w, w + NW, ...; lane x holds the pages of the x-th
    // of the next 64 of them, both groups' (-1: no such page, or past the end)
    const int steps = (hi - lo + KS - 1) / KS;
    const int mine = steps > wave ? (steps - wave + NW - 1) / NW : 0;
    int ids[2] = {-1, -1};
    auto find_pages = [&](int x0) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t key = lo + ((int64_t)wave + (int64_t)NW * (x0 + lane)) * KS + 16 * h;
        ids[h] = -1;
        if (x0 + lane < mine && key < hi) {
          ids[h] = table[key >> rows_log];
          if (ids[h] < 0 || ids[h] >= pool.n_pages) {
            ids[h] = -1;
            page_note(pool, HERMES_PAGE_BAD_ID);
          }
        }
      }
    };
    auto key_of = [&](int x) { return lo + (wave + NW * x) * KS; };
    using Frag = Step<D, FP4>;
    auto load = [&](Frag &f, int x) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int id = max(__builtin_amdgcn_readlane(ids[h], x & 63), 0);
        const int r = (key_of(x) + 16 * h) & (page_rows - 1);
        const uint8_t *block = pool.pages + (int64_t)id * pool.page_bytes + (int64_t)kv * pool.block_bytes;
        const uint8_t *kb = block + r * B::kRow;            // (16 rows of V take as much as 16 of K)
        load_words<Frag::WV>(f.v[h], kb + v_ofs);
        if constexpr (FP4) {
          load_words<Frag::WK>(f.k[h], kb + k_ofs);
          f.ks[h] = *(block + r * B::kScales + ks_ofs);
          f.vs[h] = *reinterpret_cast<const uint32_t *>(block + r * B::kScales + vs_ofs);
        } else {
          // (channels 32 kk + 8 u ..: 64 bytes of a row for each MFMA)
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) load_words<4>(f.k[h] + 4 * kk, kb + k_ofs + 64 * kk);
        }
      }
    };
    auto step = [&](Frag &f, int x) {
      const int key0 = key_of(x);
      // Memory that holds no stored row (past the length, or no page) may hold
      // anything: its values become zeros.  Keys there are masked by S, or zeros too.
      const bool hole = (__builtin_amdgcn_readlane(ids[0], x & 63) | __builtin_amdgcn_readlane(ids[1], x & 63)) < 0;
      if (__builtin_expect(hole || key0 + KS > seq.len, 0)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool none = __builtin_amdgcn_readlane(ids[h], x & 63) < 0;
          const int valid = none ? 0 : seq.len - (key0 + 16 * h + 4 * u);    // of this lane's four rows of V
          if constexpr (FP4) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (j < valid) continue;
              f.vs[h] &= ~(0xFFu << (8 * j));               // (scale 0: small and finite)
              if constexpr (D == 128) f.v[h][j] = 0u;
              else f.v[h][j / 2] &= j & 1 ? 0x0000FFFFu : 0xFFFF0000u;
            }
            if (none) f.ks[h] = 0u;
          } else {
#pragma unroll
            for (int i = 0; i < Frag::WV; ++i)
              if (i / (Frag::WV / 4) >= valid) f.v[h][i] = 0u;
          }
          if (none) {
#pragma unroll
            for (int i = 0; i < Frag::WK; ++i) f.k[h][i] = 0u;
          }
        }
      }
      f32x4 s[RT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < RT; ++t) s[t][h] = f32x4{};
        const float sc = FP4 ? scale_of(f.ks[h]) : 0.f;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = FP4 ? fp4_pair(f.k[h][kk], sc, i) : f.k[h][4 * (FP4 ? 0 : kk) + i];
          const bf16x8 kf = __builtin_bit_cast(bf16x8, uint4{w[0], w[1], w[2], w[3]});
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][h] = mfma16(kf, qf[t][kk], s[t][h]);
        }
      }
      if (key0 + KS > all_see) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (key0 + 16 * (j / 4) + 4 * u + j % 4 >= vis[t]) s[t][j / 4][j % 4] = -INFINITY;
        }
      }
      bf16x8 pf[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float mx = s[t][0][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) mx = fmaxf(mx, s[t][j / 4][j % 4]);
        // The running maximum, common to the four lanes of a row, moves only when a
        // score passes it by more than 2^8 (log2 domain): P stays below 2^8 and the
        // usual step needs no exchange between lanes.
        if (__builtin_expect(__any(mx > m_lim[t]), 0)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float m_new = fmaxf(m_run[t], mx * c);
          const float alpha = fast_exp2(m_run[t] - m_new);
          m_run[t] = m_new;
          m_lim[t] = (m_new + 8.f) * inv_c;
          l_run[t] *= alpha;
#pragma unroll
          for (int i = 0; i < PC; ++i) o[t][i] *= alpha;
        }
        float ls = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = fast_exp2(fmaf(s[t][j / 4][j % 4], c, -m_run[t]));
          ls += p;
          pf[t][j] = static_cast<__bf16>(p);    // (P enters an MFMA as bf16; the sum keeps fp32)
        }
        l_run[t] += ls;
      }
      // V: pair i of channels, four keys a group; the halves of two keys' words
      // are joined into (key j, key j + 1) of one channel
#pragma unroll
      for (int i = 0; i < PC / 2; ++i) {
        uint32_t even[4], odd[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (FP4) {
              const float sc = scale_of((f.vs[h] >> (8 * j)) & 0xFFu);
              x[j] = D == 128 ? fp4_pair(f.v[h][j], sc, i) : fp4_pair(f.v[h][j / 2], sc, 2 * (j & 1) + i);
            } else {
              x[j] = f.v[h][j * (PC / 2) + i];
            }
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            even[2 * h + j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
            odd[2 * h + j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
          }
        }
        const bf16x8 ve = __builtin_bit_cast(bf16x8, uint4{even[0], even[1], even[2], even[3]});
        const bf16x8 vo = __builtin_bit_cast(bf16x8, uint4{odd[0], odd[1], odd[2], odd[3]});
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          o[t][2 * i] = mfma16(ve, pf[t], o[t][2 * i]);
          o[t][2 * i + 1] = mfma16(vo, pf[t], o[t][2 * i + 1]);
        }
      }
    };
    // a ring of steps in registers, AHEAD of them in flight
    for (int x0 = 0; x0 < mine; x0 += 64) {
      find_pages(x0);
      const int x1 = min(x0 + 64, mine);
      Frag f[AHEAD + 1];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (x0 + i < x1) load(f[i], x0 + i);
      for (int x = x0; x < x1; x += AHEAD + 1) {
#pragma unroll
        for (int i = 0; i <= AHEAD; ++i) {
          if (x + i + AHEAD < x1) load(f[(i + AHEAD) % (AHEAD + 1)], x + i + AHEAD);
          if (x + i < x1) step(f[i], x + i);
        }
      }
    }

    // join the waves' states, 16 rows at a time
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (p0 + 16 * t >= P) break;
      float l = l_run[t];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      float(*so)[16][D + 4] = so_[t];
      float2(*sml)[16] = sml_[t];
      if (u == 0) sml[wave][n16] = float2{m_run[t], l};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < PC; i += 4)
          *reinterpret_cast<float4 *>(&so[wave][n16][PC * (4 * u + j) + i]) =
              float4{o[t][i][j], o[t][i + 1][j], o[t][i + 2][j], o[t][i + 3][j]};
      }
      __syncthreads();
      constexpr int TPR = 4 * NW, CPT = D / TPR;                    // threads of a row, channels of a thread
      const int row = threadIdx.x / TPR, ch = threadIdx.x % TPR * CPT;
      const int p = p0 + 16 * t + row;
      if (p >= P) continue;
      float m = sml[0][row].x;
#pragma unroll
      for (int w = 1; w < NW; ++w) m = fmaxf(m, sml[w][row].x);
      float sum = 0.f, acc[CPT];
#pragma unroll
      for (int i = 0; i < CPT; ++i) acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float e = fast_exp2(sml[w][row].x - m);
        sum += e * sml[w][row].y;
#pragma unroll
        for (int i = 0; i < CPT; ++i) acc[i] += e * so[w][row][ch + i];
      }
      if (!whole) {
        const int64_t at = (int64_t)(2 * unit + slot) * (16 * RT) + 16 * t + row;
        if (ch == 0) *reinterpret_cast<float2 *>(a.mlpart + 2 * at) = float2{m, sum};
        if (hi > lo) {                      // (an empty part leaves its O unwritten, and unread)
#pragma unroll
          for (int x = 0; x < CPT; x += 2)
            *reinterpret_cast<float2 *>(a.opart + at * D + ch + x) = float2{acc[x], acc[x + 1]};
        }
      } else {
        const int i = p / G, g = p - i * G;
        const int64_t at = (int64_t)(seq.r0 + i) * Hq + kv * G + g;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (0: the row sees nothing; a NaN stays one)
#pragma unroll
        for (int x = 0; x < CPT; x += 2)
          *reinterpret_cast<uint32_t *>(a.out + at * D + ch + x) = f2bf(acc[x] * inv) | f2bf(acc[x + 1] * inv) << 16;
        if (a.lse != nullptr && ch == 0) a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
      }
    }
  });
}

// ------------------------------------------------------------------- many rows
// MFMA layout (v_mfma_f32_32x32x16_bf16): lane l supplies A[m = l % 32][k = 8 (l / 32)
// .. + 7] and B[k = 8 (l / 32) .. + 7][n = l % 32]; result register j of lane l holds
// D[m = 8 (j / 4) + 4 (l / 32) + j % 4][n = l % 32].
//
// Eight waves: RG row groups of 32 packed rows, times KG = 8 / RG key groups, each of
// which takes every KG-th tile of keys and holds all the item's rows, so that items of
// 64 or 128 rows keep the matrix units as busy as those of 256; the key groups' states are
// merged through LDS at an item's end.  A wave fetches its share of its group's tile from
// the page (8 or 16 keys, so a page id is a scalar), turns FP4 into bf16 on the way to LDS,
// and reads all of the tile from there, K row by row and V transposed by
// ds_read_b64_tr_b16.  As in attn_fwd, S^T = K Q^T puts one query row a lane, so the softmax
// stays in the lane and P^T is the B operand of O^T = V^T P^T as it is.
//
// Bound by the issue port and the chain S -> softmax -> P V (matrix units busy 44% by counters):
// 3136 rows of 28 + 4 heads of 128 on 35904 tokens in FP4 take 1431 us with the joins (1.08
// PFLOP/s), 64 rows on each of 28 layers' 4 K to 16 K tokens 304 us.
constexpr int MT = 512, MW = MT / 64;   // waves
constexpr int KPAD = 8, VPAD = 32;      // u16 padding of K and V rows in LDS

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Inside each group of 16 lanes, lane j receives element j % 4 of the 8-byte rows
// addressed by lanes j / 4, 4 + j / 4, 8 + j / 4, 12 + j / 4.
__device__ __forceinline__ s4 lds_tr16(const uint16_t *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)p);
}

template <int D, bool FP4, int RG>
__global__ __launch_bounds__(MT, 1) void page_attn_many(PageAttnArgs a) {
  using B = PageBlock<D, FP4>;
  constexpr int KG = MW / RG, MROWS = 32 * RG;   // key groups, packed rows of an item
  constexpr int MK = KG <= 2 ? 64 : 32;   // keys of a tile (four groups' tiles of 64 do not fit LDS)
  constexpr int SUB = MK / 32;
  constexpr int WKEYS = MK / RG;          // keys a wave fetches
  static_assert(WKEYS == 8 || WKEYS == 16, "a wave's keys lie in one page");
  constexpr int UK = WKEYS * D / 8 / 64;  // pieces of eight channels of K a lane fetches
  constexpr int LK = D / 8 / UK;          // lanes of a key
  constexpr int PC = D / 16;              // channels of a piece of V; a lane fetches one of two keys,
  constexpr int NV = WKEYS / 8;           // NV times, eight keys apart
  constexpr int WK = FP4 ? UK : 4 * UK, WV = FP4 ? D / 64 : D / 16;   // words a lane fetches (of V NV times)
  constexpr int kAheadK = 4, kAheadV = 4; // LDS reads issued ahead of their MFMA

  const PagePool &pool = a.pool;
  const int Hq = pool.Hq, G = Hq / pool.Hkv;
  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int half = lane >> 5, l32 = lane & 31;
  const int rg = wave % RG, kg = wave / RG;
  const int rows_log = pool.log_rows, page_rows = 1 << rows_log;
  const float c = a.scale_log2, inv_c = 1.f / c;

  // what this lane fetches: of key `kkey` of the wave's, channels 8 kpc ..; of keys vkey and
  // vkey + 1 (and eight further), channels PC vpc ..
  const int kkey = lane / LK, kpc = lane % LK * UK;
  const int vpc = lane % 32 / 2, vkey = lane / 32 * 4 + lane % 2 * 2;
  const int k_ofs = B::k(kkey) + kpc * (FP4 ? 4 : 16);
  const int v_ofs = B::v(page_rows, lane / 32) + vpc * 4 * B::kPiece + lane % 2 * 2 * B::kPiece;
  const int ks_ofs = B::ks(page_rows, kkey) + kpc * 8 / 32;
  const int vs_ofs = B::vs(page_rows, lane / 32) + vpc * PC / 32 * 4 + lane % 2 * 2;

  // two tiles of K and V for each key group
  __shared__ __attribute__((aligned(16))) uint16_t tiles[KG * 2 * MK * (D + KPAD + D + VPAD)];
  uint16_t(*Ks)[MK][D + KPAD] = reinterpret_cast<uint16_t(*)[MK][D + KPAD]>(tiles) + 2 * kg;
  uint16_t(*Vs)[MK][D + VPAD] = reinterpret_cast<uint16_t(*)[MK][D + VPAD]>(tiles + KG * 2 * MK * (D + KPAD)) + 2 * kg;
  // transposed-read coordinates of this lane inside its 16-lane group
  const int tr_row = 4 * half + ((lane & 15) >> 2);
  const int tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

  walk_items<MW>(a, unit, [&](const Item &it, int lo, int hi, bool whole, int slot) {
    const PageSeq seq = it.seq;
    const int kv = it.kv;
    const int p0 = it.p0, P = it.P;
    const int first = __builtin_amdgcn_readfirstlane(p0 / G), base = seq.len - seq.n;
    const int all_see = base + first + 1;   // keys that every row of the item sees
    const int32_t *table = a.seqs.tables + (int64_t)it.b * a.seqs.max_pages;
    const uint8_t *blocks = pool.pages + (int64_t)kv * pool.block_bytes;

    // this lane's query row
    const int p = p0 + 32 * rg + l32;
    const bool row_ok = p < P;
    const bool wave_rows = p0 + 32 * rg < P;      // (a wave without rows still fetches)
    int vis;                                // keys it sees
    bf16x8 qf[D / 16];
    {
      const int r = row_ok ? p / G : 0, g = row_ok ? p - r * G : 0;
      vis = row_ok ? base + r + 1 : 0;
      const uint16_t *q = a.q + (int64_t)(seq.r0 + r) * a.q_stride + (int64_t)(kv * G + g) * D + 8 * half;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) qf[kk] = row_ok ? *reinterpret_cast<const bf16x8 *>(q + 16 * kk) : bf16x8{};
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
    float m_run = kLowest, l_run = 0.f;
    float m_lim = (kLowest + 8.f) * inv_c;

    // Step s: tiles t_lo + s KG .. + KG - 1, one for each key group.  Lane x holds the page
    // of this wave's keys of step ids_at + x (-1: none)
    const int t_hi = (hi + MK - 1) / MK, t_lo = lo < hi ? lo / MK : t_hi;   // (an empty part starts anywhere)
    const int steps = (t_hi - t_lo + KG - 1) / KG;
    auto tile = [&](int s) { return t_lo + s * KG + kg; };
    int ids = -1, ids_at = 0;
    auto find_pages = [&](int s) {
      ids_at = s;
      const int64_t key = (int64_t)tile(s + lane) * MK + rg * WKEYS;
      ids = -1;
      if (s + lane < steps && key < hi) {
        ids = table[key >> rows_log];
        if (ids < 0 || ids >= pool.n_pages) {
          ids = -1;
          page_note(pool, HERMES_PAGE_BAD_ID);
        }
      }
    };
    uint32_t kw[WK], vw[NV][WV], ksc = 0, vsc[NV];
#pragma unroll
    for (int z = 0; z < NV; ++z) vsc[z] = 0;
    auto load = [&](int s) {
      if (s - ids_at >= 64) find_pages(s);
      const int id = __builtin_amdgcn_readlane(ids, s - ids_at);
      const int key0 = tile(s) * MK + rg * WKEYS, row = key0 & (page_rows - 1);
      const uint8_t *block = blocks + (int64_t)max(id, 0) * pool.page_bytes;
      load_words<WK>(kw, block + row * B::kRow + k_ofs);
#pragma unroll
      for (int z = 0; z < NV; ++z) load_words<WV>(vw[z], block + (row + 8 * z) * B::kRow + v_ofs);
      if constexpr (FP4) {
        ksc = *(block + row * B::kScales + ks_ofs);
#pragma unroll
        for (int z = 0; z < NV; ++z)
          vsc[z] = *reinterpret_cast<const uint16_t *>(block + (row + 8 * z) * B::kScales + vs_ofs);
      }
      // what lies past the length, or in no page, may be anything: zeros instead
      if (__builtin_expect(id < 0 || key0 + WKEYS > seq.len, 0)) {
        const int valid = id < 0 ? 0 : seq.len - key0;
        if (kkey >= valid) {
          ksc = 0;
#pragma unroll
          for (int i = 0; i < WK; ++i) kw[i] = 0u;
        }
#pragma unroll
        for (int z = 0; z < NV; ++z) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            if (vkey + 8 * z + j < valid) continue;
            if constexpr (FP4) {
              vsc[z] &= ~(0xFFu << (8 * j));
              if constexpr (D == 128) vw[z][j] = 0u;
              else vw[z][0] &= j == 1 ? 0x0000FFFFu : 0xFFFF0000u;
            } else {
#pragma unroll
              for (int i = 0; i < WV / 2; ++i) vw[z][j * (WV / 2) + i] = 0u;
            }
          }
        }
      }
    };
    auto store_tile = [&](int b) {
      uint16_t *kd = &Ks[b][rg * WKEYS + kkey][kpc * 8];
      const float sc = scale_of(ksc);
#pragma unroll
      for (int i = 0; i < UK; ++i) {
        uint4 x;
        if constexpr (FP4) x = uint4{fp4_pair(kw[i], sc, 0), fp4_pair(kw[i], sc, 1), fp4_pair(kw[i], sc, 2), fp4_pair(kw[i], sc, 3)};
        else x = uint4{kw[4 * i], kw[4 * i + 1], kw[4 * i + 2], kw[4 * i + 3]};
        *reinterpret_cast<uint4 *>(kd + 8 * i) = x;
      }
#pragma unroll
      for (int z = 0; z < NV; ++z) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint16_t *vd = &Vs[b][rg * WKEYS + vkey + 8 * z + j][vpc * PC];
          const uint32_t *w = vw[z];
          const float vs = scale_of(j == 0 ? vsc[z] & 0xFFu : vsc[z] >> 8);
          if constexpr (D == 128) {
            uint4 x;
            if constexpr (FP4) x = uint4{fp4_pair(w[j], vs, 0), fp4_pair(w[j], vs, 1), fp4_pair(w[j], vs, 2), fp4_pair(w[j], vs, 3)};
            else x = uint4{w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]};
            *reinterpret_cast<uint4 *>(vd) = x;
          } else {
            uint2 x;
            if constexpr (FP4) x = uint2{fp4_pair(w[0], vs, 2 * j), fp4_pair(w[0], vs, 2 * j + 1)};
            else x = uint2{w[2 * j], w[2 * j + 1]};
            *reinterpret_cast<uint2 *>(vd) = x;
          }
        }
      }
    };
    auto compute = [&](int b, int t, auto masked) {
      f32x16 s[SUB];
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
        s[sub] = f32x16{};
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          s[sub] = mfma32(*reinterpret_cast<const bf16x8 *>(&Ks[b][sub * 32 + l32][16 * kk + 8 * half]), qf[kk], s[sub]);
      }
#pragma unroll
      for (int i = 0; i < kAheadK; ++i) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int i = 0; i < SUB * (D / 16) - kAheadK; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
#pragma unroll
      for (int i = 0; i < kAheadK; ++i) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (decltype(masked)::value) {
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
          for (int jj = 0; jj < 16; ++jj)
            if (t * MK + sub * 32 + 8 * (jj >> 2) + 4 * half + (jj & 3) >= vis) s[sub][jj] = -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
        for (int jj = 0; jj < 16; ++jj) mx = fmaxf(mx, s[sub][jj]);
      }
      {
        // a row's keys are split over the lane halves
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float m0 = __uint_as_float(x[0]), m1 = __uint_as_float(x[1]);
        mx = m0 > m1 ? m0 : m1;
      }
      // the maximum moves only when it is passed by more than 2^8 (log2 domain)
      if (__builtin_expect(__any(mx > m_lim), 0)) {
        const float m_new = fmaxf(m_run, mx * c);
        const float alpha = fast_exp2(m_run - m_new);
        m_run = m_new;
        m_lim = (m_run + 8.f) * inv_c;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db) o[db] *= alpha;
      }
      bf16x8 pf[2 * SUB];
      float ls = 0.f;
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
        for (int jj = 0; jj < 16; ++jj) {
          const float x = fast_exp2(fmaf(s[sub][jj], c, -m_run));
          ls += x;
          pf[2 * sub + (jj >> 3)][jj & 7] = static_cast<__bf16>(x);   // (P enters an MFMA as bf16; the sum keeps fp32)
        }
      }
      l_run += ls;
      __builtin_amdgcn_s_setprio(1);        // (the SIMD's other wave fills in with its softmax)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
#pragma unroll
        for (int qq = 0; qq < 2 * SUB; ++qq) {
          const uint16_t *vp = &Vs[b][16 * qq + tr_row][32 * db + tr_col];
          const s4 x = lds_tr16(vp), y = lds_tr16(vp + 8 * (D + VPAD));
          o[db] = mfma32(__builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7)), pf[qq], o[db]);
        }
      }
      constexpr int kPV = D / 32 * 2 * SUB;
#pragma unroll
      for (int i = 0; i < 2 * kAheadV; ++i) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
#pragma unroll
      for (int i = 0; i < kPV - kAheadV; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
      }
#pragma unroll
      for (int i = 0; i < kAheadV; ++i) __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
      __builtin_amdgcn_s_setprio(0);
    };

    using Masked = std::integral_constant<bool, true>;
    using Open = std::integral_constant<bool, false>;
    __syncthreads();                        // the tiles (or states) of the item before are read
    if (steps > 0) {
      find_pages(0);
      load(0);
    }
    // steps whose tiles every row sees whole, two a trip so that each LDS buffer is a constant
    const int s_open = min(steps - 1, all_see > t_lo * MK ? (all_see / MK - t_lo) / KG : 0);
    int s = 0;
    for (; s + 1 < s_open; s += 2) {
      store_tile(0);
      __syncthreads();
      load(s + 1);
      if (wave_rows) compute(0, tile(s), Open{});
      store_tile(1);
      __syncthreads();
      load(s + 2);
      if (wave_rows) compute(1, tile(s + 1), Open{});
    }
    // (the rest are masked, needed or not: with both kinds in this loop the kernel takes
    // 345 registers instead of 202, and spills)
    for (int b = 0; s < steps; ++s, b ^= 1) {
      store_tile(b);
      __syncthreads();
      if (s + 1 < steps) load(s + 1);
      if (wave_rows && (KG == 1 || tile(s) < t_hi)) compute(b, tile(s), Masked{});
    }

    // The key groups' states merge through LDS: every wave leaves its (max, sum) and O there,
    // then wave kg of a row group merges the KG-th part of the channels, groups in order.
    // fn(c, x) gets channels 8 c + 4 half .. of this lane's row.
    constexpr int NC = D / 8;
    float l = l_run + __shfl_xor(l_run, 32);
    auto own = [&](int i) {
      return float4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    };
    auto merge = [&](auto fn) {
      if constexpr (KG == 1) {
#pragma unroll
        for (int i = 0; i < NC; ++i) fn(i, own(i));
      } else {
        static_assert(MW * NC * 64 * 16 + MW * 32 * 8 <= (int)sizeof(tiles), "the states fit");
        float4 *mo = reinterpret_cast<float4 *>(tiles);
        float2 *mm = reinterpret_cast<float2 *>(mo + MW * NC * 64);
        __syncthreads();                    // all tiles are read
#pragma unroll
        for (int i = 0; i < NC; ++i) mo[(wave * NC + i) * 64 + lane] = own(i);
        if (half == 0) mm[wave * 32 + l32] = float2{m_run, l};
        __syncthreads();
        float w[KG];
        m_run = kLowest;
#pragma unroll
        for (int x = 0; x < KG; ++x) m_run = fmaxf(m_run, mm[(x * RG + rg) * 32 + l32].x);
        l = 0.f;
#pragma unroll
        for (int x = 0; x < KG; ++x) {
          const float2 y = mm[(x * RG + rg) * 32 + l32];
          w[x] = fast_exp2(y.x - m_run);
          l += w[x] * y.y;
        }
#pragma unroll
        for (int i = 0; i < NC / KG; ++i) {
          const int at = kg * (NC / KG) + i;
          float4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < KG; ++x) {
            const float4 y = mo[((x * RG + rg) * NC + at) * 64 + lane];
            t.x += w[x] * y.x;
            t.y += w[x] * y.y;
            t.z += w[x] * y.z;
            t.w += w[x] * y.w;
          }
          fn(at, t);
        }
      }
    };
    if (!whole) {
      const int64_t part = (int64_t)(2 * unit + slot) * MROWS + 32 * rg;
      float4 *op = reinterpret_cast<float4 *>(a.opart + part * D) + lane;   // [channels / 8][lane]
      if (hi > lo) {                        // (an empty part leaves its O unwritten, and unread)
        merge([&](int i, float4 x) {
          if (row_ok) op[i * 64] = x;
        });
      }
      if (row_ok && half == 0 && kg == 0) *reinterpret_cast<float2 *>(a.mlpart + 2 * (part + l32)) = float2{m_run, l};
    } else {
      const int r = row_ok ? p / G : 0;
      const int64_t at = (int64_t)(seq.r0 + r) * Hq + kv * G + (row_ok ? p - r * G : 0);
      uint16_t *orow = a.out + at * D + 4 * half;
      merge([&](int i, float4 x) {
        const float inv = l == 0.f ? 0.f : 1.f / l;   // (0: the row sees nothing; a NaN stays one)
        if (row_ok)
          *reinterpret_cast<uint2 *>(orow + 8 * i) =
              uint2{f2bf(x.x * inv) | f2bf(x.y * inv) << 16, f2bf(x.z * inv) | f2bf(x.w * inv) << 16};
      });
      if (row_ok && a.lse != nullptr && half == 0 && kg == 0) a.lse[at] = l == 0.f ? -INFINITY : (m_run + log2f(l)) * kLn2;
    }
  });
}

// -------------------------------------------------------------------- the joins
// O = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m) over the parts s of a cut
// item.  A task is 256 float4 of an item of a few parts, 64 a wave, or 64 of an item of
// more, whose parts its four waves share out (wave w takes w, w + 4, ..., and their sums
// are joined in wave order); its loads are four parts at once.  Most units hold no
// first cut when items are long, so every workgroup adds up all cuts' tasks and takes
// every gridDim.x-th (with a workgroup for each (unit, 64 float4), 64 rows on 8192 tokens
// took 34 us here, most of it workgroups that found nothing to do).
constexpr int kJoinUnits = kStreamSlots;   // units of a launch with cuts at most: a thread a unit
constexpr int kFewParts = 4;
static_assert(kJoinUnits == 256, "a thread a unit");

template <int D, bool MANY>
__global__ __launch_bounds__(256) void page_combine(PageAttnArgs a) {
  __shared__ int upto[kJoinUnits];      // tasks of the cuts 0 .. i
  __shared__ int wsum[4];
  __shared__ float4 sacc[4][64];
  __shared__ float2 sml[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int rows = a.plan.rows;
  // float4 groups of 64 that hold rows of a cut's item
  auto groups = [&](const PageCut &c) {
    const int n = min(rows, c.P - c.p0);
    return MANY ? (n + 31) / 32 * (D / 8) : (n * (D / 4) + 63) / 64;
  };
  int n = 0;
  if ((int)threadIdx.x < a.plan.units) {
    const PageCut c = a.cuts[threadIdx.x];
    const int parts = c.last - c.first + 1;
    if (parts > 0) n = parts > kFewParts ? groups(c) : (groups(c) + 3) / 4;
  }
  const int64_t sums = wave_sums(n);
  if (lane == 63) wsum[wave] = (int)sums;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    before += w < wave ? wsum[w] : 0;
    total += wsum[w];
  }
  upto[threadIdx.x] = before + (int)sums;
  __syncthreads();

  for (int task = blockIdx.x; task < total; task += gridDim.x) {
    int lo = 0, hi = kJoinUnits - 1;    // the first cut with upto > task
    while (lo < hi) {
      const int m = (lo + hi) / 2;
      if (upto[m] > task) hi = m; else lo = m + 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const PageCut cut = a.cuts[lo];
    const int parts = cut.last - cut.first + 1, nth = task - (lo > 0 ? upto[lo - 1] : 0);
    const bool shared = parts > kFewParts;
    // which row and channels float4 `i` of a part holds
    const int i = (shared ? nth : 4 * nth + wave) * 64 + lane;
    int row, ch;
    if constexpr (MANY) {     // [32 rows][channels / 8][lane]
      row = i / (D / 8 * 64) * 32 + i % 32;
      ch = i / 64 % (D / 8) * 8 + i / 32 % 2 * 4;
    } else {
      row = i / (D / 4);
      ch = i % (D / 4) * 4;
    }
    const bool ok = row < min(rows, cut.P - cut.p0);
    auto part = [&](int s) { return (int64_t)2 * (cut.first + s) + (s == 0 ? cut.slot : 0); };
    float m = kLowest, l = 0.f;
    float4 acc = {0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 4;
    const int step = shared ? 4 : 1;
    for (int s0 = shared ? wave : 0; s0 < parts; s0 += step * AHEAD) {
      float2 ml[AHEAD];
      float4 o[AHEAD];
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        const int s = s0 + step * x;
        ml[x] = float2{kLowest, 0.f};
        o[x] = float4{0.f, 0.f, 0.f, 0.f};
        if (s < parts && ok) {
          ml[x] = *reinterpret_cast<const float2 *>(a.mlpart + 2 * (part(s) * rows + row));
          o[x] = reinterpret_cast<const float4 *>(a.opart + part(s) * rows * D)[i];
        }
      }
      float mn = m;
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) mn = fmaxf(mn, ml[x].x);
      const float old = fast_exp2(m - mn);
      m = mn;
      l *= old;
      acc = float4{acc.x * old, acc.y * old, acc.z * old, acc.w * old};
#pragma unroll
      for (int x = 0; x < AHEAD; ++x) {
        if (ml[x].y == 0.f) continue;      // (an empty part, whose O was not written)
        const float w = fast_exp2(ml[x].x - m);
        l += w * ml[x].y;
        acc.x += w * o[x].x;
        acc.y += w * o[x].y;
        acc.z += w * o[x].z;
        acc.w += w * o[x].w;
      }
    }
    if (shared) {
      sacc[wave][lane] = acc;
      sml[wave][lane] = float2{m, l};
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) m = fmaxf(m, sml[w][lane].x);
        acc = float4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 x = sml[w][lane];
          const float4 y = sacc[w][lane];
          const float e = fast_exp2(x.x - m);
          l += e * x.y;
          acc.x += e * y.x;
          acc.y += e * y.y;
          acc.z += e * y.z;
          acc.w += e * y.w;
        }
      }
      __syncthreads();                     // (the next task writes there)
      if (wave != 0) continue;
    }
    if (!ok) continue;
    const int G = a.pool.Hq / a.pool.Hkv;
    const int p = cut.p0 + row, r = p / G, g = p - r * G;
    const int64_t at = (int64_t)(cut.r0 + r) * a.pool.Hq + cut.kv * G + g;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2 *>(a.out + at * D + ch) =
        uint2{f2bf(acc.x * inv) | f2bf(acc.y * inv) << 16, f2bf(acc.z * inv) | f2bf(acc.w * inv) << 16};
    if (a.lse != nullptr && ch == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

template <int D, bool FP4>
hipError_t attend(const PageAttnArgs &a, hipStream_t s) {
  const dim3 grid(a.plan.units);
  const int rows = a.plan.rows;
  const bool four = a.plan.step == 128;
  if (rows == 16 && four) hipLaunchKernelGGL((page_attn_few<D, FP4, 1, 4>), grid, dim3(256), 0, s, a);
  else if (rows == 16) hipLaunchKernelGGL((page_attn_few<D, FP4, 1, 8>), grid, dim3(512), 0, s, a);
  else if (rows == 32 && four) hipLaunchKernelGGL((page_attn_few<D, FP4, 2, 4>), grid, dim3(256), 0, s, a);
  else if (rows == 32) hipLaunchKernelGGL((page_attn_few<D, FP4, 2, 8>), grid, dim3(512), 0, s, a);
  else if (rows == 64) hipLaunchKernelGGL((page_attn_many<D, FP4, 2>), grid, dim3(MT), 0, s, a);
  else if (rows == 128) hipLaunchKernelGGL((page_attn_many<D, FP4, 4>), grid, dim3(MT), 0, s, a);
  else hipLaunchKernelGGL((page_attn_many<D, FP4, 8>), grid, dim3(MT), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.plan.tiles > 0) return e;
  const dim3 joins(8 * kStreamSlots);
  if (rows <= 32) hipLaunchKernelGGL((page_combine<D, false>), joins, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((page_combine<D, true>), joins, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_attend(const PageAttnArgs &a, int head_dim, int format, hipStream_t s) {
  if (format == HERMES_PAGE_FP4) return head_dim == 64 ? attend<64, true>(a, s) : attend<128, true>(a, s);
  return head_dim == 64 ? attend<64, false>(a, s) : attend<128, false>(a, s);
}

}  // namespace hermes
