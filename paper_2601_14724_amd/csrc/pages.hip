// Rows into pages and back, for gfx950:
//
// page_append  rotates new keys and queries to their positions and stores keys
//              and values in their sequence's pages, in bf16 or FP4;
// page_pack    stores a context's compact caches (keys already rotated);
// page_read    gives stored rows back as bf16.
//
// All three move each row once and are bound by HBM where there are many rows, by
// latency where there are few.  The 64 lanes of a wave hold 64 pieces of eight
// channels (16 bytes) of a row, that is 512 / d heads at a time.
//
// Rotation: x'_j = x_j cos a_j - x_{j + d/2} sin a_j, x'_{j + d/2} = x_{j + d/2}
// cos a_j + x_j sin a_j, a_j = p theta^(-2j/d), all in fp64 (positions of a long
// stream pass 2^17, where an fp32 angle is off by 2^-7), rounded to fp32 and then
// bf16 as the re-indexing rotation does.  One sine and cosine a lane and row: lane
// f has frequency f % (d/2), and the row's heads share them through LDS.
//
// FP4: a block of 32 channels lies in four neighbouring lanes.  Its scale 2^e is
// the least with amax <= 7 x 2^e: with amax = m 2^E, 1 <= m < 2, e is E - 2, or E - 1
// if m > 1.75, which on the bits of a bf16 magnitude is ((bits + 31) >> 7) - 2
// (m > 1.75 exactly if the 7 mantissa bits are 97 or more).  The hardware
// conversion rounds to nearest, ties to even, and saturates, for every bf16 value
// (all 65536, at scales from 2^-119 to 2^125, agree with the definition).
#include "pages_internal.h"

namespace hermes {
namespace {

constexpr int NT = 256;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ double bf16_to_f64(uint16_t b) {
  return (double)__builtin_bit_cast(float, (uint32_t)b << 16);
}

// fp64 -> fp32 -> bf16, both to nearest even; on the bits, so that the compiler
// does not make one rounding of the two.
__device__ __forceinline__ uint32_t f64_to_bf16(double x) {
  const float f = (float)x;
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  // (a NaN's payload must not carry into the exponent)
  return f != f ? 0x7FC0u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ uint4 shfl_xor4(uint4 v, int m) {
  return uint4{(uint32_t)__shfl_xor((int)v.x, m), (uint32_t)__shfl_xor((int)v.y, m),
               (uint32_t)__shfl_xor((int)v.z, m), (uint32_t)__shfl_xor((int)v.w, m)};
}

// The scale byte of this lane's block of 32 channels (its four lanes agree).
__device__ __forceinline__ uint32_t fp4_scale(const uint4 &x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = max(m, w[i] & 0x7FFFu);
    m = max(m, (w[i] >> 16) & 0x7FFFu);
  }
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  m = max(m, (uint32_t)__shfl_xor((int)m, 2));
  if (m >= 0x7F80u) return 255u;            // an infinity or a NaN: the block is NaN
  return (uint32_t)min(max((int)((m + 31u) >> 7) - 2, 127 - 119), 127 + 125);
}

// The codes of eight bf16 channels.
__device__ __forceinline__ uint32_t fp4_codes(const uint4 &x, uint32_t scale) {
  const float sc = __builtin_bit_cast(float, scale << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x.x), sc, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x.y), sc, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x.z), sc, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x.w), sc, 3);
  return r;
}

__device__ __forceinline__ uint4 fp4_values(uint32_t codes, uint32_t scale) {
  const float sc = __builtin_bit_cast(float, scale << 23);
  return uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 3))};
}

// Stores eight channels (8 piece ..) of row r of a KV head's block.  Every lane
// of the wave calls it (the scales are found across lanes); `on` ones store.
template <int D, bool FP4>
__device__ __forceinline__ void store_k(uint8_t *block, int rows, int r, int piece, const uint4 &x, bool on) {
  using B = PageBlock<D, FP4>;
  if constexpr (FP4) {
    const uint32_t scale = fp4_scale(x);
    if (!on) return;
    *reinterpret_cast<uint32_t *>(block + B::k(r) + 4 * piece) = fp4_codes(x, scale);
    if (piece % 4 == 0) block[B::ks(rows, r) + piece / 4] = (uint8_t)scale;
  } else {
    if (on) *reinterpret_cast<uint4 *>(block + B::k(r) + 16 * piece) = x;
  }
}

template <int D, bool FP4>
__device__ __forceinline__ void store_v(uint8_t *block, int rows, int r, int piece, const uint4 &x, bool on) {
  using B = PageBlock<D, FP4>;
  // (at head size 64 eight channels are two pieces of V)
  uint8_t *at = block + B::v(rows, r / 4) + piece * (D == 128 ? 1 : 2) * 4 * B::kPiece + r % 4 * B::kPiece;
  if constexpr (FP4) {
    const uint32_t scale = fp4_scale(x);
    if (!on) return;
    const uint32_t c = fp4_codes(x, scale);
    if constexpr (D == 128) {
      *reinterpret_cast<uint32_t *>(at) = c;
    } else {
      *reinterpret_cast<uint16_t *>(at) = (uint16_t)c;
      *reinterpret_cast<uint16_t *>(at + 4 * B::kPiece) = (uint16_t)(c >> 16);
    }
    if (piece % 4 == 0) block[B::vs(rows, r / 4) + piece / 4 * 4 + r % 4] = (uint8_t)scale;
  } else {
    if (!on) return;
    if constexpr (D == 128) {
      *reinterpret_cast<uint4 *>(at) = x;
    } else {
      *reinterpret_cast<uint2 *>(at) = uint2{x.x, x.y};
      *reinterpret_cast<uint2 *>(at + 4 * B::kPiece) = uint2{x.z, x.w};
    }
  }
}

template <int D, bool FP4>
__device__ __forceinline__ uint4 load_k(const uint8_t *block, int rows, int r, int piece) {
  using B = PageBlock<D, FP4>;
  if constexpr (FP4)
    return fp4_values(*reinterpret_cast<const uint32_t *>(block + B::k(r) + 4 * piece), block[B::ks(rows, r) + piece / 4]);
  else
    return *reinterpret_cast<const uint4 *>(block + B::k(r) + 16 * piece);
}

template <int D, bool FP4>
__device__ __forceinline__ uint4 load_v(const uint8_t *block, int rows, int r, int piece) {
  using B = PageBlock<D, FP4>;
  const uint8_t *at = block + B::v(rows, r / 4) + piece * (D == 128 ? 1 : 2) * 4 * B::kPiece + r % 4 * B::kPiece;
  if constexpr (FP4) {
    uint32_t c;
    if constexpr (D == 128) {
      c = *reinterpret_cast<const uint32_t *>(at);
    } else {
      c = *reinterpret_cast<const uint16_t *>(at) | (uint32_t)*reinterpret_cast<const uint16_t *>(at + 4 * B::kPiece) << 16;
    }
    return fp4_values(c, block[B::vs(rows, r / 4) + piece / 4 * 4 + r % 4]);
  } else if constexpr (D == 128) {
    return *reinterpret_cast<const uint4 *>(at);
  } else {
    const uint2 x = *reinterpret_cast<const uint2 *>(at), y = *reinterpret_cast<const uint2 *>(at + 4 * B::kPiece);
    return uint4{x.x, x.y, y.x, y.y};
  }
}

// Stores rows r .. r + 3 (r a multiple of 4) in FP4 at head size 128, eight channels a
// lane, with four stores: the four rows' codes of V are neighbours, and so are four lanes'
// codes of a row of K, which the lanes of a block exchange (lane y of the four gets row
// r + y).
__device__ __forceinline__ void store_four(uint8_t *block, int rows, int r, int piece, const uint4 *x, const uint4 *y,
                                           bool on) {
  using B = PageBlock<128, true>;
  uint32_t kc[4], vc[4], ks[4], vs = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    ks[u] = fp4_scale(x[u]);
    kc[u] = fp4_codes(x[u], ks[u]);
    const uint32_t s = fp4_scale(y[u]);
    vc[u] = fp4_codes(y[u], s);
    vs |= s << (8 * u);
  }
  // a transpose of 4 x 4 over the rows (registers) and the block's lanes
  const int q = piece & 3;
#pragma unroll
  for (int b = 1; b <= 2; b *= 2) {
    const bool high = (q & b) != 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (u & b) continue;
      const uint32_t give = high ? kc[u] : kc[u | b];
      const uint32_t got = (uint32_t)__shfl_xor((int)give, b);
      if (high) kc[u] = got; else kc[u | b] = got;
    }
  }
  const uint32_t scale = q == 0 ? ks[0] : q == 1 ? ks[1] : q == 2 ? ks[2] : ks[3];
  if (!on) return;
  *reinterpret_cast<uint4 *>(block + B::k(r + q) + 16 * (piece / 4)) = uint4{kc[0], kc[1], kc[2], kc[3]};
  *reinterpret_cast<uint4 *>(block + B::v(rows, r / 4) + 16 * piece) = uint4{vc[0], vc[1], vc[2], vc[3]};
  block[B::ks(rows, r + q) + piece / 4] = (uint8_t)scale;
  if (q == 0) *reinterpret_cast<uint32_t *>(block + B::vs(rows, r / 4) + piece / 4 * 4) = vs;
}

// Finds where stacked rows are stored; every call is the whole wave's, and its results
// are the same in every lane.
struct Finder {
  const PagePool &pool;
  const PageSeqs &seqs;
  int start, len;           // with up to 63 sequences: lane b has row_start[b] and kv_len[b]
  int b;                    // else: the last row's sequence
  PageSeq seq;

  __device__ __forceinline__ Finder(const PagePool &p, const PageSeqs &s) : pool(p), seqs(s), start(0), len(0), b(-1) {
    seq = PageSeq{0, 0, 0};
    if (lanes()) {
      const int lane = threadIdx.x & 63;
      if (s.row_start != nullptr && lane <= s.n_seqs) start = s.row_start[lane];
      if (lane < s.n_seqs) len = s.kv_len[lane];
    }
  }
  __device__ __forceinline__ bool lanes() const { return seqs.n_seqs < 64; }

  // The sequence of row `row` (-1: none): the last b with row_start[b] <= row.  Each round
  // of the search the lanes probe 64 evenly spaced starts.
  __device__ __forceinline__ int seq_of(int row) const {
    if (seqs.row_start == nullptr) return row;
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = seqs.n_seqs + 1;       // the first start beyond the row lies in [lo, hi]
    if (lanes()) {
      const unsigned long long m = __ballot(lane >= hi || start > row);
      lo = m == 0ull ? hi : min((int)__builtin_ctzll(m), hi);
    } else {
      while (lo < hi) {
        const int step = (hi - lo + 63) / 64;
        const int p = lo + (lane + 1) * step - 1;
        const unsigned long long m = __ballot(p >= hi || seqs.row_start[p] > row);
        if (m == 0ull) {
          lo = hi;
        } else {
          const int k = __builtin_ctzll(m);
          const int pk = lo + (k + 1) * step - 1;
          lo += k * step;
          hi = min(hi, pk);
        }
      }
    }
    return lo > seqs.n_seqs ? -1 : __builtin_amdgcn_readfirstlane(lo - 1);
  }

  // A row's sequence b, and its token t there (t < 0: not stored); false: in none.
  __device__ __forceinline__ bool token_of(int row, int *t) {
    if (b < 0 || seqs.row_start == nullptr || lanes() || row < seq.r0 || row >= seq.r0 + seq.n) {
      b = seq_of(row);
      if (b < 0) return false;
      if (lanes()) {
        // (as page_seq, from the lanes)
        int a0 = b, a1 = b + 1;
        if (seqs.row_start != nullptr) {
          a0 = __builtin_amdgcn_readlane(start, b);
          a1 = __builtin_amdgcn_readlane(start, b + 1);
        }
        seq = page_seq_of(pool, seqs, a0, a1, __builtin_amdgcn_readlane(len, b));
      } else {
        const PageSeq x = page_seq(pool, seqs, b);
        seq = PageSeq{__builtin_amdgcn_readfirstlane(x.r0), __builtin_amdgcn_readfirstlane(x.n),
                      __builtin_amdgcn_readfirstlane(x.len)};
      }
    }
    if (row < seq.r0 || row >= seq.r0 + seq.n) return false;   // (starts that fall)
    *t = seq.len - seq.n + (row - seq.r0);
    return true;
  }

  // The page of token t of sequence b: its id as the table has it (t < 0: -1).
  __device__ __forceinline__ int id_of(int t) const {
    return t < 0 ? -1 : seqs.tables[(int64_t)b * seqs.max_pages + (t >> pool.log_rows)];
  }
  // and checked (-1: none)
  __device__ __forceinline__ int checked(int t, int id) const {
    if (t < 0) return -1;
    if (id < 0 || id >= pool.n_pages) {
      page_note(pool, HERMES_PAGE_BAD_ID);
      return -1;
    }
    return __builtin_amdgcn_readfirstlane(id);
  }
};

// A row's passes (512 / d heads of q each, then of k and v) are shared by a.share waves: one
// where the rows fill the device, four where they do not and a row's latency counts (28 + 4
// heads of 128, four waves and one: 16 rows 4.6 and 7.0 us, 1000 7.9 and 8.6, 4000 19.0 and 17.1).
constexpr int kAhead = 4;           // passes of q whose loads are on their way at once
template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_append(PageAppendArgs a) {
  constexpr int HD = D / 2, CH = D / 8, HP = 64 / CH;    // pieces of a head, heads of a pass
  __shared__ double2 trig[NT / 64][72];     // frequency f at f + f / 8: a wave reads every eighth at once
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int share = a.share, nth = wave % share;
  const int row = blockIdx.x * (NT / 64 / share) + wave / share;
  if (row >= a.seqs.n_rows) return;
  const int Hq = a.q != nullptr ? a.pool.Hq : 0, Hkv = a.pool.Hkv;
  const int q_passes = (Hq + HP - 1) / HP;
  const int piece = lane % CH, hl = lane / CH;
  const bool turn = a.rope != nullptr, second = piece >= CH / 2;
  const int f0 = 9 * (piece % (CH / 2));    // (where the piece's eight frequencies lie)
  const uint16_t *q = a.q + (int64_t)row * a.q_stride;
  const uint16_t *k = a.k + (int64_t)row * a.k_stride, *v = a.v + (int64_t)row * a.v_stride;

  const int f = lane % HD;
  const double freq = turn ? a.inv_freq[f] : 0.0;
  Finder find(a.pool, a.seqs);
  int t = -1;
  if (!find.token_of(row, &t)) return;
  // Only now the row's inputs: rows of no sequence may lie in no memory.  (Asked for before,
  // 16 rows took 4.39 us instead of 4.44, 28 x 784 rows 80 instead of 77.5.)
  int pos = 0;
  if (turn) {
    const int axis = a.axes != 3 ? 0 : f < a.section[0] ? 0 : f < a.section[0] + a.section[1] ? 1 : 2;
    pos = a.rope[(int64_t)axis * a.seqs.n_rows + row];
  }
  auto load_q = [&](uint4 *x, int pass0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = (pass0 + u * share) * HP + hl;
      if (h < Hq) x[u] = *reinterpret_cast<const uint4 *>(q + h * D + 8 * piece);
    }
  };
  uint4 x[kAhead];
  load_q(x, nth);
  const int id = find.id_of(t);
  if (turn) {
    double sn, cs;
    sincos((double)pos * freq, &sn, &cs);
    trig[wave][lane + lane / 8] = double2{cs, sn};
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  auto rotated = [&](const uint4 &x) {
    const uint4 y = shfl_xor4(x, CH / 2);             // the other half of each pair
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const double2 c = trig[wave][f0 + 2 * i + h];
        const double xd = bf16_to_f64((uint16_t)(xw[i] >> (16 * h))), yd = bf16_to_f64((uint16_t)(yw[i] >> (16 * h)));
        const double xc = __dmul_rn(xd, c.x), ys = __dmul_rn(yd, c.y);
        w[i] |= f64_to_bf16(second ? __dadd_rn(xc, ys) : __dsub_rn(xc, ys)) << (16 * h);
      }
    }
    return uint4{w[0], w[1], w[2], w[3]};
  };
  const int page_id = find.checked(t, id);
  const int rows = 1 << a.pool.log_rows, r = t & (rows - 1);
  uint8_t *page = a.pool.pages + (int64_t)max(page_id, 0) * a.pool.page_bytes;
  uint16_t *o = a.q_out + (int64_t)row * Hq * D;
  for (int pass0 = nth; pass0 < q_passes; pass0 += kAhead * share) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = (pass0 + u * share) * HP + hl;
      if (pass0 + u * share >= q_passes) break;
      const uint4 z = rotated(x[u]);
      if (h < Hq) *reinterpret_cast<uint4 *>(o + h * D + 8 * piece) = z;
    }
    load_q(x, pass0 + kAhead * share);
  }
  // (the passes of k and v go on where those of q ended, so that the waves have equal shares)
  const int first = (nth + share - q_passes % share) % share;
  for (int pass = first; pass * HP < Hkv; pass += share) {
    const int h = pass * HP + hl, e = h * D + 8 * piece;
    uint4 kx = {0u, 0u, 0u, 0u}, vx = {0u, 0u, 0u, 0u};
    if (h < Hkv) {
      kx = *reinterpret_cast<const uint4 *>(k + e);
      vx = *reinterpret_cast<const uint4 *>(v + e);
    }
    if (turn) kx = rotated(kx);
    const bool on = h < Hkv && page_id >= 0;
    uint8_t *block = page + (int64_t)h * a.pool.block_bytes;
    store_k<D, FP4>(block, rows, r, piece, kx, on);
    store_v<D, FP4>(block, rows, r, piece, vx, on);
  }
}

// A wave reads two rows, whose loads are on their way at once: 28 layers' 114688 rows of 4
// heads of 128 take 71 us (297 MB, 4.2 TB/s), with one row a wave 80 and with four 79.
constexpr int RR = 2;
template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_read(PageReadArgs a) {
  constexpr int CH = D / 8, HP = 64 / CH;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row0 = (blockIdx.x * (NT / 64) + wave) * RR;
  if (row0 >= a.seqs.n_rows) return;
  const int Hkv = a.pool.Hkv, piece = lane % CH, hl = lane / CH;
  const int rows = 1 << a.pool.log_rows;
  Finder find(a.pool, a.seqs);
  bool mine[RR];
  int t[RR], id[RR];
#pragma unroll
  for (int u = 0; u < RR; ++u) {
    t[u] = -1;
    mine[u] = row0 + u < a.seqs.n_rows && find.token_of(row0 + u, &t[u]);
    id[u] = mine[u] ? find.id_of(t[u]) : -1;
  }
#pragma unroll
  for (int u = 0; u < RR; ++u) id[u] = mine[u] ? find.checked(t[u], id[u]) : -1;
  for (int h = hl; h < Hkv; h += HP) {
    uint4 x[RR], y[RR];
#pragma unroll
    for (int u = 0; u < RR; ++u) {
      x[u] = y[u] = uint4{0u, 0u, 0u, 0u};
      if (id[u] >= 0) {
        const uint8_t *block = a.pool.pages + (int64_t)id[u] * a.pool.page_bytes + (int64_t)h * a.pool.block_bytes;
        x[u] = load_k<D, FP4>(block, rows, t[u] & (rows - 1), piece);
        y[u] = load_v<D, FP4>(block, rows, t[u] & (rows - 1), piece);
      }
    }
#pragma unroll
    for (int u = 0; u < RR; ++u) {
      if (!mine[u]) continue;
      const int64_t e = ((int64_t)(row0 + u) * Hkv + h) * D + 8 * piece;
      if (a.k != nullptr) *reinterpret_cast<uint4 *>(a.k + e) = x[u];
      if (a.v != nullptr) *reinterpret_cast<uint4 *>(a.v + e) = y[u];
    }
  }
}

// With FP4 a wave packs four rows, which lie in one page and are one group of V's layout
// (28 layers' 114688 rows of 4 heads of 128: 59 us, 297 MB; a row a wave, 62).  bf16 rows
// leave in whole lines anyway, and take a wave each (91 us, 470 MB; four rows, 100).
template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_pack(PagePackArgs a) {
  constexpr int CH = D / 8, HP = 64 / CH, PR = FP4 ? 4 : 1;
  const int j = blockIdx.y, len = a.len[j];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.kv_len[j] = len;
  const int row0 = (blockIdx.x * (NT / 64) + wave) * PR;
  if (row0 >= len) return;
  int id = a.tables[(int64_t)j * a.max_pages + (row0 >> a.pool.log_rows)];
  const int Hkv = a.pool.Hkv, piece = lane % CH, hl = lane / CH;
  const int rows = 1 << a.pool.log_rows, r = row0 & (rows - 1);
  const uint16_t *k = a.k[j] + (int64_t)row0 * Hkv * D, *v = a.v[j] + (int64_t)row0 * Hkv * D;
  for (int h0 = 0; h0 < Hkv; h0 += HP) {
    const int h = h0 + hl, e = h * D + 8 * piece;
    uint4 x[PR], y[PR];
#pragma unroll
    for (int u = 0; u < PR; ++u) {
      x[u] = y[u] = uint4{0u, 0u, 0u, 0u};
      if (h < Hkv && row0 + u < len) {
        x[u] = *reinterpret_cast<const uint4 *>(k + (int64_t)u * Hkv * D + e);
        y[u] = *reinterpret_cast<const uint4 *>(v + (int64_t)u * Hkv * D + e);
      }
    }
    if (h0 == 0) {
      id = __builtin_amdgcn_readfirstlane(id);
      if (id < 0 || id >= a.pool.n_pages) {
        page_note(a.pool, HERMES_PAGE_BAD_ID);
        return;
      }
    }
    uint8_t *block = a.pool.pages + (int64_t)id * a.pool.page_bytes + (int64_t)h * a.pool.block_bytes;
    if constexpr (FP4 && D == 128) {
      if (row0 + PR <= len) {
        store_four(block, rows, r, piece, x, y, h < Hkv);
        continue;
      }
    }
#pragma unroll
    for (int u = 0; u < PR; ++u) {
      const bool on = h < Hkv && row0 + u < len;
      store_k<D, FP4>(block, rows, r + u, piece, x[u], on);
      store_v<D, FP4>(block, rows, r + u, piece, y[u], on);
    }
  }
}

// fn(head size, whether FP4) with both as constants
template <typename F>
hipError_t with_kind(int head_dim, int format, F &&fn) {
  using Yes = std::integral_constant<bool, true>;
  using No = std::integral_constant<bool, false>;
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (format == HERMES_PAGE_FP4) head_dim == 64 ? fn(D64{}, Yes{}) : fn(D128{}, Yes{});
  else head_dim == 64 ? fn(D64{}, No{}) : fn(D128{}, No{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_append(const PageAppendArgs &a, int head_dim, int format, hipStream_t s) {
  const int per = NT / 64 / a.share;
  const dim3 grid((unsigned)((a.seqs.n_rows + per - 1) / per));
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_append<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

hipError_t launch_page_read(const PageReadArgs &a, int head_dim, int format, hipStream_t s) {
  constexpr int per = NT / 64 * RR;
  const dim3 grid((unsigned)((a.seqs.n_rows + per - 1) / per));
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_read<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

hipError_t launch_page_pack(const PagePackArgs &a, int head_dim, int format, hipStream_t s) {
  int most = 1;                                        // (an empty layer's length is written too)
  for (int j = 0; j < a.n_list; ++j) most = max(most, a.len[j]);
  const int per = NT / 64 * (format == HERMES_PAGE_FP4 ? 4 : 1);
  const dim3 grid((unsigned)(((int64_t)most + per - 1) / per), a.n_list);
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_pack<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

}  // namespace hermes
