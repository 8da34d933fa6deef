// Rows into pages and back, for gfx950:
//
// page_append  rotates new keys and queries to their positions and stores keys
//              and values in their sequence's pages, in bf16 or FP4;
// page_pack    stores a context's compact caches (keys already rotated);
// page_read    gives stored rows back as bf16.
//
// All three move each row once and are bound by HBM where there are many rows, by
// latency where there are few.  A wave takes one row: its 64 lanes hold 64
// pieces of eight channels (16 bytes), that is 512 / d heads at a time.
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

// The sequence of stacked row `row` (-1: none), found by the whole wave: the last
// b with row_start[b] <= row, if the row lies before its end.  Each round the
// lanes probe 64 evenly spaced starts.
__device__ __forceinline__ int seq_of_row(const PageSeqs &s, int row) {
  if (s.row_start == nullptr) return row;
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = s.n_seqs + 1;            // the first start beyond the row lies in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64;
    const int p = lo + (lane + 1) * step - 1;
    const unsigned long long m = __ballot(p >= hi || s.row_start[p] > row);
    if (m == 0ull) {
      lo = hi;
    } else {
      const int k = __builtin_ctzll(m);
      const int pk = lo + (k + 1) * step - 1;
      lo += k * step;
      hi = min(hi, pk);
    }
  }
  return lo > s.n_seqs ? -1 : lo - 1;
}

// Where stacked row `row` is stored: its sequence's page and its row there.
// page < 0: nowhere.  Wave-uniform.
struct Place {
  int page, r;
  bool mine;                // the row belongs to a sequence
};
__device__ __forceinline__ Place place_of(const PagePool &p, const PageSeqs &s, int row) {
  Place x = {-1, 0, false};
  const int b = __builtin_amdgcn_readfirstlane(seq_of_row(s, row));
  if (b < 0) return x;
  const PageSeq q = page_seq(p, s, b);
  if (row < q.r0 || row >= q.r0 + q.n) return x;    // (starts that fall)
  x.mine = true;
  const int t = q.len - q.n + (row - q.r0);
  if (t < 0) return x;
  const int id = s.tables[(int64_t)b * s.max_pages + (t >> p.log_rows)];
  if (id < 0 || id >= p.n_pages) {
    page_note(p, HERMES_PAGE_BAD_ID);
    return x;
  }
  x.page = __builtin_amdgcn_readfirstlane(id);
  x.r = __builtin_amdgcn_readfirstlane(t & ((1 << p.log_rows) - 1));
  return x;
}

template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_append(PageAppendArgs a) {
  constexpr int HD = D / 2, CH = D / 8, HP = 64 / CH;    // pieces of a head, heads of a pass
  __shared__ double2 trig[NT / 64][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = blockIdx.x * (NT / 64) + wave;
  if (row >= a.seqs.n_rows) return;
  const Place at = place_of(a.pool, a.seqs, row);
  if (!at.mine) return;
  const int Hq = a.pool.Hq, Hkv = a.pool.Hkv;
  const int piece = lane % CH, hl = lane / CH;
  const bool turn = a.rope != nullptr, second = piece >= CH / 2;
  const int f0 = 8 * (piece % (CH / 2));
  if (turn) {
    const int f = lane % HD;
    const int axis = a.axes != 3 ? 0 : f < a.section[0] ? 0 : f < a.section[0] + a.section[1] ? 1 : 2;
    const int p = a.rope[(int64_t)axis * a.seqs.n_rows + row];
    double sn, cs;
    sincos((double)p * a.inv_freq[f], &sn, &cs);
    trig[wave][lane] = double2{cs, sn};
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
        const double2 t = trig[wave][f0 + 2 * i + h];
        const double xd = bf16_to_f64((uint16_t)(xw[i] >> (16 * h))), yd = bf16_to_f64((uint16_t)(yw[i] >> (16 * h)));
        const double xc = __dmul_rn(xd, t.x), ys = __dmul_rn(yd, t.y);
        w[i] |= f64_to_bf16(second ? __dadd_rn(xc, ys) : __dsub_rn(xc, ys)) << (16 * h);
      }
    }
    return uint4{w[0], w[1], w[2], w[3]};
  };
  if (a.q != nullptr) {
    const uint16_t *q = a.q + (int64_t)row * a.q_stride;
    uint16_t *o = a.q_out + (int64_t)row * Hq * D;
    for (int h0 = 0; h0 < Hq; h0 += HP) {
      const int e = (h0 + hl) * D + 8 * piece;
      const bool on = h0 + hl < Hq;
      uint4 x = {0u, 0u, 0u, 0u};
      if (on) x = *reinterpret_cast<const uint4 *>(q + e);
      x = rotated(x);
      if (on) *reinterpret_cast<uint4 *>(o + e) = x;
    }
  }
  if (at.page < 0) return;
  const int rows = 1 << a.pool.log_rows;
  uint8_t *page = a.pool.pages + (int64_t)at.page * a.pool.page_bytes;
  const uint16_t *k = a.k + (int64_t)row * a.k_stride, *v = a.v + (int64_t)row * a.v_stride;
  for (int h0 = 0; h0 < Hkv; h0 += HP) {
    const int h = h0 + hl, e = h * D + 8 * piece;
    const bool on = h < Hkv;
    uint4 x = {0u, 0u, 0u, 0u}, y = {0u, 0u, 0u, 0u};
    if (on) {
      x = *reinterpret_cast<const uint4 *>(k + e);
      y = *reinterpret_cast<const uint4 *>(v + e);
    }
    if (turn) x = rotated(x);
    uint8_t *block = page + (int64_t)h * a.pool.block_bytes;
    store_k<D, FP4>(block, rows, at.r, piece, x, on);
    store_v<D, FP4>(block, rows, at.r, piece, y, on);
  }
}

template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_read(PageReadArgs a) {
  constexpr int CH = D / 8, HP = 64 / CH;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = blockIdx.x * (NT / 64) + wave;
  if (row >= a.seqs.n_rows) return;
  const Place at = place_of(a.pool, a.seqs, row);
  if (!at.mine) return;
  const int Hkv = a.pool.Hkv, piece = lane % CH, hl = lane / CH;
  const int rows = 1 << a.pool.log_rows;
  const uint8_t *page = a.pool.pages + (int64_t)max(at.page, 0) * a.pool.page_bytes;
  for (int h = hl; h < Hkv; h += HP) {
    const int64_t e = ((int64_t)row * Hkv + h) * D + 8 * piece;
    const uint8_t *block = page + (int64_t)h * a.pool.block_bytes;
    uint4 x = {0u, 0u, 0u, 0u}, y = {0u, 0u, 0u, 0u};
    if (at.page >= 0) {
      x = load_k<D, FP4>(block, rows, at.r, piece);
      y = load_v<D, FP4>(block, rows, at.r, piece);
    }
    if (a.k != nullptr) *reinterpret_cast<uint4 *>(a.k + e) = x;
    if (a.v != nullptr) *reinterpret_cast<uint4 *>(a.v + e) = y;
  }
}

template <int D, bool FP4>
__global__ __launch_bounds__(NT) void page_pack(PagePackArgs a) {
  constexpr int CH = D / 8, HP = 64 / CH;
  const int j = blockIdx.y, len = a.len[j];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.kv_len[j] = len;
  const int row = blockIdx.x * (NT / 64) + wave;
  if (row >= len) return;
  const int id = a.tables[(int64_t)j * a.max_pages + (row >> a.pool.log_rows)];
  if (id < 0 || id >= a.pool.n_pages) {
    page_note(a.pool, HERMES_PAGE_BAD_ID);
    return;
  }
  const int Hkv = a.pool.Hkv, piece = lane % CH, hl = lane / CH;
  const int rows = 1 << a.pool.log_rows, r = row & (rows - 1);
  uint8_t *page = a.pool.pages + (int64_t)__builtin_amdgcn_readfirstlane(id) * a.pool.page_bytes;
  const uint16_t *k = a.k[j] + (int64_t)row * Hkv * D, *v = a.v[j] + (int64_t)row * Hkv * D;
  for (int h0 = 0; h0 < Hkv; h0 += HP) {
    const int h = h0 + hl, e = h * D + 8 * piece;
    const bool on = h < Hkv;
    uint4 x = {0u, 0u, 0u, 0u}, y = {0u, 0u, 0u, 0u};
    if (on) {
      x = *reinterpret_cast<const uint4 *>(k + e);
      y = *reinterpret_cast<const uint4 *>(v + e);
    }
    uint8_t *block = page + (int64_t)h * a.pool.block_bytes;
    store_k<D, FP4>(block, rows, r, piece, x, on);
    store_v<D, FP4>(block, rows, r, piece, y, on);
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
  const dim3 grid((unsigned)(((int64_t)a.seqs.n_rows + NT / 64 - 1) / (NT / 64)));
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_append<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

hipError_t launch_page_read(const PageReadArgs &a, int head_dim, int format, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)a.seqs.n_rows + NT / 64 - 1) / (NT / 64)));
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_read<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

hipError_t launch_page_pack(const PagePackArgs &a, int head_dim, int format, hipStream_t s) {
  int most = 1;                                        // (an empty layer's length is written too)
  for (int j = 0; j < a.n_list; ++j) most = max(most, a.len[j]);
  const dim3 grid((unsigned)(((int64_t)most + NT / 64 - 1) / (NT / 64)), a.n_list);
  return with_kind(head_dim, format, [&](auto d, auto f) {
    hipLaunchKernelGGL((page_pack<decltype(d)::value, decltype(f)::value>), grid, dim3(NT), 0, s, a);
  });
}

}  // namespace hermes
