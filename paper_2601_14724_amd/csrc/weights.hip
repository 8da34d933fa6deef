// Products of a few rows with weights in 4 bits, for gfx950:
//
// weight_pack      stores a bf16 weight as FP4 codes and scales, tile by tile
// weight_product   out = x W^T + bias + add, or of a part of the inputs x W^T in fp32
// weight_join      sums such parts
//
// A product of M <= 64 rows reads 17/32 byte of weight for 2 M operations, so HBM bounds it up
// to there.  The layout is an MFMA operand's: of a tile of 16 outputs and 128 inputs a lane holds 32
// inputs of one output in one 16-byte load.  Codes times scales are exact in bf16
// (v_cvt_scalef32_pk_bf16_fp4, two values an instruction), x is bf16, and
// v_mfma_f32_16x16x32_bf16 sums in fp32, so what is rounded is the sum alone.
//
// Measured (calls in one graph, weights not in the caches; an empty launch takes 1.8 us): 8 rows of 3584 on
// 131072 outputs 46.6 us, 5.4 TB/s; one row on 4608 5.3, on 1152 x 896 2.9; 16 on 4608 6.7; 64 on 14336 15.6;
// 32 and 64 on 131072 52 and 64.  64 rows on 14336: reading x, 103 MB from L2, is 2.6 us of that (11.3 without any);
// MFMAs are busy for 3.  The rest, by the code, is seven steps a wave that each wait for all of their loads, with one
// more step asked for and, of 128 KiB of LDS a workgroup, one wave a SIMD.
#include "tokens_internal.h"

namespace hermes {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));


// ------------------------------------------------------------------------- pack
// A wave stores the same 16 outputs of four tiles along the inputs (a quad).  The scale
// of 32 values is the least 2^e with amax <= 7 x 2^e: on the bits of a bf16
// magnitude e = ((bits + 31) >> 7) - 2 - 127 (as in the pages).  A block's 32 values lie in the
// four lanes of an output.
__global__ __launch_bounds__(256) void weight_pack(WeightPackArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= (int64_t)a.w.tiles_out * a.w.quads) return;
  const int lane = threadIdx.x & 63, q = lane / 16;
  const int nt = (int)(unit / a.w.quads), quad = (int)(unit % a.w.quads);
  const int n = 16 * nt + lane % 16;
  const uint16_t *row = a.dense + (int64_t)n * a.stride;
  uint32_t mine = 0;        // the scales of tile q of the quad
  for (int i = 0; i < 4; ++i) {
    const int kt = 4 * quad + i;
    if (kt >= a.w.tiles_in) break;
    uint32_t c[4], scales = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k0 = 128 * kt + 32 * j + 8 * q, have = n < a.w.n_out ? a.w.n_in - k0 : 0;
      uint32_t v[4] = {0, 0, 0, 0}, m = 0;
      if (have >= 8) {
        __builtin_memcpy(v, row + k0, 16);      // (a row may begin at any element)
      } else {
#pragma unroll 1
        for (int x = 0; x < have; ++x) {
          const uint32_t bits = (uint32_t)row[k0 + x] << (x % 2 * 16);
#pragma unroll
          for (int y = 0; y < 4; ++y) v[y] |= x / 2 == y ? bits : 0u;
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) m = max(m, max(v[x] & 0x7FFFu, v[x] >> 16 & 0x7FFFu));
      m = max(m, (uint32_t)__shfl_xor((int)m, 16));
      m = max(m, (uint32_t)__shfl_xor((int)m, 32));
      const uint32_t scale = m >= 0x7F80u ? 255u : (uint32_t)min(max((int)((m + 31u) >> 7) - 2, 127 - 119), 127 + 125);
      const float sc = __builtin_bit_cast(float, scale << 23);
      uint32_t r = 0;
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[0]), sc, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[1]), sc, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[2]), sc, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[3]), sc, 3);
      c[j] = r;
      scales |= scale << (8 * j);
    }
    *reinterpret_cast<uint4 *>(a.w.codes + (((int64_t)nt * a.w.tiles_in + kt) * 64 + lane) * 16) = uint4{c[0], c[1], c[2], c[3]};
    if (q == i) mine = scales;
  }
  *reinterpret_cast<uint32_t *>(a.w.scales + (unit * 16 + lane % 16) * 16 + 4 * q) = mine;
}

// ---------------------------------------------------------------------- product
__device__ __forceinline__ bf16x8 unpack(uint32_t codes, float scale) {
  const uint4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
  return __builtin_bit_cast(bf16x8, r);
}

// Four outputs n .. n + 3 of row r.
__device__ __forceinline__ void store(const WeightProductArgs &a, int64_t r, int n, f32x4 v) {
  const int64_t at = r * a.w.n_out + n;
  if (n >= a.w.n_out) return;
  const bool whole = n + 4 <= a.w.n_out && a.w.n_out % 4 == 0;
  const auto plus = [&](const uint16_t *from) {
    uint16_t b[4] = {0, 0, 0, 0};
    if (whole) {
      __builtin_memcpy(b, from, 8);
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.w.n_out) b[i] = from[i];
    }
    for (int i = 0; i < 4; ++i) v[i] += __builtin_bit_cast(float, (uint32_t)b[i] << 16);
  };
  if (a.bias != nullptr) plus(a.bias + n);
  if (a.add != nullptr) plus(a.add + at);
  if (a.fp32) {
    float *out = static_cast<float *>(a.out) + at;
    if (whole) {
      *reinterpret_cast<f32x4 *>(out) = v;
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.w.n_out) out[i] = v[i];
    }
  } else {
    uint16_t *out = static_cast<uint16_t *>(a.out) + at;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[i]));
    if (whole) {
      *reinterpret_cast<uint2 *>(out) = uint2{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16};
    } else {
      for (int i = 0; i < 4; ++i)
        if (n + i < a.w.n_out) out[i] = h[i];
    }
  }
}

// A wave's loads of a step: codes and scales of U tiles along the inputs of NT tiles of outputs
// into registers, the same inputs of x into LDS.
template <int NT, int U>
struct Step {
  u32x4 codes[U][NT];
  uint32_t scales[U][NT];
};

// Waits for all loads of this wave, those to LDS among them, and for its reads of LDS.
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);       // vmcnt 0, lgkmcnt 0
  asm volatile("" ::: "memory");
}

// 16 bytes a lane from base + lane_offset + offset (below `bytes`; zeros past it) to `to` + 16 lane.
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t bytes, uint32_t lane_offset, uint32_t offset, uint8_t *to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000),
                                           (__attribute__((address_space(3))) void *)to, 16, lane_offset, offset, 0, 0);
}

// MFMA layout (v_mfma_f32_16x16x32_bf16): lane l = 16 q + n supplies A[n][8 q ..] (weights) and
// B[8 q ..][n] (row n of x), and holds D[4 q + i][n].
//
// x reaches the lanes through LDS, a tile's 128 inputs of a row in 256 bytes, 16 lanes a row: as
// fragments straight from memory 16 neighbouring lanes' pieces lie in 16 rows, and the loads take longer than
// the weight's (64 rows on 14336 x 3584 23.8 us so, 17.3 through LDS; 8 rows on 131072 54.9 and 46.0, before
// the steps since).  Piece c of row r lies at c ^ (r % 16), so that neither the loads nor the fragments' reads meet in a
// bank.  LDS is each wave's own (waves that share outputs have different inputs), so there is no
// barrier before their sums are joined, and while a step is multiplied the next one's loads run.
//
// Common: four waves of the same inputs and of outputs of their own share one x in LDS, a quarter of
// its rows loaded by each, at a barrier a step; it is read from L2 a quarter as often and nothing is joined.  64 rows
// of 3584 on 131072 outputs 88 us without and 57 with, of 896 on 40000 16.6 and 12.1; 32 rows of 3584 on 131072 62
// and 49; 16 rows 51 and 49, on 40000 20.7 and 20.2; up to 8 rows it gains nothing (46.1 and 47.8 on 131072).
template <int RQ, int NT, int U, int W, bool Common>
__global__ __launch_bounds__(64 * W) void weight_product(WeightProductArgs a) {
  constexpr int MT = (RQ + 3) / 4;                      // tiles of 16 rows
  constexpr int kTile = RQ * 1024, kSlot = U * kTile;   // bytes of x: 4 RQ rows of a tile, of a step
  constexpr int kSlots = 2 * kSlot * (Common ? 1 : W), kSums = Common ? 0 : W * MT * NT * 1024;
  constexpr int kRoom = kSlots > kSums ? kSlots : kSums;
  constexpr int kMine = Common ? RQ / W : RQ;           // rows that this wave loads, by four
  static_assert(!Common || RQ % W == 0, "waves load equal shares");
  __shared__ __attribute__((aligned(16))) uint8_t room[kRoom];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = 1 << a.plan.log_split, groups = W >> a.plan.log_split, sub = wave & (split - 1);
  const int nt0 = ((int)blockIdx.x * groups + (wave >> a.plan.log_split)) * NT;
  const int q = lane / 16, n16 = lane % 16;
  // this wave's tiles of inputs, of those of the workgroup's part
  int r0 = (int)blockIdx.y * 16 * MT, z = 0, p0 = 0, p1 = a.w.tiles_in;
  if (a.plan.parts > 1) {
    z = blockIdx.y % a.plan.parts;
    r0 = blockIdx.y / a.plan.parts * 16 * MT;
    p0 = a.w.tiles_in * z / a.plan.parts;
    p1 = a.w.tiles_in * (z + 1) / a.plan.parts;
  }
  const int k0 = p0 + ((p1 - p0) * sub >> a.plan.log_split), k1 = p0 + ((p1 - p0) * (sub + 1) >> a.plan.log_split);
  const int whole = a.w.n_in / 128, rows = min(a.n_rows - r0, 16 * MT);
  // (an offset in the rows of a block stays below 2^32: 64 rows of up to 2^24 elements)
  const uint16_t *x0 = a.x + (int64_t)r0 * a.x_stride;
  const uint32_t x_bytes = (uint32_t)(2 * ((rows - 1) * a.x_stride + a.w.n_in));
  const int quad0 = Common ? wave * kMine : 0;
  uint32_t from[kMine];                 // this lane's piece of row 4 (quad0 + i) + q
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int r = 4 * (quad0 + i) + q;
    from[i] = (uint32_t)(min(r, rows - 1) * a.x_stride * 2) + 16 * (n16 ^ (r % 16));
  }
  uint8_t *const mine = room + (Common ? 0 : wave * 2 * kSlot);
  int at[MT];                           // this lane's row of fragments, and its place in a tile
#pragma unroll
  for (int t = 0; t < MT; ++t) at[t] = min(16 * t + n16, 4 * RQ - 1);
  const uint8_t *codes[NT], *scales[NT];
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const int64_t nt = min(nt0 + u, a.w.tiles_out - 1);
    codes[u] = a.w.codes + (nt * a.w.tiles_in * 64 + lane) * 16;
    scales[u] = a.w.scales + (nt * a.w.quads * 16 + n16) * 16;
  }
  f32x4 acc[NT][MT];
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[u][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const auto weights = [&](Step<NT, U> &s, int kt) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (kt + i >= k1) break;
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        s.codes[i][u] = *reinterpret_cast<const u32x4 *>(codes[u] + (int64_t)(kt + i) * 1024);
        s.scales[i][u] = *reinterpret_cast<const uint32_t *>(scales[u] + (int64_t)((kt + i) / 4) * 256 + (kt + i) % 4 * 4);
      }
    }
  };
  const auto load = [&](Step<NT, U> &s, int kt, int slot) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (kt + i >= k1) break;
      uint8_t *const to = mine + slot * kSlot + i * kTile;
      if (kt + i < whole) {
#pragma unroll
        for (int r = 0; r < kMine; ++r) load_to_lds(x0, x_bytes, from[r], (kt + i) * 256, to + (quad0 + r) * 1024);
        continue;
      }
      // the tile that the inputs end in: whole pieces, and zeros in place of the others
      const int left = a.w.n_in - 128 * (kt + i);
#pragma unroll
      for (int r = 0; r < kMine; ++r) {
        if (8 * (n16 ^ ((4 * (quad0 + r) + q) % 16)) + 8 <= left) {
          load_to_lds(x0, x_bytes, from[r], (kt + i) * 256, to + (quad0 + r) * 1024);
        } else {
          *reinterpret_cast<u32x4 *>(to + (quad0 + r) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
        }
      }
      if (left % 8 != 0 && lane < 4 * kMine) {  // a row's piece that the inputs end in, a lane each
        const int r = 4 * quad0 + lane;
        const uint16_t *row = x0 + min(r, rows - 1) * a.x_stride + a.w.n_in - left % 8;
        u32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
          if (e < left % 8) v[e / 2] |= (uint32_t)row[e] << (e % 2 * 16);
        *reinterpret_cast<u32x4 *>(to + r * 256 + 16 * (left / 8 ^ r % 16)) = v;
      }
    }
    weights(s, kt);
  };
  const auto multiply = [&](const Step<NT, U> &s, int kt, int slot) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (kt + i >= k1) break;
      const uint8_t *tile = mine + slot * kSlot + i * kTile;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 x[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = *reinterpret_cast<const bf16x8 *>(tile + at[t] * 256 + 16 * ((4 * j + q) ^ (at[t] % 16)));
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const bf16x8 v = unpack(s.codes[i][u][j], __builtin_bit_cast(float, (s.scales[i][u] >> (8 * j) & 255u) << 23));
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, x[t], acc[u][t], 0, 0, 0);
        }
      }
    }
  };
  if (Common || nt0 < a.w.tiles_out) {
    Step<NT, U> now, next;
    int slot = 0;
    if (k0 < k1) load(now, k0, 0);
#pragma unroll 1
    for (int kt = k0; kt < k1; kt += U) {
      wait_for_loads();
      if constexpr (Common) __syncthreads();
      if (kt + U < k1) load(next, kt + U, slot ^ 1);
      multiply(now, kt, slot);
      now = next;
      slot ^= 1;
    }
  }
  if constexpr (Common) {
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t)
        if (nt0 + u < a.w.tiles_out && 16 * t + n16 < rows) store(a, r0 + 16 * t + n16, 16 * (nt0 + u) + 4 * q, acc[u][t]);
    return;
  }
  __syncthreads();
  f32x4 *part = reinterpret_cast<f32x4 *>(room);        // [waves][NT MT][64]
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int t = 0; t < MT; ++t) part[(wave * MT * NT + u * MT + t) * 64 + lane] = acc[u][t];
  __syncthreads();
  // tile i of group g: summed over the group's waves, in their order
#pragma unroll 1
  for (int i = wave; i < groups * NT * MT; i += W) {
    const int g = i / (NT * MT), tile = i % (NT * MT);
    const int nt = (blockIdx.x * groups + g) * NT + tile / MT, r = 16 * (tile % MT) + n16;
    f32x4 v = part[(g * split * MT * NT + tile) * 64 + lane];
#pragma unroll 1
    for (int s = 1; s < split; ++s) v += part[((g * split + s) * MT * NT + tile) * 64 + lane];
    if (nt >= a.w.tiles_out || r >= rows) continue;
    if (a.plan.parts == 1) {
      store(a, r0 + r, 16 * nt + 4 * q, v);
    } else {
      *reinterpret_cast<f32x4 *>(a.sums + (((int64_t)z * a.n_rows + r0 + r) * a.w.tiles_out + nt) * 16 + 4 * q) = v;
    }
  }
}

// Four outputs of a row a thread: its parts in their order.
__global__ __launch_bounds__(256) void weight_join(WeightProductArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, wide = (int64_t)a.w.tiles_out * 4, all = wide * a.n_rows;
  if (i >= all) return;
  const f32x4 *from = reinterpret_cast<const f32x4 *>(a.sums) + i;
  f32x4 v = from[0];
#pragma unroll 4
  for (int z = 1; z < a.plan.parts; ++z) v += from[z * all];
  const int64_t r = i / wide;
  store(a, r, (int)(i - r * wide) * 4, v);
}

}  // namespace

hipError_t launch_weight_pack(const WeightPackArgs &a, hipStream_t s) {
  const int64_t units = (int64_t)a.w.tiles_out * a.w.quads;
  hipLaunchKernelGGL((weight_pack), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Rows by four, tiles of outputs a wave, steps of so many tiles of inputs, waves.  (A workgroup's x
// is 2 steps x waves x 1 KiB x rows by four: 128 KiB at 16 rows and more, so that workgroups of 64 rows
// have four waves.)
template <int RQ, int NT, int U, int W, bool Common>
static void launch_product(const WeightProductArgs &a, hipStream_t s) {
  constexpr int kRows = 16 * ((RQ + 3) / 4);
  const int groups = (W >> a.plan.log_split) * NT;
  const dim3 grid((a.w.tiles_out + groups - 1) / groups, (a.n_rows + kRows - 1) / kRows * a.plan.parts);
  hipLaunchKernelGGL((weight_product<RQ, NT, U, W, Common>), grid, dim3(64 * W), 0, s, a);
}

template <int RQ, int NT>
static void launch_product(const WeightProductArgs &a, hipStream_t s) {
  if constexpr (RQ >= 4) {
    // (two steps take 64 KiB at most: two workgroups on a CU)
    if (a.plan.common) return launch_product<RQ, NT, RQ == 16 ? (NT == 1 ? 2 : 1) : 4 / NT, 4, true>(a, s);
  }
  launch_product<RQ, NT, RQ <= 4 && NT < 4 ? 2 : 1, RQ <= 8 ? 8 : 4, false>(a, s);
}

template <int RQ>
static void launch_product(const WeightProductArgs &a, hipStream_t s) {
  if (a.plan.tiles == 1) return launch_product<RQ, 1>(a, s);
  if constexpr (RQ > 1) {       // (up to four rows have two tiles at most)
    if (a.plan.tiles == 4) return launch_product<RQ, 4>(a, s);
  }
  launch_product<RQ, 2>(a, s);
}

hipError_t launch_weight_product(const WeightProductArgs &a, hipStream_t s) {
  if (a.plan.row_quads == 1) {
    launch_product<1>(a, s);
  } else if (a.plan.row_quads == 2) {
    launch_product<2>(a, s);
  } else if (a.plan.row_quads == 4) {
    launch_product<4>(a, s);
  } else if (a.plan.row_quads == 8) {
    launch_product<8>(a, s);
  } else {
    launch_product<16>(a, s);
  }
  if (a.plan.parts > 1) {
    const int64_t threads = (int64_t)a.w.tiles_out * 4 * a.n_rows;
    hipLaunchKernelGGL(weight_join, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace hermes
