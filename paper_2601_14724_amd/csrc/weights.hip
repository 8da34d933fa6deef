// Products of a few rows with weights in 4 bits, for gfx950:
//
// weight_pack      stores a bf16 weight as FP4 codes and scales, tile by tile
// weight_product   out = x W^T + bias + add
//
// A product of M <= 64 rows reads 17/32 byte of weight for 2 M operations, so HBM bounds it up
// to there.  The layout is an MFMA operand's: of a tile of 16 outputs and 128 inputs a lane holds 32
// inputs of one output, one 16-byte load, one scale.  Codes times scales are exact in bf16
// (v_cvt_scalef32_pk_bf16_fp4, two values an instruction), x is bf16, and
// v_mfma_f32_16x16x32_bf16 sums in fp32, so what is rounded is the sum alone.
#include "tokens_internal.h"

namespace hermes {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 8;

// ------------------------------------------------------------------------- pack
// A wave stores the same 16 outputs of four tiles along the inputs (a quad).  The scale
// of 32 values is the least 2^e with amax <= 7 x 2^e: on the bits of a bf16
// magnitude e = ((bits + 31) >> 7) - 2 - 127 (as in the pages).
__global__ __launch_bounds__(256) void weight_pack(WeightPackArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= (int64_t)a.w.tiles_out * a.w.quads) return;
  const int lane = threadIdx.x & 63;
  const int nt = (int)(unit / a.w.quads), quad = (int)(unit % a.w.quads);
  const int n = 16 * nt + lane % 16;
  const uint16_t *row = a.dense + (int64_t)n * a.stride;
  uint32_t scales = 0;
  for (int i = 0; i < 4; ++i) {
    const int kt = 4 * quad + i;
    if (kt >= a.w.tiles_in) break;
    const int k0 = 128 * kt + 32 * (lane / 16);
    uint32_t v[16];         // pairs of bf16
    const int have = n < a.w.n_out ? min(a.w.n_in - k0, 32) : 0;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const uint32_t lo = 2 * j < have ? row[k0 + 2 * j] : 0u, hi = 2 * j + 1 < have ? row[k0 + 2 * j + 1] : 0u;
      v[j] = lo | hi << 16;
      m = max(m, max(lo & 0x7FFFu, hi & 0x7FFFu));
    }
    const uint32_t scale = m >= 0x7F80u ? 255u : (uint32_t)min(max((int)((m + 31u) >> 7) - 2, 127 - 119), 127 + 125);
    const float sc = __builtin_bit_cast(float, scale << 23);
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t r = 0;
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[4 * j]), sc, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[4 * j + 1]), sc, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[4 * j + 2]), sc, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, v[4 * j + 3]), sc, 3);
      c[j] = r;
    }
    *reinterpret_cast<uint4 *>(a.w.codes + (((int64_t)nt * a.w.tiles_in + kt) * 64 + lane) * 16) = uint4{c[0], c[1], c[2], c[3]};
    scales |= scale << (8 * i);
  }
  *reinterpret_cast<uint32_t *>(a.w.scales + (unit * 64 + lane) * 4) = scales;
}

// ---------------------------------------------------------------------- product
__device__ __forceinline__ bf16x8 unpack(uint32_t codes, float scale) {
  const uint4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
  return __builtin_bit_cast(bf16x8, r);
}

// Inputs k .. k + 7 of a row, zeros past the last.
__device__ __forceinline__ uint4 inputs(const uint16_t *row, int k, int n_in) {
  if (k + 8 <= n_in) return *reinterpret_cast<const uint4 *>(row + k);
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = k + 2 * i < n_in ? row[k + 2 * i] : 0u, hi = k + 2 * i + 1 < n_in ? row[k + 2 * i + 1] : 0u;
    v[i] = lo | hi << 16;
  }
  return uint4{v[0], v[1], v[2], v[3]};
}

// Four outputs n .. n + 3 of row r.
__device__ __forceinline__ void store(const WeightProductArgs &a, int64_t r, int n, f32x4 v) {
  const int64_t at = r * a.w.n_out + n;
  const bool whole = n + 4 <= a.w.n_out && a.w.n_out % 4 == 0;
  uint16_t b[4] = {0, 0, 0, 0}, d[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= a.w.n_out) continue;
    if (a.bias != nullptr) b[i] = a.bias[n + i];
    if (a.add != nullptr) d[i] = a.add[at + i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (a.bias != nullptr) v[i] += __builtin_bit_cast(float, (uint32_t)b[i] << 16);
    if (a.add != nullptr) v[i] += __builtin_bit_cast(float, (uint32_t)d[i] << 16);
  }
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

// MFMA layout (v_mfma_f32_16x16x32_bf16): lane l = 16 q + n supplies A[n][8 q ..] (weights; any order
// of the inputs that both operands agree on) and B[8 q ..][n] (row n of x), and holds D[4 q + i][n].
template <int MT, int NT>
__global__ __launch_bounds__(64 * kWaves) void weight_product(WeightProductArgs a) {
  __shared__ f32x4 part[kWaves][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int split = a.plan.split, sub = wave % split;
  const int nt0 = (blockIdx.x * (kWaves / split) + wave / split) * NT;
  const int q = lane / 16, r0 = blockIdx.y * 16 * MT;
  const uint16_t *row[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) row[t] = a.x + (int64_t)min(r0 + 16 * t + lane % 16, a.n_rows - 1) * a.x_stride;
  f32x4 acc[NT][MT];
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[u][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int q0 = (int)((int64_t)a.w.quads * sub / split), q1 = (int)((int64_t)a.w.quads * (sub + 1) / split);
  if (nt0 < a.w.tiles_out) {
    for (int quad = q0; quad < q1; ++quad) {
      uint32_t scales[NT];
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const int nt = min(nt0 + u, a.w.tiles_out - 1);
        scales[u] = *reinterpret_cast<const uint32_t *>(a.w.scales + (((int64_t)nt * a.w.quads + quad) * 64 + lane) * 4);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int kt = 4 * quad + i;
        if (kt >= a.w.tiles_in) break;
        uint4 codes[NT], xv[MT][4];
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const int nt = min(nt0 + u, a.w.tiles_out - 1);
          codes[u] = *reinterpret_cast<const uint4 *>(a.w.codes + (((int64_t)nt * a.w.tiles_in + kt) * 64 + lane) * 16);
        }
        const int k0 = 128 * kt + 32 * q;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) xv[t][j] = inputs(row[t], k0 + 8 * j, a.w.n_in);
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const float scale = __builtin_bit_cast(float, (scales[u] >> (8 * i) & 255u) << 23);
          const uint32_t c[4] = {codes[u].x, codes[u].y, codes[u].z, codes[u].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bf16x8 w = unpack(c[j], scale);
#pragma unroll
            for (int t = 0; t < MT; ++t)
              acc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, xv[t][j]), acc[u][t], 0, 0, 0);
          }
        }
      }
    }
  }
  if (split == 1) {
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int r = r0 + 16 * t + lane % 16;
        if (nt0 + u < a.w.tiles_out && r < a.n_rows) store(a, r, 16 * (nt0 + u) + 4 * q, acc[u][t]);
      }
    return;
  }
#pragma unroll
  for (int u = 0; u < NT; ++u)
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][u * MT + t][lane] = acc[u][t];
  __syncthreads();
  // tile i of group g: summed over the group's waves, in their order
  const int groups = kWaves / split;
  for (int i = wave; i < groups * NT * MT; i += kWaves) {
    const int g = i / (NT * MT), tile = i % (NT * MT);
    const int nt = (blockIdx.x * groups + g) * NT + tile / MT, r = r0 + 16 * (tile % MT) + lane % 16;
    f32x4 v = part[g * split][tile][lane];
    for (int s = 1; s < split; ++s) v += part[g * split + s][tile][lane];
    if (nt < a.w.tiles_out && r < a.n_rows) store(a, r, 16 * nt + 4 * q, v);
  }
}

}  // namespace

hipError_t launch_weight_pack(const WeightPackArgs &a, hipStream_t s) {
  const int64_t units = (int64_t)a.w.tiles_out * a.w.quads;
  hipLaunchKernelGGL((weight_pack), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_weight_product(const WeightProductArgs &a, hipStream_t s) {
  const int groups = kWaves / a.plan.split * a.plan.tiles, rows = 16 * a.plan.row_tiles;
  const dim3 grid((a.w.tiles_out + groups - 1) / groups, (a.n_rows + rows - 1) / rows), block(64 * kWaves);
  if (a.plan.row_tiles == 1) {
    hipLaunchKernelGGL((weight_product<1, 1>), grid, block, 0, s, a);
  } else if (a.plan.row_tiles == 2) {
    hipLaunchKernelGGL((weight_product<2, 1>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((weight_product<4, 1>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace hermes
