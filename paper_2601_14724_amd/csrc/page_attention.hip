// Causal attention over pages for gfx950 (MFMA bf16, 64-wide waves).
//
// page_attn_few   a few packed rows (row, query head of the KV head) against
//                 all keys of their sequence, or of a range of them
// page_combine    joins the ranges
//
// S = scale q k^T over the keys a row sees, O = softmax(S) V, in one pass over the
// keys with a running maximum and sum (fp32), lse = ln sum exp S.
//
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
#include <type_traits>

#include "pages_internal.h"

namespace hermes {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256, NW = NT / 64;
constexpr int KS = 32;                  // keys of a wave's step
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
  } else {
    static_assert(N == 2, "two words");
    const uint2 x = *reinterpret_cast<const uint2 *>(p);
    w[0] = x.x, w[1] = x.y;
  }
}

template <int D, bool FP4, int RT>
__global__ __launch_bounds__(NT, RT == 1 ? 2 : 1) void page_attn_few(PageAttnArgs a) {
  using B = PageBlock<D, FP4>;
  constexpr int KK = D / 32;                // MFMAs of S for each group of keys
  constexpr int PC = D / 16;                // channels of a piece of V
  const PagePool &pool = a.pool;
  const int Hq = pool.Hq, Hkv = pool.Hkv, G = Hq / Hkv;
  const int split = blockIdx.x % a.plan.splits, pair = blockIdx.x / a.plan.splits;
  const int kv = pair % Hkv, b = pair / Hkv;
  const PageSeq seq = page_seq(pool, a.seqs, b);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n16 = lane & 15, u = lane >> 4;
  const int64_t P = (int64_t)seq.n * G;
  const int rows_log = pool.log_rows, page_rows = 1 << rows_log;
  const int32_t *table = a.seqs.tables + (int64_t)b * a.seqs.max_pages;
  const float c = a.scale_log2, inv_c = 1.f / c;

  // lane's byte offsets in a KV head's block, from the first row of a group of 16
  const int k_ofs = n16 * B::kRow + (FP4 ? u * (D / 8) : u * 16);
  const int v_ofs = B::v(page_rows, u) + n16 * 4 * B::kPiece;
  const int ks_ofs = B::ks(page_rows, n16) + u * (D / 4) / 32;
  const int vs_ofs = B::vs(page_rows, u) + n16 * PC / 32 * 4;

  __shared__ __attribute__((aligned(16))) float so[NW][16][D + 4];
  __shared__ float2 sml[NW][16];

  for (int64_t p0 = (int64_t)blockIdx.y * (16 * RT); p0 < P; p0 += (int64_t)gridDim.y * (16 * RT)) {
    // keys [lo, hi) of this range; row i of the tile sees those below base + i + 1
    const int first = (int)(p0 / G), last = (int)((min(p0 + 16 * RT, P) - 1) / G);
    const int base = seq.len - seq.n;
    const int end = max(0, base + last + 1);
    const int lo = (int)min((int64_t)split * a.plan.range, (int64_t)end);
    const int hi = split == a.plan.splits - 1 ? end : lo + min(end - lo, a.plan.range);

    bf16x8 qf[RT][KK];
    int vis[RT];                            // keys this lane's row sees
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int64_t p = p0 + 16 * t + n16;
      const int i = p < P ? (int)(p / G) : 0, g = p < P ? (int)(p - (int64_t)i * G) : 0;
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
    auto compute = [&](Frag &f, int x, auto masked) {
      const int key0 = key_of(x);
      if constexpr (decltype(masked)::value) {
        // Memory that holds no stored row (past the length, or no page) may hold
        // anything: its values become zeros.  Keys there are masked by S, or
        // zeros too.
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
            if (none) {
              f.ks[h] = 0u;
#pragma unroll
              for (int i = 0; i < Frag::WK; ++i) f.k[h][i] = 0u;
            }
          } else {
#pragma unroll
            for (int i = 0; i < Frag::WV; ++i)
              if (i / (Frag::WV / 4) >= valid) f.v[h][i] = 0u;
            if (none) {
#pragma unroll
              for (int i = 0; i < Frag::WK; ++i) f.k[h][i] = 0u;
            }
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
      bf16x8 pf[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if constexpr (decltype(masked)::value) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key0 + 16 * h + 4 * u + j >= vis[t]) s[t][h][j] = -INFINITY;
          }
        }
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
    using Masked = std::integral_constant<bool, true>;
    using Open = std::integral_constant<bool, false>;
    auto step = [&](Frag &f, int x) {
      const bool hole = (__builtin_amdgcn_readlane(ids[0], x & 63) | __builtin_amdgcn_readlane(ids[1], x & 63)) < 0;
      if (hole || key_of(x) + KS > all_see) compute(f, x, Masked{});
      else compute(f, x, Open{});
    };
    for (int x0 = 0; x0 < mine; x0 += 64) {
      find_pages(x0);
      const int n = min(64, mine - x0);
      Frag cur, nxt;
      load(cur, x0);
      for (int x = x0; x < x0 + n; ++x) {
        if (x + 1 < x0 + n) load(nxt, x + 1);
        step(cur, x);
        cur = nxt;
      }
    }

    // join the waves, 16 rows at a time: thread (row, piece of eight channels)
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (p0 + 16 * t >= P) break;
      float l = l_run[t];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      __syncthreads();
      if (u == 0) sml[wave][n16] = float2{m_run[t], l};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < PC; i += 4)
          *reinterpret_cast<float4 *>(&so[wave][n16][PC * (4 * u + j) + i]) =
              float4{o[t][i][j], o[t][i + 1][j], o[t][i + 2][j], o[t][i + 3][j]};
      }
      __syncthreads();
      const int row = threadIdx.x / 16, piece = threadIdx.x % 16;   // (PC channels)
      const int64_t p = p0 + 16 * t + row;
      if (p >= P) continue;
      float m = sml[0][row].x;
#pragma unroll
      for (int w = 1; w < NW; ++w) m = fmaxf(m, sml[w][row].x);
      float sum = 0.f, acc[PC];
#pragma unroll
      for (int i = 0; i < PC; ++i) acc[i] = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float e = fast_exp2(sml[w][row].x - m);
        sum += e * sml[w][row].y;
#pragma unroll
        for (int i = 0; i < PC; ++i) acc[i] += e * so[w][row][PC * piece + i];
      }
      const int i = (int)(p / G), g = (int)(p - (int64_t)i * G);
      const int64_t at = (int64_t)(seq.r0 + i) * Hq + kv * G + g;
      if (a.plan.splits > 1) {
        const int64_t blk = (int64_t)split * ((int64_t)a.seqs.n_rows * Hq) + at;
        if (piece == 0) *reinterpret_cast<float2 *>(a.mlpart + 2 * blk) = float2{m, sum};
        if (hi > lo) {                      // (an empty range leaves its O unwritten, and unread)
#pragma unroll
          for (int x = 0; x < PC; x += 4)
            *reinterpret_cast<float4 *>(a.opart + blk * D + PC * piece + x) =
                float4{acc[x], acc[x + 1], acc[x + 2], acc[x + 3]};
        }
      } else {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (0: the row sees nothing; a NaN stays one)
#pragma unroll
        for (int x = 0; x < PC; x += 4)
          *reinterpret_cast<uint2 *>(a.out + at * D + PC * piece + x) =
              uint2{f2bf(acc[x] * inv) | f2bf(acc[x + 1] * inv) << 16, f2bf(acc[x + 2] * inv) | f2bf(acc[x + 3] * inv) << 16};
        if (a.lse != nullptr && piece == 0) a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
      }
    }
    __syncthreads();   // so and sml are free for the next tile
  }
}

// Joins the ranges of a row: O = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m).
// A wave takes one (row, query head).
template <int D>
__global__ __launch_bounds__(NT) void page_combine(PageAttnArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int Hq = a.pool.Hq, S = a.plan.splits;
  const int64_t total = (int64_t)a.seqs.n_rows * Hq;
  const int per = gridDim.x / a.seqs.n_seqs;    // workgroups of a sequence
  const PageSeq seq = page_seq(a.pool, a.seqs, blockIdx.x / per);
  const int64_t n = (int64_t)seq.n * Hq;
  for (int64_t x = (int64_t)(blockIdx.x % per) * NW + wave; x < n; x += (int64_t)per * NW) {
    const int64_t at = (int64_t)seq.r0 * Hq + x;
    float m = kLowest, l = 0.f;
    float2 acc = {0.f, 0.f};
    for (int s0 = 0; s0 < S; s0 += 64) {
      // lane s has range s0 + s's (max, sum)
      float2 ml = {kLowest, 0.f};
      if (s0 + lane < S) ml = *reinterpret_cast<const float2 *>(a.mlpart + 2 * ((s0 + lane) * total + at));
      float mn = ml.x;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor(mn, o));
      mn = fmaxf(mn, m);
      const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - mn);
      float ls = w * ml.y;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) ls += __shfl_xor(ls, o);
      const float old = fast_exp2(m - mn);
      l = l * old + ls;
      acc.x *= old;
      acc.y *= old;
      m = mn;
      unsigned long long live = __ballot(ml.y != 0.f);
      while (live != 0ull) {
        const int s = __builtin_ctzll(live);
        live &= live - 1;
        const float ws = __shfl(w, s);
        const float *op = a.opart + ((s0 + s) * total + at) * D;
        if constexpr (D == 128) {
          const float2 y = *reinterpret_cast<const float2 *>(op + 2 * lane);
          acc.x += ws * y.x;
          acc.y += ws * y.y;
        } else {
          acc.x += ws * op[lane];
        }
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if constexpr (D == 128)
      *reinterpret_cast<uint32_t *>(a.out + at * D + 2 * lane) = f2bf(acc.x * inv) | f2bf(acc.y * inv) << 16;
    else
      a.out[at * D + lane] = (uint16_t)f2bf(acc.x * inv);
    if (a.lse != nullptr && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

template <int D, bool FP4>
hipError_t attend(const PageAttnArgs &a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.plan.splits * a.pool.Hkv * a.seqs.n_seqs), a.plan.tiles);
  if (a.plan.rows == 16) hipLaunchKernelGGL((page_attn_few<D, FP4, 1>), grid, dim3(NT), 0, s, a);
  else if (a.plan.rows == 32) hipLaunchKernelGGL((page_attn_few<D, FP4, 2>), grid, dim3(NT), 0, s, a);
  else hipLaunchKernelGGL((page_attn_few<D, FP4, 4>), grid, dim3(NT), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.plan.splits == 1) return e;
  const int64_t rows = (int64_t)a.plan.tiles * a.plan.rows * a.pool.Hkv;   // (of a sequence, at least)
  const int64_t per = min((rows + NW - 1) / NW, max((int64_t)1, (int64_t)(1 << 24) / a.seqs.n_seqs));
  hipLaunchKernelGGL(page_combine<D>, dim3((unsigned)(per * a.seqs.n_seqs)), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_attend(const PageAttnArgs &a, int head_dim, int format, hipStream_t s) {
  if (format == HERMES_PAGE_FP4) return head_dim == 64 ? attend<64, true>(a, s) : attend<128, true>(a, s);
  return head_dim == 64 ? attend<64, false>(a, s) : attend<128, false>(a, s);
}

}  // namespace hermes
