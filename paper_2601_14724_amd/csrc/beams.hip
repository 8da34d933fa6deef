// Beam search's choice of continuations, for gfx950:
//
// beam_rows   one pass over the logits: of every chunk of 512 tokens the greatest, of
//             every run of chunks the sum of exponentials
// beam_pick   a workgroup a sequence: ln sum exp of its beams, the n_keep best chunks, and
//             the n_keep best tokens among those
//
// Only the chunks' maxima are needed to find the best tokens: if token t of chunk c is among
// the K best in the order (value descending, beam and token ascending), so is c among the K
// best chunks by (greatest value descending, beam and chunk ascending).  Else K chunks came
// before it, each with a token of a greater value than all of c's, or of c's greatest and a lower
// beam or token: K tokens before t.  So the pass over the logits keeps nothing but maxima and sums,
// and is bound by HBM, whatever the logits are.
//
// Beams meet through ln sum exp, and what is chosen are whole numbers, so it is found to about 1e-8:
// differences to a peak times log2 e in two fp32 steps (the second holds what log2 e as an
// fp32 lacks), the hardware's exponential (1 ulp), eight of them added in fp32, all else in 64 bits.
#include "tokens_internal.h"

namespace hermes {
namespace {

constexpr int kRowThreads = 256, kPickThreads = 1024;
constexpr float kLog2eHigh = 1.44269502162933349609375f;       // log2 e as an fp32, and what that lacks
constexpr float kLog2eLow = 1.92596299112661746887e-8f;
constexpr double kNone = -__builtin_inf();

template <bool FP32>
__device__ __forceinline__ float logit(const void *row, int64_t i) {
  if constexpr (FP32) return static_cast<const float *>(row)[i];
  return __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
}

// Eight logits from i on, -infinity past the last.  (Rows may begin at any element: the
// loads need no alignment beyond an element's.)
template <bool FP32>
__device__ __forceinline__ void eight(const void *row, int i, int n, float *x) {
  if (i + 8 <= n) {
    if constexpr (FP32) {
      __builtin_memcpy(x, static_cast<const float *>(row) + i, 32);
    } else {
      uint32_t v[4];
      __builtin_memcpy(v, static_cast<const uint16_t *>(row) + i, 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __builtin_bit_cast(float, v[j] << 16);
        x[2 * j + 1] = __builtin_bit_cast(float, v[j] & 0xFFFF0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = i + j < n ? logit<FP32>(row, i + j) : -__builtin_inff();
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x = fmaxf(x, __shfl_xor(x, m));
  return x;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
  return x;
}

template <bool FP32>
__device__ __forceinline__ const void *row_of(const BeamArgs &a, int64_t r) {
  return static_cast<const char *>(a.logits) + r * a.stride * (FP32 ? 4 : 2);
}

template <bool FP32>
__global__ __launch_bounds__(kRowThreads) void beam_rows(BeamArgs a) {
  const int r = blockIdx.y, lane = threadIdx.x & 63;
  const int part = blockIdx.x * (kRowThreads / 64) + (threadIdx.x >> 6);
  if (part >= a.parts || (a.done != nullptr && a.done[r] != 0)) return;
  const void *row = row_of<FP32>(a, r);
  const int c1 = min((part + 1) * a.per, a.chunks);
  float peak = -__builtin_inff();
  double sum = 0.0;
  for (int c = part * a.per; c < c1; ++c) {
    float x[8];
    eight<FP32>(row, c * kBeamChunk + 8 * lane, a.n_vocab, x);
    float m = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, x[j]);
    m = wave_max(m);
    if (lane == 0) a.top[(int64_t)r * a.chunks + c] = m;
    if (m > peak) {
      sum = peak == -__builtin_inff() ? 0.0 : sum * exp((double)peak - (double)m);
      peak = m;
    }
    // (all -infinity so far: against zero, they add nothing)
    const float base = peak == -__builtin_inff() ? 0.0f : peak;
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = x[j] - base;
      e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(d, kLog2eHigh, d * kLog2eLow));
    }
    sum += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
  }
  sum = wave_sum(sum);
  if (lane == 0) {
    a.sum[(int64_t)r * a.parts + part] = sum;
    a.peak[(int64_t)r * a.parts + part] = peak;
  }
}

// ------------------------------------------------------------------------- pick
// Candidates are (value, index) pairs in the order (value descending, index ascending);
// those of value -infinity are none.
__device__ __forceinline__ bool before(double v, int i, double w, int j) { return v > w || (v == w && i < j); }

constexpr int kList = 2048;

struct PickShared {
  double offset[kMaxBeams];         // score - ln sum exp; a done beam: its score; -infinity: offers nothing
  int32_t done[kMaxBeams];
  double best_value[64];
  int32_t best_index[64];
  double value[kList];
  int32_t index[kList];
  int32_t count;
  unsigned long long counted;
  double out_value[kMaxKeep];
  int32_t out_index[kMaxKeep];
};

// Orders as the value does (-0 and 0 alike).
__device__ __forceinline__ unsigned long long key_of(double v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// How many of `n` candidates item(i, &value, &index) satisfy `test`.
template <typename Item, typename Test>
__device__ __forceinline__ unsigned long long count_items(PickShared &s, int n, Item &&item, Test &&test) {
  __syncthreads();
  if (threadIdx.x == 0) s.counted = 0;
  __syncthreads();
  unsigned long long mine = 0;
  for (int i = threadIdx.x; i < n; i += kPickThreads) {
    double v;
    int j;
    item(i, &v, &j);
    if (v > kNone && test(v, j)) ++mine;
  }
  if (mine != 0) atomicAdd(&s.counted, mine);
  __syncthreads();
  return s.counted;
}

// The `keep` first of n candidates, in order, to s.out_value and s.out_index; how many there are.
//
// The first of each of 64 groups of candidates: the keep-th of those is a bound that at least
// `keep` candidates reach, and few more do (the keep-th of 64 groups' greatest).  Those are listed, and
// each counts the ones before it.  Where more reach the bound than the list holds, the bound
// is raised to the keep-th candidate itself, bit by bit.
template <typename Item>
__device__ __forceinline__ int pick(PickShared &s, int keep, int n, Item &&item) {
  const int tid = threadIdx.x;
  double bv = kNone;
  int bi = INT32_MAX;
  for (int i = tid; i < n; i += kPickThreads) {
    double v;
    int j;
    item(i, &v, &j);
    if (before(v, j, bv, bi)) bv = v, bi = j;
  }
#pragma unroll
  for (int m = 1; m < 16; m *= 2) {
    const double v = __shfl_xor(bv, m);
    const int j = __shfl_xor(bi, m);
    if (before(v, j, bv, bi)) bv = v, bi = j;
  }
  if (tid == 0) s.count = 0;
  if (tid % 16 == 0) s.best_value[tid / 16] = bv, s.best_index[tid / 16] = bi;
  __syncthreads();
  double edge = s.best_value[tid & 63];
  int edge_index = s.best_index[tid & 63];
  {
    int rank = 0;
    for (int j = 0; j < 64; ++j) {
      const double v = s.best_value[j];
      const int x = s.best_index[j];
      // (empty groups are alike: they take their place in the line)
      rank += before(v, x, edge, edge_index) || (v == edge && x == edge_index && j < (tid & 63));
    }
    const int src = __builtin_ctzll(__ballot(rank == keep - 1));
    edge = __shfl(edge, src);
    edge_index = __shfl(edge_index, src);
  }
  for (int round = 0;; ++round) {
    for (int i = tid; i < n; i += kPickThreads) {
      double v;
      int j;
      item(i, &v, &j);
      if (v > kNone && !before(edge, edge_index, v, j)) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.value[at] = v, s.index[at] = j;
      }
    }
    __syncthreads();
    if (s.count <= kList || round > 0) break;
    unsigned long long k = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long next = k | 1ull << bit;
      if (count_items(s, n, item, [&](double v, int) { return key_of(v) >= next; }) >= (unsigned long long)keep) k = next;
    }
    const unsigned long long more = count_items(s, n, item, [&](double v, int) { return key_of(v) > k; });
    int last = 0;           // of the candidates that tie, the lowest indexes
    for (int bit = 30; bit >= 0; --bit) {
      const int next = last | 1 << bit;
      if (more + count_items(s, n, item, [&](double v, int j) { return key_of(v) == k && j < next; }) < (unsigned long long)keep)
        last = next;
    }
    edge = __builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
    edge_index = last;
    __syncthreads();
    if (tid == 0) s.count = 0;
    __syncthreads();
  }
  const int count = min(s.count, kList);
  for (int c = tid; c < count; c += kPickThreads) {
    const double v = s.value[c];
    const int j = s.index[c];
    int rank = 0;
    for (int o = 0; o < count; ++o) rank += before(s.value[o], s.index[o], v, j);
    if (rank < keep) s.out_value[rank] = v, s.out_index[rank] = j;
  }
  __syncthreads();
  return min(count, keep);
}

template <bool FP32>
__global__ __launch_bounds__(kPickThreads) void beam_pick(BeamArgs a) {
  __shared__ PickShared s;
  __shared__ int32_t chosen[kMaxKeep];
  const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int64_t row0 = (int64_t)seq * a.n_beams;
  for (int b = tid >> 6; b < a.n_beams; b += kPickThreads / 64) {
    const int64_t r = row0 + b;
    const double score = a.score[r];
    const int done = a.done != nullptr && a.done[r] != 0;
    double offset = score;
    if (!done) {
      float peak = -__builtin_inff();
      for (int p = lane; p < a.parts; p += 64) peak = fmaxf(peak, a.peak[r * a.parts + p]);
      peak = wave_max(peak);
      double sum = 0.0;     // (a NaN or an infinity of the row makes it a NaN)
      for (int p = lane; p < a.parts; p += 64) {
        const double x = a.sum[r * a.parts + p];
        const float at = a.peak[r * a.parts + p];
        sum += at == peak ? x : x * exp((double)at - (double)peak);
      }
      sum = wave_sum(sum);
      offset = score - ((double)peak + log(sum));
    }
    if (lane == 0) {
      s.offset[b] = __builtin_isfinite(offset) ? offset : kNone;
      s.done[b] = done;
    }
  }
  __syncthreads();
  const int pad_chunk = a.pad_token / kBeamChunk;
  const int n_chunks = pick(s, a.n_keep, a.n_beams * a.chunks, [&](int i, double *v, int *index) {
    const int b = i / a.chunks, c = i - b * a.chunks;
    const double offset = s.offset[b];
    *index = i;
    if (s.done[b]) {
      *v = c == pad_chunk ? offset : kNone;
    } else {
      *v = offset == kNone ? kNone : offset + (double)a.top[row0 * a.chunks + i];
    }
  });
  if (tid < n_chunks) chosen[tid] = s.out_index[tid];
  __syncthreads();
  const int n = pick(s, a.n_keep, n_chunks * kBeamChunk, [&](int i, double *v, int *index) {
    const int x = chosen[i / kBeamChunk], b = x / a.chunks;
    const int t = (x - b * a.chunks) * kBeamChunk + i % kBeamChunk;
    *index = b * a.n_vocab + t;
    *v = kNone;
    if (t >= a.n_vocab) return;
    if (s.done[b]) {
      if (t == a.pad_token) *v = s.offset[b];
    } else {
      *v = s.offset[b] + (double)logit<FP32>(row_of<FP32>(a, row0 + b), t);
    }
  });
  if (tid < a.n_keep) {
    const bool some = tid < n;
    const int x = some ? s.out_index[tid] : 0, b = x / a.n_vocab, t = x - b * a.n_vocab;
    const int64_t at = (int64_t)seq * a.n_keep + tid;
    a.score_out[at] = some ? (float)s.out_value[tid] : -__builtin_inff();
    a.parent_out[at] = some ? b : -1;
    a.token_out[at] = some ? t : -1;
    if (a.done_out != nullptr) a.done_out[at] = some && (s.done[b] || t == a.end_token);
  }
}

}  // namespace

hipError_t launch_beam_select(const BeamArgs &a, bool fp32, hipStream_t s) {
  const dim3 rows((a.parts + kRowThreads / 64 - 1) / (kRowThreads / 64), a.n_seqs * a.n_beams), one(a.n_seqs);
  if (fp32) {
    hipLaunchKernelGGL((beam_rows<true>), rows, dim3(kRowThreads), 0, s, a);
    hipLaunchKernelGGL((beam_pick<true>), one, dim3(kPickThreads), 0, s, a);
  } else {
    hipLaunchKernelGGL((beam_rows<false>), rows, dim3(kRowThreads), 0, s, a);
    hipLaunchKernelGGL((beam_pick<false>), one, dim3(kPickThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace hermes
