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
#include <type_traits>

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

// Moves between lanes: of 16 lanes, x ^ 1, x ^ 2, 7 - x, 15 - x; then the wave.
template <int Ctrl>
__device__ __forceinline__ int moved(int x) {
  return __builtin_amdgcn_update_dpp(x, x, Ctrl, 0xF, 0xF, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kRow15 = 0x142, kRow31 = 0x143;

// The greatest of the wave's, in lane 63.
__device__ __forceinline__ float wave_max(float x) {
  const auto with = [&](int y) { x = __builtin_fmaxf(x, __builtin_bit_cast(float, y)); };
  with(moved<kXor1>(__builtin_bit_cast(int, x)));
  with(moved<kXor2>(__builtin_bit_cast(int, x)));
  with(moved<kHalfMirror>(__builtin_bit_cast(int, x)));
  with(moved<kMirror>(__builtin_bit_cast(int, x)));
  with(moved<kRow15>(__builtin_bit_cast(int, x)));
  with(moved<kRow31>(__builtin_bit_cast(int, x)));
  return x;
}

template <int Ctrl, int Rows = 0xF>
__device__ __forceinline__ double moved(double x) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)u, Ctrl, Rows, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), Ctrl, Rows, 0xF, false);
  return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
// The sum of the wave's, in lane 63.
__device__ __forceinline__ double wave_sum(double x) {
  x += moved<kXor1>(x);
  x += moved<kXor2>(x);
  x += moved<kHalfMirror>(x);
  x += moved<kMirror>(x);
  x += moved<kRow15, 0xA>(x);
  return x + moved<kRow31, 0xC>(x);
}

__device__ __forceinline__ float last_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
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
  // P chunks at once: their loads and their maxima's moves are independent
  const auto take = [&](int c, auto number) {
    constexpr int P = decltype(number)::value;
    float x[P][8], m[P], all;
#pragma unroll
    for (int i = 0; i < P; ++i) eight<FP32>(row, (c + i) * kBeamChunk + 8 * lane, a.n_vocab, x[i]);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      m[i] = x[i][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) m[i] = __builtin_fmaxf(m[i], x[i][j]);
      m[i] = wave_max(m[i]);
      if (lane == 63) a.top[(int64_t)r * a.chunks + c + i] = m[i];
      all = i == 0 ? m[0] : __builtin_fmaxf(all, m[i]);
    }
    all = last_lane(all);
    if (all > peak) {
      sum = peak == -__builtin_inff() ? 0.0 : sum * exp((double)peak - (double)all);
      peak = all;
    }
    // (all -infinity so far: against zero, they add nothing)
    const float base = peak == -__builtin_inff() ? 0.0f : peak;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = x[i][j] - base;
        e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(d, kLog2eHigh, d * kLog2eLow));
      }
      sum += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
    }
  };
  int c = part * a.per;
  for (; c + 4 <= c1; c += 4) take(c, std::integral_constant<int, 4>{});
  for (; c < c1; ++c) take(c, std::integral_constant<int, 1>{});
  sum = wave_sum(sum);
  if (lane == 63) {
    a.sum[(int64_t)r * a.parts + part] = sum;
    a.peak[(int64_t)r * a.parts + part] = peak;
  }
}

// ------------------------------------------------------------------------- pick
// Candidates are (value, index) pairs in the order (value descending, index ascending);
// those of value -infinity are none.
__device__ __forceinline__ bool before(double v, int i, double w, int j) { return v > w || (v == w && i < j); }

constexpr int kList = 2048, kPickWaves = kPickThreads / 64;
static_assert(kPickThreads == 64 * 16, "64 groups of 16 threads");

struct PickShared {
  double offset[kMaxBeams];         // score - ln sum exp; a done beam: its score; -infinity: offers nothing
  int32_t done[kMaxBeams];
  int32_t beam[kMaxKeep], token[kMaxKeep];   // the chosen chunks: beam and first token
  double best_value[64], edge_value;
  int32_t best_index[64], edge_index;
  double value[kList];
  int32_t index[kList];
  int32_t count;
  unsigned long long counted;
  double out_value[kMaxKeep];
  int32_t out_index[kMaxKeep];
};

struct Candidate {
  double v;
  int i;
};
template <int Ctrl>
__device__ __forceinline__ Candidate first_of(const Candidate &x) {
  const Candidate y{moved<Ctrl>(x.v), moved<Ctrl>(x.i)};
  return before(y.v, y.i, x.v, x.i) ? y : x;
}
// The sum over 16 lanes.
__device__ __forceinline__ int row_sum(int x) {
  x += moved<kXor1>(x);
  x += moved<kXor2>(x);
  x += moved<kHalfMirror>(x);
  return x + moved<kMirror>(x);
}

// Orders as the value does (-0 and 0 alike).
__device__ __forceinline__ unsigned long long key_of(double v) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, v + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// A set of candidates is a function that calls another with (value, index) of each of this
// thread's; those of value -infinity do not count.

// How many satisfy `test`.
template <typename Each, typename Test>
__device__ __forceinline__ unsigned long long count_of(PickShared &s, const Each &each, Test &&test) {
  __syncthreads();
  if (threadIdx.x == 0) s.counted = 0;
  __syncthreads();
  unsigned long long mine = 0;
  each([&](double v, int i) { mine += v > kNone && test(v, i); });
  if (mine != 0) atomicAdd(&s.counted, mine);
  __syncthreads();
  return s.counted;
}

// The keep-th candidate, bit by bit.
template <typename Each>
__device__ Candidate find_edge(PickShared &s, int keep, const Each &each) {
  unsigned long long k = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const unsigned long long next = k | 1ull << bit;
    if (count_of(s, each, [&](double v, int) { return key_of(v) >= next; }) >= (unsigned long long)keep) k = next;
  }
  const unsigned long long more = count_of(s, each, [&](double v, int) { return key_of(v) > k; });
  int last = 0;             // of the candidates that tie, the lowest indexes
  for (int bit = 30; bit >= 0; --bit) {
    const int next = last | 1 << bit;
    if (more + count_of(s, each, [&](double v, int i) { return key_of(v) == k && i < next; }) < (unsigned long long)keep)
      last = next;
  }
  return Candidate{__builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k), last};
}

// The `keep` first candidates, in order, to s.out_value and s.out_index; how many there are.
//
// The first of each of 64 groups of candidates: the keep-th of those is a bound that at least
// `keep` candidates reach, and few more do.  Those are listed, and 16 threads each count the ones
// before it.  Where more reach the bound than the list holds, the bound is raised to the keep-th
// candidate itself (whole rows of ties: some 100 us).
template <typename Each>
__device__ __forceinline__ int pick(PickShared &s, int keep, const Each &each) {
  const int tid = threadIdx.x, group = tid / 16, slice = tid % 16;
  Candidate best{kNone, INT32_MAX};
  each([&](double v, int i) {
    if (before(v, i, best.v, best.i)) best = Candidate{v, i};
  });
  best = first_of<kXor1>(best);
  best = first_of<kXor2>(best);
  best = first_of<kHalfMirror>(best);
  best = first_of<kMirror>(best);
  if (tid == 0) s.count = 0;
  if (slice == 0) s.best_value[group] = best.v, s.best_index[group] = best.i;
  __syncthreads();
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int g = slice + 16 * j;
    const double v = s.best_value[g];
    const int x = s.best_index[g];
    // (empty groups are alike: they take their place in the line)
    rank += before(v, x, best.v, best.i) || (v == best.v && x == best.i && g < group);
  }
  rank = row_sum(rank);
  if (rank == keep - 1 && slice == 0) s.edge_value = best.v, s.edge_index = best.i;
  __syncthreads();
  Candidate edge{s.edge_value, s.edge_index};
  for (int round = 0;; ++round) {
    each([&](double v, int i) {
      if (v > kNone && !before(edge.v, edge.i, v, i)) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.value[at] = v, s.index[at] = i;
      }
    });
    __syncthreads();
    if (s.count <= kList || round > 0) break;
    edge = find_edge(s, keep, each);
    __syncthreads();
    if (tid == 0) s.count = 0;
    __syncthreads();
  }
  const int count = min(s.count, kList);
  for (int c0 = 0; c0 < count; c0 += 64) {
    const int c = min(c0 + group, count - 1);
    const Candidate x{s.value[c], s.index[c]};
    int first = 0;
    for (int o = slice; o < count; o += 16) first += before(s.value[o], s.index[o], x.v, x.i);
    first = row_sum(first);
    if (slice == 0 && c0 + group < count && first < keep) s.out_value[first] = x.v, s.out_index[first] = x.i;
  }
  __syncthreads();
  return min(count, keep);
}

template <bool FP32>
__global__ __launch_bounds__(kPickThreads) void beam_pick(BeamArgs a) {
  __shared__ PickShared s;
  const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row0 = (int64_t)seq * a.n_beams;
  const float *top = a.top + row0 * a.chunks;
  // a beam's chunks belong to `share` waves
  int share = kPickWaves;
  while (share > 1 && share * a.n_beams > kPickWaves) share /= 2;
  const int first_chunk = wave % share * 64 + lane;
  // (asked for now, so that it is near when the sums are done)
  const float near = wave / share < a.n_beams && first_chunk < a.chunks ? top[wave / share * a.chunks + first_chunk] : 0.0f;
  for (int b = wave; b < a.n_beams; b += kPickWaves) {
    const int64_t r = row0 + b;
    const double score = a.score[r];
    const int done = a.done != nullptr && a.done[r] != 0;
    double offset = score;
    if (!done) {
      const double *sums = a.sum + r * a.parts;
      const float *peaks = a.peak + r * a.parts;
      float peak = -__builtin_inff();
      for (int p = lane; p < a.parts; p += 64) peak = __builtin_fmaxf(peak, peaks[p]);
      peak = last_lane(wave_max(peak));
      double sum = 0.0;     // (a NaN or an infinity of the row makes it a NaN)
      for (int p = lane; p < a.parts; p += 64) {
        const double x = sums[p];
        const float at = peaks[p];
        sum += at == peak ? x : x * exp((double)at - (double)peak);
      }
      offset = score - ((double)peak + log(wave_sum(sum)));
    }
    if (lane == 63) {
      s.offset[b] = __builtin_isfinite(offset) ? offset : kNone;
      s.done[b] = done;
    }
  }
  asm volatile("" ::"v"(near));
  __syncthreads();
  const int n_chunks = pick(s, a.n_keep, [&](auto &&take) {
    for (int b = wave / share; b < a.n_beams; b += kPickWaves / share) {
      const double offset = s.offset[b];
      if (offset == kNone) continue;
      if (s.done[b]) {
        if (first_chunk == 0) take(offset, b * a.chunks + a.pad_token / kBeamChunk);
        continue;
      }
      for (int c = first_chunk; c < a.chunks; c += 64 * share) take(offset + (double)top[b * a.chunks + c], b * a.chunks + c);
    }
  });
  if (tid < n_chunks) {
    const int i = s.out_index[tid], b = i / a.chunks;
    s.beam[tid] = b;
    s.token[tid] = (i - b * a.chunks) * kBeamChunk;
  }
  __syncthreads();
  const int n = pick(s, a.n_keep, [&](auto &&take) {
    for (int k = wave; k < n_chunks; k += kPickWaves) {
      const int b = s.beam[k], t = s.token[k] + 8 * lane;
      const double offset = s.offset[b];
      if (s.done[b]) {
        if (lane == 0) take(offset, b * a.n_vocab + a.pad_token);
        continue;
      }
      float x[8];
      eight<FP32>(row_of<FP32>(a, row0 + b), t, a.n_vocab, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) take(offset + (double)x[j], b * a.n_vocab + t + j);
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
