// Beam search's choice of continuations, for gfx950:
//
// beam_rows   one pass over the logits: of every chunk of 512 tokens the greatest, of
//             every part of a row the sum of exponentials
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
// Beams meet through ln sum exp, and what is chosen are whole numbers, so it is found closer than in fp32:
// differences to the greatest logit times log2 e in two fp32 steps (the second holds what log2 e as an
// fp32 lacks), the hardware's exponential (1 ulp), eight of them added in fp32, all else in 64 bits.
// Half an ulp of a difference of 8 to 16, and of its 11 to 23 octaves, are 2^-21 and 2^-20 ln 2; with the exponential's
// ulp and three additions that is 1.4e-6 of a term.  Terms so far below their wave's greatest weigh little but where
// a wave takes very many: 1e-6 of a row of 2^20 tokens at worst (7.2e-7 measured), 1.5e-6 of 2^30 (1.1e-6 of 2^27),
// in rows of two values.  Logits that differ average it out: 1e-8.  (Differences and arguments in 64 bits are off by
// 2e-7, and take 18.3 us for 17.5 of 16 x 8 beams.)
//
// Measured: 16 sequences of eight beams over 131072 tokens in bf16, 34 MB, 9.7 us (88 vector instructions
// for 512 logits, its eight exponentials four issue slots each) and 9.5 for the choice; 32 of 16 in fp32,
// 268 MB, 45 us (6 TB/s; part of it stays in the Infinity Cache) and 13.6.  The choice is a
// workgroup a sequence, a chain of loads, moves and barriers: 7.7 us where it is short.  Its code is kept
// small: it runs once, so that every line is fetched (62 KB of unrolled loops took 8.7 us for 7.3).
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

// Eight logits from i on, -infinity past the last (Whole: there is none).  Rows may begin at any
// element: the loads need no alignment beyond an element's.
template <bool FP32, bool Whole>
__device__ __forceinline__ void eight(const void *row, int i, int n, float *x) {
  if (Whole || i + 8 <= n) {
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
  for (int j = 0; j < 8; ++j) {
    const float y = logit<FP32>(row, min(i + j, n - 1));
    x[j] = i + j < n ? y : -__builtin_inff();
  }
}

// Moves between lanes: of 16 lanes, x ^ 1, x ^ 2, 7 - x, 15 - x, x - 4 and x - 8 around; then the wave.
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kTurn4 = 0x124, kTurn8 = 0x128;
constexpr int kRow15 = 0x142, kRow31 = 0x143;
template <int Ctrl, int Rows = 0xF>
__device__ __forceinline__ int moved(int x) {
  return __builtin_amdgcn_update_dpp(0, x, Ctrl, Rows, 0xF, Rows == 0xF);
}
template <int Ctrl, int Rows = 0xF>
__device__ __forceinline__ double moved(double x) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  const uint32_t lo = moved<Ctrl, Rows>((int)u), hi = moved<Ctrl, Rows>((int)(u >> 32));
  return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}

// An int that orders as the float does (NaN apart), and back.
__device__ __forceinline__ int order_of(float x) {
  const int u = __builtin_bit_cast(int, x);
  return u ^ (u >> 31 & 0x7FFFFFFF);
}
__device__ __forceinline__ float float_of(int k) { return __builtin_bit_cast(float, k ^ (k >> 31 & 0x7FFFFFFF)); }

template <int Ctrl>
__device__ __forceinline__ int greater(int x) { return max(x, moved<Ctrl>(x)); }
// The greatest of the wave's, in all lanes.
__device__ __forceinline__ int wave_max(int x) {
  x = greater<kTurn8>(greater<kTurn4>(greater<kXor2>(greater<kXor1>(x))));
  x = max(x, __shfl_xor(x, 16));
  return max(x, __shfl_xor(x, 32));
}
// Of four values the greatest of the wave's: value l % 4 in lane l.
__device__ __forceinline__ int wave_max(int a, int b, int c, int d) {
  const int lane = threadIdx.x & 63;
  const bool one = lane & 1, two = lane & 2;
  const int x = max(one ? b : a, moved<kXor1>(one ? a : b)), y = max(one ? d : c, moved<kXor1>(one ? c : d));
  int z = max(two ? y : x, moved<kXor2>(two ? x : y));
  z = greater<kTurn8>(greater<kTurn4>(z));
  z = max(z, __shfl_xor(z, 16));
  return max(z, __shfl_xor(z, 32));
}

// The sum of 16 lanes, in all of them; of the wave's, in lane 63.
__device__ __forceinline__ double row_sum(double x) {
  x += moved<kXor1>(x);
  x += moved<kXor2>(x);
  x += moved<kHalfMirror>(x);
  return x + moved<kMirror>(x);
}
__device__ __forceinline__ double wave_sum(double x) {
  x = row_sum(x);
  x += moved<kRow15, 0xA>(x);
  return x + moved<kRow31, 0xC>(x);
}

template <bool FP32>
__device__ __forceinline__ const void *row_of(const BeamArgs &a, int64_t r) {
  return static_cast<const char *>(a.logits) + r * a.stride * (FP32 ? 4 : 2);
}

template <bool FP32>
__global__ __launch_bounds__(kRowThreads) void beam_rows(BeamArgs a) {
  __shared__ double sums[kRowThreads / 64];
  __shared__ float peaks[kRowThreads / 64];
  const int r = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (a.done != nullptr && a.done[r] != 0) return;
  const void *row = row_of<FP32>(a, r);
  const int c0 = min(((int)blockIdx.x * (kRowThreads / 64) + wave) * a.per, a.chunks), c1 = min(c0 + a.per, a.chunks);
  float peak = -__builtin_inff();
  double sum = 0.0;
  float *const top = a.top + (int64_t)r * a.chunks;
  // The greatest logit so far is `now`: older sums are scaled to it.  (Times zero where there was none but
  // -infinity: a NaN that came before stays one.)
  const auto raise = [&](float now) {
    if (now > peak) {
      sum *= peak == -__builtin_inff() ? 0.0 : exp((double)peak - (double)now);
      peak = now;
    }
  };
  const auto greatest = [&](const float (&x)[8]) {
    float m = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = __builtin_fmaxf(m, x[j]);
    return order_of(m);
  };
  const auto add = [&](const float (&x)[8]) {
    // (all -infinity so far: against zero, they add nothing)
    const float base = peak == -__builtin_inff() ? 0.0f : peak;
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = x[j] - base;
      e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(d, kLog2eHigh, d * kLog2eLow));
    }
    sum += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
  };
  const int whole = min(c1, a.n_vocab / kBeamChunk);
  int c = c0;
  // four chunks at once: their loads run together, and their maxima's moves are shared
  for (; c + 4 <= whole; c += 4) {
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) eight<FP32, true>(row, (c + i) * kBeamChunk + 8 * lane, a.n_vocab, x[i]);
    const int m = wave_max(greatest(x[0]), greatest(x[1]), greatest(x[2]), greatest(x[3]));
    if (lane < 4) top[c + lane] = float_of(m);
    raise(float_of(__builtin_amdgcn_readfirstlane(greater<kXor2>(greater<kXor1>(m)))));
#pragma unroll
    for (int i = 0; i < 4; ++i) add(x[i]);
  }
#pragma unroll 1
  for (; c < c1; ++c) {
    float x[8];
    eight<FP32, false>(row, c * kBeamChunk + 8 * lane, a.n_vocab, x);
    const float m = float_of(__builtin_amdgcn_readfirstlane(wave_max(greatest(x))));
    if (lane == 0) top[c] = m;
    raise(m);
    add(x);
  }
  sum = wave_sum(sum);
  if (lane == 63) sums[wave] = sum, peaks[wave] = peak;
  __syncthreads();
  if (wave == 0) {          // (four lanes' work, done by all)
    const float at = peaks[lane % 4];
    const float all = float_of(greater<kXor2>(greater<kXor1>(order_of(at))));
    double x = sums[lane % 4];
    if (at != all) x *= exp((double)at - (double)all);
    x += moved<kXor1>(x);
    x += moved<kXor2>(x);
    if (lane == 0) {
      a.sum[(int64_t)r * a.parts + blockIdx.x] = x;
      a.peak[(int64_t)r * a.parts + blockIdx.x] = all;
    }
  }
}

// ------------------------------------------------------------------------- pick
// Candidates are (value, index) pairs in the order (value descending, index ascending);
// those of value -infinity are none.
__device__ __forceinline__ bool before(double v, int i, double w, int j) { return v > w || (v == w && i < j); }

constexpr int kList = 2048, kPickWaves = kPickThreads / 64;
constexpr int kGroup = kPickThreads / 64;   // threads of a group: 64 groups
static_assert(kGroup == 16, "reduced by four moves");

struct PickShared {
  double offset[kMaxBeams];         // score - ln sum exp; a done beam: its score; -infinity: offers nothing
  int32_t done[kMaxBeams];
  int32_t beam[kMaxKeep], token[kMaxKeep];   // the chosen chunks: beam and first token
  double best_value[64], edge_value;
  int32_t best_index[64], edge_index;
  double value[kList];
  int32_t index[kList];
  int32_t count;
  int32_t counted;
  double out_value[kMaxKeep];
  int32_t out_index[kMaxKeep];
};

struct Candidate {
  double v;
  int i;
};
template <int Ctrl>
__device__ __forceinline__ double greater(double x) { return __builtin_fmax(x, moved<Ctrl>(x)); }
// The first of a group's, the sum over a group.
__device__ __forceinline__ Candidate group_first(const Candidate &x) {
  const double v = greater<kMirror>(greater<kHalfMirror>(greater<kXor2>(greater<kXor1>(x.v))));
  int i = x.v == v ? x.i : INT32_MAX;
  i = min(i, moved<kXor1>(i));
  i = min(i, moved<kXor2>(i));
  i = min(i, moved<kHalfMirror>(i));
  return Candidate{v, min(i, moved<kMirror>(i))};
}
__device__ __forceinline__ int group_sum(int x) {
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
__device__ __forceinline__ double value_of(unsigned long long key) {
  return __builtin_bit_cast(double, key >> 63 ? key & ~(1ull << 63) : ~key);
}

// A set of candidates has end(), an index past all; count(value, upto), how many of this thread's are greater
// than value or equal with an index below upto; and above(edge, take), which calls take(value, index) of this
// thread's that may be edge or before it.  Chunks have best(), this thread's first one; tokens greatest(), this
// thread's greatest value.
// Candidates of value -infinity do not count.

// The least logit that an edge asks of a beam, or a little less: values are sums in 64 bits, and most logits
// are sorted out by one comparison in 32.
__device__ __forceinline__ float least_logit(double edge, double offset) {
  const double gap = edge - offset;
  return edge == kNone ? -__builtin_inff() : (float)(gap - 0x1p-20 * __builtin_fabs(gap) - 0x1p-40 * __builtin_fabs(offset));
}

// The keep-th candidate, bit by bit: first the greatest value that `keep` candidates reach, unless it is
// `floor`, which they are known to reach (rows of ties), then of those that tie the least index, below `end`,
// up to which there are enough.
template <typename Set>
__device__ __forceinline__ Candidate find_edge(PickShared &s, int keep, const Set &set, double floor, int end) {
  unsigned long long k = key_of(floor);
  int last = 0;
  const int index_bits = 32 - __builtin_clz(end);
#pragma unroll 1
  for (int bit = 64 + index_bits; bit >= 0; --bit) {
    const bool first = bit == 64 + index_bits, ties = bit < index_bits;
    const unsigned long long key = first ? k + 1 : ties ? k : k | 1ull << (bit - index_bits);
    const int upto = last | (ties ? 1 << bit : 0);
    __syncthreads();
    if (threadIdx.x == 0) s.counted = 0;
    __syncthreads();
    const int mine = set.count(value_of(key), ties ? upto : INT32_MAX);
    if (mine != 0) atomicAdd(&s.counted, mine);
    __syncthreads();
    const int counted = s.counted;
    if (first) {
      if (counted < keep) bit = index_bits; else k = 0;
    } else if (ties ? counted < keep : counted >= keep) {
      if (ties) last = upto; else k = key;
    }
  }
  return Candidate{value_of(k), last};
}

// A bound that at least `keep` candidates reach, and few more: of the candidates of 64 groups of threads,
// the keep-th.
template <typename Set>
__device__ __forceinline__ Candidate bound_of(PickShared &s, int keep, const Set &set) {
  const int tid = threadIdx.x, group = tid / kGroup, slice = tid % kGroup;
  const Candidate best = group_first(set.best());
  if (slice == 0) s.best_value[group] = best.v, s.best_index[group] = best.i;
  __syncthreads();
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 64 / kGroup; ++j) {
    const int g = slice + kGroup * j;
    const double v = s.best_value[g];
    const int x = s.best_index[g];
    // (empty groups are alike: they take their place in the line)
    rank += before(v, x, best.v, best.i) || (v == best.v && x == best.i && g < group);
  }
  rank = group_sum(rank);
  if (rank == keep - 1 && slice == 0) s.edge_value = best.v, s.edge_index = best.i;
  __syncthreads();
  return Candidate{s.edge_value, s.edge_index};
}

// The `keep` first of the `count` in the list, in order, to s.out_value and s.out_index.
__device__ __forceinline__ void first_of_list(PickShared &s, int keep, int count) {
  const int group = threadIdx.x / kGroup, slice = threadIdx.x % kGroup;
  for (int c0 = 0; c0 < count; c0 += 64) {
    const int c = min(c0 + group, count - 1);
    const Candidate x{s.value[c], s.index[c]};
    int first = 0;
    for (int o = slice; o < count; o += kGroup) first += before(s.value[o], s.index[o], x.v, x.i);
    first = group_sum(first);
    if (slice == 0 && c0 + group < count && first < keep) s.out_value[first] = x.v, s.out_index[first] = x.i;
  }
  __syncthreads();
}

// The `keep` first candidates, in order, to s.out_value and s.out_index; how many there are.  At least
// `keep` reach the edge (or all do): those that do are listed, and a group of threads each counts the
// ones before it.  Where tokens are many, the edge is raised first: of the threads' first ones the keep-th is a
// bound, and a thread has few behind it (28 of 14 x 543 tokens for 21 sequences, where the least chunk has few: 218 us
// or more without, 27 with; 6 of 3 x 278 for 11, where nothing bounds them, 104 and 12; 1024 firsts at most).  Where
// they are still more than the list holds, it is raised to the keep-th candidate itself (eight of 4 x 32000 equal
// tokens: 81 us in all).  s.count is zero.
constexpr int kShort = 256;
template <typename Set>
__device__ __forceinline__ int pick(PickShared &s, int keep, const Set &set, Candidate edge) {
  const int tid = threadIdx.x;
  const auto clear = [&]() {
    __syncthreads();
    if (tid == 0) s.count = 0;
    __syncthreads();
  };
  const auto add = [&](double v, int i) {
    const int at = atomicAdd(&s.count, 1);
    if (at < kList) s.value[at] = v, s.index[at] = i;
  };
  // (a step lists candidates, or threads' first ones; the list is put in order at one place, for less code)
  bool firsts = Set::kRaise && edge.v == kNone, raised = firsts || !Set::kRaise;
#pragma unroll 1
  for (int most = raised ? kList : kShort;;) {
    if (Set::kRaise && firsts) {
      if constexpr (Set::kRaise) {
        const double v = set.greatest();
        if (v > kNone && v >= edge.v) add(v, tid);
      }
    } else {
      set.above(edge.v, [&](double v, int i) {
        if (v > kNone && !before(edge.v, edge.i, v, i)) add(v, i);
      });
    }
    __syncthreads();
    const int count = min(s.count, kList);
    if (!firsts && s.count > most) {
      clear();
      if (raised) {
        edge = find_edge(s, keep, set, edge.v, set.end());
        most = INT32_MAX;
      } else {
        firsts = raised = true;
        most = kList;
      }
      continue;
    }
    first_of_list(s, keep, count);
    if (!firsts) return min(count, keep);
    edge = Candidate{count < keep ? edge.v : s.out_value[keep - 1], INT32_MAX};
    firsts = false;
    clear();
  }
}

// Chunks, each of the value of its greatest token.  A beam's lie in `share` waves.
struct Chunks {
  static constexpr bool kRaise = false;     // (their edge is such a bound)
  const PickShared &s;
  const BeamArgs &a;
  const float *top;         // of the sequence
  int wave, lane, share;

  // place(b, offset): a beam with chunks of this wave's; done(...): one that is done, to one of its threads
  template <typename Place, typename Done>
  __device__ __forceinline__ void walk(Place &&place, Done &&done) const {
#pragma unroll 1
    for (int b = wave / share; b < a.n_beams; b += kPickWaves / share) {
      const double offset = s.offset[b];
      if (offset == kNone) continue;
      if (s.done[b] == 0) {
        place(b, offset);
      } else if (wave % share == 0 && lane == 0) {
        done(offset, b * a.chunks + a.pad_token / kBeamChunk);
      }
    }
  }
  __device__ __forceinline__ Candidate best() const {
    Candidate x{kNone, INT32_MAX};
    const auto with = [&](double v, int i) {
      if (before(v, i, x.v, x.i)) x = Candidate{v, i};
    };
    walk([&](int b, double offset) {
      const float *from = top + b * a.chunks;
      float m = -__builtin_inff();
      int at = 0;
#pragma unroll 4
      for (int c = wave % share * 64 + lane; c < a.chunks; c += 64 * share) {
        const float y = from[c];
        if (y > m) m = y, at = c;
      }
      with(offset + (double)m, b * a.chunks + at);
    }, with);
    return x;
  }
  __device__ __forceinline__ int end() const { return a.n_beams * a.chunks; }
  __device__ __forceinline__ int count(double value, int upto) const {
    int n = 0;
    above(value, [&](double v, int i) { n += v > value || (v == value && i < upto); });
    return n;
  }
  template <typename Take>
  __device__ __forceinline__ void above(double edge, Take &&take) const {
    walk([&](int b, double offset) {
      const float *from = top + b * a.chunks;
      const float least = least_logit(edge, offset);
#pragma unroll 4
      for (int c = wave % share * 64 + lane; c < a.chunks; c += 64 * share) {
        const float y = from[c];
        if (y >= least) take(offset + (double)y, b * a.chunks + c);
      }
    }, take);
  }
};

// Tokens of the chosen chunks: a chunk is a group's, of 16 threads, with four times eight neighbours each.
template <bool FP32>
struct Tokens {
  static constexpr bool kRaise = true;
  const BeamArgs &a;
  const void *row;          // of the chunk
  double offset;            // -infinity: no chunk
  int first, b, done;       // its first token, its beam, whether that is done
  float x[4][8];

  __device__ __forceinline__ Tokens(const PickShared &s, const BeamArgs &a_, int64_t row0, int n_chunks) : a(a_) {
    const int n = threadIdx.x / kGroup;
    b = n < n_chunks ? s.beam[n] : 0;
    offset = n < n_chunks ? s.offset[b] : kNone;
    first = n < n_chunks ? s.token[n] + 8 * (threadIdx.x % kGroup) : 0;
    done = s.done[b];
    row = row_of<FP32>(a, row0 + b);
    if (offset == kNone || done) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) eight<FP32, false>(row, first + 128 * k, a.n_vocab, x[k]);
  }
  __device__ __forceinline__ double greatest() const {
    if (offset == kNone) return kNone;
    if (done) return threadIdx.x % kGroup == 0 ? offset : kNone;
    float m = x[0][0];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, x[k][j]);
    return offset + (double)m;
  }
  __device__ __forceinline__ int end() const { return a.n_beams * a.n_vocab; }
  __device__ __forceinline__ int count(double value, int upto) const {
    if (offset == kNone) return 0;
    const int i0 = b * a.n_vocab;
    if (done) return threadIdx.x % kGroup == 0 && (offset > value || (offset == value && i0 + a.pad_token < upto));
    int n = 0;
#pragma unroll 1
    for (int k = 0; k < 4; ++k) {       // (read again: x stays in registers for few)
      float y[8];
      eight<FP32, false>(row, first + 128 * k, a.n_vocab, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) {     // (past the vocabulary: -infinity, below all values asked for)
        const double v = offset + (double)y[j];
        n += v > value || (v == value && i0 + first + 128 * k + j < upto);
      }
    }
    return n;
  }
  template <typename Take>
  __device__ __forceinline__ void above(double edge, Take &&take) const {
    if (offset == kNone) return;
    if (done) {
      if (threadIdx.x % kGroup == 0) take(offset, b * a.n_vocab + a.pad_token);
      return;
    }
    const float least = least_logit(edge, offset);
    uint32_t bits = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) bits |= x[k][j] >= least ? 1u << (8 * k + j) : 0u;
    // (few: read again, as registers have no index)
#pragma unroll 1
    for (; bits != 0; bits &= bits - 1) {
      const int j = __builtin_ctz(bits), t = first + j / 8 * 128 + j % 8;
      if (t < a.n_vocab) take(offset + (double)logit<FP32>(row, t), b * a.n_vocab + t);
    }
  }
};

template <bool FP32>
__global__ __launch_bounds__(kPickThreads) void beam_pick(BeamArgs a) {
  __shared__ PickShared s;
  const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row0 = (int64_t)seq * a.n_beams;
  int share = kPickWaves;
  while (share > 1 && share * a.n_beams > kPickWaves) share /= 2;
  // ln sum exp: 16 lanes a beam, a part each (all lanes go through, for the moves between them)
#pragma unroll 1
  for (int b0 = 0; b0 < a.n_beams; b0 += kPickThreads / 16) {
    const int b = min(b0 + tid / 16, a.n_beams - 1), p = tid % 16;
    const int64_t r = row0 + b;
    const float at = p < a.parts ? a.peak[r * a.parts + p] : -__builtin_inff();
    double sum = p < a.parts ? a.sum[r * a.parts + p] : 0.0;
    const double score = a.score[r];
    const int done = a.done != nullptr && a.done[r] != 0;
    const float peak = float_of(greater<kTurn8>(greater<kTurn4>(greater<kXor2>(greater<kXor1>(order_of(at))))));
    if (at != peak) sum *= exp((double)at - (double)peak);
    sum = row_sum(sum);     // (a NaN or an infinity of the row makes it a NaN)
    const double offset = done ? score : score - ((double)peak + log(sum));
    if (p == 0) {
      s.offset[b] = __builtin_isfinite(offset) ? offset : kNone;
      s.done[b] = done;
    }
  }
  if (tid == 0) s.count = 0;
  __syncthreads();
  const Chunks chunks{s, a, a.top + row0 * a.chunks, wave, lane, share};
  const int n_chunks = pick(s, a.n_keep, chunks, bound_of(s, a.n_keep, chunks));
  if (tid < n_chunks) {
    const int i = s.out_index[tid], b = i / a.chunks;
    s.beam[tid] = b;
    s.token[tid] = (i - b * a.chunks) * kBeamChunk;
  }
  // Each chosen chunk has a token of its value: with n_keep of them, that of the last is a bound.
  Candidate edge{s.out_value[a.n_keep - 1], INT32_MAX};
  if (tid == 0) s.count = 0;
  __syncthreads();
  const Tokens<FP32> tokens(s, a, row0, n_chunks);
  if (n_chunks < a.n_keep) edge.v = kNone;      // (all chunks were chosen)
  const int n = pick(s, a.n_keep, tokens, edge);
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
  const dim3 rows(a.parts, a.n_seqs * a.n_beams), one(a.n_seqs);
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
