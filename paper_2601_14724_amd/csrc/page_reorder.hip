// Pages of beams after a choice of continuations, for gfx950 (see hermes_page_reorder).
//
// page_reorder   a group (the beams of one sequence in one layer) a workgroup, or several
//                workgroups: each finds the group's new tables, the first writes
//                them, and all share the copies of partly filled pages
//
// A group's room is a range of pages, so that which of them the new tables hold is a bitmap
// in LDS, and a free page a clear bit: no lists or counts are kept between calls, and
// what no beam goes on with is free without being told so.  One launch: the groups need
// nothing of each other.
//
// Few bytes move (tables, and a page's live rows for every beam whose parent has another child), so small
// calls are a chain: parents and lengths, the parents' tables, free pages, copies (one layer of four beams 3.4 us
// without copies and 5.2 with, 1.8 of it an empty launch).  Large ones are bound by the copies, 1 to 16 KiB at random
// places, which go piece by piece (see there): 28 layers of 64 beams move 23 MB, 12.3 us, of which 4.3 are the chain.
#include "tokens_internal.h"

namespace hermes {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

struct ReorderShared {
  uint32_t held[kRoomPages / 32];   // pages of the room that a new table holds
  int32_t parent[kMaxBeams], len[kMaxBeams];   // len: of the old beams, then of the new ones
  int32_t full[kMaxBeams];          // shared pages
  int32_t last[kMaxBeams];          // the parent's partly filled page
  int32_t total[kMaxBeams];         // entries of the new table
  int32_t target[kMaxBeams];        // page that `last` is copied to (-1: none)
  int32_t copied[kMaxBeams];        // the beams that have one
  int32_t copies;
  int32_t free[64 * 32];            // free pages of 64 words of `held`
};

// The sum over the lanes up to this one.
template <int Ctrl, int Rows>
__device__ __forceinline__ int plus(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, Ctrl, Rows, 0xF, false);
}
__device__ __forceinline__ int sum_up_to(int x) {
  x = plus<0x118, 0xF>(plus<0x114, 0xF>(plus<0x112, 0xF>(plus<0x111, 0xF>(x))));
  return plus<0x143, 0xC>(plus<0x142, 0xA>(x));
}

__global__ __launch_bounds__(kThreads) void page_reorder(PageReorderArgs a) {
  __shared__ ReorderShared s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % a.n_groups, share = blockIdx.x / a.n_groups, B = a.n_beams, rows = 1 << a.pool.log_rows;
  const int64_t row0 = (int64_t)g * B;
  // (asked for at once; the lengths are given to the children through LDS)
  int p = -1, n = 0;
  if (tid < B) {
    p = a.parent[(int64_t)(g % a.n_seqs) * B + tid];
    n = a.kv_len[row0 + tid];
  }
  int room = a.room[2 * g], pages = a.room[2 * g + 1];
  if (room < 0 || pages < 0 || pages > kRoomPages || (int64_t)room + pages > a.pool.n_pages) {
    room = pages = 0;
    if (tid == 0) page_note(a.pool, HERMES_PAGE_BAD_ID);
  }
  for (int i = tid; i < (pages + 31) / 32; i += kThreads) s.held[i] = 0;
  if (wave == 0) {
    s.len[lane] = n;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    if (p < -1 || p >= B) {
      p = -1;
      page_note(a.pool, HERMES_PAGE_BAD_PARENT);
    }
    n = p < 0 ? 0 : s.len[p];
    if (n < 0 || n > (int64_t)a.max_pages << a.pool.log_rows) {
      n = 0;
      page_note(a.pool, HERMES_PAGE_BAD_LENGTH);
    }
    const int full = n >> a.pool.log_rows;
    const int want = p < 0 ? 0 : (int)(((int64_t)n + a.grow + rows - 1) >> a.pool.log_rows);
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    s.parent[lane] = p;
    s.len[lane] = n;
    s.full[lane] = full;
    s.total[lane] = min(want, a.max_pages);
    if (want > a.max_pages) page_note(a.pool, HERMES_PAGE_NO_ROOM);
    if (share == 0 && lane < B) a.kv_len_out[row0 + lane] = n;
  }
  __syncthreads();
  // Shared pages, a beam a wave; and the partly filled ones.
  int last = -1;
  if (tid < B && (s.len[tid] & (rows - 1)) != 0) last = a.tables[(row0 + s.parent[tid]) * a.max_pages + s.full[tid]];
  for (int b = wave; b < B; b += kWaves) {
    const int32_t *from = a.tables + (row0 + max(s.parent[b], 0)) * a.max_pages;
    int32_t *to = a.tables_out + (row0 + b) * a.max_pages;
    const int full = s.full[b], total = s.total[b], end = share == 0 ? a.max_pages : full;
    for (int e0 = 0; e0 < end; e0 += 256) {
      int id[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + 64 * k + lane;
        id[k] = e < full ? from[e] : -1;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + 64 * k + lane;
        const unsigned at = (unsigned)id[k] - (unsigned)room;
        if (e < full && at < (unsigned)pages) atomicOr(&s.held[at / 32], 1u << (at % 32));
        // (entries that get a page of their own are written below)
        if (share == 0 && e < end && (e < full || e >= total)) to[e] = id[k];
      }
    }
  }
  if (tid < B) s.last[tid] = last;
  __syncthreads();
  // The first wave, a lane a beam: who goes on in its parent's last page, then the free pages, of which a beam
  // gets the begin-th to the one before the end-th.
  if (wave == 0) {
    const bool part = lane < B && (s.len[lane] & (rows - 1)) != 0;
    const unsigned in_room = (unsigned)last - (unsigned)room;
    bool keep = part && in_room < (unsigned)pages && (s.held[in_room / 32] >> (in_room % 32) & 1) == 0;
    for (int b = 0; b < B; ++b) {     // (of beams with the same last page the first one)
      const int other = __builtin_amdgcn_readlane(part ? last : -1, b);
      if (b < lane && other == last) keep = false;
    }
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    if (keep) {
      atomicOr(&s.held[in_room / 32], 1u << (in_room % 32));
      if (share == 0) a.tables_out[(row0 + lane) * a.max_pages + s.full[lane]] = last;
    }
    const int need = lane < B ? s.total[lane] - s.full[lane] - keep : 0;
    const int end = sum_up_to(need), all = __builtin_amdgcn_readlane(end, 63), begin = end - need;
    const int64_t own = (row0 + lane) * a.max_pages + s.full[lane] + keep;      // the first entry that gets one
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    int given = 0, target = -1;
    for (int w0 = 0; w0 * 32 < pages && given < all; w0 += 64) {
      const int w = w0 + lane, left = pages - 32 * w;
      uint32_t clear = left <= 0 ? 0u : ~s.held[w];
      if (left > 0 && left < 32) clear &= (1u << left) - 1u;
      const int found = __builtin_popcount(clear), upto = sum_up_to(found), most = __builtin_amdgcn_readlane(upto, 63);
      for (int i = upto - found; clear != 0 && given + i < all; clear &= clear - 1, ++i)
        s.free[i] = room + 32 * w + __builtin_ctz(clear);
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      for (int i = max(begin, given); i < min(end, given + most); ++i) {
        const int id = s.free[i - given];
        if (share == 0) a.tables_out[own + i - begin] = id;
        if (i == begin && part && !keep) target = id;
      }
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
      given += most;
    }
    if (given < all) {
      for (int i = max(begin, given); i < end; ++i)
        if (share == 0) a.tables_out[own + i - begin] = -1;
      if (lane == 0) page_note(a.pool, HERMES_PAGE_NO_ROOM);
    }
    s.target[lane] = target;
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    const bool copy = target >= 0 && last >= 0 && last < a.pool.n_pages;
    if (target >= 0 && !copy) page_note(a.pool, HERMES_PAGE_BAD_ID);
    const unsigned long long copies = __ballot(copy);
    if (copy) s.copied[__builtin_popcountll(copies & ((1ull << lane) - 1))] = lane;
    if (lane == 0) s.copies = __builtin_popcountll(copies);
  }
  __syncthreads();
  // Copies: of every KV head's block the starts of K and of V with their scales (see PageBlock), a wave
  // each.  (Four pieces a lane are meant to be in flight.  As compiled, the conditional loads are waited for one by one
  // and three of the four go through scratch memory, 80 bytes a lane: 15.9 MB written where pages and tables
  // are 11.6, 28 layers of 64 beams.)
  const int jobs = s.copies * a.pool.Hkv * 2;
  for (int j = share * kWaves + wave; j < jobs; j += a.shares * kWaves) {
    const int b = s.copied[j / (2 * a.pool.Hkv)], part = j % 2, h = j / 2 % a.pool.Hkv;
    const int n4 = ((s.len[b] & (rows - 1)) + 3) & ~3;
    const int wide = n4 * a.row_bytes / 16, fine = n4 * a.scale_bytes / 8;   // pieces
    const int64_t head = (int64_t)h * a.pool.block_bytes, codes = head + (int64_t)part * rows * a.row_bytes;
    const int64_t scales = head + (int64_t)rows * (2 * a.row_bytes + part * a.scale_bytes);
    const uint8_t *from = a.pool.pages + s.last[b] * a.pool.page_bytes;
    uint8_t *to = a.pool.pages + s.target[b] * a.pool.page_bytes;
    for (int x0 = lane; x0 < wide; x0 += 256) {
      uint4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (x0 + 64 * k < wide) v[k] = *reinterpret_cast<const uint4 *>(from + codes + 16 * (x0 + 64 * k));
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (x0 + 64 * k < wide) *reinterpret_cast<uint4 *>(to + codes + 16 * (x0 + 64 * k)) = v[k];
    }
    for (int x = lane; x < fine; x += 64)
      *reinterpret_cast<uint2 *>(to + scales + 8 * x) = *reinterpret_cast<const uint2 *>(from + scales + 8 * x);
  }
}

}  // namespace

hipError_t launch_page_reorder(const PageReorderArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((page_reorder), dim3(a.n_groups * a.shares), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace hermes
